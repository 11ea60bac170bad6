"""Products and FFNs of few rows whose widths take several steps of the kernels'
rings: a wave has 2 blocks of 128 k on the way and comes back for every 16th block
(every 8th in a down product of at most 16 blocks)."""
import pytest
import torch

import scaled_ref as ref
from paper_2410_12247_amd import moe
from test_scaled import BF16, F32, HALF, cuda, dispatch, ffn_inputs, gen, gpu, run_gemm


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("R,N,K", [(1, 256, 2048), (3, 192, 2112), (16, 320, 4160), (7, 5120, 2240),
                                   (16, 4160, 6144), (2, 64, 16448)])
def test_gemm_of_many_steps(R, N, K, dtype):
    g = gen(R + N + K)
    # (small integers at every 7th k: sums stay below 2^24)
    xq, wq = ref.small_integers(g, R, K), ref.small_integers(g, N, K)
    xq[:, torch.arange(K) % 7 != 0] = 0
    xs, ws = ref.scale_bytes(g, R, K, -2, 2), ref.scale_bytes(g, ref.blocks(N), K, -2, 2)
    want = ref.widen(xq, xs, 1) @ ref.widen(wq, ws, 128).T
    assert torch.equal(run_gemm(xq, xs, wq, ws, dtype), want.to(F32).to(dtype))


@gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T,E,k,H,I,pop", [
    (1, 8, 2, 2240, 1344, None),           # gate and up, and the down product of four waves
    (2, 8, 2, 4160, 3648, None),           # and of eight
    (1, 8, 2, 192, 4160, None),
    (13, 4, 1, 2112, 1088, None),
    (24, 4, 1, 2112, 1344, [1, 0, 0, 0]),  # one expert has every row: two rounds of them
    (48, 16, 4, 2112, 192, [9] + [1] * 15)])
def test_ffn_of_many_steps(T, E, k, H, I, pop, dtype):
    g = gen(T + H + I)
    off, slot, cap = dispatch(g, T, E, k, 0, E, pop)
    d = moe.dims(T, H, I, E, k)
    t = ffn_inputs(g, T, H, I, E)
    ws = torch.empty(moe.scaled_workspace_bytes(d), dtype=torch.uint8, device="cuda")
    y = torch.full((cap, H), 33.0, dtype=dtype, device="cuda")
    moe.ffn_group_scaled(d, 0, E, cuda(off), cuda(slot), *t, y, ws)
    got, x = y.cpu().double(), ref.widen(t[0], t[1], 1)
    for e in range(E):
        lo, hi = int(off[e]), int(off[e + 1])
        if lo == hi:
            continue
        want, bound = ref.ffn_rows(x[(slot[lo:hi] // k).long()],
                                   *[ref.widen(t[i][e], t[i + 1][e], 128) for i in (2, 4, 6)])
        off_by = (got[lo:hi] - want).abs()
        assert bool((off_by <= bound + HALF(dtype) * (want.abs() + bound)).all())
        # the bound lets every value next to a rounding border flip; few do
        assert float(off_by.norm() / want.norm()) < 0.02
