"""Block-scaled products whose workgroups take several tiles each: what a tile
leaves behind for the next one (row indices of a gather, operands and scales
requested ahead, LDS areas used again) against 64-bit results."""
import pytest
import torch

import scaled_ref as ref
from paper_2410_12247_amd import moe
from test_scaled import BF16, F32, HALF, cuda, ffn_inputs, gen, gpu, run_gemm


def local_dispatch(g, T, k, EL, cap):
    """Every slot of every token on the EL local experts: (offsets, sorted_slot)."""
    ids = torch.rand((T, EL), generator=g).topk(k, 1).indices.flatten()
    order = torch.argsort(ids, stable=True).int()
    off = torch.zeros(EL + 1, dtype=torch.int32)
    off[1:] = torch.bincount(ids, minlength=EL).cumsum(0)
    assert len(order) == cap
    return off, order


# The form is chosen by the rows expected under uniform routing; all slots on the
# local experts are 1.5 to 30 times those, two tiles and more for each of 256
# workgroups.  Tiles of 256 x 256 (with tails), 192 x 256, 128 x 256, 128 x 128 and
# 64 x 128 (token x weight rows), of 2, 2, 2, 3 and 4 LDS buffers; K of fewer pairs
# than those, as many, and more, with and without half a pair at the end.
TILES = {"256x256": (16, 4, 16, 4101, 2112), "192x256": (4, 1, 1, 8001, 4160),
         "128x256": (160, 6, 20, 1300, 2112), "128x128": (40, 4, 8, 900, 2112),
         "64x128": (256, 8, 8, 700, 1088)}
KS = {"256x256": (64, 128, 192, 256, 384), "192x256": (192, 256, 320),
      "128x256": (64, 128, 192, 256, 384), "128x128": (64, 128, 192, 256, 320, 384, 512),
      "64x128": (320, 384, 448, 512, 576, 640)}


@gpu
@pytest.mark.parametrize("tile,K", [(t, k) for t in TILES for k in KS[t]])
def test_group_gemm_of_many_tiles(tile, K):
    E, k, EL, T, N = TILES[tile]
    g = gen(T + N + K)
    d = moe.dims(T, 64, 64, E, k, 0, EL)
    cap = T * min(k, EL)
    off, slot = local_dispatch(g, T, k, EL, cap)
    xq, xs = ref.small_integers(g, T, K), ref.scale_bytes(g, T, K)
    wq = ref.small_integers(g, EL, N, K)
    ws = torch.stack([ref.scale_bytes(g, ref.blocks(N), K) for _ in range(EL)])
    rows = (slot // k).long()
    x = ref.widen(xq, xs, 1)
    want = torch.cat([x[rows[int(off[e]):int(off[e + 1])]] @ ref.widen(wq[e], ws[e], 128).T
                      for e in range(EL)]).to(F32)
    dev = [cuda(t) for t in (off, slot, xq, xs, wq, ws)]
    y = torch.full((cap, N), 55.0, device="cuda")
    moe.gemm_group_scaled(d, 0, EL, *dev, y)
    assert torch.equal(y.cpu(), want)
    y = torch.full((cap, N), 55.0, dtype=BF16, device="cuda")
    moe.gemm_group_scaled(d, 0, EL, *dev, y)
    assert torch.equal(y.cpu(), want.to(BF16))
    # the same rows in dispatch order
    y.fill_(55)
    moe.gemm_group_scaled(d, 0, EL, dev[0], None, cuda(xq[rows]), cuda(xs[rows]), *dev[4:], y)
    assert torch.equal(y.cpu(), want.to(BF16))


# Gate and up tiles of 64, 128 and 256 token rows: local experts, slots and tokens
# as above, I, and the widths H that keep them.
FFN_TILES = {64: (160, 6, 20, 500, 1088), 128: (40, 4, 8, 900, 2112), 256: (16, 4, 16, 2051, 1600)}


@gpu
@pytest.mark.parametrize("H", [64, 128, 192, 256, 384])
@pytest.mark.parametrize("tile", FFN_TILES)
def test_ffn_of_many_tiles(tile, H):
    """An expert alone leaves a workgroup one tile and has the same bits."""
    E, k, EL, T, I = FFN_TILES[tile]
    g = gen(T + H)
    d = moe.dims(T, H, I, E, k, 0, EL)
    cap = T * k
    off, slot = local_dispatch(g, T, k, EL, cap)
    t = ffn_inputs(g, T, H, I, EL)
    ws = torch.empty(moe.scaled_workspace_bytes(d), dtype=torch.uint8, device="cuda")
    offd, slotd, rows = cuda(off), cuda(slot), (slot // k).long()
    ys = [torch.full((cap, H), 33.0, device="cuda") for _ in range(3)]
    moe.ffn_group_scaled(d, 0, EL, offd, slotd, *t, ys[0], ws)
    for e in range(EL):
        moe.ffn_group_scaled(d, e, 1, offd, slotd, *t, ys[1], ws)
    rc = cuda(rows)
    moe.ffn_group_scaled(d, 0, EL, offd, None, t[0].view(torch.uint8)[rc], t[1][rc], *t[2:], ys[2],
                         ws)
    assert torch.equal(ys[0], ys[1]) and torch.equal(ys[0], ys[2])
    # some rows of some experts against 64 bits
    got, x = ys[0].cpu().double(), ref.widen(t[0], t[1], 1)
    for e in (0, EL // 3, EL - 1):
        lo, hi = int(off[e]), int(off[e + 1])
        at = torch.unique(torch.cat([torch.tensor([lo, hi - 1]),
                                     torch.randint(lo, hi, (8,), generator=g)]))
        want, bound = ref.ffn_rows(x[rows[at]], *[ref.widen(t[i][e], t[i + 1][e], 128)
                                                  for i in (2, 4, 6)])
        assert bool(((got[at] - want).abs() <= bound + HALF(F32) * (want.abs() + bound)).all())


@gpu
@pytest.mark.parametrize("R,N,K", [(2200, 16448, 192), (1801, 16448, 320), (5801, 6208, 64)])
def test_gemm_of_many_tiles(R, N, K):
    g = gen(R + N + K)
    xq, wq = ref.small_integers(g, R, K), ref.small_integers(g, N, K)
    xs, ws = ref.scale_bytes(g, R, K), ref.scale_bytes(g, ref.blocks(N), K)
    want = (ref.widen(xq, xs, 1) @ ref.widen(wq, ws, 128).T).to(F32)
    for dtype in (F32, BF16):
        assert torch.equal(run_gemm(xq, xs, wq, ws, dtype), want.to(dtype))
