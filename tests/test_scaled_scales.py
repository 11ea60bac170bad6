"""Scale bytes over their whole range: one operand's far from the other's, the
product of both in the middle, so that every result is an ordinary number."""
import pytest
import torch

import scaled_ref as ref
from paper_2410_12247_amd import moe
from test_scaled import (F32, HALF, cuda, dispatch, ffn_inputs, gen, gpu, large_values, product,
                         run_gemm)
from test_scaled_tiles import local_dispatch

# exponents of x and of w, four of each
FAR = [(-127, 120), (120, -127), (124, -110), (-126, 124)]


def operand(g, e, *shape):
    """Any finite values below the middle, ones of 128 to 448 above it: products of
    2^-2 and more, before the scales' product of 2^-10 to 2^20."""
    return ref.e4m3_random(g, *shape) if e < 0 else large_values(g, *shape)


@gpu
@pytest.mark.parametrize("ex,ew", FAR)
@pytest.mark.parametrize("R", [3, 30, 90, 400])
def test_gemm_of_far_scales(R, ex, ew):
    g = gen(R + ex)
    N, K = 192, 320
    xq, wq = operand(g, ex, R, K), operand(g, ew, N, K)
    xs = ref.scale_bytes(g, R, K, ex, ex + 3)
    ws = ref.scale_bytes(g, ref.blocks(N), K, ew, ew + 3)
    want, bound = product(ref.widen(xq, xs, 1), ref.widen(wq, ws, 128), F32)
    got = run_gemm(xq, xs, wq, ws, F32).double()
    assert bool(((got - want).abs() <= bound).all())


# few rows, gate and up tiles of 64 rows and (the last) of 128; H with and without half a block
@gpu
@pytest.mark.parametrize("ex,ew", FAR)
@pytest.mark.parametrize("T,H,I", [(1, 192, 192), (40, 192, 192), (40, 128, 192), (40, 448, 192),
                                   (200, 192, 192), (1100, 192, 1024)])
def test_ffn_of_far_scales(T, H, I, ex, ew):
    E, k = 4, 2
    g = gen(T + H + ex)
    off, slot, cap = dispatch(g, T, E, k, 0, E, None)
    d = moe.dims(T, H, I, E, k)
    x, xs = operand(g, ex, T, H), ref.scale_bytes(g, T, H, ex, ex + 3)
    stacks = []
    for n, kk, e in ((I, H, ew), (I, H, ew), (H, I, -8)):
        q = operand(g, e, E, n, kk)
        stacks += [q, torch.stack([ref.scale_bytes(g, ref.blocks(n), kk, e, e + 3)
                                   for _ in range(E)])]
    ws = torch.empty(moe.scaled_workspace_bytes(d), dtype=torch.uint8, device="cuda")
    y = torch.zeros((cap, H), device="cuda")
    moe.ffn_group_scaled(d, 0, E, cuda(off), cuda(slot), *map(cuda, (x, xs, *stacks)), y, ws)
    got, xw = y.cpu().double(), ref.widen(x, xs, 1)
    for e in range(E):
        lo, hi = int(off[e]), int(off[e + 1])
        if lo == hi:
            continue
        w = [ref.widen(stacks[i][e], stacks[i + 1][e], 128) for i in (0, 2, 4)]
        rows = (slot[lo:hi] // k).long()
        want, bound = ref.ffn_rows(xw[rows], *w)
        assert bool(((got[lo:hi] - want).abs() <= bound + HALF(F32) * (want.abs() + bound)).all())


@gpu
@pytest.mark.parametrize("H", [128, 192, 576])
def test_far_scales_stay_in_their_rows(H):
    """A few tokens with far scales in an FFN whose workgroups take several tiles of
    64 rows: these are right, and the others have the bits they have without them."""
    E, k, EL, T, I = 160, 6, 20, 500, 1088
    g = gen(H)
    off, slot = local_dispatch(g, T, k, EL, T * k)
    d = moe.dims(T, H, I, E, k, 0, EL)
    t = ffn_inputs(g, T, H, I, EL)
    ws = torch.empty(moe.scaled_workspace_bytes(d), dtype=torch.uint8, device="cuda")
    ys = [torch.zeros((T * k, H), device="cuda") for _ in range(2)]
    moe.ffn_group_scaled(d, 0, EL, cuda(off), cuda(slot), *t, ys[0], ws)
    far = torch.tensor([0, 77, 311, T - 1])
    t[1][far[:2].cuda(), 0] = 3     # 2^-124: nothing beside the row's other blocks
    t[1][far[2].cuda(), :] = 0      # all of a row
    t[1][far[3].cuda(), 0] = 248    # 2^121, gate and up values of 2^120
    moe.ffn_group_scaled(d, 0, EL, cuda(off), cuda(slot), *t, ys[1], ws)
    token = slot // k
    mine = torch.isin(token, far.int())
    assert torch.equal(ys[0].cpu()[~mine], ys[1].cpu()[~mine])
    got, x = ys[1].cpu().double(), ref.widen(t[0], t[1], 1)
    for e in range(EL):
        at = torch.arange(int(off[e]), int(off[e + 1]))
        at = at[mine[at] & (token[at] != T - 1)]  # (the last one's products leave fp32)
        if len(at) == 0:
            continue
        want, bound = ref.ffn_rows(x[token[at].long()],
                                   *[ref.widen(t[i][e], t[i + 1][e], 128) for i in (2, 4, 6)])
        assert bool(((got[at] - want).abs() <= bound + HALF(F32) * (want.abs() + bound)).all())
    assert not bool(torch.isfinite(got[token == T - 1]).all())
