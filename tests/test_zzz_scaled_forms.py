"""Which kernel the sizes of the 8-bit operators' tests reach, read from a trace of
the call: a rule that changes shows here which tests have lost their form."""
import re

import pytest
import torch

import scaled_ref as ref
from paper_2410_12247_amd import moe
from test_scaled import BF16, F32, FFNS, GROUPS, gpu
from test_scaled_tiles import FFN_TILES, KS, TILES


def kernels(call):
    """The names of the call's kernels, in order."""
    from torch.profiler import ProfilerActivity, profile
    call()  # (nothing of the first call's set-up)
    torch.cuda.synchronize()
    with profile(activities=[ProfilerActivity.CUDA]) as p:
        call()
        torch.cuda.synchronize()
    events = sorted(p.events(), key=lambda e: e.time_range.start)
    names = [re.search(r"(\w+_kernel<[^>]*>)", e.name) for e in events]
    return [m.group(1) for m in names if m]


def zeros(*shape):
    return torch.zeros(shape, dtype=torch.uint8, device="cuda")


def product(R, N, K, dtype=BF16):
    y = torch.empty((R, N), dtype=dtype, device="cuda")
    a = zeros(R, K), zeros(R, ref.pitch(K)), zeros(N, K), zeros(ref.blocks(N), ref.pitch(K))
    return kernels(lambda: moe.gemm_scaled(*a, y))


def stacks(EL, *shapes):
    return [t for n, k in shapes for t in (zeros(EL, n, k), zeros(EL, ref.blocks(n), ref.pitch(k)))]


def group(T, E, k, e0, EL, N, K):
    d = moe.dims(T, 64, 64, E, k, e0, EL)
    cap = T * min(k, EL)
    off, slot = (torch.zeros(n, dtype=torch.int32, device="cuda") for n in (EL + 1, cap))
    y = torch.empty((cap, N), dtype=BF16, device="cuda")
    a = zeros(T, K), zeros(T, ref.pitch(K)), *stacks(EL, (N, K))
    return kernels(lambda: moe.gemm_group_scaled(d, 0, EL, off, slot, *a, y))


def ffn(T, E, k, e0, EL, H, I):
    d = moe.dims(T, H, I, E, k, e0, EL)
    cap = T * min(k, EL)
    off, slot = (torch.zeros(n, dtype=torch.int32, device="cuda") for n in (EL + 1, cap))
    y = torch.empty((cap, H), dtype=BF16, device="cuda")
    ws = zeros(moe.scaled_workspace_bytes(d))
    a = zeros(T, H), zeros(T, ref.pitch(H)), *stacks(EL, (I, H), (I, H), (H, I))
    return kernels(lambda: moe.ffn_group_scaled(d, 0, EL, off, slot, *a, y, ws))


ONE, TWO = "stream_kernel<2, false, 1, 8, 2>", "stream_kernel<2, false, 2, 8, 2>"
GATE_UP = "stream_kernel<0, false, 2, 8, 2>"
DOWN = {w: f"stream_kernel<2, true, 2, {w}, 2>" for w in (4, 8)}


def tile(bm, bn):
    return f"tile_kernel<2, {bm}, {bn}>"


def gate_up(bm):
    return f"tile_kernel<0, {bm}, 256>"


@gpu
@pytest.mark.parametrize("R,N,K,name", [
    (1, 64, 64, ONE), (16, 192, 1344, ONE), (16, 33024, 4096, TWO), (16, 5120, 2240, TWO),
    (17, 64, 320, "mid_kernel<2>"), (300, 704, 1088, "mid_kernel<2>"), (700, 1024, 320, tile(64, 128)),
    (1100, 1472, 192, tile(128, 128)), (2000, 2112, 320, tile(128, 256)),
    (2500, 3904, 320, tile(192, 256)), (1801, 16448, 320, tile(192, 256)),
    (2950, 4160, 192, tile(256, 256)), (2068, 8192, 64, tile(256, 256)),
    (2200, 16448, 192, tile(256, 256)), (5801, 6208, 64, tile(256, 256))])
def test_product(R, N, K, name):
    assert product(R, N, K) == [name]
    assert product(R, N, K, F32) == [name.replace("<2", "<1")]


@gpu
def test_group_products():
    forms = [ONE, ONE, "mid_kernel<2>", "mid_kernel<2>", "mid_kernel<2>", tile(128, 128),
             "mid_kernel<2>", tile(128, 128), tile(128, 128), tile(128, 128), tile(128, 256),
             tile(256, 256), tile(256, 256), tile(128, 128), ONE]
    assert [group(*c[:-1]) for c in GROUPS] == [[f] for f in forms]


@gpu
@pytest.mark.parametrize("name", TILES)
def test_group_products_of_many_tiles(name):
    E, k, EL, T, N = TILES[name]
    bm, bn = map(int, name.split("x"))
    for K in KS[name]:
        assert group(T, E, k, 0, EL, N, K) == [tile(bm, bn)], K


@gpu
def test_ffns():
    forms = [[GATE_UP, DOWN[4]], [GATE_UP, DOWN[4]], [gate_up(64), "mid_kernel<2>"],
             [gate_up(64), "mid_kernel<2>"], [gate_up(64), "mid_kernel<2>"],
             [gate_up(64), "mid_kernel<2>"], [gate_up(128), tile(64, 128)],
             [gate_up(256), tile(64, 128)]]
    assert [ffn(*c[:-1]) for c in FFNS] == forms


@gpu
@pytest.mark.parametrize("bm", FFN_TILES)
def test_gate_up_of_many_tiles(bm):
    E, k, EL, T, I = FFN_TILES[bm]
    for H in (64, 128, 192, 256, 384):
        assert ffn(T, E, k, 0, EL, H, I)[0] == gate_up(bm), H


@gpu
@pytest.mark.parametrize("T,E,k,H,I,names", [
    (1, 8, 2, 2240, 1344, [GATE_UP, DOWN[4]]), (2, 8, 2, 4160, 3648, [GATE_UP, DOWN[8]]),
    (48, 16, 4, 2112, 192, [GATE_UP, DOWN[4]]), (49, 16, 4, 2112, 192, [gate_up(64), tile(128, 256)]),
    (40, 4, 2, 192, 192, [gate_up(64), "mid_kernel<2>"]),
    (200, 4, 2, 192, 192, [gate_up(64), "mid_kernel<2>"]),
    (1100, 4, 2, 192, 1024, [gate_up(128), tile(64, 128)])])
def test_ffn(T, E, k, H, I, names):
    assert ffn(T, E, k, 0, E, H, I) == names


@gpu
@pytest.mark.parametrize("T,narrow,wide", [(16, TWO, TWO), (17, "mid_kernel<2>", TWO),
                                           (32, tile(128, 128), TWO),
                                           (33, tile(128, 128), tile(64, 128))])
def test_products_around_the_borders_of_few_rows(T, narrow, wide):
    assert group(T, 32, 4, 0, 8, 1088, 192) == [narrow]
    assert group(T, 32, 4, 0, 8, 20480, 4096) == [wide]
