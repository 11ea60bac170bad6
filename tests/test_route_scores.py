"""Routing by scores (softmax or sigmoid, bias, groups, top-k, weights) and its
gradient through the Python binding, against the 64-bit definition; what the
calls refuse; a layer routed by them."""
import ctypes
import math

import numpy as np
import pytest
import torch

import route_scores_ref as ref
from paper_2410_12247_amd import moe

gpu = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
FAKE = ctypes.c_void_p(4096)  # never dereferenced
ODD = ctypes.c_void_p(4096 + 1)
SCORE = {True: moe.SCORE_SIGMOID, False: moe.SCORE_SOFTMAX}


def last():
    return moe.lib().moe_last_error().decode()


# ---- refusals: host only --------------------------------------------------


@pytest.mark.parametrize("backward", [False, True])
def test_refusals(backward):
    L = moe.lib()
    d = moe.dims(5, 64, 64, 12, 3)

    def call(d=d, r=moe.routing(0, 4, 2), z=FAKE, t=1, ids=FAKE, w=FAKE, bias=None, dz=FAKE):
        rp = ctypes.byref(r) if r is not None else None
        dp = ctypes.byref(d) if d is not None else None
        if backward:
            return L.moe_route_scores_backward(dp, rp, z, t, ids, w, dz, None)
        return L.moe_route_scores(dp, rp, z, t, bias, ids, w, None)
    bad = [dict(d=None), dict(r=None), dict(r=moe.routing(2)), dict(r=moe.routing(-1)),
           dict(r=moe.routing(0, 5, 1)), dict(r=moe.routing(0, 0, 0)),
           dict(r=moe.routing(0, 4, 0)), dict(r=moe.routing(0, 4, 5)),
           dict(r=moe.routing(0, 6, 1)),  # two experts in the group kept
           dict(r=moe.routing(0, 4, 2, 2)), dict(r=moe.routing(0, 4, 2, 0, math.inf)),
           dict(r=moe.routing(0, 4, 2, 0, math.nan)), dict(t=2), dict(t=-1), dict(z=None),
           dict(ids=None), dict(w=None), dict(z=ODD), dict(ids=ODD), dict(w=ODD), dict(t=0, z=ODD)]
    bad += [dict(dz=None), dict(dz=ODD)] if backward else [dict(bias=ODD)]
    for b in bad:
        assert call(**b) == 1, (b, last())
    assert call(d=moe.dims(5, 64, 64, 257, 3)) == 2
    assert call(d=moe.dims(5, 64, 64, 12, 9)) == 2
    assert call(d=moe.dims(1 << 28, 64, 64, 12, 3)) == 2
    assert call(d=moe.dims(0, 64, 64, 12, 3), z=None, ids=None, w=None, dz=None) == 0


def test_logits_refusals():
    L = moe.lib()
    d = moe.dims(5, 64, 64, 12, 3)

    def call(d=d, x=FAKE, w=FAKE, z=FAKE):
        return L.moe_route_logits(ctypes.byref(d), x, w, z, None)
    for b in (dict(x=None), dict(w=None), dict(z=None), dict(x=ctypes.c_void_p(4096 + 2)),
              dict(w=ODD), dict(z=ODD), dict(d=moe.dims(5, 65, 64, 12, 3))):
        assert call(**b) == 1, (b, last())
    assert call(d=moe.dims(0, 64, 64, 12, 3), x=None) == 0


def test_binding_refuses_what_it_cannot_pass():
    d, r = moe.dims(4, 64, 64, 8, 2), moe.routing()
    z = torch.zeros((4, 8))
    with pytest.raises(ValueError, match="contiguous device tensor"):
        moe.route_scores(d, r, z, None, z, z)
    with pytest.raises(ValueError):
        moe.route_scores_backward(d, r, z, z, z, z)
    with pytest.raises(ValueError):
        moe.route_logits(d, z, z, z)


def test_reference_gradient_is_the_difference_quotient():
    rng = np.random.default_rng(3)
    for sigmoid in (False, True):
        for renorm in (False, True):
            z = rng.standard_normal((1, 9))
            ids = np.array([[2, 7, 7, -1]])
            on = ids[0, :3]
            dw = rng.standard_normal((1, 4))
            dz = ref.route_backward(z, ids, dw, sigmoid, renorm, 1.7)
            for e in range(9):
                h = np.zeros(9)
                h[e] = 1e-6
                hi, lo = (ref.weights_of(z[0] + f * h, on, sigmoid, renorm, 1.7) for f in (1, -1))
                # central differences: h^2 / 6 times a third derivative below 10, plus
                # 2^-52 / h of rounding
                assert abs((hi - lo) @ dw[0, :3] / 2e-6 - dz[0, e]) < 1e-8


# ---- choice and weights -----------------------------------------------------

RULES = [  # experts, top_k, groups, top_groups
    (1, 1, 1, 1), (2, 2, 1, 1), (7, 3, 1, 1), (8, 2, 1, 1), (16, 4, 4, 2), (60, 4, 1, 1),
    (63, 8, 7, 3), (64, 6, 1, 1), (64, 8, 64, 8), (65, 5, 5, 1), (96, 6, 4, 2), (100, 8, 50, 5),
    (128, 8, 1, 1), (129, 1, 3, 2), (160, 6, 8, 3), (161, 5, 7, 3), (200, 3, 5, 2), (255, 8, 15, 4),
    (256, 8, 8, 4), (256, 8, 1, 1), (256, 2, 256, 3), (256, 8, 2, 1)]


def make(seed, T, E, dtype, masked=0, sigmoid=False):
    g = torch.Generator().manual_seed(seed)
    z = torch.randn((T, E), generator=g) * 1.5 - (1 if sigmoid else 0)
    z[:, torch.randperm(E, generator=g)[:masked]] = -math.inf
    return z.to(dtype).cuda()


def run(z, bias, k, sigmoid, groups, top_groups, pair, renorm, scale, stream=None):
    T, E = z.shape
    ids = torch.full((T, k), -7, dtype=torch.int32, device="cuda")
    w = torch.full((T, k), -7.0, device="cuda")
    d = moe.dims(T, 64, 64, E, k, renormalize=renorm)
    r = moe.routing(SCORE[sigmoid], groups, top_groups,
                    moe.GROUP_TOP_TWO if pair else moe.GROUP_MAX, scale)
    moe.route_scores(d, r, z, bias, ids, w, stream)
    return ids, w


def check(z, bias, k, **rules):
    ids, w = run(z, bias, k, **rules)
    rid, rw = ref.route(z.double().cpu().numpy(), None if bias is None else
                        bias.double().cpu().numpy(), k, **rules)
    np.testing.assert_array_equal(ids.cpu().numpy(), rid)
    # computed in 64 bits and rounded once: 2^-24, and 2^-30 for the 64-bit steps
    got = w.double().cpu().numpy()
    np.testing.assert_array_equal(np.isnan(got), np.isnan(rw))
    ok = ~np.isnan(rw)
    # below fp32's normal range a rounding is half of 2^-149
    assert (np.abs(got - rw)[ok] <= np.abs(rw[ok]) * (2.0 ** -24 + 2.0 ** -30) + 2.0 ** -150).all()
    return ids, w


@gpu
@pytest.mark.parametrize("rule", RULES, ids=lambda r: "x".join(map(str, r)))
@pytest.mark.parametrize("sigmoid", [False, True], ids=["softmax", "sigmoid"])
def test_choice_and_weights(rule, sigmoid):
    E, k, G, top = rule
    for i, (T, dtype, bias, pair, renorm, masked) in enumerate([
            (1, F32, True, True, True, 0), (5, BF16, False, False, False, 0),
            (37, F32, False, True, True, E // 8), (66, BF16, True, False, False, E // 3),
            (130, F32, True, True, False, 0), (33, F32, False, False, True, E // 2)]):
        z = make(100 * E + i, T, E, dtype, masked, sigmoid)
        b = torch.randn(E, generator=torch.Generator().manual_seed(i)).mul(0.1).cuda() \
            if bias else None
        check(z, b, k, sigmoid=sigmoid, groups=G, top_groups=top, pair=pair, renorm=renorm,
              scale=2.5 if i % 2 else 1.0)


@gpu
@pytest.mark.parametrize("sigmoid", [False, True], ids=["softmax", "sigmoid"])
@pytest.mark.parametrize("bias", [False, True], ids=["plain", "bias"])
def test_ties_go_to_the_lowest(sigmoid, bias):
    """Logits of three values, a bias of two: most choices are equal."""
    for E, k, G, top in ((8, 2, 1, 1), (64, 8, 8, 2), (200, 6, 10, 3), (256, 8, 1, 1)):
        g = torch.Generator().manual_seed(E)
        z = torch.randint(0, 3, (50, E), generator=g).float().cuda()
        b = (torch.randint(0, 2, (E,), generator=g) * 0.5).cuda() if bias else None
        for pair in (False, True):
            check(z, b, k, sigmoid=sigmoid, groups=G, top_groups=top, pair=pair, renorm=True,
                  scale=1.0)
    z = torch.zeros((3, 256), device="cuda")
    z[1] = -0.0
    z[2, ::2] = -0.0
    ids, _ = run(z, None, 8, sigmoid, 1, 1, False, True, 1.0)
    assert (ids.cpu() == torch.arange(8)).all()


@gpu
def test_near_choices_are_told_apart():
    """Scores that differ by less than fp32 can hold, and biases that make
    choices of different scores meet within 2^-40."""
    E, k = 256, 8
    g = torch.Generator().manual_seed(1)
    z = 1 + torch.arange(E).float() * 2.0 ** -23  # neighbours in fp32
    z = torch.stack([z[torch.randperm(E, generator=g)] for _ in range(40)]).cuda()
    for sigmoid in (False, True):
        for bias in (None, torch.zeros(E, device="cuda"), torch.full((E,), 0.3, device="cuda")):
            check(z, bias, k, sigmoid=sigmoid, groups=1, top_groups=1, pair=False, renorm=False,
                  scale=1.0)
            check(z, bias, k, sigmoid=sigmoid, groups=16, top_groups=4, pair=True, renorm=True,
                  scale=1.0)
    # choices near 1 from the bias' side: fp32(1 - s) differs from 1 - s by up to 2^-25
    z = make(5, 1, E, F32, sigmoid=True)
    b = (1 - torch.sigmoid(z[0].double())).float()
    check(z.expand(9, E).contiguous(), b, k, sigmoid=True, groups=8, top_groups=4, pair=True,
          renorm=True, scale=1.0)


@gpu
@pytest.mark.parametrize("sigmoid", [False, True], ids=["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [False, True], ids=["raw", "renorm"])
def test_rows_with_little_left(sigmoid, renorm):
    """Rows whose mask leaves nothing, one expert, or one group; the lowest finite
    value as a mask; far logits."""
    E, k = 48, 4
    low = torch.finfo(F32).min
    z = make(9, 12, E, F32).cpu()
    z[0] = -math.inf
    z[1] = -math.inf
    z[1, 47] = 0.5
    z[2, 6:] = -math.inf
    z[3] = low
    z[4] = low
    z[4, 5] = 3.0
    z[5] = 80.0
    z[5, 3] = -80.0
    z[6] *= 300  # s underflows beside the largest
    z[7] = -700 + z[7]
    z[8] = torch.finfo(F32).max
    z[9, ::2] = torch.finfo(F32).tiny
    for bias in (None, torch.linspace(-0.2, 0.2, E).cuda()):
        for G, top, pair in ((1, 1, False), (8, 2, False), (8, 2, True), (8, 8, True)):
            check(z.cuda(), bias, k, sigmoid=sigmoid, groups=G, top_groups=top, pair=pair,
                  renorm=renorm, scale=1.0)


@gpu
@pytest.mark.parametrize("sigmoid", [False, True], ids=["softmax", "sigmoid"])
def test_large_logits(sigmoid):
    """Logits from 2^20 to 2^100, where a product with log2(e) is rounded by more than
    the exponent's range."""
    E, k = 96, 6
    z = make(13, 81, E, F32).cpu()
    z *= (2.0 ** torch.arange(20, 101)).float()[:, None]
    z[::2, 1:] = make(14, 41, E - 1, F32).cpu()  # one large beside ordinary ones
    z[::4, 0] = z[::4, 0].abs()
    for T in (81, 81 * 203):
        zt = z.repeat(T // 81, 1).cuda()
        for dtype in (F32, BF16):
            for bias in (None, torch.linspace(0.1, -0.1, E).cuda()):
                for G, top, pair in ((1, 1, False), (8, 3, False), (8, 3, True)):
                    rules = dict(sigmoid=sigmoid, groups=G, top_groups=top, pair=pair,
                                 renorm=True, scale=1.0)
                    ids, w = check(zt[:81].to(dtype), bias, k, **rules)
                    ids2, w2 = run(zt.to(dtype), bias, k, **rules)
                    assert torch.equal(ids2, ids.repeat(T // 81, 1))
                    assert torch.equal(w2, w.repeat(T // 81, 1))


@gpu
@pytest.mark.parametrize("sigmoid", [False, True], ids=["softmax", "sigmoid"])
def test_infinities_and_nan(sigmoid):
    E, k = 40, 3
    z = make(11, 8, E, F32).cpu()
    z[1, 17] = math.nan
    z[2, :] = math.nan
    z[3, 5] = math.inf
    z[4, 5] = z[4, 30] = math.inf
    z[5, 4] = math.nan
    z[5, 6:] = -math.inf
    z[6, 3] = math.nan
    z[6, 39] = math.inf
    for dtype in (F32, BF16):
        for bias in (None, torch.linspace(0.1, -0.1, E).cuda()):
            check(z.to(dtype).cuda(), bias, k, sigmoid=sigmoid, groups=5, top_groups=2, pair=True,
                  renorm=True, scale=1.0)
    # a bias that switches off, forces, or is NaN
    b = torch.zeros(E)
    b[3], b[4], b[20] = -math.inf, math.inf, math.nan
    z = make(12, 30, E, F32)
    for G, top in ((1, 1), (5, 2)):
        ids, _ = check(z, b.cuda(), k, sigmoid=sigmoid, groups=G, top_groups=top, pair=True,
                       renorm=False, scale=1.0)
        assert not ((ids == 3) | (ids == 20)).any() and (ids[:, 0] == 4).all()


@gpu
@pytest.mark.parametrize("T", [4096, 70001])
def test_many_tokens(T):
    z = make(21, T, 256, F32, sigmoid=True)
    b = torch.randn(256, generator=torch.Generator().manual_seed(2)).mul(0.1).cuda()
    ids, w = run(z, b, 8, True, 8, 4, True, True, 2.5)
    at = torch.arange(0, T, 97)
    rid, rw = ref.route(z[at.cuda()].double().cpu().numpy(), b.double().cpu().numpy(), 8,
                        sigmoid=True, groups=8, top_groups=4, pair=True, renorm=True, scale=2.5)
    np.testing.assert_array_equal(ids[at.cuda()].cpu().numpy(), rid)
    np.testing.assert_allclose(w[at.cuda()].cpu().numpy(), rw, rtol=2.0 ** -23)
    assert (ids >= 0).all() and (ids.sort(1).values.diff(dim=1) > 0).all()
    ids2, w2 = run(z, b, 8, True, 8, 4, True, True, 2.5)
    assert torch.equal(ids, ids2) and torch.equal(w, w2)


@gpu
@pytest.mark.parametrize("E,k,G,top", [(65, 5, 1, 1), (100, 8, 1, 1), (128, 8, 4, 2),
                                       (160, 6, 8, 3), (161, 5, 7, 3), (200, 3, 1, 1),
                                       (256, 8, 8, 4), (256, 7, 2, 1), (256, 8, 16, 5)])
def test_rules_over_many_tokens(E, k, G, top):
    T = 16387
    b = torch.randn(E, generator=torch.Generator().manual_seed(2)).mul(0.1).cuda()
    b[E // 2], b[3] = -math.inf, math.nan
    at = torch.cat([torch.arange(0, T, 211), torch.arange(T - 9, T)]).cuda()
    for i, (sigmoid, bias, pair, renorm, dtype, masked) in enumerate([
            (True, b, True, True, F32, 0), (False, None, False, False, F32, 0),
            (False, b, True, False, F32, 5), (True, None, True, False, BF16, 0),
            (False, None, True, True, BF16, 9), (True, b, False, False, BF16, 0)]):
        z = make(E + i, T, E, dtype, masked, sigmoid)
        z[211 * 3, 7], z[211 * 5] = math.nan, -math.inf
        z[T - 2, :9] = 1.5  # ties
        rules = dict(sigmoid=sigmoid, groups=G, top_groups=top, pair=pair, renorm=renorm, scale=1.5)
        ids, w = run(z, bias, k, **rules)
        rid, rw = ref.route(z[at].double().cpu().numpy(),
                            None if bias is None else b.double().cpu().numpy(), k, **rules)
        np.testing.assert_array_equal(ids[at].cpu().numpy(), rid)
        np.testing.assert_allclose(w[at].cpu().numpy(), rw, rtol=2.0 ** -23, atol=2.0 ** -150)
        # the tokens in parts of few: the same
        ids2, w2 = run(z[:5000], bias, k, **rules)
        assert torch.equal(ids[:5000], ids2)
        assert torch.equal(w[:5000].view(torch.int32), w2.view(torch.int32))


def compare(z, bias, k, at, **rules):
    """run() over all tokens against 64 bits at some."""
    ids, w = run(z, bias, k, **rules)
    rid, rw = ref.route(z[at].double().cpu().numpy(),
                        None if bias is None else bias.double().cpu().numpy(), k, **rules)
    np.testing.assert_array_equal(ids[at].cpu().numpy(), rid)
    np.testing.assert_allclose(w[at].cpu().numpy(), rw, rtol=2.0 ** -23, atol=2.0 ** -150)


@gpu
@pytest.mark.parametrize("sigmoid", [False, True], ids=["softmax", "sigmoid"])
@pytest.mark.parametrize("E,k,G,top", [(256, 8, 8, 4), (256, 8, 1, 1), (160, 6, 8, 3),
                                       (200, 3, 5, 2), (12, 4, 3, 2)])
def test_biases_of_any_size(E, k, G, top, sigmoid):
    """Finite biases on either side of 4: as a common offset, at one expert or at some
    among small ones, and so large that scores vanish beside them."""
    g = torch.Generator().manual_seed(E)
    small = torch.randn(E, generator=g) * 0.1
    some = small.clone()
    some[::5], some[1::7], some[3] = -10.0, 20.0, 1e3
    one = small.clone()
    one[E // 3] = -10.0
    biases = [small + c for c in (3.5, -3.5, 3.9, 4.1, -4.1, 20.0, -20.0)]
    biases += [one, -one, some, -some, torch.full((E,), 1e30), torch.full((E,), -3e38)]
    for T in (37, 16387):
        z = make(E + T, T, E, F32, 0, sigmoid)
        at = torch.arange(0, T, 37 if T < 100 else 1021).cuda()
        at = torch.cat([torch.arange(30).cuda(), at, torch.arange(T - 3, T).cuda()])
        for i, b in enumerate(biases):
            compare(z.to(BF16) if i % 4 == 3 else z, b.cuda(), k, at, sigmoid=sigmoid, groups=G,
                    top_groups=top, pair=i % 2 == 0, renorm=i % 3 == 0, scale=2.0)


@gpu
@pytest.mark.parametrize("T", [997, 16387])
def test_what_fp32_does_not_decide(T):
    """Softmax scores with a bias of their size, and logits of which the last chosen
    lie far below the largest: many tokens, or all, are done in 64 bits."""
    at = torch.arange(0, T, T // 60).cuda()
    for E, k, G, top in ((256, 8, 8, 4), (256, 8, 1, 1), (160, 6, 8, 3)):
        g = torch.Generator().manual_seed(E)
        z = torch.randn((T, E), generator=g).cuda()
        b = (torch.randn(E, generator=g) / E).cuda()
        for pair in (False, True):
            for renorm in (False, True):
                rules = dict(sigmoid=False, groups=G, top_groups=top, pair=pair, renorm=renorm,
                             scale=1.0)
                compare(z * 0.3, b, k, at, **rules)
                compare(z * 0.001, b, k, at, **rules)
                compare(z * 8, None, k, at, **rules)
                compare(z * 8, b, k, at, **rules)
                compare(z * 8, None, k, at, **{**rules, "sigmoid": True})


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_any_address(dtype):
    """Logits and outputs at any address of their type, the bytes around untouched."""
    for E, k in ((60, 4), (64, 8), (161, 5), (256, 8)):
        z = make(E, 19, E, dtype)
        want = check(z, None, k, sigmoid=False, groups=1, top_groups=1, pair=False, renorm=False,
                     scale=1.0)
        for off in (1, 2, 3):
            flat = torch.zeros(19 * E + 8, dtype=dtype, device="cuda")
            zo = flat[off:off + 19 * E].view(19, E)
            zo.copy_(z)
            ids = torch.full((19 * k + 8,), -9, dtype=torch.int32, device="cuda")
            w = torch.full((19 * k + 8,), -9.0, device="cuda")
            part = slice(off, off + 19 * k)
            d, r = moe.dims(19, 64, 64, E, k, renormalize=False), moe.routing()
            moe.route_scores(d, r, zo, None, ids[part].view(19, k), w[part].view(19, k))
            assert torch.equal(ids[part].view(19, k), want[0])
            assert torch.equal(w[part].view(19, k), want[1])
            for t in (ids, w):
                assert (t[:off] == -9).all() and (t[off + 19 * k:] == -9).all()


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_many_tokens_at_any_address(dtype):
    """The same choices and weights where rows do not load four at a time."""
    T, E, k = 16390, 160, 6
    z = make(15, T, E, dtype)
    flat = torch.zeros(T * E + 8, dtype=dtype, device="cuda")
    zo = flat[1:1 + T * E].view(T, E)
    zo.copy_(z)
    for sigmoid, renorm in ((True, True), (False, False)):
        rules = dict(sigmoid=sigmoid, groups=8, top_groups=3, pair=True, renorm=renorm, scale=2.0)
        want, got = run(z, None, k, **rules), run(zo, None, k, **rules)
        assert torch.equal(got[0], want[0])
        assert ((got[1] - want[1]).abs() <= 2.0 ** -23 * want[1]).all()
        rid, _ = ref.route(z[:40].double().cpu().numpy(), None, k, **rules)
        np.testing.assert_array_equal(got[0][:40].cpu().numpy(), rid)


# ---- gradient ---------------------------------------------------------------


def back(z, ids, dw, sigmoid, renorm, scale):
    T, E = z.shape
    dz = torch.full_like(z, 7.0)
    d = moe.dims(T, 64, 64, E, ids.shape[1], renormalize=renorm)
    moe.route_scores_backward(d, moe.routing(SCORE[sigmoid], scale=scale), z, ids, dw, dz)
    return dz


def check_back(z, ids, dw, sigmoid, renorm, scale):
    dz = back(z, ids, dw, sigmoid, renorm, scale).double().cpu().numpy()
    zn, idn, dwn = z.double().cpu().numpy(), ids.cpu().numpy(), dw.double().cpu().numpy()
    want = ref.route_backward(zn, idn, dwn, sigmoid, renorm, scale)
    # one rounding to the output's type; the terms in fp32 or better, each within
    # 2^-20 of the largest |G| (s, q <= 1), and differences of them.  bf16 keeps
    # fp32's exponents.
    half = 2.0 ** -24 if z.dtype == F32 else 2.0 ** -8
    g = np.abs(dwn * scale).max(1, keepdims=True)
    assert (np.abs(dz - want) <= half * np.abs(want) + 2.0 ** -20 * g).all()
    return dz


@gpu
@pytest.mark.parametrize("rule", RULES, ids=lambda r: "x".join(map(str, r)))
@pytest.mark.parametrize("sigmoid", [False, True], ids=["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [False, True], ids=["raw", "renorm"])
def test_gradient(rule, sigmoid, renorm):
    E, k, G, top = rule
    for T, dtype, masked in ((1, F32, 0), (6, BF16, 0), (67, F32, E // 3)):
        z = make(E + T, T, E, dtype, masked, sigmoid)
        ids, _ = run(z, None, k, sigmoid, G, top, False, renorm, 2.5)
        dw = torch.randn((T, k), generator=torch.Generator().manual_seed(T)).cuda()
        check_back(z, ids, dw, sigmoid, renorm, 2.5)


@gpu
@pytest.mark.parametrize("sigmoid", [False, True], ids=["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [False, True], ids=["raw", "renorm"])
def test_gradient_of_odd_choices(sigmoid, renorm):
    """No expert, ids out of range, one expert twice, far logits, rows switched off."""
    z = make(31, 9, 70, F32).cpu()
    z[5] = -math.inf
    z[6] = 60 * z[6]
    z[7, 4:] = -math.inf
    ids = torch.randint(0, 70, (9, 5), generator=torch.Generator().manual_seed(1)).int()
    ids[0] = -1
    ids[1, 2:] = -1
    ids[2] = torch.tensor([70, 71, 2 ** 31 - 1, -2 ** 31, 4])
    ids[3, :] = 9
    ids[4] = torch.tensor([8, 9, 8, 9, 8])
    ids[5] = -1
    ids[7] = torch.tensor([0, 1, 2, 3, -1])
    dw = torch.randn((9, 5), generator=torch.Generator().manual_seed(2))
    dz = check_back(z.cuda(), ids.cuda(), dw.cuda(), sigmoid, renorm, 1.5)
    assert (dz[0] == 0).all() and (dz[5] == 0).all()


def exact_gradient(z, ids, dw, sigmoid, renorm, scale):
    """dz and the sum of its terms' magnitudes without a difference of sums:
    s_e sum_i s_i (g_e - g_i) over all experts, g the gradient of their weights; over
    the chosen slots with s of those alone where renormalised (times 1 - s of a
    sigmoid's logit); in the host's longest type."""
    f = np.longdouble
    z, g = z.astype(f), dw.astype(f) * f(scale)
    dz, size = np.zeros(z.shape, f), np.zeros(z.shape, f)
    for t in range(len(z)):
        on = ids[t] >= 0
        at = ids[t][on]
        if not len(at):
            continue
        if not renorm:
            gt = np.zeros(z.shape[1], f)
            np.add.at(gt, at, g[t][on])
        if sigmoid and not renorm:
            dz[t] = gt / (1 + np.exp(-z[t])) / (1 + np.exp(z[t]))
            size[t] = np.abs(dz[t])
            continue
        zt, gt = (z[t][at], g[t][on]) if renorm else (z[t], gt)
        s = 1 / (1 + np.exp(-zt)) if sigmoid else np.exp(zt - zt.max())
        s = s / s.sum()
        terms = (gt[:, None] - gt) * s * s[:, None]
        if sigmoid:
            terms = terms / (1 + np.exp(zt))[:, None]
        if renorm:
            np.add.at(dz[t], at, terms.sum(1))
            np.add.at(size[t], at, np.abs(terms).sum(1))
        else:
            dz[t], size[t] = terms.sum(1), np.abs(terms).sum(1)
    return dz, size


@gpu
@pytest.mark.parametrize("sigmoid", [False, True], ids=["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [False, True], ids=["raw", "renorm"])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_gradient_of_confident_tokens(sigmoid, renorm, dtype):
    """One logit, or two, ahead of the others by up to 80: what is left of 1 - s there."""
    for E, k in ((8, 1), (8, 2), (61, 3), (160, 6), (256, 8)):
        z = make(E + k, 99, E, F32).cpu() * 0.5
        gap = torch.arange(99) % 33 * 2.5
        z[torch.arange(99), torch.arange(99) * 7 % E] += gap
        z[66:, 5] = z[66:].amax(1)  # two of them
        z = z.to(dtype).cuda()
        ids, _ = run(z, None, k, sigmoid, 1, 1, False, renorm, 2.5)
        ids[40:45, -1] = -1
        if k > 2:
            ids[45:50, -1] = ids[45:50, 0]  # one expert twice
        dw = torch.randn((99, k), generator=torch.Generator().manual_seed(E)).cuda()
        dz = back(z, ids, dw, sigmoid, renorm, 2.5).double().cpu().numpy()
        want, size = exact_gradient(z.double().cpu().numpy(), ids.cpu().numpy(),
                                    dw.double().cpu().numpy(), sigmoid, renorm, 2.5)
        # terms in 64 bits (exponentials to 2^-37, sums of 256 of them), at most three
        # roundings to fp32, one to bf16; below fp32's normal range half of its step
        half = 3 * 2.0 ** -24 + (2.0 ** -8 if dtype == BF16 else 0)
        step = 2.0 ** (-134 if dtype == BF16 else -149)
        assert (np.abs(dz - want) <= half * np.abs(want) + 2.0 ** -35 * size + step).all(), (E, k)


@gpu
@pytest.mark.parametrize("sigmoid", [False, True], ids=["softmax", "sigmoid"])
@pytest.mark.parametrize("renorm", [False, True], ids=["raw", "renorm"])
def test_gradient_is_the_difference_quotient(sigmoid, renorm):
    z = make(41, 4, 20, F32, sigmoid=sigmoid)
    ids, _ = run(z, None, 3, sigmoid, 1, 1, False, renorm, 1.5)
    dw = torch.randn((4, 3), generator=torch.Generator().manual_seed(7)).cuda()
    dz = back(z, ids, dw, sigmoid, renorm, 1.5).double().cpu().numpy()
    zn, idn = z.double().cpu().numpy(), ids.cpu().numpy()
    for t in range(4):
        for e in range(20):
            h = np.zeros(20)
            h[e] = 1e-5
            hi, lo = (ref.weights_of(zn[t] + f * h, idn[t], sigmoid, renorm, 1.5)
                      for f in (1, -1))
            q = (hi - lo) @ dw[t].double().cpu().numpy() / 2e-5
            # h^2 of the differences, 2^-52 / h of their rounding, 2^-20 |G| of the kernel
            assert abs(q - dz[t, e]) < 1e-9 + 2.0 ** -20 * 1.5 * float(dw[t].abs().max())


@gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("renorm", [False, True], ids=["raw", "renorm"])
def test_gradient_at_any_address(dtype, renorm):
    """Logits and their gradient at any address of their type; the elements around stay."""
    for E, k in ((7, 3), (64, 6), (161, 5), (256, 8)):
        z = make(E, 19, E, dtype)
        ids, _ = run(z, None, k, False, 1, 1, False, renorm, 1.0)
        dw = torch.randn((19, k), generator=torch.Generator().manual_seed(E)).cuda()
        want = back(z, ids, dw, False, renorm, 1.0)
        d = moe.dims(19, 64, 64, E, k, renormalize=renorm)
        for a, b in ((1, 0), (0, 3), (2, 1)):
            flat = torch.full((2, 19 * E + 8), 5.0, dtype=dtype, device="cuda")
            zo, dz = (flat[i, o:o + 19 * E].view(19, E) for i, o in ((0, a), (1, b)))
            zo.copy_(z)
            moe.route_scores_backward(d, moe.routing(), zo, ids, dw, dz)
            assert torch.equal(dz, want)
            assert (flat[1, :b] == 5).all() and (flat[1, b + 19 * E:] == 5).all()


@gpu
def test_gradient_of_many_tokens():
    z = make(51, 70001, 256, F32, sigmoid=True)
    ids, _ = run(z, None, 8, True, 8, 4, True, True, 2.5)
    dw = torch.randn((70001, 8), generator=torch.Generator().manual_seed(7)).cuda()
    dz = back(z, ids, dw, True, True, 2.5)
    at = torch.arange(0, 70001, 997).cuda()
    want = ref.route_backward(z[at].double().cpu().numpy(), ids[at].cpu().numpy(),
                              dw[at].double().cpu().numpy(), True, True, 2.5)
    g = 2.5 * dw[at].abs().amax(1, keepdim=True).double().cpu().numpy()
    assert (np.abs(dz[at].double().cpu().numpy() - want) <= 2.0 ** -20 * g).all()
    rest = torch.ones_like(dz, dtype=torch.bool).scatter_(1, ids.long(), False)
    assert (dz[rest] == 0).all()


@gpu
@pytest.mark.parametrize("E,k,renorm", [(256, 8, False), (160, 6, False), (61, 3, False),
                                        (256, 8, True)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_softmax_gradient_of_many_tokens(E, k, renorm, dtype):
    T = 40003
    z = make(52, T, E, dtype)
    z[5 * 997] = -math.inf
    z[6 * 997, E // 2:] = -math.inf
    ids, _ = run(z, None, k, False, 1, 1, False, renorm, 1.5)
    dw = torch.randn((T, k), generator=torch.Generator().manual_seed(7)).cuda()
    dz = back(z, ids, dw, False, renorm, 1.5)
    at = torch.cat([torch.arange(0, T, 997), torch.arange(T - 5, T)]).cuda()
    want = ref.route_backward(z[at].double().cpu().numpy(), ids[at].cpu().numpy(),
                              dw[at].double().cpu().numpy(), False, renorm, 1.5)
    # of the definition's difference s (g - s g): 2^-50 of |G|; of the kernel's values at
    # most three roundings to fp32, one to bf16
    half = 3 * 2.0 ** -24 + (2.0 ** -8 if dtype == BF16 else 0)
    g = 1.5 * dw[at].abs().amax(1, keepdim=True).double().cpu().numpy()
    err = np.abs(dz[at].double().cpu().numpy() - want)
    assert (err <= half * np.abs(want) + 2.0 ** -33 * g).all()
    assert dz.isfinite().all()
    if renorm:
        rest = torch.ones_like(dz, dtype=torch.bool).scatter_(1, ids.clamp(min=0).long(), False)
        assert (dz[rest] == 0).all()
    dz2 = back(z[:5000], ids[:5000], dw[:5000], False, renorm, 1.5)
    assert torch.equal(dz[:5000], dz2)


@gpu
def test_gradient_of_nan_logits():
    """A NaN reaches the gradient of its token alone."""
    z = make(61, 6, 32, F32)
    ids, _ = run(z, None, 4, False, 1, 1, False, False, 1.0)
    z[2, 5] = math.nan
    dw = torch.ones((6, 4), device="cuda")
    dz = back(z, ids, dw, False, False, 1.0)
    assert dz[2].isnan().all() and not dz[[0, 1, 3, 4, 5]].isnan().any()


# ---- logits, streams, graphs, a layer ----------------------------------------


@gpu
@pytest.mark.parametrize("T,H,E", [(1, 64, 1), (3, 256, 8), (17, 64, 60), (300, 512, 160),
                                   (1027, 256, 256), (9000, 128, 33), (20000, 64, 256)])
def test_route_logits_are_moe_routes(T, H, E):
    """Their top-k by a plain softmax is moe_route's, bit for bit."""
    g = torch.Generator().manual_seed(T)
    x = torch.randn((T, H), generator=g).to(BF16).cuda()
    wr = (torch.randn((E, H), generator=g) * 0.05).cuda()
    z = torch.full((T, E), 7.0, device="cuda")
    k = min(E, 6)
    d = moe.dims(T, H, 64, E, k, renormalize=True)
    moe.route_logits(d, x, wr, z)
    want = x.double() @ wr.double().t()
    size = x.double().abs() @ wr.double().abs().t()
    assert ((z - want).abs() <= H * 2.0 ** -24 * size).all()  # a chain of H fp32 roundings
    ids, w = run(z, None, k, False, 1, 1, False, True, 1.0)
    ids2, w2 = torch.empty_like(ids), torch.empty_like(w)
    moe.route(d, x, wr, None, ids2, w2)
    assert torch.equal(ids, ids2)
    assert ((w - w2).abs() <= 2.0 ** -23 * w2).all()


@gpu
@pytest.mark.parametrize("T,H,E", [(16380, 64, 256), (16385, 64, 256), (33000, 128, 250),
                                   (20000, 192, 16), (16384, 64, 17), (5000, 64, 100)])
def test_route_logits_of_many_tokens(T, H, E):
    """On either side of where tiles grow; the rows around stay as they were."""
    g = torch.Generator().manual_seed(T)
    x = torch.randn((T, H), generator=g).to(BF16).cuda()
    wr = (torch.randn((E, H), generator=g) * 0.05).cuda()
    flat = torch.full(((T + 2) * E,), 7.0, device="cuda")
    z = flat[E:-E].view(T, E)
    moe.route_logits(moe.dims(T, H, 64, E, 1), x, wr, z)
    want = x.double() @ wr.double().t()
    size = x.double().abs() @ wr.double().abs().t()
    assert ((z - want).abs() <= H * 2.0 ** -24 * size).all()  # a chain of H fp32 roundings
    assert (flat[:E] == 7).all() and (flat[-E:] == 7).all()


@gpu
def test_other_stream_and_captured_graph():
    T, E, k = 333, 160, 6
    z = make(71, T, E, F32)
    rules = dict(sigmoid=False, groups=8, top_groups=3, pair=False, renorm=False, scale=16.0)
    want = run(z, None, k, **rules)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = run(z, None, k, **rules, stream=side)
    side.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    d, r = moe.dims(T, 64, 64, E, k, renormalize=False), moe.routing(0, 8, 3, 0, 16.0)
    ids, w, dz = torch.empty_like(want[0]), torch.empty_like(want[1]), torch.empty_like(z)
    dw = torch.randn((T, k), device="cuda")
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        moe.route_scores(d, r, z, None, ids, w)
        moe.route_scores_backward(d, r, z, ids, dw, dz)
    for seed in (72, 73, 74):
        z.copy_(make(seed, T, E, F32))
        dw.copy_(torch.randn((T, k), generator=torch.Generator().manual_seed(seed)))
        graph.replay()
        want = run(z, None, k, **rules)
        wdz = back(z, want[0], dw, False, False, 16.0)
        torch.cuda.synchronize()
        assert torch.equal(ids, want[0]) and torch.equal(w, want[1]) and torch.equal(dz, wdz)


@gpu
def test_layer_routed_by_groups():
    """Logits, routing, dispatch, experts and combine together, with experts
    switched off so that some tokens have fewer than k: against 64 bits."""
    T, H, I, E, k = 150, 128, 192, 24, 5
    g = torch.Generator().manual_seed(81)
    x = torch.randn((T, H), generator=g).to(BF16).cuda()
    wr = (torch.randn((E, H), generator=g) * 0.1).cuda()
    wg, wu = ((torch.randn((E, I, H), generator=g) * 0.05).to(BF16).cuda() for _ in range(2))
    wd = (torch.randn((E, H, I), generator=g) * 0.05).to(BF16).cuda()
    bias = (torch.randn(E, generator=g) * 0.1).cuda()
    bias[8:] = -math.inf  # two groups of four are left, the two that are kept
    d = moe.dims(T, H, I, E, k)
    r = moe.routing(moe.SCORE_SIGMOID, 6, 2, moe.GROUP_TOP_TWO, 2.0)
    z = torch.empty((T, E), device="cuda")
    ids = torch.empty((T, k), dtype=torch.int32, device="cuda")
    w = torch.empty((T, k), device="cuda")
    moe.route_logits(d, x, wr, z)
    z[:10, :6] = -math.inf  # these tokens have two experts
    moe.route_scores(d, r, z, bias, ids, w)
    assert (ids[:10, 2:] == -1).all() and (ids[10:] >= 0).all()

    def i32(*s):
        return torch.empty(s, dtype=torch.int32, device="cuda")
    counts, off, slot, row = i32(E), i32(E + 1), i32(T * k), i32(T * k)
    xp = torch.empty((T * k, H), dtype=BF16, device="cuda")
    ws = torch.empty(moe.workspace_bytes(d), dtype=torch.uint8, device="cuda")
    moe.permute(d, ids, x, counts, off, slot, row, xp, ws)
    act = torch.empty((T * k, I), dtype=BF16, device="cuda")
    yp = torch.empty((T * k, H), device="cuda")
    moe.ffn_group(d, 0, E, off, xp, wg, wu, wd, act, yp)
    y = torch.empty((T, H), device="cuda")
    moe.combine(d, 0, E, yp, ids, row, w, y, False)
    want = torch.zeros((T, H), dtype=torch.float64, device="cuda")
    for e in range(E):
        t, j = torch.nonzero(ids == e, as_tuple=True)
        xe = x[t].double()
        gate, up = xe @ wg[e].double().t(), xe @ wu[e].double().t()
        h = gate * torch.sigmoid(gate) * up
        want.index_add_(0, t, w[t, j, None].double() * (h @ wd[e].double().t()))
    # the activations are rounded to bf16: 2^-8 a term at worst, far less in a norm
    assert float((y - want).norm() / want.norm()) < 5e-3
    assert float((y - want).abs().max()) < 2e-2
