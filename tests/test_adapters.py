"""Low-rank adapters of many requests beside a shared projection, and their
gradient, through the Python binding against 64 bits; what the calls refuse; a
layer with adapters beside its products."""
import ctypes
import weakref

import pytest
import torch

from paper_2410_12247_amd import moe

gpu = pytest.mark.gpu
BF16, F32, F64 = torch.bfloat16, torch.float32, torch.float64
FAKE = ctypes.c_void_p(4096)  # never dereferenced
ODD = ctypes.c_void_p(4096 + 2)
HALF = {BF16: 2.0 ** -8, F32: 2.0 ** -24}  # a rounding to the type


def last():
    return moe.lib().moe_last_error().decode()


def handle(count=3, rank=16, n=128, k=64, a=FAKE, b=FAKE, scale=None):
    return moe.Adapters(count, rank, n, k, a, b, scale)


# ---- refusals: host only --------------------------------------------------

BAD = [(dict(count=0), 1), (dict(count=-1), 1), (dict(count=257), 2), (dict(rank=0), 1),
       (dict(rank=-8), 1), (dict(rank=12), 1), (dict(rank=264), 2), (dict(n=0), 1),
       (dict(n=100), 1), (dict(k=32), 1), (dict(k=(1 << 20) + 64), 1)]


@pytest.mark.parametrize("change,status", BAD)
def test_bad_adapters(change, status):
    L, ad = moe.lib(), ctypes.byref(handle(**change))
    assert L.moe_adapter_workspace_bytes(4, ad) == 0 and L.moe_adapter_backward_bytes(4, ad) == 0
    big = 1 << 40
    assert L.moe_adapter_rows(4, ad, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, 0, FAKE, big,
                              None) == status, last()
    assert L.moe_adapter_backward(4, ad, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, 0, FAKE, FAKE, 0,
                                  FAKE, big, None) == status, last()


def test_workspaces():
    L = moe.lib()
    rows = [0, 1, 2, 17, 64, 100, 511, 512, 1000, 1985, 1986, 2299, 2300, 4096, 5000, 40000,
            70000, 1 << 20]
    for fn, ad in ((f, handle(rank=r, n=4096, k=2048))
                   for f in (L.moe_adapter_workspace_bytes, L.moe_adapter_backward_bytes)
                   for r in (8, 64, 128, 256)):
        need = [fn(r, ctypes.byref(ad)) for r in rows]
        assert need == sorted(need) and need[0] > 0  # one for some rows serves fewer
        assert fn(-1, ctypes.byref(ad)) == 0 and fn(1 << 31, ctypes.byref(ad)) == 0
        assert fn(4, None) == 0


@pytest.mark.parametrize("rank", [8, 16, 32, 64, 128, 136, 256])
def test_the_gradients_workspace_serves_both(rank):
    """On either side of where either direction's tiles become tall."""
    for n, k in ((64, 64), (64, 512), (1344, 64), (8192, 64), (4096, 4096)):
        for count in (1, 8, 256):
            ad = handle(count, rank, n, k)
            edges = [-(-(18 << 20) // (n + k)), -(-(1 << 30) // ((n + k) * (rank + 24))),
                     64 * count, 1, 300, 40000]
            for rows in (r + d for r in edges for d in (-1, 0, 1) if r + d > 0):
                both = moe.adapter_workspace_bytes(rows, ad), moe.adapter_backward_bytes(rows, ad)
                assert 0 < both[0] <= both[1], (n, k, count, rows)


def test_refusals():
    L = moe.lib()
    need = L.moe_adapter_workspace_bytes(4, ctypes.byref(handle()))

    def call(rows=4, ad=handle(), off=FAKE, order=FAKE, place=FAKE, x=FAKE, base=FAKE,
             y=ctypes.c_void_p(8192), t=0, ws=FAKE, size=need):
        return L.moe_adapter_rows(rows, ctypes.byref(ad) if ad else None, off, order, place, x,
                                  base, y, t, ws, size, None)
    for b in (dict(rows=-1), dict(ad=None), dict(ad=handle(a=None)), dict(ad=handle(b=None)),
              dict(ad=handle(a=ODD)), dict(ad=handle(b=ODD)), dict(ad=handle(scale=ODD)),
              dict(off=None), dict(off=ODD), dict(order=None), dict(order=ODD), dict(place=None),
              dict(place=ODD), dict(x=None), dict(x=ODD), dict(base=ODD), dict(y=None),
              dict(y=ODD), dict(t=2), dict(t=-1), dict(ws=ODD), dict(base=None, place=None)):
        assert call(**b) == 1, (b, last())
    assert call(rows=1 << 31) == 2
    # 2^32 lanes and more in a launch
    wide = handle(rank=136, n=1 << 20, k=64)
    assert call(rows=1 << 17, ad=wide) == 2 and call(rows=1 << 15, ad=wide) == 3
    assert call(rows=1 << 29) == 2 and call(rows=(1 << 31) - 1, ad=handle(rank=8, n=64)) == 2
    assert L.moe_adapter_workspace_bytes(1 << 17, ctypes.byref(wide)) == 0
    assert call(size=need - 1) == 3 and call(ws=None) == 3
    assert call(rows=0, off=None, order=None, x=None, y=None, ws=None) == 0


def test_backward_refusals():
    L = moe.lib()
    need = L.moe_adapter_backward_bytes(4, ctypes.byref(handle()))

    def call(rows=4, ad=handle(), off=FAKE, order=FAKE, place=FAKE, x=FAKE, dy=FAKE, base=FAKE,
             dx=ctypes.c_void_p(8192), t=0, da=FAKE, db=FAKE, acc=0, ws=FAKE, size=need):
        return L.moe_adapter_backward(rows, ctypes.byref(ad) if ad else None, off, order, place, x,
                                      dy, base, dx, t, da, db, acc, ws, size, None)
    for b in (dict(rows=-1), dict(ad=None), dict(ad=handle(a=None)), dict(ad=handle(b=ODD)),
              dict(off=None), dict(order=None), dict(order=ODD), dict(place=None), dict(x=None),
              dict(x=ODD), dict(dy=None), dict(dy=ODD), dict(base=ODD), dict(dx=None),
              dict(dx=ODD), dict(t=3), dict(da=None), dict(db=None), dict(da=ODD), dict(db=ODD),
              dict(acc=2), dict(acc=-1), dict(ws=ODD), dict(dx=None, base=None, da=None, db=None)):
        assert call(**b) == 1, (b, last())
    assert call(rows=1 << 31) == 2
    assert call(size=need - 1) == 3 and call(ws=None) == 3
    assert call(rows=0, da=None, db=None, off=None, dy=None, ws=None) == 0


def test_binding_refuses_what_it_cannot_pass():
    a, b = torch.zeros((2, 8, 64), dtype=BF16), torch.zeros((2, 64, 8), dtype=BF16)
    with pytest.raises(ValueError, match="contiguous device tensor"):
        moe.adapters(a, b)
    with pytest.raises(ValueError):
        moe.adapters(a[0], b)


# ---- forward ----------------------------------------------------------------


def i32(*s):
    return torch.empty(s, dtype=torch.int32, device="cuda")


def order_of(ids, count):
    """offsets, sorted_slot, slot_row of the rows' adapters (-1: none)."""
    R = ids.numel()
    d = moe.dims(R, 64, 64, count, 1)
    counts, off, slot, row = i32(count), i32(count + 1), i32(R), i32(R)
    ws = torch.empty(moe.workspace_bytes(d), dtype=torch.uint8, device="cuda")
    moe.permute(d, ids.view(R, 1), None, counts, off, slot, row, None, ws)
    return off, slot, row


def pick(seed, R, count, none=0.2, skew=False):
    g = torch.Generator().manual_seed(seed)
    u = torch.rand(R, generator=g)
    ids = ((u ** 3 if skew else u) * count).int().clamp(max=count - 1)
    return torch.where(torch.rand(R, generator=g) < none, -1, ids).int().cuda()


class Problem:
    def __init__(self, seed, R, n, k, rank, count, ids=None, scaled=True):
        g = torch.Generator().manual_seed(seed)

        def normal(*s, size=1.0):
            return (torch.randn(s, generator=g) * size).to(BF16).cuda()
        self.R, self.n, self.k, self.rank, self.count = R, n, k, rank, count
        self.x, self.dy = normal(R, k), normal(R, n)
        self.a, self.b = normal(count, rank, k, size=k ** -0.5), normal(count, n, rank, size=0.1)
        self.scale = (0.25 + 2 * torch.rand(count, generator=g)).cuda() if scaled else None
        self.ids = pick(seed, R, count) if ids is None else ids
        self.order = order_of(self.ids, count)
        self.ad = moe.adapters(self.a, self.b, self.scale)

    def normal(self, seed, cols, dtype):
        g = torch.Generator().manual_seed(seed)
        return torch.randn((self.R, cols), generator=g).to(dtype).cuda()

    def factor(self, e):
        return 1.0 if self.scale is None else self.scale[e].double()

    def rows_of(self):
        for e in range(self.count):
            at = torch.nonzero(self.ids == e)[:, 0]
            if len(at):
                yield e, at


def guarded(nbytes):
    """A workspace between untouched bytes."""
    flat = torch.full((nbytes + 512,), 0xA5, dtype=torch.uint8, device="cuda")
    return flat, flat[256:256 + nbytes]


def intact(flat):
    return bool((flat[:256] == 0xA5).all() and (flat[-256:] == 0xA5).all())


def forward(p, base, dtype, y=None, place=True, ws=None, stream=None):
    y = torch.full((p.R, p.n), 9.0, dtype=dtype, device="cuda") if y is None else y
    flat, own = guarded(moe.adapter_workspace_bytes(p.R, p.ad))
    off, slot, row = p.order
    moe.adapter_rows(p.ad, off, slot, row if place else None, p.x, base, y,
                     own if ws is None else ws, stream)
    if stream is None:
        assert intact(flat)
    return y


def check_forward(p, y, base):
    """fp32 sums of k and of rank terms: at most (k + 3 rank + 8) roundings of the
    sum of magnitudes; A x cut into bf16 parts, exact in three for fp32, within
    2^-15 in two for bf16; one rounding to y's type."""
    want = torch.zeros((p.R, p.n), dtype=F64, device="cuda")
    slack = torch.zeros_like(want)
    if base is not None:
        want += base
    for e, at in p.rows_of():
        a, b, f = p.a[e].double(), p.b[e].double(), p.factor(e)
        x = p.x[at].double()
        u = x @ a.t()
        want[at] += f * (u @ b.t())
        size = f * ((x.abs() @ a.abs().t()) @ b.abs().t())
        slack[at] += (p.k + 3 * p.rank + 8) * 2.0 ** -24 * size
        if y.dtype == BF16:
            slack[at] += 2.0 ** -15 * f * (u.abs() @ b.abs().t())
    none = p.ids < 0
    assert torch.equal(y[none].double(), want[none])
    err = (y.double() - want).abs()
    assert (err <= HALF[y.dtype] * want.abs() * (1 + 2.0 ** -8) + 2 * slack).all(), \
        float((err - HALF[y.dtype] * want.abs() - slack).max())


SHAPES = [  # rows, n, k, rank, count
    (1, 64, 64, 8, 1), (1, 576, 1344, 16, 4), (2, 128, 192, 24, 2), (15, 64, 128, 32, 3),
    (16, 192, 64, 8, 1), (17, 64, 320, 40, 1), (33, 320, 576, 16, 200), (63, 128, 64, 64, 1),
    (64, 64, 2048, 16, 64), (65, 448, 64, 72, 1), (130, 64, 64, 128, 2), (257, 1344, 448, 16, 5),
    (300, 64, 704, 200, 3), (256, 128, 128, 8, 256), (500, 192, 128, 256, 4),
    (700, 256, 256, 64, 7), (1100, 704, 64, 32, 2), (3000, 64, 128, 8, 3),
    # either side of where a workgroup sums over k itself
    (1, 128, 12288, 8, 2), (3, 64, 6208, 16, 2), (16, 192, 2048, 32, 1), (16, 128, 2112, 32, 3),
    (90, 4096, 128, 16, 2), (200, 4160, 64, 24, 40), (1400, 1536, 128, 16, 7),
    # up to and beyond the rows from which on gradients are joined
    (127, 576, 64, 8, 3), (128, 64, 1088, 24, 130), (128, 128, 64, 48, 1), (129, 64, 128, 8, 200),
    (255, 128, 64, 24, 2), (256, 64, 576, 72, 2), (256, 64, 64, 16, 1)]


@gpu
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_rows(shape, dtype):
    p = Problem(sum(shape), *shape)
    base = p.normal(1, p.n, dtype)
    y = forward(p, base, dtype)
    check_forward(p, y, base)
    z = forward(p, None, dtype)
    check_forward(p, z, None)
    # in place: the same bits, rows without an adapter as they were
    w = base.clone()
    forward(p, w, dtype, y=w, place=False)
    assert torch.equal(w, y)


# Many rows: rows, n, k, rank, count, skewed (few adapters of many rows); the latter ones in
# tall tiles: from 18 * 2^20 values of (n + k) rows on, the gradient from 2^30 of
# (n + k) (rank + 24) rows on, and 64 rows an adapter
MANY = [(1536, 64, 64, 8, 24, False), (1537, 576, 320, 24, 24, True), (1663, 64, 448, 32, 1, True),
        (2047, 128, 576, 64, 7, True), (2500, 704, 704, 128, 2, True),
        (3001, 64, 1024, 136, 4, True), (4097, 128, 512, 120, 9, True), (9000, 192, 192, 48, 1, False),
        (4600, 64, 7936, 8, 24, False), (4300, 6080, 2112, 16, 25, True),
        (3001, 320, 8000, 24, 24, True), (2403, 7872, 448, 32, 1, True),
        (2500, 64, 8192, 40, 5, False), (3100, 4096, 2112, 64, 7, True),
        (2800, 1344, 5440, 72, 3, False), (2600, 5696, 1728, 128, 2, True),
        (4097, 4160, 512, 120, 60, True), (9200, 192, 2048, 48, 1, False),
        (16500, 64, 1088, 64, 128, True), (2303, 4096, 4096, 16, 36, False),
        (2304, 4096, 4096, 16, 36, False), (2304, 4096, 4096, 16, 37, False),
        (70, 64, 1 << 19, 16, 1, False), (65, 1 << 19, 64, 24, 1, False)]


def many(shape, seed=0):
    R, n, k, rank, count, skew = shape
    return Problem(R + seed, R, n, k, rank, count, pick(R, R, count, 0.1, skew))


@gpu
@pytest.mark.parametrize("shape", MANY, ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_many_rows(shape, dtype):
    p = many(shape)
    base = p.normal(1, p.n, dtype)
    y = forward(p, base, dtype)
    check_forward(p, y, base)
    check_forward(p, forward(p, None, dtype), None)
    w = base.clone()
    forward(p, w, dtype, y=w, place=False)
    assert torch.equal(w, y)


@gpu
@pytest.mark.parametrize("none", [0.0, 1.0])
@pytest.mark.parametrize("count,which", [(1, 0), (5, 0), (5, 4), (256, 255)])
def test_one_adapter_for_all_or_none(none, count, which):
    for R in (1, 40, 333):
        ids = torch.full((R,), -1 if none else which, dtype=torch.int32, device="cuda")
        p = Problem(R, R, 128, 192, 16, count, ids, scaled=False)
        base = p.normal(1, p.n, BF16)
        check_forward(p, forward(p, base, BF16), base)
        check_forward(p, forward(p, None, F32), None)


@gpu
def test_neighbours_do_not_matter():
    """A row's bits do not depend on the other rows' adapters or values, and
    infinities and NaN stay in their row."""
    p = Problem(5, 200, 128, 256, 24, 6)
    base = p.normal(1, p.n, F32)
    want = forward(p, base, F32)
    x = p.x.clone()
    bad = torch.zeros(200, dtype=torch.bool, device="cuda")
    bad[3::7] = True
    p.x[3::7, 5] = float("nan")
    p.x[10::14, 5] = float("inf")
    bad[10::14] = True
    got = forward(p, base, F32)
    assert torch.equal(got[~bad], want[~bad])
    assert not got[bad & (p.ids >= 0)].isfinite().any()
    assert torch.equal(got[bad & (p.ids < 0)], want[bad & (p.ids < 0)])
    p.x.copy_(x)
    ids = torch.where(torch.arange(200, device="cuda") % 2 == 0, p.ids, (p.ids + 3) % 6).int()
    p.ids, p.order = ids, order_of(ids, 6)
    got = forward(p, base, F32)
    assert torch.equal(got[::2], want[::2])


@gpu
def test_large_values():
    """Sums near fp32's largest value and far below 1."""
    p = Problem(6, 40, 64, 64, 8, 2, scaled=False)
    for size in (2.0 ** 60, 2.0 ** -60):
        p.x = (p.x.float() * size).to(BF16)
        z = forward(p, None, F32)
        check_forward(p, z, None)
        p.x = (p.x.float() / size).to(BF16)


@gpu
def test_bad_indices_are_passed_over():
    """Offsets and rows outside the batch: cut or passed over by the kernels'
    own checks, nothing outside the outputs is touched."""
    p = Problem(8, 100, 128, 64, 16, 4)
    off, slot, row = p.order
    base = p.normal(1, p.n, BF16)
    want = forward(p, base.clone(), BF16, y=None)
    worse = slot.clone()
    worse[3], worse[4], worse[5] = -1, 100, 2 ** 31 - 1
    p.order = (off, worse, row)
    got = base.clone()
    forward(p, got, BF16, y=got)
    touched = torch.zeros(100, dtype=torch.bool, device="cuda")
    touched[slot[3:6].long()] = True
    assert torch.equal(got[~touched], want[~touched]) and torch.equal(got[touched], base[touched])
    wild = off.clone()
    wild[-1], wild[0] = 2 ** 31 - 1, -5
    p.order = (wild, slot, row)
    got = base.clone()
    forward(p, got, BF16, y=got)
    assert got.isfinite().all()
    p.order = (off.flip(0).contiguous(), slot, row)  # no adapter has rows
    got = base.clone()
    forward(p, got, BF16, y=got)
    da, db, dx = (torch.empty(s, device="cuda") for s in ((4, 16, 64), (4, 128, 16), (100, 64)))
    backward(p, None, dx, da, db)
    zigzag = torch.tensor([0, 100, 0, 100, 0], dtype=torch.int32, device="cuda")
    for o, order in ((wild, slot), (zigzag, slot), (off, worse)):
        p.order = (o, order, row)
        backward(p, None, dx, da, db)
        forward(p, got, BF16, y=got)
    torch.cuda.synchronize()


def whole_order(ids, count):
    """offsets, sorted_slot, slot_row with the rows of no adapter behind the others."""
    key = torch.where(ids < 0, count, ids)
    slot = torch.argsort(key, stable=True)
    off = torch.zeros(count + 1, dtype=torch.int32, device="cuda")
    off[1:] = torch.bincount(key, minlength=count + 1)[:count].cumsum(0)
    row = torch.empty_like(ids)
    row[slot] = torch.arange(len(ids), dtype=torch.int32, device="cuda")
    row[ids < 0] = -1
    return off, slot.int(), row


@gpu
@pytest.mark.parametrize("R,n", [(1, 128), (100, 128), (700, 192), (5000, 5696)])
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_rows_out_of_order_are_rows_of_no_adapter(R, n, dtype):
    """Bad entries of sorted_slot, and offsets that end early, late or fall: every
    output is written, as for rows without an adapter where no place is theirs."""
    p = Problem(18, R, n, 128, 16, 4)
    p.ids[0] = 2
    off, slot, row = whole_order(p.ids, 4)
    used, ids = int(off[-1]), p.ids.clone()
    bad = torch.arange(0, used, 7, device="cuda")
    worse = slot.clone()
    worse[bad] = torch.tensor([-1, R, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32,
                              device="cuda").repeat(len(bad))[:len(bad)]
    without = ids.clone()
    without[slot[bad].long()] = -1
    short, late = off.clone(), off.clone()
    short[-1] = max(int(off[-2]), used - 3)
    fewer = ids.clone()
    fewer[slot[int(short[-1]):used].long()] = -1
    late[0], late[-1] = -5, 2 ** 31 - 1  # the last adapter has the others' rows too
    place = row.clone()
    place[slot[used:].long()] = torch.arange(used, R, dtype=torch.int32, device="cuda")
    for order, has in (((off, slot, row), ids), ((off, worse, row), without),
                       ((short, slot, row), fewer),
                       ((late, slot, place), torch.where(ids < 0, 3, ids)),
                       ((off.flip(0).contiguous(), slot, row), torch.full_like(ids, -1))):
        p.order, p.ids = order, has
        for base, dx0 in ((p.normal(1, n, dtype), p.normal(2, 128, dtype)), (None, None)):
            check_forward(p, forward(p, base, dtype), base)
            dx, da, db = grads(p, dtype)
            backward(p, dx0, dx, da, db)
            check_backward(p, dx0, dx, da, db)
            if base is not None:
                forward(p, base, dtype, y=base, place=False)
                check_forward(p, base, p.normal(1, n, dtype))


@gpu
def test_offsets_past_32_bits():
    """x and y of more than 4 GiB."""
    R, n, k = 40000, 65536, 64
    g = torch.Generator(device="cuda").manual_seed(1)
    ids = (torch.arange(R, device="cuda") % 3 - 1).int()
    p = Problem(9, 64, n, k, 8, 2)  # the weights
    p.R, p.ids, p.order = R, ids, order_of(ids, 2)
    p.x = torch.randn((R, k), generator=g, device="cuda").to(BF16)
    y = torch.zeros((R, n), dtype=BF16, device="cuda")
    forward(p, y, BF16, y=y)
    at = torch.tensor([0, 1, 2, 20000, 32768, 39997, 39998, 39999], device="cuda")
    q = Problem(9, 64, n, k, 8, 2)
    q.R, q.ids, q.x = len(at), ids[at], p.x[at]
    check_forward(q, y[at], None)
    del y
    dy = torch.randn((R, n), generator=g, device="cuda", dtype=BF16)
    p.dy, dx = dy, torch.zeros((R, k), device="cuda")
    backward(p, dx, dx, None, None)
    for r in (1, 2, 39998, 39997):
        e = int(ids[r])
        v = dy[r].double() @ p.b[e].double()
        w = p.factor(e) * (v @ p.a[e].double())
        s = p.factor(e) * ((dy[r].double().abs() @ p.b[e].double().abs()) @ p.a[e].double().abs())
        assert ((dx[r] - w).abs() <= (n + 40) * 2.0 ** -24 * s).all()


# ---- gradient ---------------------------------------------------------------


def backward(p, base, dx, da, db, accumulate=False, ws=None, stream=None):
    flat, own = guarded(moe.adapter_backward_bytes(p.R, p.ad))
    off, slot, row = p.order
    moe.adapter_backward(p.ad, off, slot, row, p.x, p.dy, base, dx, da, db,
                         own if ws is None else ws, accumulate, stream)
    if stream is None:
        assert intact(flat)


def grads(p, dtype):
    return (torch.full((p.R, p.k), 9.0, dtype=dtype, device="cuda"),
            torch.full((p.count, p.rank, p.k), 9.0, device="cuda"),
            torch.full((p.count, p.n, p.rank), 9.0, device="cuda"))


def check_backward(p, base, dx, da, db, da0=None, db0=None):
    """dx as the forward pass with the roles of A and B turned; da and db: fp32 sums
    of n (or k) and of the rows, their factors exact."""
    wx = torch.zeros((p.R, p.k), dtype=F64, device="cuda")
    sx = torch.zeros_like(wx)
    wa = torch.zeros(p.a.shape, dtype=F64, device="cuda")
    wb = torch.zeros(p.b.shape, dtype=F64, device="cuda")
    sa, sb = torch.zeros_like(wa), torch.zeros_like(wb)
    if base is not None:
        wx += base
    for e, at in p.rows_of():
        a, b, f = p.a[e].double(), p.b[e].double(), p.factor(e)
        x, dy = p.x[at].double(), p.dy[at].double()
        u, v = x @ a.t(), dy @ b
        ua, va = x.abs() @ a.abs().t(), dy.abs() @ b.abs()
        wx[at] += f * (v @ a)
        sx[at] += (p.n + 3 * p.rank + 8) * 2.0 ** -24 * f * (va @ a.abs())
        if dx is not None and dx.dtype == BF16:
            sx[at] += 2.0 ** -15 * f * (v.abs() @ a.abs())
        wa[e] = f * (v.t() @ x)
        wb[e] = f * (dy.t() @ u)
        sa[e] = (p.n + 3 * len(at) + 16) * 2.0 ** -24 * f * (va.t() @ x.abs())
        sb[e] = (p.k + 3 * len(at) + 16) * 2.0 ** -24 * f * (dy.abs().t() @ ua)
    if dx is not None:
        assert torch.equal(dx[p.ids < 0].double(), wx[p.ids < 0])
        assert ((dx.double() - wx).abs() <= HALF[dx.dtype] * (1 + 2.0 ** -8) * wx.abs()
                + 2 * sx).all()
    for got, want, s, was in ((da, wa, sa, da0), (db, wb, sb, db0)):
        if got is None:
            continue
        if was is not None:
            want = want + was
            s = s + 2.0 ** -23 * (want.abs() + was.abs())
        assert ((got.double() - want).abs() <= 2.0 ** -24 * want.abs() + 2 * s).all()


@gpu
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_gradients(shape, dtype):
    p = Problem(sum(shape) + 1, *shape)
    base = p.normal(1, p.k, dtype)
    dx, da, db = grads(p, dtype)
    backward(p, base, dx, da, db)
    check_backward(p, base, dx, da, db)
    # twice the same bits; in place; each half alone; added
    dx2, da2, db2 = grads(p, dtype)
    backward(p, base, dx2, da2, db2)
    assert torch.equal(dx, dx2) and torch.equal(da, da2) and torch.equal(db, db2)
    w = base.clone()
    backward(p, w, w, None, None)
    assert torch.equal(w, dx)
    da2.fill_(9.0), db2.fill_(9.0)
    backward(p, None, None, da2, db2)
    assert torch.equal(da, da2) and torch.equal(db, db2)
    da0, db0 = torch.randn_like(da), torch.randn_like(db)
    da2.copy_(da0), db2.copy_(db0)
    backward(p, None, dx2, da2, db2, accumulate=True)
    check_backward(p, None, dx2, da2, db2, da0, db0)


@gpu
@pytest.mark.parametrize("shape", MANY, ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_gradients_of_tall_tiles(shape, dtype):
    p = many(shape, 1)
    base = p.normal(1, p.k, dtype)
    dx, da, db = grads(p, dtype)
    backward(p, base, dx, da, db)
    check_backward(p, base, dx, da, db)
    w = base.clone()
    backward(p, w, w, None, None)
    assert torch.equal(w, dx)
    da2, db2 = torch.full_like(da, 9.0), torch.full_like(db, 9.0)
    backward(p, None, None, da2, db2)
    assert torch.equal(da, da2) and torch.equal(db, db2)
    da0, db0 = torch.randn_like(da), torch.randn_like(db)
    da2.copy_(da0), db2.copy_(db0)
    backward(p, None, dx, da2, db2, accumulate=True)
    check_backward(p, None, dx, da2, db2, da0, db0)


@gpu
@pytest.mark.parametrize("R,n", [(90, 192), (2100, 192), (5000, 5696)])
def test_gradients_pass_over_bad_rows(R, n):
    """Entries of sorted_slot outside the rows take no part in da and db, whatever
    row 0 holds."""
    p = Problem(17, R, n, 128, 16, 3)
    off, slot, row = p.order
    bad = torch.arange(3, int((p.ids >= 0).sum()), 11, device="cuda")
    worse = slot.clone()
    worse[bad] = torch.tensor([-1, R, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32,
                              device="cuda").repeat(len(bad))[:len(bad)]
    keep = p.ids.clone()
    keep[slot[bad].long()] = -1
    if keep[0] >= 0:  # row 0 takes no part
        worse[torch.nonzero(slot[:off[-1]] == 0)[0, 0]] = keep[0] = -1
    for e in (float("nan"), 1.0):
        p.x[0] = p.dy[0] = e
        p.order = (off, worse, row)
        da, db = grads(p, F32)[1:]
        backward(p, None, None, da, db)
        p.ids, was = keep, p.ids
        check_backward(p, None, None, da, db)
        p.ids = was


@gpu
@pytest.mark.parametrize("R,count", [(5000, 1), (4096, 3), (1537, 2)])
def test_gradients_of_many_rows(R, count):
    """Adapters whose rows are cut into several sums, beside some with one or none."""
    for seed, skew in ((1, False), (2, True)):
        p = Problem(R, R, 192, 128, 16, count + 2,
                    pick(seed, R, count, 0.1, skew))  # the last two have none
        dx, da, db = grads(p, F32)
        backward(p, None, dx, da, db)
        check_backward(p, None, dx, da, db)
        assert (da[count:] == 0).all() and (db[count:] == 0).all()


@gpu
@pytest.mark.parametrize("R,used", [(1, [37]), (5, [0, 255]), (128, [254]), (40, []), (256, [9]),
                                    (300, [3, 77])])
def test_gradients_of_idle_adapters(R, used):
    """Zeros for every adapter without rows, wherever it lies; nothing where they add."""
    ids = torch.tensor([used[i % len(used)] if used else -1 for i in range(R)],
                       dtype=torch.int32, device="cuda")
    p = Problem(15, R, 576, 64, 16, 256, ids)
    for dtype in (BF16, F32):
        dx, da, db = grads(p, dtype)
        backward(p, None, dx, da, db)
        check_backward(p, None, dx, da, db)
        da2, db2 = torch.full_like(da, 9.0), torch.full_like(db, 9.0)
        backward(p, None, None, da2, db2)
        assert torch.equal(da, da2) and torch.equal(db, db2)
        da2.fill_(3.0), db2.fill_(3.0)
        backward(p, None, dx, da2, db2, accumulate=True)
        idle = torch.ones(256, dtype=torch.bool, device="cuda")
        idle[used] = False
        assert (da2[idle] == 3).all() and (db2[idle] == 3).all()


@gpu
def test_gradients_of_no_rows():
    p = Problem(3, 4, 128, 64, 16, 3)
    da, db = grads(p, F32)[1:]
    d0 = torch.empty((0, 64), dtype=BF16, device="cuda")
    y0 = torch.empty((0, 128), dtype=BF16, device="cuda")
    e = i32(0)
    ws = torch.empty(256, dtype=torch.uint8, device="cuda")
    off = torch.zeros(4, dtype=torch.int32, device="cuda")
    moe.adapter_backward(p.ad, off, e, e, d0, y0, None, d0, da, db, ws, accumulate=True)
    assert (da == 9).all() and (db == 9).all()
    moe.adapter_backward(p.ad, off, e, e, d0, y0, None, d0, da, db, ws)
    assert (da == 0).all() and (db == 0).all()
    moe.adapter_rows(p.ad, off, e, e, d0, None, y0, ws)


@gpu
def test_gradients_are_difference_quotients():
    """The derivative of sum(dy * y) along random directions, y in 64 bits: y is
    linear in x, A and B each, so a difference of any width is exact."""
    p = Problem(12, 90, 128, 192, 24, 3)
    dx, da, db = grads(p, F32)
    backward(p, None, dx, da, db)

    def loss(x, a, b):
        return sum(p.factor(e) * (p.dy[at].double() * (x[at] @ a[e].t() @ b[e].t())).sum()
                   for e, at in p.rows_of())
    at = [p.x.double(), p.a.double(), p.b.double()]
    for i, grad in enumerate((dx, da, db)):
        step = torch.randn(at[i].shape, generator=torch.Generator().manual_seed(i)).cuda().double()
        q = loss(*[v + step if j == i else v for j, v in enumerate(at)]) - loss(*at)
        # each gradient's fp32 error is below 2^-15 of its norm by the bounds above
        assert abs(q - (grad.double() * step).sum()) <= 2.0 ** -15 * grad.norm() * step.norm()


def whole_numbers(seed, R, n, k, rank, count, turned):
    """A problem of whole numbers whose every sum is below 2^24, so exact in fp32 in any
    order.  The rank's values stand in pairs of nearly equal ones with weights 1 and -1:
    their sums over k (of dy over n where turned) have 16 to 20 bits and outputs some ten."""
    p = Problem(seed, R, n, k, rank, count, pick(seed, R, count, 0.2 if R > 1 else 0.0))
    g = torch.Generator().manual_seed(seed + 1)

    def ints(most, *s):
        return torch.randint(-most, most + 1, s, generator=g)
    K, N = (n, k) if turned else (k, n)
    rows, long = ints(255, R, K), ints(min(127, int(2 ** 24 * 1.8 / (140 * K))), count, rank, K)
    long[:, 1::2] = long[:, ::2]
    at = torch.randint(0, K, (count, rank // 2, 3), generator=g)
    long[:, 1::2].scatter_add_(2, at, ints(1, *at.shape))
    pair, sign = torch.randint(0, rank // 2, (count, N, 1), generator=g), ints(1, count, N, 1)
    wide = torch.zeros((count, N, rank), dtype=torch.int64)
    wide.scatter_(2, 2 * pair, sign).scatter_(2, 2 * pair + 1, -sign)
    assert int((rows.abs() @ long.abs().flatten(0, 1).t()).max()) < 2 ** 24
    if turned:
        p.dy.copy_(rows), p.b.copy_(long.transpose(1, 2)), p.a.copy_(wide.transpose(1, 2))
    else:
        p.x.copy_(rows), p.a.copy_(long), p.b.copy_(wide)
    p.scale.copy_(2.0 ** ints(2, count))
    return p, ints(256, R, N).double().cuda()


# one workgroup's own sums; short tiles, of ranks that fill whole instructions and that do
# not; tall ones
WHOLE = [(1, 576, 1344, 16, 4), (16, 192, 2048, 32, 1), (40, 128, 4096, 32, 3),
         (200, 320, 704, 24, 6), (300, 512, 704, 200, 3), (1100, 704, 576, 64, 2),
         (2403, 7872, 448, 32, 1), (3100, 4096, 2112, 64, 7), (2600, 5696, 1728, 128, 2),
         (2500, 512, 8192, 40, 5)]


@gpu
@pytest.mark.parametrize("shape", WHOLE, ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_sums_keep_their_bits(shape, dtype):
    """Where the rank's terms cancel, outputs are what is left, rounded once: A x is
    held, and multiplied, in fp32's 24 bits whatever the output's type."""
    p, base = whole_numbers(sum(shape), *shape, turned=False)
    d = torch.zeros((p.R, p.n), dtype=F64, device="cuda")
    most = 0.0
    for e, at in p.rows_of():
        u = p.x[at].double() @ p.a[e].double().t()
        most = max(most, float(u.abs().max()))
        d[at] = p.factor(e) * (u @ p.b[e].double().t())
    assert most >= 2 ** 16  # more bits than two bf16 parts hold
    assert torch.equal(forward(p, None, dtype), d.to(dtype))
    assert torch.equal(forward(p, base.to(dtype), dtype), (d + base).to(dtype))


@gpu
@pytest.mark.parametrize("shape", WHOLE, ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_gradient_sums_keep_their_bits(shape, dtype):
    """The same of dy B in dx, beside the gradients of A and B and by itself."""
    p, base = whole_numbers(sum(shape) + 1, *shape, turned=True)
    d = torch.zeros((p.R, p.k), dtype=F64, device="cuda")
    most = 0.0
    for e, at in p.rows_of():
        v = p.dy[at].double() @ p.b[e].double()
        most = max(most, float(v.abs().max()))
        d[at] = p.factor(e) * (v @ p.a[e].double())
    assert most >= 2 ** 16
    dx, da, db = grads(p, dtype)
    backward(p, None, dx, da, db)
    assert torch.equal(dx, d.to(dtype))
    dx.fill_(9.0)
    backward(p, base.to(dtype), dx, None, None)
    assert torch.equal(dx, (d + base).to(dtype))


# ---- streams, graphs, workspaces, a layer -------------------------------------


@gpu
def test_other_stream_and_captured_graph():
    p = Problem(21, 150, 192, 256, 16, 5)
    base = p.normal(1, p.n, BF16)
    ws = torch.empty(moe.adapter_backward_bytes(p.R, p.ad), dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    want = forward(p, base, BF16)
    side.wait_stream(torch.cuda.current_stream())
    got = forward(p, base, BF16, ws=ws, stream=side)
    side.synchronize()
    assert torch.equal(got, want)
    y = torch.empty_like(base)
    dx, da, db = grads(p, BF16)
    off, slot, row = p.order
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        moe.adapter_rows(p.ad, off, slot, row, p.x, base, y, ws)
        moe.adapter_backward(p.ad, off, slot, row, p.x, p.dy, None, dx, da, db, ws)
    for seed in (1, 2, 3):
        p.ids = pick(seed, p.R, p.count, 0.3, seed == 2)  # another batch: the same buffers
        for t, v in zip((off, slot, row), order_of(p.ids, p.count)):
            t.copy_(v)
        p.x.copy_(p.normal(seed, p.k, BF16))
        p.dy.copy_(p.normal(seed + 9, p.n, BF16))
        torch.cuda.synchronize()
        graph.replay()
        check_forward(p, y, base)
        check_backward(p, None, dx, da, db)
        dx2, da2, db2 = grads(p, BF16)
        backward(p, None, dx2, da2, db2)
        torch.cuda.synchronize()
        assert torch.equal(dx, dx2) and torch.equal(da, da2) and torch.equal(db, db2)


@gpu
@pytest.mark.parametrize("rows,width", [(1700, 576), (2300, 8192)])
def test_many_rows_captured_and_beside_another_call(rows, width):
    """Two calls at once on streams and workspaces of their own; both captured."""
    p, q = many((rows + 10, 320, width, 32, 7, True)), many((rows, width, 320, 96, 2, False))
    want = [forward(p, None, F32), *grads(p, BF16), forward(q, None, BF16), *grads(q, F32)]
    backward(p, None, *want[1:4])
    backward(q, None, *want[5:8])
    got = [torch.full_like(t, 9.0) for t in want]
    ws = [torch.full((moe.adapter_backward_bytes(t.R, t.ad),), 0xFF, dtype=torch.uint8,
                     device="cuda") for t in (p, q)]

    def run(stream=None):
        forward(q, None, BF16, y=got[4], ws=ws[1], stream=stream)
        backward(q, None, *got[5:8], ws=ws[1], stream=stream)
        forward(p, None, F32, y=got[0], ws=ws[0], stream=torch.cuda.current_stream())
        backward(p, None, *got[1:4], ws=ws[0], stream=torch.cuda.current_stream())
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    run(side)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    with torch.cuda.graph(graph):
        side.wait_stream(torch.cuda.current_stream())
        run(side)
        torch.cuda.current_stream().wait_stream(side)
    for i in range(3):
        for t in got:
            t.fill_(float(i))
        for w in ws:
            w.fill_(0xFF)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, got))


@gpu
def test_adapters_are_let_go():
    """A handle keeps its tensors while it lives, and no longer."""
    a, b = (torch.zeros(s, dtype=BF16, device="cuda") for s in ((2, 8, 64), (2, 64, 8)))
    ad, seen = moe.adapters(a, b), weakref.ref(a)
    del a, b
    assert seen() is not None
    del ad
    assert seen() is None


@gpu
def test_gradient_without_x():
    p = Problem(24, 20, 128, 64, 16, 2)
    dx = grads(p, BF16)[0]
    backward(p, None, dx, None, None)
    p.x, x = None, p.x
    dx2 = torch.zeros_like(dx)
    backward(p, None, dx2, None, None)
    assert torch.equal(dx, dx2)
    with pytest.raises(moe.MoEError):
        backward(p, None, dx2, *grads(p, BF16)[1:])


@gpu
def test_a_larger_workspace_of_other_contents():
    """One for many rows serves few, whatever it holds."""
    p = Problem(22, 37, 128, 64, 32, 4)
    want = forward(p, None, F32)
    dx, da, db = grads(p, F32)
    backward(p, None, dx, da, db)
    ws = torch.full((moe.adapter_backward_bytes(5000, p.ad),), 0xFF, dtype=torch.uint8,
                    device="cuda")  # NaN everywhere
    assert torch.equal(forward(p, None, F32, ws=ws), want)
    ws.fill_(0xFF)
    dx2, da2, db2 = grads(p, F32)
    backward(p, None, dx2, da2, db2, ws=ws)
    assert torch.equal(dx, dx2) and torch.equal(da, da2) and torch.equal(db, db2)


@gpu
def test_binding_refuses_other_shapes():
    p = Problem(23, 8, 128, 64, 16, 2)
    off, slot, row = p.order
    y = torch.empty((8, 128), dtype=BF16, device="cuda")
    ws = torch.empty(moe.adapter_workspace_bytes(8, p.ad), dtype=torch.uint8, device="cuda")
    moe.adapter_rows(p.ad, off, slot, row, p.x, None, y, ws)
    for bad in ((off[:2], slot, row, p.x, None, y), (off, slot[:4], row, p.x, None, y),
                (off, slot, row, p.x[:, :32], None, y), (off, slot, row, p.x.float(), None, y),
                (off, slot, row, p.x, y.float(), y), (off, slot, row, p.x, None, y[:4]),
                (off, slot, row, p.x, None, y.half()), (off, slot, row, p.x, None, y.t()),
                (off.long(), slot, row, p.x, None, y)):
        with pytest.raises(ValueError):
            moe.adapter_rows(p.ad, *bad, ws)
    with pytest.raises(moe.MoEError):
        moe.adapter_rows(p.ad, off, slot, row, p.x, None, y, ws[:16])


@gpu
def test_layer_with_adapters():
    """A routed layer whose batch mixes requests: grouped routing, experts and
    combine, a dense FFN beside them, and each row's adapter beside the whole layer
    (x to y, fp32, in place); then the adapters' gradient."""
    T, H, I, E, k, C = 130, 128, 192, 16, 4, 6
    g = torch.Generator().manual_seed(31)
    p = Problem(31, T, H, H, 16, C)
    wr = (torch.randn((E, H), generator=g) * 0.1).cuda()
    wg, wu, sg, su = ((torch.randn((E, I, H), generator=g) * 0.05).to(BF16).cuda()
                      for _ in range(4))
    wd, sd = ((torch.randn((E, H, I), generator=g) * 0.05).to(BF16).cuda() for _ in range(2))
    d = moe.dims(T, H, I, E, k)
    z, w = torch.empty((T, E), device="cuda"), torch.empty((T, k), device="cuda")
    ids, counts, off, slot, row = i32(T, k), i32(E), i32(E + 1), i32(T * k), i32(T * k)
    moe.route_logits(d, p.x, wr, z)
    moe.route_scores(d, moe.routing(moe.SCORE_SIGMOID, 4, 2, moe.GROUP_TOP_TWO, 1.5), z, None, ids,
                     w)
    xp = torch.empty((T * k, H), dtype=BF16, device="cuda")
    wsp = torch.empty(moe.workspace_bytes(d), dtype=torch.uint8, device="cuda")
    moe.permute(d, ids, p.x, counts, off, slot, row, xp, wsp)
    act, yp = torch.empty((T * k, I), dtype=BF16, device="cuda"), torch.empty((T * k, H),
                                                                               device="cuda")
    moe.ffn_group(d, 0, E, off, xp, wg, wu, wd, act, yp)
    y = torch.empty((T, H), device="cuda")
    moe.ffn_dense(T, H, I, p.x, sg[0], su[0], sd[0], torch.empty((T, I), dtype=BF16,
                                                                 device="cuda"), y)
    moe.combine(d, 0, E, yp, ids, row, w, y, True)
    base = y.clone()
    forward(p, y, F32, y=y)
    check_forward(p, y, base)

    def ffn(x, a, b, c):
        gate, up = x @ a.double().t(), x @ b.double().t()
        return (gate * torch.sigmoid(gate) * up) @ c.double().t()
    want = ffn(p.x.double(), sg[0], su[0], sd[0])
    for e in range(E):
        t, j = torch.nonzero(ids == e, as_tuple=True)
        want.index_add_(0, t, w[t, j, None].double() * ffn(p.x[t].double(), wg[e], wu[e], wd[e]))
    for e, at in p.rows_of():
        want[at] += p.factor(e) * (p.x[at].double() @ p.a[e].double().t() @ p.b[e].double().t())
    # the experts' activations are rounded to bf16: 2^-8 a term at worst
    assert float((y - want).norm() / want.norm()) < 5e-3
    dx, da, db = grads(p, F32)
    backward(p, base, dx, da, db)
    check_backward(p, base, dx, da, db)
