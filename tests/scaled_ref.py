"""Plain 64-bit implementations of the block-scaled 8-bit operators, on the
CPU, and the bounds their results are held to.

Bounds.  A rounding is off by at most half a step: 2^-8 of the value for bf16,
2^-24 for fp32.  The 8-bit matrix instruction adds products in groups of eight
consecutive k, each product cut to 13 bits below the group's largest exponent;
a product's own exponent is at least the sum of its factors', so the group's
error is at most 8 * 2^-13 * max |product| (``group_bound``).  Everything after
that is fp32 additions."""
import numpy as np
import torch

BLOCK = 128
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def pitch(k):
    return 4 * -(-k // 512)


def blocks(k):
    return -(-k // BLOCK)


def _decode_table():
    t = np.empty(256)
    for b in range(256):
        s, e, m = b >> 7, (b >> 3) & 15, b & 7
        v = np.ldexp(1 + m / 8, e - 7) if e else np.ldexp(m / 8, -6)
        t[b] = np.nan if (b & 127) == 127 else (-v if s else v)
    return torch.from_numpy(t)


DECODE = _decode_table()


def decode(q):
    """e4m3 bits or tensors -> fp64 values."""
    return DECODE[q.cpu().view(torch.uint8).long()]


def round_e4m3(v):
    """fp64 |v| <= 448 to the nearest e4m3 value, ties to even."""
    a = v.abs()
    _, x = torch.frexp(a)
    step = torch.ldexp(torch.ones_like(a), torch.clamp(x - 1, min=-6) - 3)
    return torch.round(v / step) * step  # torch.round: ties to even


def exponent(amax):
    """Smallest e in [-127, 127] with amax <= 448 * 2^e; 0 for 0."""
    m, x = torch.frexp(amax)
    e = (x - 9 + (m > 0.875)).clamp(-127, 127)
    return torch.where(amax > 0, e, torch.zeros_like(e))


def tiles(v, tall):
    """[n, k] -> [n/tall, tall, k/128, 128], zero padded."""
    n, k = v.shape
    p = torch.zeros((-(-n // tall) * tall, blocks(k) * BLOCK), dtype=v.dtype)
    p[:n, :k] = v
    return p.view(-1, tall, blocks(k), BLOCK)


def quant(v, tall):
    """(e4m3 values, exponents [n/tall, blocks]) of fp64 v."""
    t = tiles(v, tall)
    e = exponent(t.abs().amax((1, 3)))
    f = torch.ldexp(torch.ones((), dtype=torch.float64), e)[:, None, :, None]
    return round_e4m3(t / f).reshape(-1, t.shape[2] * BLOCK)[:v.shape[0], :v.shape[1]], e


def widen(q, scales, tall):
    """Values of e4m3 q [n, k] with scale bytes [n/tall, pitch]."""
    n, k = q.shape
    f = torch.ldexp(torch.ones((), dtype=torch.float64),
                    scales.cpu().view(torch.uint8)[:, :blocks(k)].int() - 127)
    f = f.repeat_interleave(tall, 0)[:n].repeat_interleave(BLOCK, 1)[:, :k]
    return decode(q) * f


def spread(q, e, tall):
    """Values of quant()'s answer."""
    n, k = q.shape
    f = torch.ldexp(torch.ones((), dtype=torch.float64), e)
    return q * f.repeat_interleave(tall, 0)[:n].repeat_interleave(BLOCK, 1)[:, :k]


def group_bound(x, w):
    """[R, N]: 2^-10 times the sum over groups of eight k of the largest
    |product|, plus the fp32 additions of the groups' sums."""
    R, K = x.shape
    a, b = x.abs(), w.abs()
    top = torch.zeros((R, w.shape[0]), dtype=torch.float64)
    for g in range(0, K, 8):
        p = torch.zeros_like(top)
        for j in range(g, g + 8):
            p = torch.maximum(p, a[:, j, None] * b[None, :, j])
        top += p
    return 2.0 ** -10 * top + (K / 8 + 8) * 2.0 ** -24 * (a @ b.T)


def e4m3_random(gen, *shape):
    """Random finite e4m3 bits."""
    b = torch.randint(0, 256, shape, generator=gen, dtype=torch.int32)
    return torch.where((b & 127) == 127, b - 1, b).to(torch.uint8)


def small_integers(gen, *shape):
    """e4m3 bits of -3 .. 3: every sum of their products is exact."""
    v = torch.randint(-3, 4, shape, generator=gen).float()
    return v.to(torch.float8_e4m3fn).view(torch.uint8)


def scale_bytes(gen, rows, k, lo=-3, hi=3, fill=0xEE):
    """Random scale rows 2^lo .. 2^hi, the padding filled with `fill`."""
    s = torch.full((rows, pitch(k)), fill, dtype=torch.uint8)
    s[:, :blocks(k)] = torch.randint(127 + lo, 128 + hi, (rows, blocks(k)),
                                     generator=gen).to(torch.uint8)
    return s


def silu(g):
    return g * torch.sigmoid(g)


def ffn_rows(x, wg, wu, wd):
    """(y, bound) of one expert's rows in fp64: y = wd Q(silu(g) u).  The
    bound: an error d of h (from g, u and the fp32 SwiGLU) moves Q(h) by at
    most what rounding h - d and h + d instead gives, under the exponents that
    their largest values ask for."""
    g, u = x @ wg.T, x @ wu.T
    dg, du = group_bound(x, wg), group_bound(x, wu)
    h = silu(g) * u
    # |silu'| < 1.1, |silu(g)| <= |g|; the fp32 evaluation: exp2's argument is
    # rounded (2^-24 |g| log2 e in the exponent), six operations of 1 ulp
    d = 1.1 * dg * (u.abs() + du) + (silu(g).abs()) * du \
        + h.abs() * 2.0 ** -23 * (6 + 1.5 * g.abs())
    q, e = quant(h, 1)
    hq = spread(q, e, 1)
    move = torch.zeros_like(h)
    lo, hi = (h.abs() - d).clamp(min=0), h.abs() + d
    elo, ehi = exponent(tiles(lo, 1).amax((1, 3))), exponent(tiles(hi, 1).amax((1, 3)))
    for ee in (elo, ehi):
        f = torch.ldexp(torch.ones((), dtype=torch.float64), ee)
        f = f.repeat_interleave(BLOCK, 1)[:, :h.shape[1]]
        for v in (h - d, h + d):
            r = round_e4m3((v / f).clamp(-448, 448)) * f
            move = torch.maximum(move, (r - hq).abs())
    return hq @ wd.T, move @ wd.abs().T + group_bound(hq.abs() + move, wd)
