"""The token operators in 64 bits, with bounds on how far a kernel may be off, element by element.

Bounds: u = 2^-24.  A sum of n products in fp32 is off by at most (n + 8) u times the sum of the products' magnitudes (products of bfloat16
are exact; every addition rounds once; eight for a split's and a chain's joining).  A value stored in type t is off by half a step, 2^-8 of it for
bfloat16, 2^-24 for fp32.  An activation's slope is at most 1.13, its derivative's 1.1; its own evaluation goes through e^-t with t rounded: (4 |t| + 16) u of
its value."""
import math

import torch

U = 2.0 ** -24
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}
ACTS = ("none", "relu", "relu6", "silu", "gelu")


def f64(t):
    return t.to(torch.float64)


def act(z, name):
    """(act(z), act'(z), argument of the exponential)"""
    if name == "none":
        return z, torch.ones_like(z), torch.zeros_like(z)
    if name == "relu":
        return z.clamp(min=0), (z > 0).double(), torch.zeros_like(z)
    if name == "relu6":
        return z.clamp(0, 6), ((z > 0) & (z < 6)).double(), torch.zeros_like(z)
    if name == "silu":
        p = torch.sigmoid(z)
        return z * p, p * (1 + z * (1 - p)), z
    k, c = math.sqrt(8 / math.pi), 0.044715
    t = k * (z + c * z ** 3)
    p = torch.sigmoid(t)
    return z * p, p + z * p * (1 - p) * k * (1 + 3 * c * z * z), t


def act_err(a, t, ez):
    return 1.13 * ez + (4 * t.abs() + 16) * U * a.abs()


def dact_err(z, t):
    return (4 * t.abs() + 16) * U * (1 + z.abs())


def product(a, b, ea=None, eb=None):
    """a [m, k] times b [n, k] transposed, and its bound for operands off by ea, eb"""
    y = a @ b.t()
    e = (a.shape[1] + 8) * U * (a.abs() @ b.abs().t())
    if ea is not None:
        e = e + ea @ b.abs().t()
    if eb is not None:
        e = e + a.abs() @ eb.t()
    return y, e


def stored(y, e, dtype):
    return e + HALF[dtype] * (y.abs() + e)


def groups(x):
    rows, cols = x.shape
    g = -(-cols // 32)
    v = torch.zeros(rows, g * 32, dtype=x.dtype, device=x.device)
    v[:, :cols] = x
    return v.view(rows, g, 32)


def act8_scales(x):
    """exponents of the groups' scales, by the definition: the smallest power of two, 2^-127 at least, with which the largest finite magnitude is at most 448"""
    v = groups(f64(x)).abs()
    top = torch.where(v.isfinite(), v, torch.zeros_like(v)).amax(2)
    e = torch.full_like(top, -127.0)
    for k in range(-126, 121):
        e = torch.where(top > 448 * 2.0 ** (k - 1), torch.full_like(e, float(k)), e)
    return e


def act8(x):
    """(values of the 8-bit form, exponents): to nearest even with three bits behind the leading one, steps of 2^-9 below 2^-6"""
    e = act8_scales(x)
    v = groups(f64(x)) / torch.exp2(e)[..., None]
    m = v.abs()
    k = torch.floor(torch.log2(m.clamp(min=2.0 ** -6)))
    k = torch.where(torch.exp2(k) > m.clamp(min=2.0 ** -6), k - 1, k)
    step = torch.exp2(k - 3)
    q = torch.round(v / step) * step
    q = torch.where(v.isfinite(), q, torch.full_like(q, float("nan")))
    return (q * torch.exp2(e)[..., None]).reshape(x.shape[0], -1)[:, :x.shape[1]], e


def act8_decode(q, s):
    """values from the bytes"""
    sign = 1.0 - 2.0 * (q >> 7).double()
    ex, man = ((q >> 3) & 15).double(), (q & 7).double()
    v = torch.where(ex == 0, man * 2.0 ** -9, (1 + man / 8) * torch.exp2(ex - 7)) * sign
    v = torch.where((q & 127) == 127, torch.full_like(v, float("nan")), v)
    return v * torch.exp2(s.double() - 127).repeat_interleave(32, 1)[:, :q.shape[1]]


def act8_encode(x):
    """(q, s) bytes of the 8-bit form"""
    val, e = act8(x)
    cols = x.shape[1]
    codes = torch.arange(256, device=x.device, dtype=torch.uint8)[None]
    table = act8_decode(codes, torch.full((1, 8), 127, dtype=torch.uint8, device=x.device))[0]
    v = val / torch.exp2(e).repeat_interleave(32, 1)[:, :cols]
    pos = table[:127]
    q = torch.searchsorted(pos.contiguous(), v.abs().contiguous()).clamp(max=126).to(torch.uint8)
    q = torch.where(v < 0, q | 128, q)
    q = torch.where(v.isnan(), torch.full_like(q, 127), q)
    return q, (e + 127).to(torch.uint8)


def close(got, want, bound, what):
    got = f64(got)
    off = (got - want).abs()
    bad = ~(off <= 1.01 * bound + 1e-300)
    assert not bool(bad.any()), (what, int(bad.sum()), float(off[bad].max()), float((off / bound.clamp(min=1e-300)).max()), got.shape,
                                 torch.nonzero(bad)[:4].tolist())
