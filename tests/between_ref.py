"""Joins with norms, dropout, the gated recurrence and log probabilities in 64 bits, each value with a bound on how far a kernel may be off.

A number of type V is a value and its bound; every operation on two of them rounds once to 32 bits (u = 2^-24 of the result) and passes its operands' bounds on.
Sums over n values of a row are made by 64 lanes at least, n / 64 additions one behind the other and some thirty between lanes, chains and blocks: (n / 64 + 32) u of the sum
of magnitudes, whatever their order.  Square roots, divisions and reciprocals are off by 2 u at most, exponentials by 2 u and by the rounding of their
argument, twice: 2 u of it.  A value stored in type t is off by half a step more (token_ref.HALF).  Below 2^-126 steps are no smaller than there, 2^-149 in fp32 and 2^-133 in
bfloat16: half of one of the latter where it is stored, and of the former there and at the multiplication in front (SMALLEST)."""
import math

import torch

from token_ref import HALF, U, close, f64  # noqa: F401

SMALLEST = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -134 + 2.0 ** -149}


class V:
    def __init__(self, v, e=None):
        self.v = v.double() if hasattr(v, "double") else torch.tensor(float(v), dtype=torch.float64, device="cuda")
        self.e = torch.zeros_like(self.v) if e is None else e

    @staticmethod
    def of(x):
        return x if isinstance(x, V) else V(x)

    def rounded(self, k=1.0):
        return V(self.v, self.e + k * U * (self.v.abs() + self.e))

    def __add__(self, o):
        o = V.of(o)
        return V(self.v + o.v, self.e + o.e).rounded()

    def __sub__(self, o):
        o = V.of(o)
        return V(self.v - o.v, self.e + o.e).rounded()

    def __mul__(self, o):
        o = V.of(o)
        return V(self.v * o.v, self.v.abs() * o.e + o.v.abs() * self.e + self.e * o.e).rounded()

    __radd__, __rmul__ = __add__, __mul__

    def sum(self, dim, keepdim=True, n=None):
        n = self.v.shape[dim] if n is None else n
        return V(self.v.sum(dim, keepdim=keepdim), self.e.sum(dim, keepdim=keepdim) + (n / 64 + 32) * U * self.v.abs().sum(dim, keepdim=keepdim))

    def where(self, cond):
        z = torch.zeros_like(self.v)
        return V(torch.where(cond, self.v, z), torch.where(cond, self.e, z))

    def stored(self, dtype):
        return self.v, self.e + HALF[dtype] * (self.v.abs() + self.e) + SMALLEST[dtype]


def check(got, want, what):
    v, e = want.stored(got.dtype)
    close(got, v, e, what)


# ---- the generator -----------------------------------------------------------------------------------------------
def philox(counter, key):
    """ten rounds on Python's whole numbers"""
    c, (k0, k1) = list(counter), key
    for _ in range(10):
        a, b = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
        c = [(b >> 32) ^ c[1] ^ k0, b & 0xffffffff, (a >> 32) ^ c[3] ^ k1, a & 0xffffffff]
        k0, k1 = (k0 + 0x9E3779B9) & 0xffffffff, (k1 + 0xBB67AE85) & 0xffffffff
    return c


def mask(rows, cols, p, seed, site, row0):
    """(where values are kept, the factor of these)"""
    import numpy as np
    j, r = np.meshgrid(np.arange(-(-cols // 8), dtype=np.uint64), np.arange(rows, dtype=np.uint64) + np.uint64(row0))
    low, sh = np.uint64(0xffffffff), np.uint64(32)
    c = [j, np.full_like(j, site), r & low, r >> sh]
    k0, k1 = seed & 0xffffffff, (seed >> 32) & 0xffffffff
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> sh) ^ c[1] ^ np.uint64(k0), b & low, (a >> sh) ^ c[3] ^ np.uint64(k1), a & low]
        k0, k1 = (k0 + 0x9E3779B9) & 0xffffffff, (k1 + 0xBB67AE85) & 0xffffffff
    u = np.stack([h for w in c for h in (w & np.uint64(0xffff), w >> np.uint64(16))], 2).reshape(rows, -1)[:, :cols]
    q = math.floor(p * 65536 + 0.5)
    return torch.from_numpy((u >= q)).cuda(), 65536 / (65536 - q)


# ---- the join ------------------------------------------------------------------------------------------------------
def inverse_root(var, eps):
    """1 / sqrt(var + eps)"""
    t = var + V(eps, torch.tensor(U * eps, dtype=torch.float64, device="cuda"))
    r = 1 / torch.sqrt(t.v)
    return V(r, 0.5 * r * t.e / (t.v - t.e).clamp(min=0.5 * eps)).rounded(4)


def norm(v, layer, eps):
    """(normed, inverse deviation)"""
    n = v.v.shape[1]
    if layer:
        v = v - v.sum(1) * V(1 / n).rounded(1)
    r = inverse_root((v * v).sum(1) * V(1 / n).rounded(1), eps)
    return v * r, r


def norm_back(dv, vh, r, layer):
    n = dv.v.shape[1]
    t = dv - vh * ((dv * vh).sum(1) * V(1 / n).rounded(1))
    if layer:
        t = t - dv.sum(1) * V(1 / n).rounded(1)
    return r * t


def join(x, b, layer, post, eps, scale, pw, pb, qw, qb, gate, gate_rows, keep, up, dy=None, dn=None):
    """pre weights pw, pb; post weights qw, qb; any operand None: not there.  -> dict of V"""
    rows, width = (x if x is not None else b).shape
    y = V(f64(x)) if x is not None else V(torch.zeros(rows, width, dtype=torch.float64, device="cuda"))
    out, one = {}, torch.ones(1, width, dtype=torch.float64, device="cuda")
    if b is not None:
        bh, br = norm(V(f64(b)), layer, eps) if post else (V(f64(b)), None)
        c = bh
        if post:
            c = bh * (f64(qw) if qw is not None else one) + (f64(qb) if qb is not None else 0 * one)
        g = f64(gate)[torch.arange(rows, device="cuda") // gate_rows] if gate is not None else torch.ones(rows, width, dtype=torch.float64, device="cuda")
        s = V(scale, torch.tensor(abs(scale) * U, dtype=torch.float64, device="cuda"))
        sg = s * V(g)
        if keep is not None:
            k = V(torch.full((1, 1), up, dtype=torch.float64, device="cuda")).rounded()
            drop = lambda t: (t * k).where(keep)                                                # noqa: E731
        else:
            drop = lambda t: t                                                                  # noqa: E731
        y = y + sg * drop(c)
    yh, yr = norm(y, layer, eps)
    w = f64(pw) if pw is not None else one
    out["y"], out["n"] = y, yh * w + (f64(pb) if pb is not None else 0 * one)
    if dy is None and dn is None:
        return out
    d = V(f64(dy)) if dy is not None else V(torch.zeros(rows, width, dtype=torch.float64, device="cuda"))
    if dn is not None:
        n = V(f64(dn))
        d = d + norm_back(n * w, yh, yr, layer)
        out["dpre_w"], out["dpre_bias"] = (n * yh).sum(0, n=64 * rows), n.sum(0, n=64 * rows)
    out["dx"] = d
    if b is not None:
        dc = drop(sg * d)
        dg = s * drop(c) * d
        if gate is not None:
            groups = gate.shape[0]
            at = torch.arange(rows, device="cuda") // gate_rows
            add = lambda t: torch.zeros(groups, width, dtype=torch.float64, device="cuda").index_add_(0, at, t)          # noqa: E731
            n = 64 * min(gate_rows, rows)
            out["dgate"] = V(add(dg.v), add(dg.e) + (n / 64 + 32) * U * add(dg.v.abs()))
        if post:
            out["dpost_w"], out["dpost_bias"] = (dc * bh).sum(0, n=64 * rows), dc.sum(0, n=64 * rows)
            dc = norm_back(dc * (f64(qw) if qw is not None else one), bh, br, layer)
        out["db"] = dc
    return out


# ---- the recurrence --------------------------------------------------------------------------------------------------
# Whatever chunks it is cut into, a state is the sum of the same terms a[t] ... a[s+1] c x[s], and each step multiplies one rounding of a factor and two of a
# product or sum into it: bounds go through the recurrence with the sum of the terms' magnitudes.
def scan(f, x, g, h0, starts, form, act, dy=None, dh_end=None):
    import token_ref as R
    f, x = f64(f), f64(x)
    e = torch.exp(-f.abs())
    a = torch.where(f >= 0, 1 / (1 + e), e / (1 + e))
    rest = torch.where(f >= 0, e / (1 + e), 1 / (1 + e))
    rel = (2 * f.abs() + 16) * U                                     # of a, 1 - a, c and c's derivative
    c, dc = {"add": (torch.ones_like(a), torch.zeros_like(a)), "mix": (rest, -a * rest),
             "unit": ((rest * (1 + a)).sqrt(), -a * a * (rest / (1 + a)).sqrt())}[form]
    rows, width = f.shape
    zero = torch.zeros(rows, width, dtype=torch.float64, device=f.device)
    h, eh, before, eb, seqs = zero.clone(), zero.clone(), zero.clone(), zero.clone(), len(starts) - 1
    end, ee = torch.zeros(seqs, width, dtype=torch.float64, device=f.device), torch.zeros(seqs, width, dtype=torch.float64, device=f.device)
    for s in range(seqs):
        v = f64(h0[s]) if h0 is not None else zero[0]
        m, q = v.abs(), torch.zeros_like(v)
        for t in range(starts[s], starts[s + 1]):
            before[t], eb[t] = v, q
            u = c[t] * x[t]
            q = a[t] * q + (rel[t] + 3 * U) * (a[t] * m + u.abs())
            v, m = a[t] * v + u, a[t] * m + u.abs()
            h[t], eh[t] = v, q
        end[s], ee[s] = v, q
    H = V(h, eh)
    out = {"h_end": V(end, ee)}
    if g is not None:
        ga, gd, garg = R.act(f64(g), act)
        G, D = V(ga, R.act_err(ga, garg, 0)), V(gd, R.dact_err(f64(g), garg))
    out["y"] = H * G if g is not None else H
    if dy is None:
        return out
    dy = V(f64(dy))
    into = dy * G if g is not None else dy
    lam, el = zero.clone(), zero.clone()
    dh0, e0 = end * 0, end * 0
    for s in range(seqs):
        v = f64(dh_end[s]) if dh_end is not None else zero[0]
        m, q = v.abs(), torch.zeros_like(v)
        for t in range(starts[s + 1] - 1, starts[s] - 1, -1):
            v, m, q = v + into.v[t], m + into.v[t].abs(), q + into.e[t] + U * (m + into.v[t].abs())
            lam[t], el[t] = v, q
            q = a[t] * q + (rel[t] + 3 * U) * a[t] * m
            v, m = a[t] * v, a[t] * m
        dh0[s], e0[s] = v, q
    L = V(lam, el)
    A = lambda t: V(t, rel * t.abs())                                # noqa: E731
    out.update(dh0=V(dh0, e0), dx=L * A(c), df=L * (V(before, eb) * A(a * rest) + V(x) * A(dc)))
    if g is not None:
        out["dg"] = dy * H * D
    return out


# ---- log probabilities -------------------------------------------------------------------------------------------------
def logp(logits, scale, ids, pad_id, dlogp=None, dentropy=None):
    """rows without a NaN or +inf"""
    z = f64(logits)
    rows, vocab = z.shape
    there = (z > -math.inf)
    some = there.any(1, keepdim=True)
    m = torch.where(some, z.amax(1, keepdim=True), torch.zeros_like(z[:, :1]))
    t = torch.where(there, (z - m) * scale, torch.full_like(z, -math.inf))
    tf = torch.where(there, t, torch.zeros_like(t))
    et = 3 * U * tf.abs()
    x = torch.exp(t)
    ex = x * (2 * U * tf.abs() + 4 * U + et) + 1e-37                 # exponentials below the smallest number vanish
    s1 = V(x, torch.where(there, ex, torch.zeros_like(x))).sum(1)
    l = torch.log(s1.v)
    L = V(torch.where(some, l, torch.zeros_like(l)), torch.where(some, s1.e / s1.v + 4 * U * (l.abs() + 1), torch.zeros_like(l)))
    lp = V(torch.where(there, tf - L.v, torch.full_like(t, -math.inf)), torch.where(there, et + L.e + U * (tf - L.v).abs(), torch.zeros_like(t)))
    p = torch.exp(lp.v)
    fin = torch.where(there, lp.v, torch.zeros_like(lp.v))
    s2 = V(x * tf, torch.where(there, ex * tf.abs() + x * et + U * (x * tf).abs(), torch.zeros_like(x))).sum(1)
    ent = -(p * fin).sum(1, keepdim=True)
    q = s2.v / s1.v.clamp(min=1e-300)
    E = V(ent, torch.where(some, L.e + s2.e / s1.v + q.abs() * s1.e / s1.v + 4 * U * (q.abs() + L.v.abs()), torch.zeros_like(l)))
    ids = ids.long()[:, None]
    inside = (ids >= 0) & (ids < vocab)
    at = ids.clamp(0, vocab - 1)
    given = lambda v, none: torch.where(ids == pad_id, torch.zeros_like(l), torch.where(inside, v.gather(1, at), torch.full_like(l, none)))   # noqa: E731
    out = {"logp": V(given(torch.where(some, lp.v, torch.full_like(lp.v, -math.inf)), math.nan)[:, 0], given(lp.e, 0.0)[:, 0]), "entropy": V(E.v[:, 0], E.e[:, 0])}
    out["lse"] = V(torch.where(some, m * scale + l, torch.full_like(l, -math.inf))[:, 0], torch.where(some, L.e + 2 * U * ((m * scale).abs() + l.abs()), torch.zeros_like(l))[:, 0])
    out["lp"] = lp
    if dlogp is None and dentropy is None:
        return out
    w = torch.where(inside & (ids != pad_id), f64(dlogp)[:, None], torch.zeros_like(l)) if dlogp is not None else torch.zeros_like(l)
    hw = f64(dentropy)[:, None] if dentropy is not None else torch.zeros_like(l)
    P = V(p, p * (lp.e + 2 * U * fin.abs() + 4 * U) + 1e-37)
    Q = V(w) + V(hw) * (V(fin, torch.where(there, lp.e, torch.zeros_like(lp.e))) + E)
    hit = torch.zeros_like(z).scatter_(1, at, torch.where(inside & (ids != pad_id), w, torch.zeros_like(w)))
    d = (V(hit) - P * Q) * V(torch.tensor(float(scale), dtype=torch.float64, device="cuda"))
    d = V(torch.where(some, d.v, torch.zeros_like(d.v)), torch.where(some, d.e, torch.zeros_like(d.e)))
    out["dlogits"] = d
    return out


def top(logits, k):
    """the k largest logits above -inf, of equal ones the lower column first; -1 where there is none"""
    z = f64(logits)
    order = torch.sort(torch.where(z.isnan(), torch.full_like(z, -math.inf), z), dim=1, descending=True, stable=True)
    ids = torch.where(order[0] > -math.inf, order[1], torch.full_like(order[1], -1))[:, :k]
    if ids.shape[1] < k:
        ids = torch.cat((ids, ids.new_full((ids.shape[0], k - ids.shape[1]), -1)), 1)
    return ids.int()
