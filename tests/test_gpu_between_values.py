"""Joins, the recurrence and log probabilities with values that are no ordinary ones: logits far from zero, scales that leave little of a row, infinities and NaN in one of several sequences.
Bounds are those of between_ref.py, which hold for any finite logits."""
import math

import pytest

from test_gpu_between import ACT_CODE, DTYPES, env, gen_of, logp_case, put, stream  # noqa: F401
from test_gpu_token import given, matrix, types

pytestmark = pytest.mark.gpu
ROWS = [(4, 1000, 0), (3, 5000, 20), (300, 700, 5), (2, 40000, 0), (5, 33001, 3)]              # rows by one block and by several, with and without alternatives


def step(dtype, at):
    """the distance of numbers of the type at this one"""
    return 2.0 ** (math.floor(math.log2(abs(at))) - (23 if dtype == "f32" else 7))


# ---- log probabilities ------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("at", [1e5, -1e5, 2.3e6, -2.3e6, 1e7, -1e7, 3e7, -1e9, 1e9, -1e20, 1e30])
@pytest.mark.parametrize("rows,vocab,k", ROWS)
def test_logp_far_from_zero(env, dtype, at, rows, vocab, k):
    """all the same, spread over thirty of the type's steps, and half of a row there (an ordinary mask where it is negative)"""
    torch = env[0]
    g, d = gen_of(torch, rows, vocab, at), step(dtype, at)
    z = at + d * torch.randint(0, 30, (rows, vocab), generator=g, device="cuda").double()
    z[0] = at
    z[1, ::2] = torch.randn(z[1, ::2].shape, generator=g, device="cuda").double()
    for scale in (1.0, 0.5 / d):                                    # powers of two
        logp_case(env, dtype, rows, vocab, k, scale=scale, logits=z)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("scale", [1e3, 1e4, 1e5, 1e6, 1e7, 1e8])
@pytest.mark.parametrize("rows,vocab,k", ROWS)
def test_logp_of_ordinary_logits_with_a_large_scale(env, dtype, scale, rows, vocab, k):
    """sampling at a temperature next to nothing"""
    logp_case(env, dtype, rows, vocab, k, scale=scale)
    g = gen_of(env[0], rows, vocab, scale)
    z = 4 + env[0].randint(0, 40, (rows, vocab), generator=g, device="cuda").double() * step(dtype, 4.0)           # neighbours, so that more than one counts
    logp_case(env, dtype, rows, vocab, k, scale=scale, logits=z)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,vocab,k", ROWS)
def test_logp_of_a_scale_next_to_the_types_largest(env, dtype, rows, vocab, k):
    """log2 e times it is no number of 32 bits any more; logits so small that they are a few units apart all the same"""
    torch = env[0]
    g = gen_of(torch, rows, vocab)
    z = 2.0 ** -126 * torch.randint(0, 12, (rows, vocab), generator=g, device="cuda").double()
    z[-1] = 0
    logp_case(env, dtype, rows, vocab, k, scale=1.5 * 2.0 ** 127, logits=z, dlogp_there=False, dent_there=False)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,vocab", [(4, 30), (300, 60), (2, 5000)])
def test_logp_of_logits_farther_apart_than_the_type_reaches(env, dtype, rows, vocab):
    """3e38 and -3e38: the log probability, a quarter of their difference, is a number all the same"""
    torch = env[0]
    z = torch.zeros(rows, vocab, device="cuda")
    z[:, 1], z[:, 2::2], z[:, -1] = 3e38, -3e38, -math.inf
    z[0, 1] = -3e38
    ids = torch.arange(rows, device="cuda") % 4
    ids[1] = vocab - 1
    for k in (0, min(vocab, 64)):
        logp_case(env, dtype, rows, vocab, k, scale=0.25, logits=z, ids=ids)
    logp_case(env, dtype, rows, vocab, 3, scale=1e-37, logits=z, ids=ids)


# ---- the recurrence ------------------------------------------------------------------------------------------------------
def scan_both(env, a, names, rows, seqs, width, dt):
    """results of the forward and the backward, each in a buffer of its own"""
    torch, P, _ = env
    res = {}
    for name, ld in names:
        res[name] = torch.full((seqs, width), 777.0, device="cuda") if name in ("h_end", "dh0") else torch.full((rows, width), 777.0, dtype=dt, device="cuda")
        put(a, **{name: res[name], ld: width})
    for back, call in ((False, P.scan_forward), (True, P.scan_backward)):
        ws, ok = given(a, torch, P.scan_workspace(a, back))
        call(a, stream(torch))
        torch.cuda.synchronize()
        ok()
    return res


# sequences in one chunk, in several, in one launch, in three, in more chunks than a column's threads keep; long ones in front, in the middle and behind
PACKED = [([5, 10, 6], 20), ([1] * 40, 9), ([30, 0, 33, 20], 66), ([100, 28], 131), ([200, 150, 300], 70), ([3, 700, 2, 60], 20), ([600, 1, 600], 130), ([0, 90, 0, 0, 400, 31, 0], 33), ([64, 64, 64], 40),
          ([5000, 70, 4000], 4), ([9000, 9000], 3)]
EVEN = [([1] * 40, 9), ([10] * 3, 20), ([64] * 2, 131), ([64] * 3, 40), ([600] * 3, 130), ([9000] * 2, 3)]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("form", ["add", "mix", "unit"])
@pytest.mark.parametrize("lens,width,uniform", [(*c, False) for c in PACKED] + [(*c, True) for c in EVEN], ids=lambda v: str(v).replace(" ", "")[:40])
def test_scan_keeps_what_is_not_finite_in_its_sequence(env, dtype, form, lens, width, uniform):
    """an infinity or NaN in any operand of one sequence: all others have the bits that they have without it; rows of no sequence hold NaN"""
    torch, P, _ = env
    tdt, code = types(P, torch, dtype)
    starts = [0 if uniform else 2]
    for n in lens:
        starts.append(starts[-1] + n)
    rows, seqs, act = starts[-1] + (0 if uniform else 3), len(lens), "" if form == "mix" else "silu"
    g = gen_of(torch, lens, width, form)
    m = {k: matrix(torch, g, rows, width, tdt, 2.0 if k == "f" else 1.0) for k in ("f", "x", "g", "dy")}
    m.update({k: matrix(torch, g, seqs, width, torch.float32) for k in ("h0", "dh_end")})
    for k in ("f", "x", "g", "dy"):                                 # rows of no sequence
        m[k][:starts[0]], m[k][starts[-1]:] = math.nan, math.nan
    dev = torch.tensor(starts, dtype=torch.int32, device="cuda")
    a = P.scan_args(rows=rows, width=width, seqs=seqs, dtype=code, form={"add": P.SCAN_ADD, "mix": P.SCAN_MIX, "unit": P.SCAN_UNIT}[form], act=ACT_CODE[act or "none"])
    put(a, **({"length": lens[0]} if uniform else {"starts": dev}))
    if not act:
        del m["g"]
    for k, ld in (("f", "ldf"), ("x", "ldx"), ("g", "ldg"), ("dy", "lddy"), ("h0", "ldh0"), ("dh_end", "lddhe")):
        if k in m:
            put(a, **{k: m[k], ld: width})
    names = [("y", "ldy"), ("h_end", "ldhe"), ("df", "lddf"), ("dx", "lddx"), ("dh0", "lddh0")] + [("dg", "lddg")] * bool(act)
    want = scan_both(env, a, names, rows, seqs, width, tdt)
    assert all(bool(v.isfinite().all()) for v in want.values())
    for s in sorted({0, seqs // 2, seqs - 1}):
        if not lens[s]:
            continue
        b, e = starts[s], starts[s + 1]
        others = torch.ones(rows, dtype=torch.bool, device="cuda")
        others[b:e] = False
        for k in m:
            for bad in (math.nan, math.inf, -math.inf):
                states = k in ("h0", "dh_end")
                at = (s if states else b if bad != bad else (b + e) // 2 if bad > 0 else e - 1)
                old = m[k][at].clone()
                m[k][at] = bad
                got = scan_both(env, a, names, rows, seqs, width, tdt)
                m[k][at] = old
                for name, r in got.items():
                    same = [q for q in range(seqs) if q != s] if name in ("h_end", "dh0") else others
                    assert torch.equal(r[same], want[name][same]), (name, k, bad, s)


@pytest.mark.parametrize("form", ["add", "mix", "unit"])
def test_scan_gates_keep_their_places(env, form):
    """a, 1 - a and c(a) of gates from one end to the other in single precision, and their derivatives, from single steps.  e^-|f| is off by 2 u of the exponential, one rounding and 0.05 |f| u
    (4 u at 80), its quotient by 1 + e by 4 u more, c by no more than that and a root's 2 u; two products and the store round: 16 u of a result that is one product, and of the sum of the
    magnitudes of two.  Below 2^-100 a product's operands may have lost places."""
    torch, P, B = env
    f = torch.cat([torch.linspace(-80, 80, 4001, device="cuda"), torch.randn(4095, device="cuda") * 8])[None].contiguous()
    n = f.shape[1]
    g = gen_of(torch, form)
    x, h0, dy = (torch.randn(1, n, generator=g, device="cuda") for _ in range(3))
    y, end, df, dx, dh0 = (torch.empty(1, n, device="cuda") for _ in range(5))
    a = P.scan_args(rows=1, length=1, seqs=1, width=n, dtype=P.F32, form={"add": P.SCAN_ADD, "mix": P.SCAN_MIX, "unit": P.SCAN_UNIT}[form], f=f, ldf=n, x=x, ldx=n, h0=h0, ldh0=n, y=y, ldy=n,
                    h_end=end, ldhe=n, dy=dy, lddy=n, df=df, lddf=n, dx=dx, lddx=n, dh0=dh0, lddh0=n)
    P.scan_forward(a, stream(torch))
    P.scan_backward(a, stream(torch))
    torch.cuda.synchronize()
    z, x, h0, dy = (t.double() for t in (f, x, h0, dy))
    s, r = torch.sigmoid(z), torch.sigmoid(-z)
    c = {"add": torch.ones_like(s), "mix": r, "unit": (r * (1 + s)).sqrt()}[form]
    dc = {"add": torch.zeros_like(s), "mix": -s * r, "unit": -s * s * (r / (1 + s)).sqrt()}[form]
    for name, got, terms in (("y", y, (s * h0, c * x)), ("h_end", end, (s * h0, c * x)), ("dx", dx, (dy * c,)), ("dh0", dh0, (dy * s,)), ("df", df, (dy * s * r * h0, dy * dc * x))):
        B.close(got, sum(terms), 16 * B.U * sum(t.abs() for t in terms) + 2.0 ** -124, name)
