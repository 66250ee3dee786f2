"""Joins with norms, dropout, the gated recurrence and log probabilities against their formulas in 64 bits (between_ref.py): every type, form and direction, at the
sizes where vectors, wavefronts, blocks and chunks end, with strides and offsets of every alignment."""
import math
import zlib

import pytest

from test_gpu_token import given, matrix, out, types

pytestmark = pytest.mark.gpu
DTYPES = ["f32", "bf16"]
ACT_CODE = {"none": 0, "relu": 1, "relu6": 2, "silu": 3, "gelu": 4}


@pytest.fixture(scope="module")
def env():
    import torch
    import paper_2110_02781_amd as P
    import between_ref as B
    return torch, P, B


def gen_of(torch, *key):
    return torch.Generator(device="cuda").manual_seed(zlib.crc32(repr(key).encode()))


def stream(torch):
    return torch.cuda.current_stream().cuda_stream


def put(a, **kw):
    for k, v in kw.items():
        setattr(a, k, v.data_ptr() if hasattr(v, "data_ptr") else v)


# ---- dropout --------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols,p,slack,skip", [(1, 1, 0.5, 0, 0), (1, 8, 0.1, 0, 0), (3, 7, 0.3, 2, 1), (5, 9, 0.0, 0, 0), (130, 1001, 0.1, 3, 3), (2, 4096, 0.9, 0, 0), (700, 64, 0.25, 0, 1)])
def test_dropout(env, dtype, rows, cols, p, slack, skip):
    torch, P, B = env
    tdt, code = types(P, torch, dtype)
    g = gen_of(torch, rows, cols)
    x, r, dy = (matrix(torch, g, rows, cols, tdt, 1.0, slack, skip) for _ in range(3))
    x[0, 0] = math.inf                                              # dropped or not
    (y, y_ok), (dx, dx_ok) = (out(torch, rows, cols, tdt, slack, skip) for _ in range(2))
    seed, site, row0 = 0xfedcba9876543210, 0x80000001, (1 << 40) + 77
    a = P.dropout_args(rows=rows, cols=cols, dtype=code, p=p, seed=seed, site=site, row0=row0, x=x, ldx=x.stride(0), residual=r, ldr=r.stride(0), y=y, ldy=y.stride(0), dy=dy,
                       lddy=dy.stride(0), dx=dx, lddx=dx.stride(0))
    P.dropout_forward(a, stream(torch))
    P.dropout_backward(a, stream(torch))
    torch.cuda.synchronize()
    keep, up = B.mask(rows, cols, p, seed, site, row0)
    up = up if p else 1.0
    want = torch.where(keep, B.f64(x) * up, 0.0)
    fin = want.isfinite()
    assert bool((y[~fin] == math.inf).all())
    e = 2 * B.U * want.abs() + B.U * (want + B.f64(r)).abs()
    B.close(y[fin], (want + B.f64(r))[fin], (e + B.HALF[tdt] * ((want + B.f64(r)).abs() + e))[fin], "y")
    want = torch.where(keep, B.f64(dy) * up, 0.0)
    B.close(dx, want, 2 * B.U * want.abs() + B.HALF[tdt] * want.abs() * (1 + 1e-6), "dx")
    y_ok(), dx_ok()


def test_dropout_goes_by_row_numbers_and_the_seed_in_memory(env):
    """parts of a batch have the whole batch's mask; a captured call follows the seed in memory; in place"""
    torch, P, _ = env
    rows, cols, s = 96, 200, stream(torch)
    x = torch.ones(rows, cols, device="cuda")
    whole, parts = torch.empty_like(x), torch.empty_like(x)
    at = torch.tensor([5], dtype=torch.int64, device="cuda")
    kw = dict(cols=cols, dtype=P.F32, p=0.3, site=3, x=x, ldx=cols, ldy=cols)
    P.dropout_forward(P.dropout_args(rows=rows, y=whole, seed=40, **kw), s)
    for r0, r1 in ((0, 1), (1, 50), (50, 96)):
        P.dropout_forward(P.dropout_args(rows=r1 - r0, row0=r0, y=parts[r0:], seed=35, seed_dev=at, **kw), s)          # 35 + 5
    assert torch.equal(whole, parts) and 0.25 < float((whole == 0).float().mean()) < 0.35
    same = x.clone()
    a = P.dropout_args(rows=rows, cols=cols, dtype=P.F32, p=0.3, site=3, seed=35, seed_dev=at, x=same, ldx=cols, y=same, ldy=cols)
    P.dropout_forward(a, s)
    assert torch.equal(same, whole)
    a.seed = 30
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        P.dropout_forward(a, torch.cuda.current_stream().cuda_stream)
    for k in (10, 11, 10):
        at.fill_(k)
        same.fill_(1)
        graph.replay()
        torch.cuda.synchronize()
        if k == 10:
            assert torch.equal(same, whole)
        else:
            assert not torch.equal(same, whole) and 0.25 < float((same == 0).float().mean()) < 0.35


# ---- the join ---------------------------------------------------------------------------------------------------------
def join_case(env, dtype, rows, width, layer=False, post=True, gate="row", gate_rows=1, p=0.0, x_there=True, b_there=True, weights=True, dy_there=True, dn_there=True, accumulate=0,
              slack=0, skip=0, gate_f32=False, scale=0.5):
    torch, P, B = env
    tdt, code = types(P, torch, dtype)
    g = gen_of(torch, rows, width, layer, post, gate)
    mat = lambda r, std=1.0, dt=tdt: matrix(torch, g, r, width, dt, std, slack, skip)                     # noqa: E731
    x, b = (mat(rows) if x_there else None), (mat(rows, 2.0) if b_there else None)
    if x_there and width > 3:
        x[:, 3] *= 8
    vec = lambda mean, std: mean + std * torch.randn(width, generator=g, device="cuda")                  # noqa: E731
    pw, pb, qw, qb = (vec(1, 0.1), vec(0, 0.1), vec(1, 0.2), vec(0, 0.1)) if weights else (None,) * 4
    gt, gdt = None, torch.float32 if gate_f32 or dtype == "f32" else tdt
    gate_rows = {"none": 0, "row": 1, "all": rows}.get(gate, gate_rows)
    if gate != "none" and b_there:
        gt = matrix(torch, g, -(-rows // gate_rows), width, gdt, 1.0, slack, skip)
    dy, dn = (mat(rows) if dy_there else None), (mat(rows) if dn_there else None)
    seed, site, row0 = 1234567890123, 5, 1 << 33
    keep, up = B.mask(rows, width, p, seed, site, row0) if p else (None, 1.0)
    a = P.join_args(rows=rows, width=width, dtype=code, norm=int(layer), post=int(post), eps=1e-5, scale=scale, p=p, seed=seed, site=site, row0=row0)
    oks, res = [], {}

    def result(name, r, dt, ld):
        m, ok = out(torch, r, width, dt, slack if ld else 0, skip)
        oks.append(ok)
        res[name] = m
        put(a, **{name: m})
        if ld:
            put(a, **{ld: m.stride(0)})
        return m
    for name, ld, m in (("x", "ldx", x), ("b", "ldb", b), ("gate", "ldg", gt), ("dy", "lddy", dy), ("dn", "lddn", dn)):
        if m is not None:
            put(a, **{name: m, ld: m.stride(0)})
    if gt is not None:
        put(a, gate_rows=gate_rows, gate_dtype=P.F32 if gdt == torch.float32 else P.BF16)
    if weights:
        put(a, pre_w=pw, pre_bias=pb)
        if post:
            put(a, post_w=qw, post_bias=qb)
    result("y", rows, tdt, "ldy")
    result("n", rows, tdt, "ldn")
    P.join_forward(a, stream(torch))
    want = B.join(x, b, layer, post, 1e-5, scale, pw, pb, qw if post else None, qb if post else None, gt, gate_rows, keep, up, dy, dn)
    torch.cuda.synchronize()
    for k in ("y", "n"):
        B.check(res[k], want[k], k)
    back = ["dx"] + ["db"] * b_there + ["dgate"] * (gt is not None) + ["dpre_w", "dpre_bias"] * dn_there + ["dpost_w", "dpost_bias"] * (b_there and post)
    for k in back:
        if k in ("dx", "db"):
            result(k, rows, tdt, "ldd" + k[1:])
        elif k == "dgate":
            result(k, gt.shape[0], gdt, "lddg")
        else:
            result(k, 1, torch.float32, None)
    if accumulate:
        a.accumulate = 1
        for k in back[1 + b_there:]:
            if k == "dgate":
                if gdt != torch.float32:
                    continue
                a.gate_accumulate = 1
            res[k].fill_(0.75)
    ws, ws_ok = given(a, torch, P.join_workspace(a))
    oks.append(ws_ok)
    P.join_backward(a, stream(torch))
    torch.cuda.synchronize()
    for k in back:
        w = want[k]
        if accumulate and k not in ("dx", "db") and (k != "dgate" or gdt == torch.float32):
            w = w + B.V(0.75)
        B.check(res[k], B.V(w.v.view(res[k].shape), w.e.view(res[k].shape)), k)
    for ok in oks:
        ok()
    return a, res


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,width,slack,skip", [(1, 1, 0, 0), (1, 8, 0, 0), (3, 7, 1, 1), (2, 9, 0, 0), (70, 64, 0, 0), (5, 511, 2, 3), (5, 512, 0, 0), (6, 513, 0, 0), (130, 1001, 7, 1),
                                                   (9, 2048, 0, 0), (3, 2049, 0, 1), (7, 4096, 0, 0), (3, 8200, 0, 0), (2, 16384, 0, 0), (2, 16385, 0, 0), (2, 33001, 0, 1), (2, 40000, 0, 0)])
def test_join_sizes(env, dtype, rows, width, slack, skip):
    join_case(env, dtype, rows, width, slack=slack, skip=skip, p=0.2 if rows % 2 else 0.0, layer=width % 2 == 1)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("layer", [False, True])
@pytest.mark.parametrize("post", [False, True])
@pytest.mark.parametrize("gate,gate_rows", [("none", 0), ("row", 1), ("all", 0), ("group", 3), ("group", 64), ("group", 5000)])
def test_join_forms(env, dtype, layer, post, gate, gate_rows):
    join_case(env, dtype, 67, 200, layer, post, gate, gate_rows, p=0.1 if layer else 0.0, gate_f32=gate == "all")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("kw", [dict(x_there=False), dict(b_there=False), dict(weights=False), dict(dy_there=False), dict(dn_there=False), dict(accumulate=1), dict(accumulate=1, gate="all", gate_f32=True),
                                dict(accumulate=1, gate="group", gate_rows=7, gate_f32=True), dict(scale=-2.0, p=0.6), dict(b_there=False, post=False, dn_there=False)], ids=str)
def test_join_parts(env, dtype, kw):
    join_case(env, dtype, 40, 136, **kw)


@pytest.mark.parametrize("gate,gate_rows", [("row", 1), ("group", 2), ("group", 700), ("group", 1500), ("all", 0)])
def test_join_many_rows(env, gate, gate_rows):
    """rows dealt to several blocks: groups inside a block's range and over several blocks, the last group short"""
    join_case(env, "bf16", 5003, 96, True, True, gate, gate_rows, p=0.1, gate_f32=gate_rows == 700)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("width", [4104, 6001, 8192])
@pytest.mark.parametrize("layer,gate,weights", [(True, "row", True), (False, "none", False), (True, "all", True), (False, "group", False)])
def test_join_of_the_longest_rows_that_are_held(env, dtype, width, layer, gate, weights):
    """column sums in LDS, up to four of them; five go another way"""
    join_case(env, dtype, 37, width, layer, True, gate, 5, p=0.1, weights=weights, gate_f32=gate == "all")


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows", [1, 2, 3, 4, 5, 7])
@pytest.mark.parametrize("width", [7, 64, 121, 128, 129, 240, 256, 257])
def test_join_rows_that_share_a_wavefront(env, dtype, rows, width):
    """up to 128 columns four rows are in a wavefront, up to 256 two: some of them past the last row"""
    join_case(env, dtype, rows, width, width % 3 == 0, rows % 2 == 0, "group", 3, p=0.25 if rows > 2 else 0.0)


@pytest.mark.parametrize("width", [20, 32, 160])
@pytest.mark.parametrize("gate,gate_rows", [("none", 0), ("row", 1), ("group", 3), ("group", 9), ("group", 5000), ("all", 0)])
def test_join_ranges_that_share_a_wavefront(env, width, gate, gate_rows):
    """more rows than there are ranges, so that a range has several and the last ones of a wavefront fewer or none"""
    join_case(env, "f32", 18005, width, width == 20, True, gate, gate_rows, p=0.1)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("tail", range(1, 8))
@pytest.mark.parametrize("front", [8, 248, 1016])
def test_join_last_columns(env, dtype, tail, front):
    """a row's last columns, fewer than eight, with rows one behind another and with space between them"""
    join_case(env, dtype, 9, front + tail, tail % 2 == 0, True, "row", p=0.1)
    join_case(env, dtype, 5, front + tail, False, False, "group", 2, slack=tail, skip=tail % 3, gate_f32=True)


def test_join_in_place_and_twice(env):
    torch, P, _ = env
    for width in (200, 40000):
        a, res = join_case(env, "bf16", 33, width, p=0.1)
        y, n, dx, db = (res[k].clone() for k in ("y", "n", "dx", "db"))
        keep = {}
        x = torch.empty(33, width, dtype=torch.bfloat16, device="cuda")
        # the operands' values from a y that is written into x's buffer, then into b's: the inputs come from the first case's generator again
        g = gen_of(torch, 33, width, False, True, "row")
        xs, bs = (matrix(torch, g, 33, width, torch.bfloat16, s) for s in (1.0, 2.0))
        xs[:, 3] *= 8
        rest = [torch.randn(width, generator=g, device="cuda") for _ in range(4)]
        pw, pb, qw, qb = (m + s * r for (m, s), r in zip(((1, 0.1), (0, 0.1), (1, 0.2), (0, 0.1)), rest))
        gt = matrix(torch, g, 33, width, torch.bfloat16)
        dy, dn = (matrix(torch, g, 33, width, torch.bfloat16) for _ in range(2))
        keep.update(pw=pw, pb=pb, qw=qw, qb=qb, gt=gt, dn=dn)
        for into in ("x", "b"):
            x2, b2 = xs.clone(), bs.clone()
            put(a, x=x2, b=b2, ldx=width, ldb=width, pre_w=pw, pre_bias=pb, post_w=qw, post_bias=qb, gate=gt, ldg=width, y=x2 if into == "x" else b2, ldy=width, n=x, ldn=width)
            P.join_forward(a, stream(torch))
            torch.cuda.synchronize()
            assert torch.equal(x2 if into == "x" else b2, y) and torch.equal(x, n)
        put(a, x=xs, b=bs, dy=dy, lddy=width, dn=dn, lddn=width, dx=dy, lddx=width)
        ws, _ = given(a, torch, P.join_workspace(a))
        P.join_backward(a, stream(torch))
        torch.cuda.synchronize()
        assert torch.equal(dy, dx) and torch.equal(res["db"], db)


def test_join_without_rows(env):
    torch, P, _ = env
    w = torch.full((4, 24), 3.0, device="cuda")
    kw = dict(rows=0, width=24, dtype=P.F32, post=1, dpre_w=w[0], dpre_bias=w[1], dpost_w=w[2], dpost_bias=w[3])
    P.join_backward(P.join_args(accumulate=1, **kw), stream(torch))
    assert bool((w == 3).all())
    P.join_backward(P.join_args(**kw), stream(torch))
    assert bool((w == 0).all())


# ---- the recurrence ------------------------------------------------------------------------------------------------------
def scan_case(env, dtype, lens, width, form="mix", act="silu", uniform=False, h0_there=True, dh_there=True, slack=0, skip=0, behind=0, front=0, in_place=False, shift=0.0, spread=2.0):
    torch, P, B = env
    tdt, code = types(P, torch, dtype)
    starts = [front]
    for n in lens:
        starts.append(starts[-1] + n)
    rows, seqs = starts[-1] + behind, len(lens)
    g = gen_of(torch, rows, width, seqs, form)
    mat = lambda std=1.0: matrix(torch, g, rows, width, tdt, std, slack, skip)                            # noqa: E731
    f, x, dy = mat(spread), mat(), mat()
    f += shift
    gt = mat() if act else None
    state = lambda: matrix(torch, g, seqs, width, torch.float32, 1.0, slack, skip)                        # noqa: E731
    h0, dh_end = (state() if h0_there else None), (state() if dh_there else None)
    want = B.scan(f, x, gt, h0, starts, form, act or "none", dy, dh_end)
    code_of = {"add": P.SCAN_ADD, "mix": P.SCAN_MIX, "unit": P.SCAN_UNIT}
    a = P.scan_args(rows=rows, width=width, seqs=seqs, dtype=code, form=code_of[form], act=ACT_CODE[act or "none"])
    dev = torch.tensor(starts, dtype=torch.int32, device="cuda")
    if uniform:
        a.length = lens[0] if lens else 0
    else:
        put(a, starts=dev)
    res, oks = {}, []
    for name, ld, m in (("f", "ldf", f), ("x", "ldx", x), ("g", "ldg", gt), ("h0", "ldh0", h0), ("dy", "lddy", dy), ("dh_end", "lddhe", dh_end)):
        if m is not None:
            put(a, **{name: m, ld: m.stride(0)})

    def result(name, r, dt, ld):
        res[name], ok = out(torch, r, width, dt, slack, skip)
        oks.append(ok)
        put(a, **{name: res[name], ld: res[name].stride(0)})
    result("y", rows, tdt, "ldy")
    if in_place:
        put(a, h_end=h0, ldhe=h0.stride(0))
        res["h_end"] = h0
    else:
        result("h_end", seqs, torch.float32, "ldhe")
    kept = h0.clone() if h0_there else None
    ws, ws_ok = given(a, torch, P.scan_workspace(a, False))
    P.scan_forward(a, stream(torch))
    torch.cuda.synchronize()
    mine = slice(front, rows - behind)

    def same(name, v, many):
        r = res[name]
        if many:
            assert bool((r[:front] == 777).all()) and bool((r[rows - behind:] == 777).all()), name
            r, v = r[mine], B.V(v.v[mine], v.e[mine])
        if r.numel():
            B.check(r, v, name)
    same("y", want["y"], True)
    same("h_end", want["h_end"], False)
    ws_ok()
    if in_place:
        put(a, h0=kept, ldh0=kept.stride(0))
    for name, ld in (("df", "lddf"), ("dx", "lddx")) + ((("dg", "lddg"),) if act else ()):
        result(name, rows, tdt, ld)
    if in_place:
        put(a, dh0=dh_end, lddh0=dh_end.stride(0))
        res["dh0"] = dh_end
    else:
        result("dh0", seqs, torch.float32, "lddh0")
    ws, ws_ok = given(a, torch, P.scan_workspace(a, True))
    P.scan_backward(a, stream(torch))
    torch.cuda.synchronize()
    for name in ("df", "dx") + (("dg",) if act else ()):
        same(name, want[name], True)
    same("dh0", want["dh0"], False)
    ws_ok()
    for ok in oks:
        ok()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("form", ["add", "mix", "unit"])
@pytest.mark.parametrize("act", ["", "none", "silu", "gelu", "relu"])
def test_scan_forms(env, dtype, form, act):
    scan_case(env, dtype, [5, 40, 1, 70], 66, form, act)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("lens,width,slack,skip", [([1], 1, 0, 0), ([1], 130, 0, 1), ([31], 64, 0, 0), ([32], 3, 1, 1), ([33], 128, 0, 0), ([64], 127, 0, 0), ([65], 129, 3, 3),
                                                   ([200], 33, 0, 0), ([32, 32, 32], 40, 0, 0), ([31, 1, 32, 1, 31], 40, 2, 1), ([700], 20, 0, 0), ([0, 100, 0, 0, 3, 64, 0], 70, 0, 1),
                                                   ([0], 5, 0, 0), ([0, 0, 0], 64, 0, 0), ([1] * 70, 20, 0, 0), ([2, 0] * 80, 9, 0, 0), ([1100, 7, 900], 6, 0, 0)])
def test_scan_lengths(env, dtype, lens, width, slack, skip):
    scan_case(env, dtype, lens, width, "mix" if width % 2 else "unit", "silu" if len(lens) % 2 else "", slack=slack, skip=skip)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("seqs,length", [(1, 1), (70, 1), (5, 7), (3, 32), (3, 33), (4, 100), (2, 513), (3, 0), (40, 16)])
def test_scan_uniform(env, dtype, seqs, length):
    scan_case(env, dtype, [length] * seqs, 77, "mix", "gelu", uniform=True)


@pytest.mark.parametrize("kw", [dict(behind=5), dict(front=3, behind=70), dict(front=40), dict(h0_there=False, dh_there=False), dict(h0_there=False), dict(dh_there=False), dict(in_place=True),
                                dict(in_place=True, front=2, behind=1)], ids=str)
def test_scan_edges(env, kw):
    for lens in ([40, 0, 3, 100, 1], [300], [2, 3, 4]):
        scan_case(env, "f32", lens, 70, "unit", "silu", **kw)


def test_scan_long_memory(env):
    """factors next to 1 (what is forgotten is far below their last place), factors next to 0, infinite gates"""
    for form in ("add", "mix", "unit"):
        scan_case(env, "f32", [300, 90], 8, form, "", shift=9.0, spread=3.0)
        scan_case(env, "f32", [130], 8, form, "", shift=-20.0, spread=10.0)
    torch, P, B = env
    f = torch.tensor([[math.inf, -math.inf, 200.0, -200.0]] * 70, device="cuda")
    x, h0 = torch.ones(70, 4, device="cuda"), torch.full((1, 4), 3.0, device="cuda")
    y, df = torch.empty(70, 4, device="cuda"), torch.empty(70, 4, device="cuda")
    a = P.scan_args(rows=70, length=70, width=4, seqs=1, dtype=P.F32, form=P.SCAN_UNIT, f=f, ldf=4, x=x, ldx=4, h0=h0, ldh0=4, y=y, ldy=4, dy=x, lddy=4, df=df, lddf=4)
    ws, _ = given(a, torch, max(P.scan_workspace(a), P.scan_workspace(a, True)))
    P.scan_forward(a, stream(torch))
    assert y[-1].tolist() == [3.0, 1.0, 3.0, 1.0]
    P.scan_backward(a, stream(torch))
    assert bool((df == 0).all())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows", [63, 65, 100, 127, 128, 129, 160])
def test_scan_few_rows(env, dtype, rows):
    """up to 128 rows go in one launch: one sequence, several, and h_end and dh0 in their operands' buffers"""
    scan_case(env, dtype, [rows], 130)
    scan_case(env, dtype, [rows // 2, 0, rows - rows // 2 - 9, 5], 67, "unit", "gelu", front=1, behind=3)
    scan_case(env, dtype, [rows - 20, 20], 64, in_place=True)
    scan_case(env, dtype, [rows], 33, "add", "", uniform=True)


@pytest.mark.parametrize("width", [1, 2, 3, 5, 63, 65, 127, 129, 131, 255, 257, 385])
def test_scan_odd_widths(env, width):
    """a last column without a second one: beside others in its wavefront, alone in it, alone altogether; states in their operands' buffers"""
    scan_case(env, "bf16", [40, 0, 3, 90], width, slack=1, in_place=True)
    scan_case(env, "bf16", [1] * 20, width, "unit", "gelu", in_place=True, uniform=True)
    scan_case(env, "bf16", [300, 17], width, "add", "", front=2, behind=1)
    scan_case(env, "bf16", [50, 0, 60], width, "mix", "relu", slack=2, skip=1, in_place=True)


@pytest.mark.parametrize("empty", [0, 61, 62, 63, 64, 65, 130])
@pytest.mark.parametrize("tail", [1, 300])
def test_scan_many_empty_sequences_together(env, empty, tail):
    """around as many starts inside a chunk as a wavefront has lanes, with and without rows behind them"""
    scan_case(env, "f32", [3] + [0] * empty + [1, 0, 20] + [0] * empty + [2, tail], 70, behind=3, front=2)
    scan_case(env, "f32", [0] * empty + [tail] + [0] * empty, 70)


@pytest.mark.parametrize("seqs", [63, 64, 65, 127, 129, 4095, 4097, 9000])
def test_scan_starts_by_count(env, seqs):
    """the search among as many starts as fill its steps, and one more or less"""
    scan_case(env, "f32", [1 + (i % 7 == 3) for i in range(seqs)], 5, front=1)


def test_scan_bad_starts_stay_inside(env):
    """starts that fall or lie outside: undefined results, and nothing else is touched"""
    torch, P, _ = env
    rows, width = 100, 40
    for starts in ([0, 50, 20, 100], [-5, 300, 40, 1000], [100, 0, 100, 0], [-(1 << 31), (1 << 31) - 1, 0, 100]):
        dev = torch.tensor(starts, dtype=torch.int32, device="cuda")
        f, x = (torch.randn(rows, width, device="cuda") for _ in range(2))
        h0 = torch.randn(3, width, device="cuda")
        (y, ok1), (he, ok2), (df, ok3), (dh0, ok4) = out(torch, rows, width, torch.float32), out(torch, 3, width, torch.float32), out(torch, rows, width, torch.float32), out(torch, 3, width, torch.float32)
        a = P.scan_args(rows=rows, width=width, seqs=3, dtype=P.F32, starts=dev, f=f, ldf=width, x=x, ldx=width, h0=h0, ldh0=width, y=y, ldy=width, h_end=he, ldhe=width, dy=x, lddy=width, df=df,
                        lddf=width, dh0=dh0, lddh0=width, dh_end=h0, lddhe=width)
        for back, call in ((False, P.scan_forward), (True, P.scan_backward)):
            ws, ok = given(a, torch, P.scan_workspace(a, back))
            call(a, stream(torch))
            torch.cuda.synchronize()
            ok()
        ok1(), ok2(), ok3(), ok4()


# ---- log probabilities ------------------------------------------------------------------------------------------------------
def logp_case(env, dtype, rows, vocab, k=0, scale=1.0, slack=0, skip=0, ids64=False, logits=None, ids=None, pad_id=-1, dlogp_there=True, dent_there=True, in_place=False):
    torch, P, B = env
    tdt, code = types(P, torch, dtype)
    g = gen_of(torch, rows, vocab, k)
    z = matrix(torch, g, rows, vocab, tdt, 3.0, slack, skip)
    if logits is not None:
        z.copy_(logits)
    if ids is None:
        ids = torch.randint(0, vocab, (rows,), generator=g, device="cuda")
    ids = ids.to(torch.int64 if ids64 else torch.int32)
    dlogp, dent = (torch.randn(rows, generator=g, device="cuda") for _ in range(2))
    want = B.logp(z, scale, ids, pad_id, dlogp if dlogp_there else None, dent if dent_there else None)
    top = B.top(z, k) if k else None
    res = {n: torch.full((rows + 1,), 777.0, device="cuda") for n in ("logp", "entropy", "lse")}
    stats = torch.full((rows + 1, 2), 777.0, device="cuda")
    a = P.logp_args(rows=rows, vocab=vocab, dtype=code, ids64=int(ids64), scale=scale, pad_id=pad_id, logits=z, ldl=z.stride(0), ids=ids, stats=stats, top=k, **res)
    tops = [torch.full((rows + 1, max(k, 1)), -7, dtype=torch.int32, device="cuda"), torch.full((rows + 1, max(k, 1)), 777.0, device="cuda")]
    put(a, top_ids=tops[0], top_logp=tops[1])
    ws, ws_ok = given(a, torch, P.logp_workspace(a))
    P.logp_forward(a, stream(torch))
    torch.cuda.synchronize()
    ws_ok()
    for n, r in res.items():
        assert float(r[rows]) == 777, n
        fin = want[n].v.isfinite()
        got = r[:rows]
        assert torch.equal(got.isnan(), want[n].v.isnan()) and torch.equal(got.isinf(), want[n].v.isinf()), n
        B.check(got[fin], B.V(want[n].v[fin], want[n].e[fin]), n)
    assert bool((stats[rows] == 777).all()) and bool((tops[0][rows] == -7).all())
    if k:
        assert torch.equal(tops[0][:rows], top), (tops[0][:rows] != top).nonzero()[:5].tolist()
        at = top.long().clamp(min=0)
        v, e = want["lp"].v.gather(1, at), want["lp"].e.gather(1, at)
        got = tops[1][:rows]
        assert bool((got[top < 0] == -math.inf).all())
        B.check(got[top >= 0], B.V(v[top >= 0], e[top >= 0]), "top_logp")
    if not (dlogp_there or dent_there):
        return
    dz, dz_ok = out(torch, rows, vocab, tdt, slack, skip)
    if in_place:
        dz, dz_ok = z, lambda: None
    put(a, dlogits=dz, lddl=dz.stride(0), dlogp=dlogp if dlogp_there else 0, dentropy=dent if dent_there else 0)
    P.logp_backward(a, stream(torch))
    torch.cuda.synchronize()
    B.check(dz, want["dlogits"], "dlogits")
    dz_ok()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,vocab,k,slack,skip", [(1, 1, 1, 0, 0), (3, 1, 4, 1, 1), (1, 7, 7, 0, 0), (2, 9, 64, 0, 0), (5, 64, 3, 0, 0), (1, 2048, 5, 0, 0), (1, 2049, 20, 0, 0), (3, 5001, 5, 3, 1),
                                                     (2, 8192, 1, 0, 0), (1, 40000, 64, 0, 0), (2, 33001, 20, 7, 3), (300, 1000, 5, 0, 0), (1300, 333, 4, 0, 1), (1100, 4100, 3, 0, 0), (4, 131072, 50, 0, 0),
                                                     (1, 160001, 8, 0, 1), (1030, 16385, 2, 0, 0)])
def test_logp_sizes(env, dtype, rows, vocab, k, slack, skip):
    logp_case(env, dtype, rows, vocab, k, slack=slack, skip=skip, scale=1.25 if rows % 2 else 1.0, ids64=rows % 2 == 0)


@pytest.mark.parametrize("kw", [dict(dent_there=False), dict(dlogp_there=False), dict(in_place=True), dict(in_place=True, scale=0.3), dict(dent_there=False, dlogp_there=False)], ids=str)
@pytest.mark.parametrize("dtype", DTYPES)
def test_logp_parts(env, dtype, kw):
    logp_case(env, dtype, 37, 700, 3, **kw)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,vocab", [(6, 50), (6, 5000), (1500, 3000)])
def test_logp_masks_and_ties(env, dtype, rows, vocab):
    """rows without a token, with one, of the type's lowest value, all the same; ids that are padding or no token's"""
    torch = env[0]
    z = torch.randn(rows, vocab, device="cuda")
    z[0] = -math.inf
    z[1] = -math.inf
    z[1, vocab // 2] = 2.0
    z[2] = torch.finfo(torch.bfloat16).min
    z[3] = 0.0
    z[3, ::2] = -0.0
    z[4, : vocab // 2] = -math.inf
    z[5] = torch.arange(vocab, device="cuda") // 8 / 64                                    # rising, in ties of eight
    ids = torch.zeros(rows, dtype=torch.int64)
    ids[:6] = torch.tensor([0, vocab // 2, vocab - 1, -1, 0, vocab])
    logp_case(env, dtype, rows, vocab, 20, logits=z, ids=ids.cuda())
    logp_case(env, dtype, rows, vocab, 3, logits=z, ids=(ids - 5).cuda(), pad_id=-6, scale=0.5, ids64=True)


@pytest.mark.parametrize("dtype", DTYPES)
def test_logp_ties_in_many_segments(env, dtype):
    """one value everywhere, and few of them: more candidates than a block keeps, within segments and where they are joined"""
    torch = env[0]
    for vocab in (131072, 50001):
        z = torch.zeros(2, vocab, device="cuda")
        z[1] = (torch.arange(vocab, device="cuda") % 3).float()
        logp_case(env, dtype, 2, vocab, 64, logits=z)


@pytest.mark.parametrize("rows,vocab", [(5, 90), (5, 6000), (1200, 700)])
def test_logp_rows_that_are_not_numbers(env, rows, vocab):
    torch, P, B = env
    z = torch.randn(rows, vocab, device="cuda")
    z[0, 7], z[1, 8], z[2, 9] = math.nan, math.inf, -math.inf
    ids = torch.zeros(rows, dtype=torch.int32, device="cuda")
    o = {n: torch.empty(rows, device="cuda") for n in ("logp", "entropy", "lse")}
    stats, ti, tl = torch.empty(rows, 2, device="cuda"), torch.empty(rows, 3, dtype=torch.int32, device="cuda"), torch.empty(rows, 3, device="cuda")
    dz, one = torch.empty(rows, vocab, device="cuda"), torch.ones(rows, device="cuda")
    a = P.logp_args(rows=rows, vocab=vocab, dtype=P.F32, logits=z, ldl=vocab, ids=ids, stats=stats, top=3, top_ids=ti, top_logp=tl, dlogp=one, dentropy=one, dlogits=dz, lddl=vocab, **o)
    ws, _ = given(a, torch, P.logp_workspace(a))
    P.logp_forward(a, stream(torch))
    P.logp_backward(a, stream(torch))
    torch.cuda.synchronize()
    for r in (*o.values(), tl, dz):
        assert bool(r[:2].isnan().all()) and not bool(r[2:].isnan().any())
    assert torch.equal(ti, B.top(z, 3)) and int(ti[1, 0]) == 8 and 7 not in ti[0].tolist()
