"""Token operators (table lookup, linear layers, gated feed-forward blocks, 8-bit activations) against their formulas in 64 bits, at the sizes
where tiles, vectors and groups end, with strides and offsets of every alignment."""
import pytest

pytestmark = pytest.mark.gpu

ACT_CODE = {"none": 0, "relu": 1, "relu6": 2, "silu": 3, "gelu": 4}
DTYPES = ["f32", "bf16"]


@pytest.fixture(scope="module")
def env():
    import torch
    import paper_2110_02781_amd as P
    import token_ref as R
    return torch, P, R


def types(P, torch, name):
    return (torch.float32, P.F32) if name == "f32" else (torch.bfloat16, P.BF16)


def matrix(torch, gen, rows, cols, dtype, std=1.0, slack=0, skip=0):
    """rows `cols + slack` apart, the first `skip` elements into its buffer"""
    buf = torch.full((skip + rows * (cols + slack) + 8,), float("nan"), device="cuda", dtype=dtype)
    m = buf[skip:skip + rows * (cols + slack)].view(rows, cols + slack)[:, :cols]
    m.copy_(torch.randn(rows, cols, generator=gen, device="cuda") * std)
    return m


def out(torch, rows, cols, dtype, slack=0, skip=0):
    """a result's place in a buffer of sentinels, and a check that nothing else was written"""
    buf = torch.full((skip + rows * (cols + slack) + 64,), 777.0, device="cuda", dtype=dtype)
    m = buf[skip:skip + rows * (cols + slack)].view(rows, cols + slack)
    def untouched():
        assert bool((buf[:skip] == 777).all()) and bool((m[:, cols:] == 777).all()) and bool((buf[skip + rows * (cols + slack):] == 777).all())
    return m[:, :cols], untouched


def space(torch, n):
    return torch.full((max(n, 1) + 256,), 0xA5, dtype=torch.uint8, device="cuda")


def given(a, torch, n):
    """workspace of exactly n bytes: what lies behind must stay"""
    ws = space(torch, n)
    a.ws, a.ws_bytes = ws.data_ptr(), n
    def intact():
        assert bool((ws[n:] == 0xA5).all())
    return ws, intact


# rows, n_in, n_out, slack, skip: one element to several tiles, reductions off the step and the vector, few rows and the first number past them, split
# reductions, the large tile
LINEAR = [(1, 1, 1, 0, 0), (1, 64, 16, 0, 0), (2, 7, 3, 1, 1), (16, 129, 33, 0, 0), (17, 129, 33, 0, 3), (5, 4104, 40, 8, 0), (33, 4097, 21, 0, 0),
          (130, 64, 128, 0, 0), (129, 200, 130, 5, 0), (300, 331, 203, 0, 1), (64, 72, 520, 8, 8)]
BIG = [(4090, 4088, 4072, 0, 0), (4095, 4089, 4001, 8, 1)]


def linear_case(env, dtype, act, rows, k, n, slack, skip, bias=True, res=True, grad=None, accumulate=0, x8=False, seed=1):
    torch, P, R = env
    tdt, code = types(P, torch, dtype)
    gen = torch.Generator(device="cuda").manual_seed(seed + rows * 7 + k * 3 + n)
    x, w = matrix(torch, gen, rows, k, tdt, 1.0, slack, skip), matrix(torch, gen, n, k, tdt, k ** -0.5, slack, skip)
    b = torch.randn(n, generator=gen, device="cuda") if bias else None
    r = matrix(torch, gen, rows, n, tdt, 1.0, slack, skip) if res else None
    y, y_ok = out(torch, rows, n, tdt, slack, skip)
    z, z_ok = out(torch, rows, n, tdt, slack, skip)
    sp = torch.cuda.current_stream().cuda_stream
    a = P.linear_args(rows=rows, n_in=k, n_out=n, dtype=code, act=ACT_CODE[act], x=x, ldx=x.stride(0), w=w, ldw=w.stride(0), bias=0 if b is None else b,
                      residual=0 if r is None else r, ldr=0 if r is None else r.stride(0), y=y, ldy=y.stride(0), z=z, ldz=z.stride(0))
    xv = R.f64(x)
    if x8:
        q, s = R.act8_encode(x)
        xv = R.act8_decode(q, s)
        a.x, a.ldx, a.x_scales, a.ldxs = q.data_ptr(), k, s.data_ptr(), s.shape[1]
    ws, ws_ok = given(a, torch, P.linear_workspace(a))
    P.linear_forward(a, sp)
    torch.cuda.synchronize()
    zx, ez = R.product(xv, R.f64(w))
    if bias:
        zx, ez = zx + b.double(), ez + R.U * (zx.abs() + b.double().abs())
    v, _, t = R.act(zx, act)
    e = R.act_err(v, t, ez)
    if res:
        e = e + R.U * (v.abs() + R.f64(r).abs())
        v = v + R.f64(r)
    R.close(z, zx, R.stored(zx, ez, tdt), "z")
    R.close(y, v, R.stored(v, e, tdt), "y")
    for ok in (y_ok, z_ok, ws_ok):
        ok()
    # backward, of the z that was kept
    gname = grad or dtype
    gdt, gcode = types(P, torch, gname)
    dy = matrix(torch, gen, rows, n, tdt, 1.0, slack, skip)
    dx, dx_ok = out(torch, rows, k, tdt, slack, skip)
    dw, dw_ok = out(torch, n, k, gdt, 0, skip)
    db, db_ok = out(torch, 1, n, gdt, 0, skip)
    if accumulate:
        dw.fill_(0.5)
        db.fill_(-0.25)
    a.dy, a.lddy, a.dx, a.lddx, a.dw, a.dbias = dy.data_ptr(), dy.stride(0), dx.data_ptr(), dx.stride(0), dw.data_ptr(), db.data_ptr()
    a.grad_dtype, a.accumulate = gcode, accumulate
    ws, ws_ok = given(a, torch, P.linear_workspace(a, True))
    P.linear_backward(a, sp)
    torch.cuda.synchronize()
    zk = R.f64(z)
    _, d, t = R.act(zk, act)
    g = R.f64(dy) * d
    eg = R.f64(dy).abs() * R.dact_err(zk, t) + R.U * g.abs() if act != "none" else torch.zeros_like(g)
    dbx, eb = g.sum(0)[None], (eg.sum(0) + (rows + 8) * R.U * g.abs().sum(0))[None]
    if act != "none":
        eg = R.stored(g, eg, tdt)
    dxx, ex = R.product(g, R.f64(w).t(), eg)
    dwx, ew = R.product(g.t(), xv.t(), eg.t())
    if accumulate:
        dwx, ew, dbx, eb = dwx + 0.5, ew + R.U * (dwx.abs() + 0.5), dbx - 0.25, eb + R.U * (dbx.abs() + 0.25)
    R.close(dx, dxx, R.stored(dxx, ex, tdt), "dx")
    R.close(dw, dwx, R.stored(dwx, ew, gdt), "dw")
    R.close(db, dbx, R.stored(dbx, eb, gdt), "db")
    for ok in (dx_ok, dw_ok, db_ok, ws_ok):
        ok()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,k,n,slack,skip", LINEAR)
def test_linear(env, dtype, rows, k, n, slack, skip):
    linear_case(env, dtype, "gelu", rows, k, n, slack, skip)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("act", ["none", "relu", "relu6", "silu"])
def test_linear_activations(env, dtype, act):
    for rows in (9, 70):
        linear_case(env, dtype, act, rows, 96, 77, 0, 0, bias=act != "none", res=act != "relu")


class routes:
    """the tiles that the products inside took, by family: {"tok_linear": {"256", ...}, ...}"""

    def __init__(self, P):
        self.P, self.took = P, {}

    def __enter__(self):
        self.P.ktrace_begin(-512)
        return self.took

    def __exit__(self, *_):
        for r in self.P.ktrace_end():
            if r["name"].startswith("__route "):
                tile, rest = r["name"][8:].split(" tok_")
                self.took.setdefault("tok_" + rest.split()[0], set()).add(tile)


@pytest.mark.parametrize("rows,k,n,slack,skip", BIG)
def test_linear_large_tile(env, rows, k, n, slack, skip):
    with routes(env[1]) as took:
        linear_case(env, "bf16", "silu", rows, k, n, slack, skip)
    assert took == {"tok_linear": {"256"}, "tok_wgrad": {"256"}}, took


# rows of whole vectors that start on 4 bytes but not on 16: read as they lie, in every product and tile
FOUR = [("bf16", 130, 136, 264, 2, 2), ("bf16", 300, 328, 200, 6, 4), ("bf16", 70, 4096, 40, 2, 6), ("f32", 130, 132, 260, 1, 1), ("f32", 301, 332, 204, 3, 2),
        ("f32", 70, 2048, 40, 5, 3), ("bf16", 33, 64, 8, 2, 2)]


@pytest.mark.parametrize("dtype,rows,k,n,slack,skip", FOUR)
def test_rows_on_four_bytes(env, dtype, rows, k, n, slack, skip):
    linear_case(env, dtype, "silu", rows, k, n, slack, skip)
    ffn_case(env, dtype, "silu", 1, rows, k, n, slack, skip)


@pytest.mark.parametrize("slack,skip", [(2, 2), (6, 4)])
def test_rows_on_four_bytes_large_tile(env, slack, skip):
    with routes(env[1]) as took:
        linear_case(env, "bf16", "silu", 4090, 4088, 4072, slack, skip)
        ffn_case(env, "bf16", "silu", 2, 4090, 4088, 4096, slack, skip)
    assert took == {k: {"256"} for k in ("tok_glu", "tok_glu_bwd", "tok_linear", "tok_wgrad")}, took


@pytest.mark.parametrize("act", ["none", "relu", "relu6", "silu", "gelu"])
@pytest.mark.parametrize("rows,n", [(4360, 4104), (4410, 4132), (4500, 4100)])
def test_large_tile_epilogues(env, act, rows, n):
    """Every activation behind whole large tiles, with and without bias and residual, both stashes; the last tiles have rows, fours of columns and groups of 32 outside."""
    for bias, res in ((True, True), (True, False), (False, True), (False, False)):
        with routes(env[1]) as took:
            linear_case(env, "bf16", act, rows, 72, n, 0, 0, bias=bias, res=res)
        assert "256" in took["tok_linear"], took
    for save in (0, 1, 2):
        with routes(env[1]) as took:
            ffn_case(env, "bf16", act, save, rows, 72, n, 0, 0)
        assert "256" in took["tok_glu"] and (save == 0 or "256" in took["tok_glu_bwd"]), took


@pytest.mark.parametrize("accumulate", [0, 1])
def test_linear_fp32_gradients(env, accumulate):
    linear_case(env, "bf16", "none", 200, 120, 90, 0, 0, grad="f32", accumulate=accumulate)
    linear_case(env, "f32", "silu", 41, 64, 90, 3, 0, accumulate=accumulate)
    linear_case(env, "bf16", "gelu", 3000, 40, 24, 0, 0, grad="f32", accumulate=accumulate)      # rows split over blocks


@pytest.mark.parametrize("dtype", DTYPES)
def test_linear_input_in_8_bits(env, dtype):
    linear_case(env, dtype, "silu", 37, 100, 64, 0, 0, x8=True)
    linear_case(env, dtype, "none", 12, 64, 33, 0, 0, x8=True)


# rows, width, hidden, slack, skip
FFN = [(1, 1, 1, 0, 0), (1, 128, 64, 0, 0), (3, 65, 31, 1, 1), (16, 128, 100, 0, 0), (17, 96, 33, 0, 0), (40, 131, 261, 3, 1), (130, 64, 128, 0, 0),
       (300, 72, 200, 8, 0)]


def ffn_case(env, dtype, act, save, rows, d, f, slack, skip, grad=None, accumulate=0, x8=False, dx_residual=1, min_scale=1.0):
    torch, P, R = env
    tdt, code = types(P, torch, dtype)
    gen = torch.Generator(device="cuda").manual_seed(rows * 5 + d * 3 + f)
    x = matrix(torch, gen, rows, d, tdt, 1.0, slack, skip)
    wg, wu = (matrix(torch, gen, f, d, tdt, d ** -0.5, slack, skip) for _ in range(2))
    wd = matrix(torch, gen, d, f, tdt, f ** -0.5, slack, skip)
    y, y_ok = out(torch, rows, d, tdt, slack, skip)
    sp = torch.cuda.current_stream().cuda_stream
    a = P.ffn_args(rows=rows, width=d, hidden=f, dtype=code, act=ACT_CODE[act], x=x, ldx=x.stride(0), w_gate=wg, ldwg=wg.stride(0), w_up=wu,
                   ldwu=wu.stride(0), w_down=wd, ldwd=wd.stride(0), residual=x, ldr=x.stride(0), y=y, ldy=y.stride(0))
    xv = R.f64(x)
    if x8:
        q, s = R.act8_encode(x)
        xv = R.act8_decode(q, s)
        a.x, a.ldx, a.x_scales, a.ldxs = q.data_ptr(), d, s.data_ptr(), s.shape[1]
    G = -(-f // 32)
    if save == P.SAVE_ACT8:
        kg, ku = (torch.full((rows, f), 0x55, dtype=torch.uint8, device="cuda") for _ in range(2))
        sg, su = (torch.full((rows, G), 0x55, dtype=torch.uint8, device="cuda") for _ in range(2))
        a.gate_scales, a.up_scales = sg.data_ptr(), su.data_ptr()
    else:
        kg, ku = (torch.full((rows, f), 777.0, dtype=tdt, device="cuda") for _ in range(2))
    a.save, a.gate, a.up = save, kg.data_ptr(), ku.data_ptr()
    ws, ws_ok = given(a, torch, P.ffn_workspace(a))
    P.ffn_forward(a, sp)
    torch.cuda.synchronize()
    g, eg = R.product(xv, R.f64(wg))
    u, eu = R.product(xv, R.f64(wu))
    v, _, t = R.act(g, act)
    ev = R.act_err(v, t, eg)
    h, eh = v * u, u.abs() * ev + (v.abs() + ev) * eu + R.U * (v * u).abs()
    eh = R.stored(h, eh, tdt)
    want, e = R.product(h, R.f64(wd), eh)
    e = e + R.U * (want.abs() + R.f64(x).abs())
    want = want + R.f64(x)
    R.close(y, want, R.stored(want, e, tdt), "y")
    y_ok()
    ws_ok()
    for name, k, s, val, err in (("gate", kg, sg if save == P.SAVE_ACT8 else None, g, eg), ("up", ku, su if save == P.SAVE_ACT8 else None, u, eu)):
        if save == P.SAVE_FULL:
            R.close(k, val, R.stored(val, err, tdt), name)
        elif save == P.SAVE_ACT8:
            # the group's scale is the exact maximum's, or the next where that is within the error of a border; half a step of 2^-4 or 2^-10 scales
            lo = R.act8_scales((val.abs() - err).clamp(min=0))
            hi = R.act8_scales(val.abs() + err)
            got = s.double() - 127
            assert bool((got >= lo).all()) and bool((got <= hi).all()), name
            half = torch.exp2(hi).repeat_interleave(32, 1)[:, :f] * 2.0 ** -10
            R.close(R.act8_decode(k, s), val, err + torch.maximum(2.0 ** -4 * (val.abs() + err), half), name)
    if save == P.SAVE_NONE:
        return
    # backward, of what was kept
    kept = [R.act8_decode(k, s) if save == P.SAVE_ACT8 else R.f64(k) for k, s in ((kg, sg if save == P.SAVE_ACT8 else None), (ku, su if save == P.SAVE_ACT8 else None))]
    gname = grad or dtype
    gdt, gcode = types(P, torch, gname)
    dy = matrix(torch, gen, rows, d, tdt, 1.0, slack, skip)
    dx, dx_ok = out(torch, rows, d, tdt, slack, skip)
    grads = [out(torch, n, m, gdt, 0, skip) for n, m in ((f, d), (f, d), (d, f))]
    if accumulate:
        for m, _ in grads:
            m.fill_(0.5)
    a.dy, a.lddy, a.dx, a.lddx = dy.data_ptr(), dy.stride(0), dx.data_ptr(), dx.stride(0)
    a.dw_gate, a.dw_up, a.dw_down = (m.data_ptr() for m, _ in grads)
    a.grad_dtype, a.accumulate, a.dx_residual = gcode, accumulate, dx_residual
    ws, ws_ok = given(a, torch, P.ffn_workspace(a, True))
    P.ffn_backward(a, sp)
    torch.cuda.synchronize()
    g, u = kept
    dyv = R.f64(dy)
    dh, edh = R.product(dyv, R.f64(wd).t())
    v, dv, t = R.act(g, act)
    edv, ev = R.dact_err(g, t), R.act_err(v, t, torch.zeros_like(g))
    dg, du, h = dh * u * dv, dh * v, v * u
    edg = R.stored(dg, (u * dv).abs() * edh + (dh.abs() + edh) * u.abs() * edv + 2 * R.U * dg.abs(), tdt)
    edu = R.stored(du, v.abs() * edh + (dh.abs() + edh) * ev + R.U * du.abs(), tdt)
    eh = R.stored(h, u.abs() * ev + R.U * h.abs(), tdt)
    d1, e1 = R.product(dg, R.f64(wg).t(), edg)
    d2, e2 = R.product(du, R.f64(wu).t(), edu)
    dxx, ex = d1 + d2, e1 + e2 + 2 * R.U * (d1.abs() + d2.abs())
    if dx_residual:
        dxx, ex = dxx + dyv, ex + R.U * (dxx.abs() + dyv.abs())
    R.close(dx, dxx, R.stored(dxx, ex, tdt), "dx")
    for (m, ok), (left, el, right, er), name in zip(grads, ((dg, edg, xv, None), (du, edu, xv, None), (dyv, torch.zeros_like(dyv), h, eh)), ("dwg", "dwu", "dwd")):
        w, ew = R.product(left.t(), right.t(), el.t(), er.t() if er is not None else None)
        if er is not None:
            ew = ew + el.t() @ er
        if accumulate:
            w, ew = w + 0.5, ew + R.U * (w.abs() + 0.5)
        R.close(m, w, R.stored(w, ew, gdt), name)
        ok()
    dx_ok()
    ws_ok()


@pytest.mark.parametrize("save", [1, 2])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,d,f,slack,skip", FFN)
def test_ffn(env, dtype, save, rows, d, f, slack, skip):
    ffn_case(env, dtype, "silu", save, rows, d, f, slack, skip)


@pytest.mark.parametrize("act", ["none", "relu", "relu6", "gelu"])
def test_ffn_activations(env, act):
    for dtype in DTYPES:
        ffn_case(env, dtype, act, 1, 20, 64, 72, 0, 0)
        ffn_case(env, dtype, act, 0, 7, 64, 72, 0, 0)


@pytest.mark.parametrize("save,rows,d,f", [(1, 4090, 4088, 4090), (2, 4095, 4089, 4064)])
def test_ffn_large_tile(env, save, rows, d, f):
    with routes(env[1]) as took:
        ffn_case(env, "bf16", "silu", save, rows, d, f, 0, 0)
    assert took == {k: {"256"} for k in ("tok_glu", "tok_glu_bwd", "tok_linear", "tok_wgrad")}, took


def test_ffn_split_reduction(env):
    ffn_case(env, "bf16", "gelu", 2, 24, 4100, 40, 0, 0)
    ffn_case(env, "f32", "silu", 1, 24, 40, 4100, 0, 0)
    ffn_case(env, "bf16", "silu", 2, 5, 2048, 64, 0, 0)


def test_few_rows_and_many_weights(env):
    """From nine rows on, aligned weights of 40 MB and more go through a tile; fewer, and those of odd rows, are streamed."""
    torch, P, R = env
    for rows, k, n in ((8, 4608, 4608), (9, 4608, 4608), (16, 4608, 4608), (16, 4608, 4000), (16, 4607, 4608)):
        linear_case(env, "bf16", "none", rows, k, n, 0, 0)
    ffn_case(env, "bf16", "silu", 1, 12, 2048, 5632, 0, 0)
    ffn_case(env, "bf16", "silu", 1, 12, 2047, 5631, 0, 0)


def test_ffn_options(env):
    ffn_case(env, "bf16", "silu", 2, 90, 64, 100, 0, 0, grad="f32", accumulate=1, dx_residual=0)
    ffn_case(env, "f32", "silu", 1, 90, 64, 100, 0, 0, accumulate=1)
    ffn_case(env, "bf16", "silu", 2, 33, 100, 64, 0, 0, x8=True)


@pytest.mark.parametrize("dtype", DTYPES)
def test_rows_do_not_mix(env, dtype):
    """An infinity and a NaN in one row leave the others' bits alone, whatever shares their tile; rows past the last are not read as values."""
    torch, P, R = env
    tdt, code = types(P, torch, dtype)
    sp = torch.cuda.current_stream().cuda_stream
    for rows, k, n in ((9, 72, 40), (40, 72, 140)):
        gen = torch.Generator(device="cuda").manual_seed(3)
        x, w = matrix(torch, gen, rows, k, tdt, 1.0, 1, 1), matrix(torch, gen, n, k, tdt, 0.1, 0, 0)
        ys = []
        for bad in (False, True):
            xx = x.clone() if not bad else x.clone().index_put_((torch.tensor([2, 5]).cuda(), torch.tensor([3, 71]).cuda()), torch.tensor([float("inf"), float("nan")], device="cuda", dtype=tdt))
            y = torch.empty(rows, n, dtype=tdt, device="cuda")
            a = P.linear_args(rows=rows, n_in=k, n_out=n, dtype=code, act=P.ACT_SILU, x=xx, ldx=xx.stride(0), w=w, ldw=k, y=y, ldy=n)
            ws, _ = given(a, torch, P.linear_workspace(a))
            P.linear_forward(a, sp)
            torch.cuda.synchronize()
            ys.append(y)
        keep = [r for r in range(rows) if r not in (2, 5)]
        assert torch.equal(ys[0][keep], ys[1][keep]) and bool(ys[1][5].isnan().all()) and not bool(ys[1][2].isfinite().all())


# ---- table lookup -------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("ids64", [0, 1])
def test_embed_forward(env, dtype, ids64):
    torch, P, R = env
    tdt, code = types(P, torch, dtype)
    gen = torch.Generator(device="cuda").manual_seed(5)
    for rows, vocab, width, slack, skip in ((1, 1, 1, 0, 0), (5, 10, 8, 0, 0), (37, 100, 77, 3, 1), (300, 50, 2056, 0, 0)):
        table = matrix(torch, gen, vocab, width, tdt, 1.0, slack, skip)
        ids = torch.randint(0, vocab, (rows,), generator=gen, device="cuda").to(torch.int64 if ids64 else torch.int32)
        if rows > 3:
            ids[1], ids[2] = -1, vocab
            if ids64:
                ids[3] = (1 << 32) + 1
        o, ok = out(torch, rows, width, tdt, slack, skip)
        a = P.embed_args(rows=rows, vocab=vocab, width=width, dtype=code, ids64=ids64, scale=1.5, ids=ids, table=table, ldt=table.stride(0), out=o, ldo=o.stride(0))
        P.embed_forward(a, torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        valid = (ids >= 0) & (ids < vocab)
        assert bool(o[~valid].isnan().all())
        want = R.f64(table)[ids[valid].long()] * 1.5
        R.close(o[valid], want, R.HALF[tdt] * want.abs(), "out")
        ok()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("accumulate", [0, 1])
def test_embed_backward(env, dtype, accumulate):
    """Counting in chunks, merging them, the passes of the sort, runs of one id over several blocks, ids of no row, an id left out; ids of either width."""
    torch, P, R = env
    tdt, code = types(P, torch, dtype)
    sp = torch.cuda.current_stream().cuda_stream
    for rows, vocab, width, kind in ((1, 3, 1, "any"), (63, 7, 9, "any"), (64, 500, 8, "any"), (65, 1, 16, "any"), (1000, 40, 101, "bad"), (700, 9, 2057, "one"),
                                     (8192, 5000, 8, "any"), (8193, 255, 8, "bad"), (16384, 5000, 8, "any"), (16385, 255, 8, "bad"), (20000, 256, 9, "any"), (30000, 70000, 8, "bad"), (20000, 3, 8, "one"), (73737, 70000, 8, "bad"),
                                     (65536, 300, 8, "any"), (65537, 255, 8, "bad"), (140000, 70000, 9, "any"), (150000, 256, 8, "one")):
        print(f"embed backward {dtype} {rows} {vocab} {width} {kind}", flush=True)
        gen = torch.Generator(device="cuda").manual_seed(rows)
        ids = torch.randint(0, vocab, (rows,), generator=gen, device="cuda")
        if kind == "one":
            ids[:] = vocab - 1
        pad = 1 if kind == "bad" else -1
        if kind == "bad":
            ids[::5] = vocab + 3
            ids[3::7] = -4
            ids[2::11] = pad
        ids64 = rows % 2
        if not ids64:
            ids = ids.to(torch.int32)
        dy = matrix(torch, gen, rows, width, tdt, 1.0, 3, 1)
        g, ok = out(torch, vocab, width, torch.float32, 2, 1)
        if accumulate:
            g.fill_(0.5)
        a = P.embed_args(rows=rows, vocab=vocab, width=width, dtype=code, ids64=ids64, scale=0.75, pad_id=pad, accumulate=accumulate, ids=ids, dy=dy, lddy=dy.stride(0),
                         dtable=g, lddt=g.stride(0))
        ws, ws_ok = given(a, torch, P.embed_backward_workspace(a))
        P.embed_backward(a, sp)
        torch.cuda.synchronize()
        ok()
        ws_ok()
        use = (ids >= 0) & (ids < vocab) & (ids != pad)
        # on the host: thousands of 64-bit additions to one row take the GPU's atomics seconds
        at, rows_of = ids[use].long().cpu(), R.f64(dy)[use].cpu()
        want = torch.zeros(vocab, width, dtype=torch.float64).index_add_(0, at, rows_of).cuda()
        mag = torch.zeros(vocab, width, dtype=torch.float64).index_add_(0, at, rows_of.abs()).cuda()
        many = torch.bincount(at, minlength=vocab).double().cuda()
        want, bound = want * 0.75 + 0.5 * accumulate, ((many[:, None] + 2) * mag * 0.75 + 0.5 * accumulate) * R.U + R.U * want.abs()
        R.close(g, want, bound, "dtable")
        if not accumulate:
            again = torch.empty(vocab, width, device="cuda")
            a.dtable, a.lddt = again.data_ptr(), width
            P.embed_backward(a, sp)
            torch.cuda.synchronize()
            assert torch.equal(again, g)


@pytest.mark.parametrize("rows,vocab,width", [(1, 5000, 1), (40, 5000, 1), (300, 200, 2100), (3, 40, 70000), (9000, 3000, 7), (70000, 3000, 3), (64, 64, 1024),
                                              (500, 1025, 64), (4097, 4096, 33)])
def test_embed_backward_rows_without_tokens(env, rows, vocab, width):
    """Whole numbers, so that sums are exact: rows with tokens hold their sum, all others zeros, whatever the gradient held."""
    torch, P, R = env
    sp = torch.cuda.current_stream().cuda_stream
    gen = torch.Generator(device="cuda").manual_seed(rows)
    for kind in range(4):
        print(f"rows without tokens {rows} {vocab} {width} {kind}", flush=True)
        ids = torch.randint(0, vocab, (rows,), generator=gen, device="cuda")
        if kind == 1:
            ids = ids // 2                                       # none in the upper half
        elif kind == 2:
            ids = ids * 0 + (vocab - 1)
        elif kind == 3:
            ids = ids * 0 + vocab                                # none at all
        dy = torch.randint(-4, 5, (rows, width), generator=gen, device="cuda").to(torch.bfloat16)
        g, ok = out(torch, vocab, width, torch.float32, 3, 1)
        a = P.embed_args(rows=rows, vocab=vocab, width=width, dtype=P.BF16, ids64=1, scale=1.0, pad_id=-1, ids=ids, dy=dy, lddy=width, dtable=g, lddt=g.stride(0))
        ws, ws_ok = given(a, torch, P.embed_backward_workspace(a))
        P.embed_backward(a, sp)
        torch.cuda.synchronize()
        ok()
        ws_ok()
        use = ids < vocab
        want = torch.zeros(vocab, width).index_add_(0, ids[use].cpu(), dy[use].cpu().float())
        assert torch.equal(g.cpu(), want)


# ---- 8 bits ----------------------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", DTYPES)
def test_act8(env, dtype):
    """Bytes and values by the definition, exactly."""
    torch, P, R = env
    tdt, code = types(P, torch, dtype)
    sp = torch.cuda.current_stream().cuda_stream
    for rows, cols, slack, skip in ((1, 1, 0, 0), (2, 32, 0, 0), (3, 31, 1, 1), (5, 33, 0, 0), (7, 64, 8, 0), (33, 101, 3, 1), (200, 257, 0, 0)):
        gen = torch.Generator(device="cuda").manual_seed(cols)
        x = matrix(torch, gen, rows, cols, tdt, 1.0, slack, skip)
        x.mul_(torch.exp2(torch.randint(-20, 20, (rows, cols), generator=gen, device="cuda").float()).to(tdt))
        if rows > 2:
            x[0] = 0                                             # an empty group, and everything a group can hold that is not a number
            x[1, 0], x[2, 0] = float("inf"), float("nan")
            x[1, 1:] = 448.0 if cols == 64 else 449.0
        if rows > 6:
            x[3] = 1e-39                                         # below what any scale reaches
            x[4] = torch.finfo(tdt).max
            x[5, ::3] = -0.0
            x[6] = torch.finfo(tdt).tiny
        q, s = torch.full((rows, cols + slack), 0x55, dtype=torch.uint8, device="cuda"), torch.full((rows, -(-cols // 32) + 1), 0x55, dtype=torch.uint8, device="cuda")
        y, ok = out(torch, rows, cols, tdt, slack, skip)
        a = P.act8_args(rows=rows, cols=cols, dtype=code, x=x, ldx=x.stride(0), q=q, ldq=cols + slack, scales=s, lds=s.shape[1], y=y, ldy=y.stride(0))
        P.act8_pack(a, sp)
        P.act8_unpack(a, sp)
        torch.cuda.synchronize()
        ok()
        assert bool((q[:, cols:] == 0x55).all()) and bool((s[:, -1] == 0x55).all())
        val, e = R.act8(x)
        assert torch.equal(s[:, :-1].double() - 127, e)
        got = R.act8_decode(q[:, :cols], s[:, :-1])
        assert torch.equal(got.nan_to_num(9e9), val.nan_to_num(9e9))
        assert torch.equal(y.nan_to_num(9e9), val.to(tdt).nan_to_num(9e9))
        assert torch.equal(y.isnan(), ~x.isfinite())


# ---- as a program uses them --------------------------------------------------------------------------------------------------------------
def test_gradients_against_differences(env):
    """fp32 blocks and layers: the loss's change along a direction, by central differences with steps of 2^-6.  The loss's own rounding is below 2^-18 of the
    sum of its terms' magnitudes, a difference divides it by 2^-5; the third-order term of a direction of norm 1 is below 2^-12 of the same."""
    torch, P, R = env
    sp = torch.cuda.current_stream().cuda_stream
    rows, d, f = 20, 48, 72
    gen = torch.Generator(device="cuda").manual_seed(11)
    x, wg, wu, wd = (matrix(torch, gen, n, m, torch.float32, s) for n, m, s in ((rows, d, 1.0), (f, d, d ** -0.5), (f, d, d ** -0.5), (d, f, f ** -0.5)))
    dy = matrix(torch, gen, rows, d, torch.float32)
    bufs = dict(x=x, wg=wg, wu=wu, wd=wd)
    grads = {k: torch.empty(v.shape, device="cuda") for k, v in bufs.items()}
    keep = [torch.empty(rows, f, device="cuda") for _ in range(2)]
    y = torch.empty(rows, d, device="cuda")

    def record(b):
        a = P.ffn_args(rows=rows, width=d, hidden=f, dtype=P.F32, act=P.ACT_GELU, save=P.SAVE_FULL, gate=keep[0], up=keep[1], x=b["x"], ldx=b["x"].stride(0),
                       w_gate=b["wg"], ldwg=d, w_up=b["wu"], ldwu=d, w_down=b["wd"], ldwd=f, residual=b["x"], ldr=b["x"].stride(0), y=y, ldy=d)
        ws = space(torch, P.ffn_workspace(a))
        a.ws, a.ws_bytes = ws.data_ptr(), ws.numel()
        return a, ws

    def loss(b):
        a, ws = record(b)
        P.ffn_forward(a, sp)
        torch.cuda.synchronize()
        return float((y.double() * dy.double()).sum()), float((y.double() * dy.double()).abs().sum())

    loss(bufs)
    a, ws = record(bufs)
    a.dy, a.lddy, a.dx, a.lddx, a.dx_residual = dy.data_ptr(), d, grads["x"].data_ptr(), d, 1
    a.dw_gate, a.dw_up, a.dw_down = (grads[k].data_ptr() for k in ("wg", "wu", "wd"))
    ws2 = space(torch, P.ffn_workspace(a, True))
    a.ws, a.ws_bytes = ws2.data_ptr(), ws2.numel()
    P.ffn_backward(a, sp)
    torch.cuda.synchronize()
    for k, v in bufs.items():
        way = torch.randn(v.shape, generator=gen, device="cuda")
        way = way / way.norm()
        h = 2.0 ** -6
        up, mag = loss({**bufs, k: (v + h * way).contiguous()})
        down, _ = loss({**bufs, k: (v - h * way).contiguous()})
        want = float((grads[k].double() * way.double()).sum())
        assert abs((up - down) / (2 * h) - want) <= (2.0 ** -13 + 2.0 ** -12) * mag, (k, (up - down) / (2 * h), want, mag)


def test_streams_and_graphs(env):
    """A training step of a block on a stream of its own, then captured: every replay gives the eager call's bits."""
    torch, P, R = env
    rows, d, f = 70, 136, 200
    gen = torch.Generator(device="cuda").manual_seed(2)
    bf = torch.bfloat16
    x, wg, wu, wd, dy = (matrix(torch, gen, n, m, bf, s, 1) for n, m, s in ((rows, d, 1.0), (f, d, 0.1), (f, d, 0.1), (d, f, 0.1), (rows, d, 1.0)))
    ids = torch.randint(0, 50, (rows,), generator=gen, device="cuda").to(torch.int32)
    outs = dict(y=torch.empty(rows, d, dtype=bf, device="cuda"), dx=torch.empty(rows, d, dtype=bf, device="cuda"), dg=torch.empty(f, d, device="cuda"),
                du=torch.empty(f, d, device="cuda"), dd=torch.empty(d, f, device="cuda"), dt=torch.empty(50, d, device="cuda"))
    keep = [torch.empty(rows, f, dtype=torch.uint8, device="cuda") for _ in range(2)] + [torch.empty(rows, -(-f // 32), dtype=torch.uint8, device="cuda") for _ in range(2)]
    a = P.ffn_args(rows=rows, width=d, hidden=f, dtype=P.BF16, act=P.ACT_SILU, save=P.SAVE_ACT8, gate=keep[0], up=keep[1], gate_scales=keep[2], up_scales=keep[3],
                   x=x, ldx=x.stride(0), w_gate=wg, ldwg=wg.stride(0), w_up=wu, ldwu=wu.stride(0), w_down=wd, ldwd=wd.stride(0), residual=x, ldr=x.stride(0),
                   y=outs["y"], ldy=d, dy=dy, lddy=dy.stride(0), dx=outs["dx"], lddx=d, dx_residual=1, dw_gate=outs["dg"], dw_up=outs["du"], dw_down=outs["dd"])
    e = P.embed_args(rows=rows, vocab=50, width=d, dtype=P.BF16, scale=2.0, ids=ids, dy=outs["dx"], lddy=d, dtable=outs["dt"], lddt=d)
    ws = [space(torch, max(P.ffn_workspace(a), P.ffn_workspace(a, True))), space(torch, P.embed_backward_workspace(e))]
    a.ws, a.ws_bytes, e.ws, e.ws_bytes = ws[0].data_ptr(), ws[0].numel(), ws[1].data_ptr(), ws[1].numel()

    def step(sp):
        P.ffn_forward(a, sp)
        P.ffn_backward(a, sp)
        P.embed_backward(e, sp)

    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    step(s.cuda_stream)
    torch.cuda.synchronize()
    first = {k: v.clone() for k, v in outs.items()}
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        step(s.cuda_stream)
    for i in range(4):
        for v in outs.values():
            v.fill_(3.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(first[k], outs[k]) for k in outs), i
        for v in outs.values():
            v.fill_(3.0)
        step(torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        assert all(torch.equal(first[k], outs[k]) for k in outs), i


def test_no_rows(env):
    """A batch without tokens: forwards do nothing, gradients are zero, or stay what they were when they accumulate."""
    torch, P, R = env
    sp = torch.cuda.current_stream().cuda_stream
    w = torch.ones(24, 16, device="cuda")
    for accumulate in (0, 1):
        dw, db, dt = torch.full((24, 16), 5.0, device="cuda"), torch.full((24,), 5.0, device="cuda"), torch.full((9, 16), 5.0, device="cuda")
        g = [torch.full(s, 5.0, device="cuda") for s in ((24, 16), (24, 16), (16, 24))]
        a = P.linear_args(rows=0, n_in=16, n_out=24, dtype=P.F32, w=w, ldw=16, dw=dw, dbias=db, accumulate=accumulate)
        assert P.linear_workspace(a) == 0
        P.linear_forward(a, sp)
        P.linear_backward(a, sp)
        f = P.ffn_args(rows=0, width=16, hidden=24, dtype=P.F32, act=P.ACT_SILU, save=P.SAVE_FULL, w_gate=w, ldwg=16, w_up=w, ldwu=16, w_down=w, ldwd=24, dw_gate=g[0],
                       dw_up=g[1], dw_down=g[2], accumulate=accumulate)
        P.ffn_forward(f, sp)
        P.ffn_backward(f, sp)
        e = P.embed_args(rows=0, vocab=9, width=16, dtype=P.F32, table=w, ldt=16, dtable=dt, lddt=16, accumulate=accumulate)
        P.embed_forward(e, sp)
        P.embed_backward(e, sp)
        P.act8_pack(P.act8_args(rows=0, cols=16, ldx=16, ldq=16, lds=1), sp)
        torch.cuda.synchronize()
        for t in (dw, db, dt, *g):
            assert bool((t == (5.0 if accumulate else 0.0)).all())
