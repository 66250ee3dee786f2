"""Gated feed-forward blocks and linear layers in forms that every operand has to itself: each matrix at its own row distance and offset, inputs in 8 bits
at any byte, infinities beside pad columns, calls without rows, the longest ones.  Against the formulas in 64 bits, with the bounds of token_ref."""
import pytest

import test_gpu_token as T
from test_gpu_token import env  # noqa: F401  (a fixture)

pytestmark = pytest.mark.gpu


def each_its_own(monkeypatch, *forms):
    """The matrices that a case makes, in its order, get (slack, skip) one after the other: elements between rows, and in front of the first."""
    real, left = T.matrix, list(forms)

    def matrix(torch, gen, rows, cols, dtype, std=1.0, slack=0, skip=0):
        return real(torch, gen, rows, cols, dtype, std, *left.pop(0))
    monkeypatch.setattr(T, "matrix", matrix)
    return left


# gate wider apart, up wider apart, one of them copied into rows of its own while the other lies as it does
FORMS = [((72, 0), (0, 0)), ((8, 0), (136, 8)), ((8, 1), (8, 0)), ((16, 0), (16, 1))]
# dtype, rows, width, hidden and the tile that gate and up take
GATED = [("bf16", 40, 72, 72, "64"), ("bf16", 40, 2056, 72, "64 split"), ("bf16", 1900, 72, 1032, "128"), ("bf16", 1900, 4104, 264, "128 split"),
         ("bf16", 1900, 72, 2056, "256"), ("bf16", 2500, 4104, 1032, "256 split"), ("f32", 40, 72, 72, "64"), ("f32", 40, 1032, 72, "64 split"),
         ("f32", 1900, 72, 1032, "128"), ("f32", 1900, 1032, 264, "128 split"), ("bf16", 5, 72, 40, None), ("bf16", 5, 70, 33, None)]


@pytest.mark.parametrize("dtype,rows,d,f,tile", GATED)
def test_gate_and_up_weights_at_their_own_distances(env, monkeypatch, dtype, rows, d, f, tile):
    x, down = (0, 0), (8, 0)
    for gate, up in FORMS:
        with monkeypatch.context() as m:
            left = each_its_own(m, x, gate, up, down)
            with T.routes(env[1]) as took:
                T.ffn_case(env, dtype, "silu", 0, rows, d, f, 0, 0)
        assert not left and took.get("tok_glu") == ({tile} if tile else None), took


# dtype, rows, width, hidden and the tile of dx, whose reduction goes over the gate weights and then the up weights: one part, or split so that a part begins
# with the gate's and ends with the up projection's.  The last step of the gate's is a whole one (320 and 2112 are multiples of 64).
DX = [("bf16", 4090, 2056, 320, "256"), ("bf16", 4090, 1032, 2112, "256 split"), ("bf16", 1500, 2056, 320, "128"), ("bf16", 1900, 520, 2112, "128 split"),
      ("bf16", 300, 264, 320, "64"), ("bf16", 500, 520, 1088, "64 split"), ("f32", 1500, 2056, 320, "128"), ("f32", 500, 520, 1088, "64 split")]


@pytest.mark.parametrize("save", [1, 2])
@pytest.mark.parametrize("dtype,rows,d,f,tile", DX)
def test_backward_with_weights_at_their_own_distances(env, monkeypatch, dtype, rows, d, f, tile, save):
    for gate, up in FORMS:
        with monkeypatch.context() as m:
            left = each_its_own(m, (0, 0), gate, up, (8, 0), (16, 0))
            with T.routes(env[1]) as took:
                T.ffn_case(env, dtype, "silu", save, rows, d, f, 0, 0)
        assert not left and tile in took["tok_linear"], took


@pytest.mark.parametrize("grad", ["f32", "bf16"])
@pytest.mark.parametrize("d,f", [(1, 1), (3, 5), (8, 9), (7, 1), (33, 31), (257, 1023), (16, 24)])
def test_gradients_of_a_call_without_rows(env, d, f, grad):
    """Zeros for each element and nothing behind the last one, whatever the gradients' lengths in bytes and their alignment."""
    torch, P, _ = env
    gdt, gcode = T.types(P, torch, grad)
    sp = torch.cuda.current_stream().cuda_stream
    w = torch.ones(f, d, device="cuda", dtype=torch.bfloat16)
    for skip in (0, 1, 2, 3):
        for accumulate in (0, 1) if grad == "f32" else (0,):
            made = [T.out(torch, n, m, gdt, 0, skip) for n, m in ((f, d), (1, f), (f, d), (f, d), (d, f))]
            dw, db, dg, du, dd = (m for m, _ in made)
            for m, _ in made:
                m.fill_(5.0)
            P.linear_backward(P.linear_args(rows=0, n_in=d, n_out=f, dtype=P.BF16, w=w, ldw=d, dw=dw, dbias=db, grad_dtype=gcode, accumulate=accumulate), sp)
            P.ffn_backward(P.ffn_args(rows=0, width=d, hidden=f, dtype=P.BF16, act=P.ACT_SILU, save=P.SAVE_FULL, w_gate=w, ldwg=d, w_up=w, ldwu=d, w_down=w, ldwd=f,
                                      dw_gate=dg, dw_up=du, dw_down=dd, grad_dtype=gcode, accumulate=accumulate), sp)
            torch.cuda.synchronize()
            for m, ok in made:
                assert bool((m == (5.0 if accumulate else 0.0)).all())
                ok()


@pytest.mark.parametrize("dtype", T.DTYPES)
@pytest.mark.parametrize("off", [1, 2, 3])
def test_inputs_in_8_bits_at_any_byte(env, monkeypatch, dtype, off):
    """Packed rows and scales that start `off` bytes into their buffers, with rows of an odd number of bytes: a slice of a stash."""
    torch, P, R = env
    encode, alive = R.act8_encode, []

    def inside(t):
        buf = torch.full((off + t.numel() + 16,), 0x7F, dtype=torch.uint8, device="cuda")          # NaN around the values
        buf[off:off + t.numel()] = t.flatten()
        alive.append(buf)                                        # a case hands on addresses, also after its names stand for something else
        return buf[off:off + t.numel()].view(t.shape)
    monkeypatch.setattr(R, "act8_encode", lambda x: tuple(inside(t) for t in encode(x)))
    for rows, k, n in ((1, 33, 8), (9, 101, 64), (40, 1001, 72), (70, 64, 40)):
        T.linear_case(env, dtype, "silu", rows, k, n, 0, 0, x8=True)
        T.ffn_case(env, dtype, "silu", 2, rows, k, n, 0, 0, x8=True)


# routes of gate and up, and of the gradients behind them: few rows, tiles of 64, 128 and 256, split reductions; hidden rows that end inside 16 bytes
ODD = [("bf16", 5, 72, 33), ("bf16", 40, 72, 33), ("bf16", 40, 2056, 33), ("bf16", 1900, 72, 1031), ("bf16", 1900, 72, 2051), ("f32", 40, 72, 33), ("f32", 40, 1032, 35),
       ("f32", 1900, 72, 1031)]


@pytest.mark.parametrize("dtype,rows,d,f", ODD)
def test_infinities_beside_pad_columns(env, dtype, rows, d, f):
    """An infinity in a row of x, or of dy: what is infinite by the formula is infinite, not NaN (products of positive numbers with ReLU and without an activation:
    no infinity meets a zero or one of the other sign), and the other rows keep their bits."""
    torch, P, R = env
    tdt, code = T.types(P, torch, dtype)
    gen = torch.Generator(device="cuda").manual_seed(rows + f)
    sp = torch.cuda.current_stream().cuda_stream

    def positive(n, m, std):
        return T.matrix(torch, gen, n, m, tdt, std, 3, 0).abs_().add_(std)
    x, wg, wu, wd, dy = positive(rows, d, 1.0), positive(f, d, 1 / d), positive(f, d, 1 / d), positive(d, f, 1 / f), positive(rows, d, 1.0)
    row = rows // 2

    def call(x, dy, act):
        o = dict(y=torch.empty(rows, d, dtype=tdt, device="cuda"), dx=torch.empty(rows, d, dtype=tdt, device="cuda"), dg=torch.empty(f, d, device="cuda"),
                 du=torch.empty(f, d, device="cuda"), dd=torch.empty(d, f, device="cuda"), gate=torch.empty(rows, f, dtype=tdt, device="cuda"),
                 up=torch.empty(rows, f, dtype=tdt, device="cuda"))
        a = P.ffn_args(rows=rows, width=d, hidden=f, dtype=code, act=act, save=P.SAVE_FULL, gate=o["gate"], up=o["up"], x=x, ldx=x.stride(0), w_gate=wg, ldwg=wg.stride(0),
                       w_up=wu, ldwu=wu.stride(0), w_down=wd, ldwd=wd.stride(0), y=o["y"], ldy=d, dy=dy, lddy=dy.stride(0), dx=o["dx"], lddx=d, dw_gate=o["dg"],
                       dw_up=o["du"], dw_down=o["dd"])
        ws, ok = T.given(a, torch, P.ffn_workspace(a))
        P.ffn_forward(a, sp)
        torch.cuda.synchronize()
        ok()
        ws, ok = T.given(a, torch, P.ffn_workspace(a, True))
        P.ffn_backward(a, sp)
        torch.cuda.synchronize()
        ok()
        return o
    for act in (P.ACT_NONE, P.ACT_RELU):
        plain = call(x, dy, act)
        assert all(bool(v.isfinite().all()) for v in plain.values())
        others = torch.arange(rows, device="cuda") != row
        bad = x.clone()
        bad[row, 3] = float("inf")
        got = call(bad, dy, act)
        for k in ("gate", "up", "y"):
            assert bool((got[k][row] == float("inf")).all()), k
        assert all(torch.equal(got[k][others], plain[k][others]) for k in ("gate", "up", "y", "dx"))
        bad = dy.clone()
        bad[row, 3] = float("inf")
        got = call(x, bad, act)
        assert bool((got["dx"][row] == float("inf")).all())
        assert torch.equal(got["dx"][others], plain["dx"][others]) and torch.equal(got["y"], plain["y"])
        # gradients of the gate and up weights take the row, those of the down weights in the row of the infinite column
        assert bool((got["dg"] == float("inf")).all()) and bool((got["du"] == float("inf")).all())
        assert bool((got["dd"][3] == float("inf")).all()) and torch.equal(got["dd"][4:], plain["dd"][4:])


# ---- the longest calls ------------------------------------------------------------------------------------------------------------------
def pieces(n, step=1 << 27):
    return [slice(i, min(n, i + step)) for i in range(0, n, step)]


@pytest.mark.parametrize("dtype", T.DTYPES)
def test_linear_layer_of_more_than_half_a_billion_rows(env, dtype):
    """More threads than a launch takes if the tiles were small.  One column in and out: y = x w, dx = dy w, both rounded once; dw and db of whole numbers, exact."""
    torch, P, R = env
    tdt, code = T.types(P, torch, dtype)
    sp = torch.cuda.current_stream().cuda_stream
    rows = (1 << 29) + 67
    x, dy = (torch.empty(rows, 1, dtype=tdt, device="cuda") for _ in range(2))
    for i in pieces(rows):
        at = torch.arange(i.start, i.stop, device="cuda")
        x[i, 0] = (at % 97 - 48).to(tdt)
        dy[i, 0] = ((at * 7) % 5 - 2).to(tdt) * ((at & 1023) == 0).to(tdt)          # half a million that are not zero: sums below 2^24
    w = torch.full((1, 1), 1.5, dtype=tdt, device="cuda")
    y, dx = (torch.empty(rows, 1, dtype=tdt, device="cuda") for _ in range(2))
    dw, db = torch.empty(1, 1, device="cuda"), torch.empty(1, device="cuda")
    a = P.linear_args(rows=rows, n_in=1, n_out=1, dtype=code, x=x, ldx=1, w=w, ldw=1, y=y, ldy=1, dy=dy, lddy=1, dx=dx, lddx=1, dw=dw, dbias=db)
    ws = torch.empty(max(P.linear_workspace(a), P.linear_workspace(a, True)), dtype=torch.uint8, device="cuda")
    a.ws, a.ws_bytes = ws.data_ptr(), ws.numel()
    P.linear_forward(a, sp)
    P.linear_backward(a, sp)
    torch.cuda.synchronize()
    want_w = want_b = 0
    for i in pieces(rows):
        assert torch.equal(y[i].float(), x[i].float() * 1.5) and torch.equal(dx[i].float(), dy[i].float() * 1.5)
        want_w += int((x[i].float() * dy[i].float()).long().sum())
        want_b += int(dy[i].long().sum())
    assert float(dw) == want_w and float(db) == want_b


def test_gated_block_of_more_than_half_a_billion_rows(env):
    """One column: gate = x, up = 2 x, hidden = 2 x^2, y = x^2; dhidden = dy / 2, dgate = dy x, dup = dy x / 2, dx = 2 dy x."""
    torch, P, R = env
    sp = torch.cuda.current_stream().cuda_stream
    bf, rows = torch.bfloat16, (1 << 29) + 67
    x, dy = (torch.empty(rows, 1, dtype=bf, device="cuda") for _ in range(2))
    for i in pieces(rows):
        at = torch.arange(i.start, i.stop, device="cuda")
        x[i, 0] = (at % 15 - 7).to(bf)
        dy[i, 0] = ((at * 7) % 5 - 2).to(bf) * ((at & 4095) == 0).to(bf)
    one, two, half = (torch.full((1, 1), v, dtype=bf, device="cuda") for v in (1.0, 2.0, 0.5))
    y, dx, gate, up = (torch.empty(rows, 1, dtype=bf, device="cuda") for _ in range(4))
    dw = [torch.empty(1, 1, device="cuda") for _ in range(3)]
    a = P.ffn_args(rows=rows, width=1, hidden=1, dtype=P.BF16, act=P.ACT_NONE, save=P.SAVE_FULL, gate=gate, up=up, x=x, ldx=1, w_gate=one, ldwg=1, w_up=two, ldwu=1,
                   w_down=half, ldwd=1, y=y, ldy=1, dy=dy, lddy=1, dx=dx, lddx=1, dw_gate=dw[0], dw_up=dw[1], dw_down=dw[2])
    ws = torch.empty(max(P.ffn_workspace(a), P.ffn_workspace(a, True)), dtype=torch.uint8, device="cuda")
    a.ws, a.ws_bytes = ws.data_ptr(), ws.numel()
    P.ffn_forward(a, sp)
    P.ffn_backward(a, sp)
    torch.cuda.synchronize()
    want = [0.0, 0.0, 0.0]
    for i in pieces(rows):
        xi, di = x[i].float(), dy[i].float()
        assert torch.equal(y[i].float(), xi * xi) and torch.equal(gate[i], x[i]) and torch.equal(up[i].float(), 2 * xi) and torch.equal(dx[i].float(), 2 * di * xi)
        p = float((di * xi * xi).double().sum())
        want = [want[0] + p, want[1] + p / 2, want[2] + 2 * p]
    assert [float(v) for v in dw] == want


def test_table_gradient_of_a_billion_tokens(env):
    """The most rows a call takes.  Whole numbers, so that sums are exact."""
    torch, P, R = env
    sp = torch.cuda.current_stream().cuda_stream
    rows, vocab = 1 << 30, 1 << 16
    ids, dy = torch.empty(rows, dtype=torch.int32, device="cuda"), torch.empty(rows, 1, dtype=torch.bfloat16, device="cuda")
    want = torch.zeros(vocab, device="cuda")
    for i in pieces(rows):
        at = torch.arange(i.start, i.stop, device="cuda")
        k = (at * 40503 + (at >> 16)) % vocab
        ids[i] = k
        dy[i, 0] = ((at * 13) % 7 - 3).to(torch.bfloat16)
        want.index_add_(0, k, dy[i, 0].float())
    g = torch.full((vocab, 1), 5.0, device="cuda")
    a = P.embed_args(rows=rows, vocab=vocab, width=1, dtype=P.BF16, scale=1.0, ids=ids, dy=dy, lddy=1, dtable=g, lddt=1)
    ws = torch.empty(P.embed_backward_workspace(a), dtype=torch.uint8, device="cuda")
    a.ws, a.ws_bytes = ws.data_ptr(), ws.numel()
    P.embed_backward(a, sp)
    torch.cuda.synchronize()
    assert torch.equal(g[:, 0], want)
