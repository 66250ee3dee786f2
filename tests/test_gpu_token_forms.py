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
