"""Argument checks of the token operators: refused on the host with a status and a message, before anything is launched (no GPU needed)."""
import ctypes as C

import pytest


@pytest.fixture(scope="module")
def P():
    import paper_2110_02781_amd as P
    return P


AT = 1 << 20            # an address that is only checked, never read


def linear(P, **kw):
    a = dict(rows=4, n_in=16, n_out=8, dtype=P.BF16, act=P.ACT_SILU, x=AT, ldx=16, w=AT, ldw=16, y=AT, ldy=8, z=AT, ldz=8, dy=AT, lddy=8, dx=AT, lddx=16, dw=AT,
             dbias=AT, grad_dtype=P.F32)
    a.update(kw)
    return P.linear_args(**a)


def ffn(P, **kw):
    a = dict(rows=4, width=16, hidden=40, dtype=P.BF16, act=P.ACT_SILU, save=P.SAVE_ACT8, x=AT, ldx=16, w_gate=AT, ldwg=16, w_up=AT, ldwu=16, w_down=AT, ldwd=40, y=AT,
             ldy=16, gate=AT, up=AT, gate_scales=AT, up_scales=AT, dy=AT, lddy=16, dx=AT, lddx=16, dw_gate=AT, dw_up=AT, dw_down=AT, grad_dtype=P.F32)
    a.update(kw)
    return P.ffn_args(**a)


def embed(P, **kw):
    a = dict(rows=4, vocab=10, width=16, dtype=P.BF16, ids=AT, table=AT, ldt=16, out=AT, ldo=16, dy=AT, lddy=16, dtable=AT, lddt=16)
    a.update(kw)
    return P.embed_args(**a)


def act8(P, **kw):
    a = dict(rows=4, cols=40, dtype=P.BF16, x=AT, ldx=40, q=AT, ldq=40, scales=AT, lds=2, y=AT, ldy=40)
    a.update(kw)
    return P.act8_args(**a)


BOTH = [dict(rows=-1), dict(rows=(1 << 30) + 1), dict(dtype=2), dict(dtype=-1)]
LINEAR = BOTH + [dict(act=5), dict(act=-1), dict(n_in=0), dict(n_out=0), dict(n_in=(1 << 20) + 1)]
LINEAR_FWD = LINEAR + [dict(x=0), dict(w=0), dict(y=0), dict(ldx=15), dict(ldw=15), dict(ldy=7), dict(x=AT + 1), dict(y=AT + 1), dict(bias=AT + 2),
                       dict(residual=AT, ldr=7), dict(ldz=7), dict(x_scales=AT, ldxs=0), dict(ldx=(1 << 20) + 1)]
LINEAR_BWD = LINEAR + [dict(dy=0), dict(z=0), dict(lddy=7), dict(lddx=15), dict(dw=AT + 2), dict(grad_dtype=7), dict(grad_dtype=-1), dict(dx=0, dw=0, dbias=0),
                       dict(x=0), dict(w=0)]
FFN = BOTH + [dict(act=9), dict(save=3), dict(save=-1), dict(width=0), dict(hidden=0), dict(w_gate=0), dict(w_up=0), dict(w_down=0), dict(ldwg=15), dict(ldwu=15),
              dict(ldwd=39), dict(gate=0), dict(up=0), dict(gate_scales=0), dict(up_scales=0), dict(x=0), dict(ldx=15)]
FFN_FWD = FFN + [dict(y=0), dict(ldy=15), dict(residual=AT, ldr=15)]
FFN_BWD = FFN + [dict(save=0), dict(dy=0), dict(lddy=15), dict(lddx=15), dict(dw_up=0), dict(dx=0, dw_gate=0, dw_up=0, dw_down=0), dict(grad_dtype=5)]
EMBED = BOTH + [dict(vocab=0), dict(width=0), dict(ids=0), dict(ids=AT + 2), dict(ids=AT + 4, ids64=1)]
ACT8 = BOTH + [dict(cols=0), dict(q=0), dict(scales=0), dict(ldq=39), dict(lds=1)]


def refused(P, call, args, status=-1):
    with pytest.raises(P.FtpError) as e:
        call(args, None)
    assert e.value.status == status and len(P.binding.last_error()) > 10


@pytest.mark.parametrize("bad", LINEAR_FWD, ids=str)
def test_linear_forward(P, bad):
    refused(P, P.linear_forward, linear(P, **bad))


@pytest.mark.parametrize("bad", LINEAR_BWD, ids=str)
def test_linear_backward(P, bad):
    refused(P, P.linear_backward, linear(P, **bad))


@pytest.mark.parametrize("bad", FFN_FWD, ids=str)
def test_ffn_forward(P, bad):
    refused(P, P.ffn_forward, ffn(P, **bad))


@pytest.mark.parametrize("bad", FFN_BWD, ids=str)
def test_ffn_backward(P, bad):
    refused(P, P.ffn_backward, ffn(P, **bad))


def test_embed(P):
    for bad in EMBED + [dict(table=0), dict(out=0), dict(ldt=15), dict(ldo=15), dict(table=AT + 1)]:
        refused(P, P.embed_forward, embed(P, **bad))
    for bad in EMBED + [dict(dy=0), dict(dtable=0), dict(lddy=15), dict(lddt=15), dict(dtable=AT + 2)]:
        refused(P, P.embed_backward, embed(P, **bad))
    for scale in (float("nan"), float("inf")):
        refused(P, P.embed_forward, embed(P, scale=scale), -5)
        refused(P, P.embed_backward, embed(P, scale=scale), -5)
    refused(P, P.embed_backward, embed(P))                                          # no workspace
    n = P.embed_backward_workspace(embed(P))
    refused(P, P.embed_backward, embed(P, ws=AT, ws_bytes=n - 1))
    refused(P, P.embed_backward, embed(P, ws=AT + 8, ws_bytes=n))


def test_act8(P):
    for bad in ACT8 + [dict(x=0), dict(ldx=39), dict(x=AT + 1)]:
        refused(P, P.act8_pack, act8(P, **bad))
    for bad in ACT8 + [dict(y=0), dict(ldy=39), dict(y=AT + 1)]:
        refused(P, P.act8_unpack, act8(P, **bad))


def test_accumulating_in_the_calls_type_is_not_supported(P):
    refused(P, P.linear_backward, linear(P, grad_dtype=P.BF16, accumulate=1), -3)
    refused(P, P.ffn_backward, ffn(P, grad_dtype=P.BF16, accumulate=1), -3)
    refused(P, P.linear_backward, linear(P, dtype=P.F32, grad_dtype=P.BF16))         # nor are bfloat16 gradients of fp32 weights


def test_null_records(P):
    lib = P.lib
    for f in (lib.ftp_linear_forward, lib.ftp_linear_backward, lib.ftp_ffn_forward, lib.ftp_ffn_backward, lib.ftp_act8_pack, lib.ftp_act8_unpack, lib.ftp_embed_forward,
              lib.ftp_embed_backward):
        assert f(None, None) == -1
    n = C.c_size_t(5)
    for f in (lib.ftp_linear_workspace, lib.ftp_ffn_workspace):
        assert f(None, 0, C.byref(n)) == -1
    assert lib.ftp_linear_workspace(C.byref(linear(P)), 0, None) == -1 and lib.ftp_embed_backward_workspace(C.byref(embed(P)), None) == -1 and n.value == 5
    with pytest.raises(TypeError):
        P.linear_args(row=3)


def test_workspaces(P):
    """Aligned operands need none for their copies, nor do those of few rows; what a call names is what it asks for."""
    assert P.linear_workspace(linear(P, rows=40, n_in=64, n_out=64, ldx=64, ldw=64, ldy=64, ldz=64)) == 0
    assert P.linear_workspace(linear(P, rows=4, n_in=15, n_out=8, x=AT + 2, ldx=17, ldw=15)) == 0
    odd = linear(P, rows=40, n_in=15, n_out=8, ldx=16, ldw=16)
    n = P.linear_workspace(odd)
    assert n >= (40 + 8) * 16 * 2
    refused(P, P.linear_forward, odd)
    for off in (dict(x=AT + 2), dict(ldx=17, n_in=16)):                             # an offset, rows of an odd distance
        assert P.linear_workspace(linear(P, rows=40, **off)) >= 40 * 16 * 2
    f = ffn(P)
    n = P.ffn_workspace(f, True)
    assert n >= 3 * 4 * 40 * 2
    f.ws, f.ws_bytes = AT, n - 1
    refused(P, P.ffn_backward, f)
    f.ws, f.ws_bytes = AT + 4, n
    refused(P, P.ffn_backward, f)


def test_record_layouts_match_the_header(P, tmp_path):
    """Offsets of every field, from the header by a C compiler."""
    import os
    import subprocess
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    B = P.binding
    names = {"ftp_embed_args": B.EmbedArgs, "ftp_linear_args": B.LinearArgs, "ftp_ffn_args": B.FfnArgs, "ftp_act8_args": B.Act8Args}
    src = '#include <stdio.h>\n#include "ftp.h"\nint main(void) {\n'
    for n, s in names.items():
        for field, _ in s._fields_:
            src += f'  printf("%zu\\n", offsetof({n}, {field}));\n'
        src += f'  printf("%zu\\n", sizeof({n}));\n'
    (tmp_path / "o.c").write_text(src + "  return 0;\n}\n")
    subprocess.run(["gcc", "-I", os.path.join(root, "include"), str(tmp_path / "o.c"), "-o", str(tmp_path / "o")], check=True)
    got = [int(v) for v in subprocess.run([str(tmp_path / "o")], check=True, stdout=subprocess.PIPE, text=True).stdout.split()]
    want = []
    for s in names.values():
        want += [getattr(s, f).offset for f, _ in s._fields_] + [C.sizeof(s)]
    assert got == want
