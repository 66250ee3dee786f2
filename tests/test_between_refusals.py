"""Argument checks of joins, dropout, the recurrence and log probabilities: refused on the host with a status and a message, before anything is launched (no GPU needed)."""
import ctypes as C

import pytest


@pytest.fixture(scope="module")
def P():
    import paper_2110_02781_amd as P
    return P


AT = 1 << 20            # an address that is only checked, never read
NAN, INF = float("nan"), float("inf")


def dropout(P, **kw):
    a = dict(rows=4, cols=10, dtype=P.BF16, p=0.1, x=AT, ldx=10, residual=AT, ldr=10, y=AT, ldy=10, dy=AT, lddy=10, dx=AT, lddx=10)
    return P.dropout_args(**{**a, **kw})


def join(P, **kw):
    a = dict(rows=40, width=16, dtype=P.BF16, post=1, x=AT, ldx=16, b=AT, ldb=16, gate=AT, ldg=16, gate_rows=1, gate_dtype=P.BF16, y=AT, ldy=16, n=AT, ldn=16, dy=AT, lddy=16,
             dn=AT, lddn=16, dx=AT, lddx=16, db=AT, lddb=16, dgate=AT, lddg=16, dpost_w=AT, dpre_w=AT)
    return P.join_args(**{**a, **kw})


def scan(P, **kw):
    a = dict(rows=40, width=16, seqs=4, length=10, dtype=P.BF16, act=P.ACT_SILU, f=AT, ldf=16, x=AT, ldx=16, g=AT, ldg=16, h0=AT, ldh0=16, y=AT, ldy=16, h_end=AT, ldhe=16,
             dy=AT, lddy=16, df=AT, lddf=16, dx=AT, lddx=16, dg=AT, lddg=16, dh0=AT, lddh0=16)
    return P.scan_args(**{**a, **kw})


def logp(P, **kw):
    a = dict(rows=4, vocab=10, dtype=P.BF16, logits=AT, ldl=10, ids=AT, logp=AT, entropy=AT, lse=AT, stats=AT, top=3, top_ids=AT, top_logp=AT, dlogp=AT, dentropy=AT, dlogits=AT, lddl=10)
    return P.logp_args(**{**a, **kw})


def refused(P, call, args, status=-1):
    with pytest.raises(P.FtpError) as e:
        call(args, None)
    assert e.value.status == status and len(P.binding.last_error()) > 10


SIZES = [dict(rows=-1), dict(rows=(1 << 30) + 1), dict(dtype=2), dict(dtype=-1)]
MASK = [(dict(p=1.0), -5), (dict(p=-0.1), -5), (dict(p=NAN), -5), (dict(p=0.999995), -5), (dict(row0=-1), -1), (dict(row0=(1 << 63) - 2), -1), (dict(seed_dev=AT + 4), -1)]


@pytest.mark.parametrize("bad", SIZES + [dict(cols=0), dict(cols=(1 << 20) + 1)], ids=str)
def test_dropout_sizes(P, bad):
    refused(P, P.dropout_forward, dropout(P, **bad))
    refused(P, P.dropout_backward, dropout(P, **bad))


def test_dropout(P):
    for bad, status in MASK:
        refused(P, P.dropout_forward, dropout(P, **bad), status)
        refused(P, P.dropout_backward, dropout(P, **bad), status)
    for bad in (dict(x=0), dict(y=0), dict(ldx=9), dict(ldr=9), dict(ldy=9), dict(x=AT + 1), dict(residual=AT + 1), dict(y=AT + 1), dict(ldx=(1 << 20) + 1)):
        refused(P, P.dropout_forward, dropout(P, **bad))
    for bad in (dict(dy=0), dict(dx=0), dict(lddy=9), dict(lddx=9), dict(dy=AT + 1)):
        refused(P, P.dropout_backward, dropout(P, **bad))


JOIN = SIZES + [dict(width=0), dict(width=(1 << 20) + 1), dict(norm=2), dict(norm=-1), dict(x=0, b=0), dict(ldx=15), dict(ldb=15), dict(x=AT + 1), dict(b=AT + 1), dict(post_w=AT + 2),
                dict(post_bias=AT + 1), dict(pre_w=AT + 2), dict(pre_bias=AT + 3), dict(gate_dtype=5), dict(gate_rows=0), dict(gate_rows=-3), dict(ldg=15), dict(gate=AT + 1)]


@pytest.mark.parametrize("bad", JOIN + [dict(y=0, n=0), dict(ldy=15), dict(ldn=15), dict(n=AT + 1)], ids=str)
def test_join_forward(P, bad):
    refused(P, P.join_forward, join(P, **bad))


@pytest.mark.parametrize("bad", JOIN + [dict(dy=0, dn=0), dict(lddy=15), dict(lddn=15), dict(lddx=15), dict(lddb=15), dict(lddg=15), dict(b=0), dict(post=0), dict(dn=0),
                                        dict(gate=0), dict(dpre_w=AT + 2), dict(dpost_bias=AT + 1), dict(dx=AT + 1),
                                        dict(dx=0, db=0, dgate=0, dpost_w=0, dpre_w=0)], ids=str)
def test_join_backward(P, bad):
    refused(P, P.join_backward, join(P, **bad))
    refused(P, lambda a, _: P.join_workspace(a), join(P, **bad))


def test_join_values(P):
    for call in (P.join_forward, P.join_backward):
        for bad, status in MASK + [(dict(eps=0.0), -5), (dict(eps=-1.0), -5), (dict(eps=NAN), -5), (dict(eps=INF), -5), (dict(scale=NAN), -5), (dict(scale=INF), -5)]:
            refused(P, call, join(P, **bad), status)
    refused(P, P.join_backward, join(P, gate_accumulate=1), -3)
    refused(P, P.join_forward, join(P, dtype=P.F32))                              # a bfloat16 gate of an fp32 call
    a = join(P)
    n = P.join_workspace(a)
    assert n >= 2 * 16 * 4
    refused(P, P.join_backward, a)
    for kw in (dict(ws=AT, ws_bytes=n - 1), dict(ws=AT + 8, ws_bytes=n)):
        refused(P, P.join_backward, join(P, **kw))
    assert P.join_workspace(join(P, dpost_w=0, dpre_w=0)) == 0                     # nothing is summed over the rows
    assert P.join_workspace(join(P, dpost_w=0, dpre_w=0, gate_rows=7)) > 0
    assert P.join_workspace(join(P, rows=0)) == 0


SCAN = SIZES + [dict(width=0), dict(width=(1 << 20) + 1), dict(form=3), dict(form=-1), dict(act=5), dict(act=-1), dict(seqs=-1), dict(seqs=3), dict(length=-10, rows=0, seqs=0),
                dict(length=11), dict(starts=AT + 2), dict(f=0), dict(x=0), dict(ldf=15), dict(ldx=15), dict(ldg=15), dict(ldh0=15), dict(f=AT + 1), dict(g=AT + 1), dict(h0=AT + 2)]


@pytest.mark.parametrize("bad", SCAN + [dict(y=0, h_end=0), dict(ldy=15), dict(ldhe=15), dict(h_end=AT + 1), dict(h_end=AT, ldhe=17)], ids=str)
def test_scan_forward(P, bad):
    refused(P, P.scan_forward, scan(P, **bad))


@pytest.mark.parametrize("bad", SCAN + [dict(dy=0), dict(lddy=15), dict(lddf=15), dict(lddx=15), dict(lddg=15), dict(lddh0=15), dict(dh_end=AT, lddhe=15), dict(g=0), dict(dy=AT + 1),
                                        dict(dh_end=AT, lddhe=17), dict(df=0, dx=0, dg=0, dh0=0)], ids=str)
def test_scan_backward(P, bad):
    refused(P, P.scan_backward, scan(P, **bad))


def test_scan_workspace(P):
    long = dict(rows=4000, length=1000)
    for back in (False, True):
        n = P.scan_workspace(scan(P, **long), back)
        assert n > 0
        call = P.scan_backward if back else P.scan_forward
        refused(P, call, scan(P, **long))
        for kw in (dict(ws=AT, ws_bytes=n - 1), dict(ws=AT + 8, ws_bytes=n)):
            refused(P, call, scan(P, **long, **kw))
    assert P.scan_workspace(scan(P, rows=4, length=1)) == 0                        # a step


LOGP = SIZES + [dict(vocab=0), dict(vocab=(1 << 20) + 1), dict(logits=0), dict(ldl=9), dict(logits=AT + 1), dict(ids=0), dict(ids=AT + 2), dict(ids=AT + 4, ids64=1), dict(entropy=AT + 1),
                dict(stats=AT + 2)]


@pytest.mark.parametrize("bad", LOGP + [dict(top=-1), dict(top=65), dict(top_ids=0), dict(top_logp=0), dict(top_ids=AT + 2), dict(logp=AT + 1), dict(lse=AT + 2),
                                        dict(logp=0, entropy=0, lse=0, stats=0, top=0)], ids=str)
def test_logp_forward(P, bad):
    refused(P, P.logp_forward, logp(P, **bad))


@pytest.mark.parametrize("bad", LOGP + [dict(stats=0), dict(dlogp=0, dentropy=0), dict(entropy=0), dict(dlogits=0), dict(lddl=9), dict(dlogits=AT + 1), dict(dlogp=AT + 2),
                                        dict(dentropy=AT + 1)], ids=str)
def test_logp_backward(P, bad):
    refused(P, P.logp_backward, logp(P, **bad))


def test_logp_values(P):
    for scale in (0.0, -1.0, NAN, INF):
        refused(P, P.logp_forward, logp(P, scale=scale), -5)
        refused(P, P.logp_backward, logp(P, scale=scale), -5)
    n = P.logp_workspace(logp(P, rows=1, vocab=100000, ldl=100000))
    if n:
        refused(P, P.logp_forward, logp(P, rows=1, vocab=100000, ldl=100000, ws=AT, ws_bytes=n - 1))
        refused(P, P.logp_forward, logp(P, rows=1, vocab=100000, ldl=100000, ws=AT + 8, ws_bytes=n))


def test_null_records(P):
    lib = P.lib
    for f in (lib.ftp_dropout_forward, lib.ftp_dropout_backward, lib.ftp_join_forward, lib.ftp_join_backward, lib.ftp_scan_forward, lib.ftp_scan_backward, lib.ftp_logp_forward,
              lib.ftp_logp_backward):
        assert f(None, None) == -1
    n = C.c_size_t(5)
    assert lib.ftp_join_workspace(None, C.byref(n)) == -1 and lib.ftp_scan_workspace(None, 0, C.byref(n)) == -1 and lib.ftp_logp_workspace(None, C.byref(n)) == -1 and n.value == 5
    assert lib.ftp_join_workspace(C.byref(join(P)), None) == -1
    with pytest.raises(TypeError):
        P.join_args(row=3)


def test_calls_without_rows_need_no_buffers(P):
    """nothing to launch: no GPU is touched"""
    P.dropout_forward(P.dropout_args(rows=0, cols=8, dtype=P.F32), None)
    P.join_forward(P.join_args(rows=0, width=8, dtype=P.F32), None)
    P.scan_forward(P.scan_args(rows=0, seqs=0, width=8, dtype=P.F32), None)
    P.logp_forward(P.logp_args(rows=0, vocab=8, dtype=P.F32), None)
    P.logp_backward(P.logp_args(rows=0, vocab=8, dtype=P.F32), None)


def test_record_layouts_match_the_header(P, tmp_path):
    """Offsets of every field, from the header by a C compiler."""
    import os
    import subprocess
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    B = P.binding
    names = {"ftp_dropout_args": B.DropoutArgs, "ftp_join_args": B.JoinArgs, "ftp_scan_args": B.ScanArgs, "ftp_logp_args": B.LogpArgs}
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


def test_the_generator_against_its_authors_vectors():
    """known answers of Philox4x32-10 that its authors publish: counter, key, result"""
    import between_ref as R
    for counter, key, want in (((0, 0, 0, 0), (0, 0), (0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8)),
                               ((0xffffffff,) * 4, (0xffffffff,) * 2, (0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd)),
                               ((0x243f6a88, 0x85a308d3, 0x13198a2e, 0x03707344), (0xa4093822, 0x299f31d0), (0xd16cfe09, 0x94fdcceb, 0x5001e420, 0x24126ea1))):
        assert tuple(R.philox(counter, key)) == want


def test_results_in_an_operands_buffer_have_its_rows(P):
    B = 3 << 20
    for kw in (dict(y=B, x=B, ldy=11), dict(y=B, residual=B, ldy=11), dict(y=B, x=B, ldx=12)):
        refused(P, P.dropout_forward, dropout(P, **kw))
    refused(P, P.dropout_backward, dropout(P, dx=B, dy=B, lddx=11))
    for kw in (dict(y=B, x=B, ldy=17), dict(y=B, b=B, ldb=18)):
        refused(P, P.join_forward, join(P, **kw))
    refused(P, P.join_backward, join(P, dx=B, dy=B, lddy=17))
    refused(P, P.scan_backward, scan(P, dh0=B, dh_end=B, lddhe=17))
    refused(P, P.logp_backward, logp(P, dlogits=B, logits=B, lddl=11))


@pytest.mark.parametrize("p", [1.5, 2.0, 65535.99, 65536.0, 65536.5, 131072.0, 1e10, 1e20, 1e30, 3e38, INF, -INF])
def test_probabilities_past_one(P, p):
    """also those that no whole number of 32 bits holds; without rows, so that a call that is let through launches nothing"""
    for call, a in ((P.dropout_forward, dropout(P, rows=0, p=p)), (P.dropout_backward, dropout(P, rows=0, p=p)), (P.join_forward, join(P, rows=0, p=p)), (P.join_backward, join(P, rows=0, p=p, dpost_w=0, dpre_w=0)),
                    (lambda r, _: P.join_workspace(r), join(P, rows=0, p=p))):
        refused(P, call, a, -5)
