"""What stands between the products of a token model's stage, in the directions that training and serving use: the join of a block's
output with the stream and the norms around it, dropout, a gated linear recurrence along the sequences, log probabilities of tokens.

Fields of a case
  op      "join_fwd"      c = norm(b) (with post) or b; y = x + scale * gate * drop(c); n = norm(y)
          "join_train"    the same, then dx, db and the gradients of gate and norm weights from dy and dn
          "drop_train"    y = x dropped + r, then dx from dy
          "scan_fwd"      h[t] = a[t] h[t-1] + c(a[t]) x[t], a = sigmoid(f); y = h * act(g); the state behind each sequence
          "scan_train"    the same, then df, dx, dg and the initial states' gradient
          "logp_fwd"      log probability of a token, entropy and the `top` likeliest tokens of each row of logits
          "logp_train"    log probability and entropy, then dlogits
  dtype   "f32" or "bf16": activations and their gradients
  rows    tokens; width, vocab: columns; slack: elements between the end of a row and the next one of the matrices that come in
  norm    "rms" or "layer"; post: the block's output is normed too; gate: "none", "row" (its own for each row), "group" (one for gate_rows rows) or
          "all" (one, fp32: a weight); drop: probability of the mask
  seqs    sequences, one behind the other: of rows / seqs rows each, or with cut != 0 of any lengths that this number gives, some of them empty, and
          `behind` rows behind the last one that belong to none
  form    c(a): "add" 1, "mix" 1 - a, "unit" sqrt(1 - a^2); act: of the gate g ("" without one)
  top     likeliest tokens; barred: tokens at the end of the vocabulary whose logit is -inf; temper: factor of the logits
"""
import math
import random

import torch

own = False

_T = {"f32": torch.float32, "bf16": torch.bfloat16}
_EPS = 1e-5


def listed():
    def at(name, op, rows, dtype="bf16", slack=0, **kw):
        return dict(name=name, op=op, rows=rows, dtype=dtype, slack=slack, **kw)
    return [
        # a decode step of a few requests between two blocks: latency alone
        at("join_fwd_4", "join_fwd", 4, width=4096, norm="rms", post=False, gate="none", drop=0.0),
        # training, everything at once: norms on both sides, a gate of its own for each row, dropout
        at("join_train_8192", "join_train", 8192, width=4096, norm="rms", post=True, gate="row", drop=0.1),
        # single precision, odd width, rows of a wider buffer, one gate for the rows of a sample
        at("join_train_1000_f32", "join_train", 1000, "f32", slack=7, width=1001, norm="layer", post=True, gate="group", gate_rows=130, drop=0.0),
        # a layer's dropout at training size
        at("drop_16384", "drop_train", 16384, width=4096, drop=0.1),
        # a small odd one in single precision
        at("drop_333_f32", "drop_train", 333, "f32", slack=3, width=1001, drop=0.5),
        # one token for each of 256 requests
        at("scan_step_256", "scan_fwd", 256, width=2048, seqs=256, cut=0, behind=0, form="mix", act="silu"),
        # one long prompt
        at("scan_fwd_16384", "scan_fwd", 16384, width=2048, seqs=1, cut=0, behind=0, form="mix", act="silu"),
        # training on packed sequences of all lengths
        at("scan_train_16384", "scan_train", 16384, width=2048, seqs=24, cut=5, behind=0, form="unit", act="gelu"),
        # single precision, odd sizes, empty sequences, rows that belong to none
        at("scan_train_1500_f32", "scan_train", 1500, "f32", slack=5, width=333, seqs=11, cut=3, behind=9, form="add", act=""),
        # a decode step's answer with alternatives
        at("logp_fwd_8", "logp_fwd", 8, vocab=128000, top=20, barred=0, temper=1.25),
        # a batch's log probabilities and entropy with their gradient
        at("logp_train_8192", "logp_train", 8192, vocab=32000, top=0, barred=0, temper=1.0),
        # scores of a prompt with alternatives, single precision, an odd vocabulary with places that stand for nothing
        at("logp_fwd_700_f32", "logp_fwd", 700, "f32", slack=3, vocab=5001, top=5, barred=41, temper=1.0),
    ]


# ---- drawn cases -------------------------------------------------------------------------------------------------
def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    """A size between lo and hi: often a multiple of 64, sometimes of 8, sometimes anything."""
    n, k = _log(rng, lo, hi), rng.choice((64, 64, 8, 1))
    return max(lo, n // k * k)


_MOST = 8192 * 32000 * 2.0 * 2           # bytes of the largest listed case


def draw(rng):
    op = rng.choice(("join_fwd", "join_train", "drop_train", "scan_fwd", "scan_train", "logp_fwd", "logp_train"))
    while True:
        dtype = rng.choice(("bf16", "bf16", "f32"))
        c = dict(op=op, dtype=dtype, rows=_log(rng, 1, 32768), slack=rng.choice((0, 0, 8, 5)))
        if op.startswith("join"):
            c.update(width=_size(rng, 64, 16384), norm=rng.choice(("rms", "rms", "layer")), post=rng.choice((False, True)),
                     gate=rng.choice(("none", "row", "group", "all")), drop=rng.choice((0.0, 0.0, 0.1, 0.35)))
            if c["gate"] == "group":
                c["gate_rows"] = _log(rng, 2, 4096)
        elif op.startswith("drop"):
            c.update(width=_size(rng, 32, 16384), drop=rng.choice((0.02, 0.1, 0.5)))
        elif op.startswith("scan"):
            c.update(width=_size(rng, 32, 8192), form=rng.choice(("add", "mix", "unit")), act=rng.choice(("", "silu", "gelu", "none")), cut=0, behind=0)
            kind = rng.choice(("step", "even", "cut", "cut"))
            if kind == "cut":
                c.update(seqs=min(c["rows"], _log(rng, 1, 300)), cut=rng.randint(1, 1000), behind=rng.choice((0, 0, min(7, c["rows"] - 1))))
            else:
                c["seqs"] = c["rows"] if kind == "step" else min(c["rows"], _log(rng, 1, 64))
                c["rows"] = c["rows"] // c["seqs"] * c["seqs"]
        else:
            c.update(vocab=_size(rng, 100, 160000), top=0 if op == "logp_train" else rng.choice((0, 1, 5, 20, 50)), barred=rng.choice((0, 0, 31)),
                     temper=rng.choice((1.0, 1.0, 0.7, 1.4)))
        if work(c)["bytes"] <= _MOST / 2:
            return c


# ---- what a program has in hand ------------------------------------------------------------------------------------
def _lengths(c):
    """Rows of each sequence."""
    if not c["cut"]:
        return [c["rows"] // c["seqs"]] * c["seqs"]
    rng, n = random.Random(c["cut"]), c["rows"] - c["behind"]
    cuts = [rng.randint(0, n) for _ in range(c["seqs"] - 1)]
    cuts = [cuts[i - 1] if i and rng.random() < 0.15 else v for i, v in enumerate(cuts)]            # twice the same: an empty sequence
    ends = sorted(cuts) + [n]
    return [b - a for a, b in zip([0] + ends, ends)]


def prepare(case, seed):
    dev, dt = "cuda", _T[case["dtype"]]
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    s, rows, op, slack = {"case": dict(case)}, case["rows"], case["op"], case["slack"]

    def normal(n, cols, std=1.0, mean=0.0, dtype=dt, wide=slack):
        t = torch.randn(n, cols + wide, generator=gen, device=dev, dtype=torch.float32)
        return t.mul_(std).add_(mean).to(dtype)[:, :cols]

    if op.startswith(("join", "drop")):
        d = case["width"]
        # some channels are far larger than the rest, as a stream's are
        loud = torch.exp(torch.randn(d, generator=gen, device=dev)).to(dt)
        s["mask"] = dict(seed=seed * 1000003 + 12345, site=7, row0=5000000000)
        s["x"] = normal(rows, d).mul_(loud)
        if op == "drop_train":
            s["r"], s["dy"] = normal(rows, d), normal(rows, d, 1e-2)
            return s
        s["b"] = normal(rows, d, 2.0, 0.1)
        s["scale"] = 0.5
        kind = case["gate"]
        if kind != "none":
            groups = rows if kind == "row" else -(-rows // case["gate_rows"]) if kind == "group" else 1
            s["gate"] = normal(groups, d, 0.3, 1.0, torch.float32 if kind == "all" else dt, 0)
        for name in ("pre", "post") if case["post"] else ("pre",):
            s[name + "_w"] = 1 + 0.1 * torch.randn(d, generator=gen, device=dev)
            if case["norm"] == "layer":
                s[name + "_bias"] = 0.1 * torch.randn(d, generator=gen, device=dev)
        if op == "join_train":
            s["dy"], s["dn"] = normal(rows, d, 1e-2), normal(rows, d, 1e-2)
    elif op.startswith("scan"):
        d = case["width"]
        lens = _lengths(case)
        ends = torch.tensor([0] + lens, dtype=torch.int64).cumsum(0)
        s["starts"] = ends.to(torch.int32).to(dev)
        s["longest"] = max(lens)
        # channels remember from one to some hundred tokens
        s["f"] = normal(rows, d).add_((2 + 2 * torch.randn(d, generator=gen, device=dev)).to(dt))
        s["x"] = normal(rows, d)
        if case["act"]:
            s["g"] = normal(rows, d)
        s["h0"] = torch.randn(len(lens), d, generator=gen, device=dev)
        if op == "scan_train":
            s["dy"] = normal(rows, d, 1e-2)
            s["dh_end"] = 1e-2 * torch.randn(len(lens), d, generator=gen, device=dev)
    else:
        v = case["vocab"]
        s["logits"] = normal(rows, v, 2.5)
        # what a model holds likely stands out
        peak = torch.randint(0, v, (rows, 4), generator=gen, device=dev)
        s["logits"].scatter_(1, peak, (6 + 4 * torch.rand(rows, 4, generator=gen, device=dev)).to(dt))
        if case["barred"]:
            s["logits"][:, v - case["barred"]:] = -math.inf
        ids = torch.randint(0, v - case["barred"], (rows,), generator=gen, device=dev)
        ids = torch.where(torch.rand(rows, generator=gen, device=dev) < 0.5, peak[:, 0].clamp(max=v - case["barred"] - 1), ids)
        if op == "logp_train":
            ids = torch.where(torch.rand(rows, generator=gen, device=dev) < 0.05, -1, ids)          # padding
            s["dlogp"] = torch.randn(rows, generator=gen, device=dev)
            s["dentropy"] = torch.full((rows,), -0.01, device=dev)
        s["ids"] = ids.to(torch.int32)
    return s


# ---- the plain forms ----------------------------------------------------------------------------------------------
def _kept(rows, cols, p, mask, device):
    """Where the mask of the counter-based generator (Philox, four words of 32 bits, ten rounds) keeps a value, and the factor of what is kept.
    Block j of a row's columns, eight of them, has the counter (j, site, row's number) under the key `seed`; its words hold sixteen bits for each."""
    low = 0xffffffff
    j = torch.arange(-(-cols // 8), dtype=torch.int64, device=device)[None, :]
    r = torch.arange(rows, dtype=torch.int64, device=device)[:, None] + mask["row0"]
    w = [j + 0 * r, j * 0 + 0 * r + mask["site"], (r & low) + 0 * j, (r >> 32) + 0 * j]
    k0, k1 = mask["seed"] & low, mask["seed"] >> 32
    for i in range(10):
        a, b = w[0] * 0xD2511F53, w[2] * 0xCD9E8D57                  # modulo 2^64: the high words' bits are whole
        w = [(b >> 32 & low) ^ w[1] ^ ((k0 + i * 0x9E3779B9) & low), b & low, (a >> 32 & low) ^ w[3] ^ ((k1 + i * 0xBB67AE85) & low), a & low]
    u = torch.stack([w[0] & 0xffff, w[0] >> 16, w[1] & 0xffff, w[1] >> 16, w[2] & 0xffff, w[2] >> 16, w[3] & 0xffff, w[3] >> 16], 2)
    least = int(p * 65536 + 0.5)
    return u.view(rows, -1)[:, :cols] >= least, 65536 / (65536 - least)


def _normed(v, kind):
    """(v normed, what its deviation was divided by, inverted)"""
    if kind == "layer":
        v = v - v.mean(1, keepdim=True)
    r = 1 / torch.sqrt((v * v).mean(1, keepdim=True) + _EPS)
    return v * r, r


def _norm_back(dv, v, r, kind):
    """gradient in front of a norm, of that behind it: v the normed values"""
    out = dv - v * (dv * v).mean(1, keepdim=True)
    return r * (out - dv.mean(1, keepdim=True) if kind == "layer" else out)


def _plain_join(s):
    c, dt, f32 = s["case"], _T[s["case"]["dtype"]], torch.float32
    x, b, kind = s["x"].to(f32), s["b"].to(f32), c["norm"]
    rows, d = x.shape
    branch = b
    if c["post"]:
        bh, br = _normed(b, kind)
        branch = bh * s["post_w"] + (s["post_bias"] if kind == "layer" else 0)
    factor = torch.full((1, 1), s["scale"], device=x.device)
    if c["drop"]:
        keep, up = _kept(rows, d, c["drop"], s["mask"], x.device)
        factor = torch.where(keep, s["scale"] * up, 0.0)
    per = 1 if c["gate"] == "row" else c.get("gate_rows", rows)
    gate = s["gate"].to(f32)[torch.arange(rows, device=x.device) // per] if "gate" in s else torch.ones(1, 1, device=x.device)
    y = x + factor * gate * branch
    yh, yr = _normed(y, kind)
    n = yh * s["pre_w"] + (s["pre_bias"] if kind == "layer" else 0)
    out = {"y": y.to(dt), "n": n.to(dt)}
    if c["op"] == "join_train":
        dn = s["dn"].to(f32)
        dy = s["dy"].to(f32) + _norm_back(dn * s["pre_w"], yh, yr, kind)
        dc = factor * gate * dy
        out.update(dx=dy.to(dt), dpre_w=(dn * yh).sum(0))
        if kind == "layer":
            out["dpre_bias"] = dn.sum(0)
        if "gate" in s:
            dgate = factor * branch * dy
            short = -rows % per
            dgate = torch.cat((dgate, dgate.new_zeros(short, d))) if short else dgate
            out["dgate"] = dgate.view(-1, per, d).sum(1).to(s["gate"].dtype)
        if c["post"]:
            out["dpost_w"] = (dc * bh).sum(0)
            if kind == "layer":
                out["dpost_bias"] = dc.sum(0)
            dc = _norm_back(dc * s["post_w"], bh, br, kind)
        out["db"] = dc.to(dt)
    return out


def _plain_drop(s):
    c, dt, f32 = s["case"], _T[s["case"]["dtype"]], torch.float32
    keep, up = _kept(c["rows"], c["width"], c["drop"], s["mask"], s["x"].device)
    return {"y": (torch.where(keep, s["x"].to(f32) * up, 0.0) + s["r"].to(f32)).to(dt), "dx": torch.where(keep, s["dy"].to(f32) * up, 0.0).to(dt)}


def _act(z, act):
    """(act(z), its derivative)"""
    if act == "silu":
        p = torch.sigmoid(z)
        return z * p, p * (1 + z * (1 - p))
    if act == "gelu":
        t = torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z))
        return 0.5 * z * (1 + t), 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * z * z)
    return z, torch.ones_like(z)


def _follow(a, u, longest):
    """h[t] = a[t] h[t-1] + u[t], a = 0 where a sequence starts: what lies 1, 2, 4, ... rows back is added in turn"""
    a, h, n = a.clone(), u.clone(), 1
    while n < longest:
        h[n:] += a[n:] * h[:-n]
        a[n:] = a[n:] * a[:-n]
        n *= 2
    return h


def _plain_scan(s):
    c, dt, f32 = s["case"], _T[s["case"]["dtype"]], torch.float32
    starts, dev = s["starts"].long(), s["f"].device
    n = c["rows"] - c["behind"]
    f, x = s["f"][:n].to(f32), s["x"][:n].to(f32)
    seq = torch.searchsorted(starts, torch.arange(n, device=dev), right=True) - 1
    lens = starts[1:] - starts[:-1]
    there = torch.nonzero(lens).view(-1)
    first, last = starts[there], starts[there + 1] - 1
    a, rest = torch.sigmoid(f), torch.sigmoid(-f)                    # 1 - a by itself: it may be far below a's last place
    if c["form"] == "mix":
        k, dk = rest, -a * rest
    elif c["form"] == "unit":
        k, dk = torch.sqrt(rest * (1 + a)), -a * a * torch.sqrt(rest / (1 + a))
    else:
        k, dk = torch.ones_like(a), torch.zeros_like(a)
    u, carried = k * x, a.clone()
    u[first] += a[first] * s["h0"][there]
    carried[first] = 0
    h = _follow(carried, u, s["longest"])
    h_end = s["h0"].clone()
    h_end[there] = h[last]
    g, dg = _act(s["g"][:n].to(f32), c["act"]) if c["act"] else (None, None)
    y = torch.zeros(c["rows"], c["width"], dtype=dt, device=dev)
    y[:n] = (h if g is None else h * g).to(dt)
    out = {"y": y, "h_end": h_end}
    if c["op"] == "scan_train":
        dy = s["dy"][:n].to(f32)
        e = dy if g is None else dy * g
        e = e.clone()
        e[last] += s["dh_end"][there]
        ahead = torch.zeros_like(a)
        ahead[:-1] = carried[1:]
        lam = _follow(ahead.flip(0), e.flip(0), s["longest"]).flip(0)
        back = torch.empty_like(h)
        back[1:] = h[:-1]
        back[first] = s["h0"][there]
        dh0 = s["dh_end"].clone()
        dh0[there] = (a * lam)[first]
        made = {"df": lam * (back * a * rest + x * dk), "dx": lam * k}
        if g is not None:
            made["dg"] = dy * h * dg
        whole = {name: torch.zeros(c["rows"], c["width"], dtype=dt, device=dev) for name in made}
        [whole[name][:n].copy_(v) for name, v in made.items()]
        out.update(whole, dh0=dh0)
    return out


def _plain_logp(s):
    c, dt, f32 = s["case"], _T[s["case"]["dtype"]], torch.float32
    z = s["logits"].to(f32) * c["temper"]
    top = z.amax(1, keepdim=True)
    e = torch.exp(z - top)
    total = e.sum(1, keepdim=True)
    p, lp = e / total, (z - top) - torch.log(total)
    plp = torch.where(p > 0, p * lp, 0.0)
    entropy = -plp.sum(1)
    ids = s["ids"].long()[:, None]
    given = ids >= 0
    out = {"logp": torch.where(given, lp.gather(1, ids.clamp(min=0)), 0.0)[:, 0], "entropy": entropy}
    if c["op"] == "logp_train":
        hit = torch.where(given, s["dlogp"][:, None], 0.0)
        d = -hit * p - s["dentropy"][:, None] * (plp + p * entropy[:, None])
        d.scatter_add_(1, ids.clamp(min=0), hit)
        out["dlogits"] = (d * c["temper"]).to(dt)
    elif c["top"]:
        order = torch.sort(s["logits"], dim=1, descending=True, stable=True)[1][:, :c["top"]]
        out.update(top_ids=order.to(torch.int32), top_logp=lp.gather(1, order))
    return out


def _plain(s):
    return {"join": _plain_join, "drop": _plain_drop, "scan": _plain_scan, "logp": _plain_logp}[s["case"]["op"][:4]](s)


# ---- the framework's calls -----------------------------------------------------------------------------------------
def _calls(s):
    """What a program sets up once for its buffers: argument records, outputs and workspace."""
    import paper_2110_02781_amd as P
    c = s["case"]
    op, dt, rows, code = c["op"], _T[c["dtype"]], c["rows"], P.F32 if c["dtype"] == "f32" else P.BF16
    train = op.endswith("train")
    out = {}

    def new(name, *shape, dtype=dt, zero=False):
        out[name] = (torch.zeros if zero else torch.empty)(*shape, dtype=dtype, device="cuda")
        return out[name]

    def given(a, **kw):
        for k, v in kw.items():
            setattr(a, k, v.data_ptr() if hasattr(v, "data_ptr") else v)

    def ld(name):
        return s[name].stride(0)

    def spaced(a, *needs):
        ws = torch.empty(max(needs), dtype=torch.uint8, device="cuda")
        given(a, ws=ws, ws_bytes=ws.numel())
        return ws

    if op.startswith("drop"):
        d = c["width"]
        a = P.dropout_args(rows=rows, cols=d, dtype=code, p=c["drop"], **s["mask"], x=s["x"], ldx=ld("x"), residual=s["r"], ldr=ld("r"), y=new("y", rows, d), ldy=d,
                           dy=s["dy"], lddy=ld("dy"), dx=new("dx", rows, d), lddx=d)
        return [(P.dropout_forward, a), (P.dropout_backward, a)], out, None
    if op.startswith("join"):
        d, f32 = c["width"], torch.float32
        a = P.join_args(rows=rows, width=d, dtype=code, norm=P.NORM_LAYER if c["norm"] == "layer" else P.NORM_RMS, post=int(c["post"]), eps=_EPS, scale=s["scale"], p=c["drop"],
                        **s["mask"], x=s["x"], ldx=ld("x"), b=s["b"], ldb=ld("b"), y=new("y", rows, d), ldy=d, n=new("n", rows, d), ldn=d)
        given(a, **{k: s[k] for k in ("pre_w", "pre_bias", "post_w", "post_bias") if k in s})
        if "gate" in s:
            given(a, gate=s["gate"], ldg=d, gate_rows=1 if c["gate"] == "row" else c.get("gate_rows", rows), gate_dtype=P.F32 if s["gate"].dtype == f32 else P.BF16)
        if not train:
            return [(P.join_forward, a)], out, None
        given(a, dy=s["dy"], lddy=ld("dy"), dn=s["dn"], lddn=ld("dn"), dx=new("dx", rows, d), lddx=d, db=new("db", rows, d), lddb=d)
        given(a, **{"d" + k: new("d" + k, d, dtype=f32) for k in ("pre_w", "pre_bias", "post_w", "post_bias") if k in s})
        if "gate" in s:
            given(a, dgate=new("dgate", *s["gate"].shape, dtype=s["gate"].dtype), lddg=d)
        return [(P.join_forward, a), (P.join_backward, a)], out, spaced(a, P.join_workspace(a))
    if op.startswith("scan"):
        d, n = c["width"], s["h0"].shape[0]
        forms, acts = {"add": P.SCAN_ADD, "mix": P.SCAN_MIX, "unit": P.SCAN_UNIT}, {"": 0, "none": P.ACT_NONE, "silu": P.ACT_SILU, "gelu": P.ACT_GELU}
        a = P.scan_args(rows=rows, width=d, seqs=n, dtype=code, form=forms[c["form"]], act=acts[c["act"]], f=s["f"], ldf=ld("f"), x=s["x"], ldx=ld("x"), h0=s["h0"], ldh0=d,
                        y=new("y", rows, d, zero=c["behind"] > 0), ldy=d, h_end=new("h_end", n, d, dtype=torch.float32), ldhe=d)
        if c["cut"]:
            given(a, starts=s["starts"])
        else:
            a.length = rows // n
        if c["act"]:
            given(a, g=s["g"], ldg=ld("g"))
        if not train:
            return [(P.scan_forward, a)], out, spaced(a, P.scan_workspace(a, False))
        zero = c["behind"] > 0
        given(a, dy=s["dy"], lddy=ld("dy"), dh_end=s["dh_end"], lddhe=d, df=new("df", rows, d, zero=zero), lddf=d, dx=new("dx", rows, d, zero=zero), lddx=d,
              dh0=new("dh0", n, d, dtype=torch.float32), lddh0=d)
        if c["act"]:
            given(a, dg=new("dg", rows, d, zero=zero), lddg=d)
        return [(P.scan_forward, a), (P.scan_backward, a)], out, spaced(a, P.scan_workspace(a, False), P.scan_workspace(a, True))
    v, f32 = c["vocab"], torch.float32
    a = P.logp_args(rows=rows, vocab=v, dtype=code, scale=c["temper"], logits=s["logits"], ldl=ld("logits"), ids=s["ids"], logp=new("logp", rows, dtype=f32),
                    entropy=new("entropy", rows, dtype=f32))
    if c["top"]:
        given(a, top=c["top"], top_ids=new("top_ids", rows, c["top"], dtype=torch.int32), top_logp=new("top_logp", rows, c["top"], dtype=f32))
    if not train:
        return [(P.logp_forward, a)], out, spaced(a, P.logp_workspace(a))
    stats = torch.empty(rows, 2, dtype=f32, device="cuda")
    given(a, stats=stats, dlogp=s["dlogp"], dentropy=s["dentropy"], dlogits=new("dlogits", rows, v), lddl=v)
    return [(P.logp_forward, a), (P.logp_backward, a)], out, (stats, spaced(a, P.logp_workspace(a)))


def run(state):
    if not own:
        return _plain(state)
    if "calls" not in state:
        state["calls"] = _calls(state)
    calls, out, _ = state["calls"]
    stream = torch.cuda.current_stream().cuda_stream
    for call, args in calls:
        call(args, stream)
    return out


# ---- what a pass cannot do without ---------------------------------------------------------------------------------
def work(case):
    es, rows, op = 4 if case["dtype"] == "f32" else 2, case["rows"], case["op"]
    if op.startswith("logp"):
        n = rows * case["vocab"]
        if op == "logp_train":
            return {"bytes": 2 * es * n + 24 * rows, "flops": 16 * n}
        return {"bytes": es * n + (12 + 8 * case["top"]) * rows, "flops": 8 * n}
    n, train = rows * case["width"], op.endswith("train")
    if op.startswith("drop"):
        return {"bytes": 5 * es * n, "flops": 4 * n}
    if op.startswith("scan"):
        gated = 1 if case["act"] else 0
        state = 4 * case["width"] * case["seqs"]
        return {"bytes": es * n * (3 + gated + (3 + gated if train else 0)) + state * (4 if train else 2), "flops": (40 if train else 12) * n}
    groups = {"none": 0, "row": rows, "group": -(-rows // case.get("gate_rows", 1)), "all": 1}[case["gate"]] * case["width"] * (4 if case["gate"] == "all" else es)
    weights = 4 * case["width"] * (2 if case["norm"] == "layer" else 1) * (2 if case["post"] else 1)
    return {"bytes": es * n * (8 if train else 4) + (groups + weights) * (2 if train else 1), "flops": (50 if train else 15) * n}


# ---- the definitions in 64 bits --------------------------------------------------------------------------------------
def _exact_kept(c, mask):
    """The generator once more, its products from halves of sixteen bits."""
    rows, cols, m16, m32 = c["rows"], c["width"], 0xffff, 0xffffffff
    blocks = (cols + 7) // 8

    def times(v, k):
        lo, hi = v & m16, v >> 16
        low, mid = lo * (k & m16), lo * (k >> 16) + hi * (k & m16)        # below 2^33
        t = low + ((mid & m16) << 16)
        return (hi * (k >> 16) + (mid >> 16) + (t >> 32)) & m32, t & m32
    at = torch.arange(rows * blocks, device="cuda")
    row = at // blocks + mask["row0"]
    x0, x1, x2, x3 = at % blocks, torch.full_like(at, mask["site"]), row % (1 << 32), row // (1 << 32)
    key = [mask["seed"] % (1 << 32), mask["seed"] // (1 << 32)]
    for _ in range(10):
        (h0, l0), (h1, l1) = times(x0, 0xD2511F53), times(x2, 0xCD9E8D57)
        x0, x1, x2, x3 = h1 ^ x1 ^ key[0], l1, h0 ^ x3 ^ key[1], l0
        key = [(key[0] + 0x9E3779B9) % (1 << 32), (key[1] + 0xBB67AE85) % (1 << 32)]
    u = torch.empty(rows * blocks, 8, dtype=torch.int32, device="cuda")
    for i, w in enumerate((x0, x1, x2, x3)):
        u[:, 2 * i], u[:, 2 * i + 1] = (w & m16).int(), (w >> 16).int()
    least = round(c["drop"] * 65536)
    keep = (u.view(rows, blocks * 8)[:, :cols] >= least).double()
    return keep / (1 - least / 65536)


def _exact_norm(v, kind):
    if kind == "rms":
        return v / ((v ** 2).sum(1, keepdim=True) / v.shape[1] + _EPS).sqrt()
    m = v.sum(1, keepdim=True) / v.shape[1]
    return (v - m) / (((v - m) ** 2).sum(1, keepdim=True) / v.shape[1] + _EPS).sqrt()


def _exact_join(c, s):
    f64 = torch.float64
    leaf = {k: s[k].to(f64).contiguous() for k in ("x", "b", "gate", "pre_w", "pre_bias", "post_w", "post_bias") if k in s}
    train = c["op"] == "join_train"
    for t in leaf.values():
        t.requires_grad_(train)
    factor = s["scale"] * (_exact_kept(c, s["mask"]) if c["drop"] else 1.0)
    branch = leaf["b"]
    if c["post"]:
        branch = _exact_norm(branch, c["norm"]) * leaf["post_w"] + leaf.get("post_bias", 0)
    if "gate" in leaf:
        each = {"row": 1, "group": c.get("gate_rows", 1), "all": c["rows"]}[c["gate"]]
        branch = branch * leaf["gate"].repeat_interleave(each, 0)[:c["rows"]]
    y = leaf["x"] + factor * branch
    n = _exact_norm(y, c["norm"]) * leaf["pre_w"] + leaf.get("pre_bias", 0)
    out = {"y": y.detach(), "n": n.detach()}
    if train:
        torch.autograd.backward([y, n], [s["dy"].to(f64), s["dn"].to(f64)])
        out.update({"d" + k: t.grad for k, t in leaf.items()})
    return out


def _exact_act(z, act):
    if act == "none":
        return z, z * 0 + 1
    if act == "silu":
        e = torch.exp(-z.abs())
        p = torch.where(z >= 0, 1 / (1 + e), e / (1 + e))
        return z * p, p + z * p * (1 - p)
    k0, k1 = math.sqrt(2 / math.pi), 0.044715
    p = torch.sigmoid(2 * k0 * (z + k1 * z ** 3))
    return z * p, p + z * p * (1 - p) * 2 * k0 * (1 + 3 * k1 * z ** 2)


def _exact_scan(c, s):
    """Row by row through all sequences at once, those of the most rows first."""
    f64, lens = torch.float64, _lengths(c)
    order = sorted(range(len(lens)), key=lambda i: -lens[i])
    at = [sum(lens[:i]) for i in range(len(lens))]
    place = torch.tensor([at[i] for i in order], device="cuda")
    seq = torch.tensor(order, device="cuda")
    many = [sum(1 for n in lens if n > t) for t in range(max(lens))] if len(lens) < 500 else [len(lens)] * max(lens)
    f, x = s["f"].to(f64), s["x"].to(f64)
    e = torch.exp(-f.abs())
    a = torch.where(f >= 0, 1 / (1 + e), e / (1 + e))
    rest = torch.where(f >= 0, e / (1 + e), 1 / (1 + e))
    k = {"add": torch.ones_like(a), "mix": rest, "unit": (rest + rest * a).sqrt()}[c["form"]]
    u = k * x
    before, h = torch.zeros_like(u), torch.zeros_like(u)
    state = s["h0"].to(f64)[seq]
    for t, m in enumerate(many):
        r = place[:m] + t
        before[r] = state[:m]
        state[:m] = torch.addcmul(u[r], a[r], state[:m])
        h[r] = state[:m]
    h_end = torch.empty_like(state)
    h_end[seq] = state
    n = c["rows"] - c["behind"]
    g, dg = _exact_act(s["g"].to(f64), c["act"]) if c["act"] else (1.0, None)
    out = {"y": h * g, "h_end": h_end}
    out["y"][n:] = 0
    if c["op"] == "scan_train":
        dy = s["dy"].to(f64)
        into, lam = dy * g, torch.zeros_like(u)
        back = s["dh_end"].to(f64)[seq]
        for t in range(len(many) - 1, -1, -1):
            m = many[t]
            r = place[:m] + t
            here = into[r] + back[:m]
            lam[r] = here
            back[:m] = here * a[r]
        dh0 = torch.empty_like(back)
        dh0[seq] = back
        slope = a * rest
        dk = {"add": 0 * a, "mix": -slope, "unit": -a * slope / k.clamp(min=1e-300)}[c["form"]]
        out.update(df=lam * (before * slope + x * dk), dx=lam * k, dh0=dh0)
        if c["act"]:
            out["dg"] = dy * h * dg
            out["dg"][n:] = 0
    return out


def _exact_logp(c, s):
    z = s["logits"].to(torch.float64) * c["temper"]
    lp = torch.log_softmax(z, 1)
    del z
    rows = torch.arange(c["rows"], device="cuda")
    ids = s["ids"].long()
    logp = torch.where(ids < 0, 0.0, lp[rows, ids.clamp(min=0)])
    entropy = torch.special.entr(lp.exp()).sum(1)
    out = {"logp": logp, "entropy": entropy}
    if c["op"] == "logp_train":
        w = torch.where(ids < 0, 0.0, s["dlogp"].double())
        d = lp.clamp(min=-1e4).add_(entropy[:, None]).mul_(s["dentropy"].double()[:, None]).add_(w[:, None]).mul_(-lp.exp_())
        d[rows, ids.clamp(min=0)] += w
        out["dlogits"] = d.mul_(c["temper"])
    elif c["top"]:
        out["top_ids"] = torch.argsort(s["logits"], dim=1, descending=True, stable=True)[:, :c["top"]].int()
        out["top_logp"] = lp.gather(1, out["top_ids"].long())
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"].startswith("drop"):
        k = _exact_kept(case, s["mask"])
        return {"y": s["x"].to(torch.float64) * k + s["r"].to(torch.float64), "dx": s["dy"].to(torch.float64) * k}
    return {"join": _exact_join, "scan": _exact_scan, "logp": _exact_logp}[case["op"][:4]](case, s)
