"""A token model with memory: a table, a block that mixes along the sequences by a gated recurrence, a gated feed-forward block and a head, with norms, gates and dropout between them.
Trained on packed sequences of different lengths, then asked token by token, each request with its own state.

The task is to remember: the first token of a sequence comes up again as its last, between them are others.

    python examples/token_memory.py            # needs an MI355X
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2110_02781_amd as P  # noqa: E402

TYPES = {"f32": (torch.float32, P.F32), "bf16": (torch.bfloat16, P.BF16)}


class Weight:
    """fp32 master, its accumulated gradient, and (for matrices) the copy in the model's type that the products read"""

    def __init__(self, value, dtype):
        self.master, self.grad, self.velocity = value, torch.zeros_like(value), torch.zeros_like(value)
        self.work = value.to(dtype) if value.dim() == 2 else value

    def update(self, lr, momentum=0.9):
        self.velocity.mul_(momentum).add_(self.grad)
        self.master.add_(self.velocity, alpha=-lr)
        self.grad.zero_()
        if self.work is not self.master:
            self.work.copy_(self.master)


class Model:
    def __init__(self, vocab=24, width=128, hidden=256, drop=0.05, dtype="bf16", seed=1):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.vocab, self.width, self.hidden, self.drop = vocab, width, hidden, drop
        self.dtype, self.code = TYPES[dtype]

        def matrix(n, m):
            return Weight(torch.randn(n, m, generator=gen, device="cuda") * m ** -0.5, self.dtype)

        def vector(n, mean):
            return Weight(mean + 0.05 * torch.randn(n, generator=gen, device="cuda"), self.dtype)
        d = width
        self.w = dict(table=matrix(vocab, d), mix_in=matrix(3 * d, d), mix_out=matrix(d, d), gate=matrix(hidden, d), up=matrix(hidden, d), down=matrix(d, hidden), head=matrix(vocab, d),
                      mix_bias=vector(3 * d, 0.0), norm0=vector(d, 1.0), norm1=vector(d, 1.0), norm2=vector(d, 1.0), post1=vector(d, 1.0), post2=vector(d, 1.0), scale1=vector(d, 1.0),
                      scale2=vector(d, 1.0))
        self.w["mix_bias"].master[:d] += 3.0                        # to begin with, remember some twenty tokens


class Run:
    """The calls of a batch of `rows` tokens in `seqs` sequences (starts: where they begin; None: one token each), their records made once."""

    def __init__(self, m, rows, seqs, starts=None, train=True, top=0):
        d, f, v, w, dt = m.width, m.hidden, m.vocab, m.w, m.code
        self.m, self.train, self.keep = m, train, [starts]

        def new(*shape, dtype=m.dtype):
            self.keep.append(torch.empty(*shape, dtype=dtype, device="cuda"))
            return self.keep[-1]
        self.ids, self.targets = new(rows, dtype=torch.int32), new(rows, dtype=torch.int32)
        self.seed = torch.zeros(1, dtype=torch.int64, device="cuda")          # of the dropout masks: changed in place, also between replays of a captured step
        x0, n0, mix, s, o1 = new(rows, d), new(rows, d), new(rows, 3 * d), new(rows, d), new(rows, d)
        x1, n1, o2, x2, n2 = (new(rows, d) for _ in range(5))
        self.logits, self.state = new(rows, v), torch.zeros(seqs, d, device="cuda")
        self.logp, self.entropy = new(rows, dtype=torch.float32), new(rows, dtype=torch.float32)
        self.top_ids, self.top_logp = (new(rows, top, dtype=torch.int32), new(rows, top, dtype=torch.float32)) if top else (None, None)
        drop = dict(p=m.drop if train else 0.0, seed_dev=self.seed)
        self.embed = P.embed_args(rows=rows, vocab=v, width=d, dtype=dt, scale=d ** 0.5, ids=self.ids, table=w["table"].work, ldt=d, out=x0, ldo=d)
        self.join0 = P.join_args(rows=rows, width=d, dtype=dt, x=x0, ldx=d, n=n0, ldn=d, pre_w=w["norm0"].work)
        # the recurrence's three inputs are columns of one product
        self.mix_in = P.linear_args(rows=rows, n_in=d, n_out=3 * d, dtype=dt, x=n0, ldx=d, w=w["mix_in"].work, ldw=d, bias=w["mix_bias"].work, y=mix, ldy=3 * d)
        self.scan = P.scan_args(rows=rows, width=d, seqs=seqs, length=0 if starts is not None else rows // seqs, starts=0 if starts is None else starts, dtype=dt, form=P.SCAN_UNIT,
                                act=P.ACT_SILU, f=mix[:, :d], ldf=3 * d, x=mix[:, d:], ldx=3 * d, g=mix[:, 2 * d:], ldg=3 * d, y=s, ldy=d, h_end=self.state, ldhe=d)
        if not train:
            self.scan.h0, self.scan.ldh0 = self.state.data_ptr(), d
        self.mix_out = P.linear_args(rows=rows, n_in=d, n_out=d, dtype=dt, x=s, ldx=d, w=w["mix_out"].work, ldw=d, y=o1, ldy=d)

        def join(x, b, y, n, post, gate, pre, site):
            return P.join_args(rows=rows, width=d, dtype=dt, post=1, scale=0.5, site=site, x=x, ldx=d, b=b, ldb=d, y=y, ldy=d, n=n, ldn=d, post_w=w[post].work, pre_w=w[pre].work,
                               gate=w[gate].work, ldg=d, gate_rows=max(rows, 1), gate_dtype=P.F32, **drop)
        self.join1 = join(x0, o1, x1, n1, "post1", "scale1", "norm1", 1)
        self.ffn = P.ffn_args(rows=rows, width=d, hidden=f, dtype=dt, act=P.ACT_SILU, x=n1, ldx=d, w_gate=w["gate"].work, ldwg=d, w_up=w["up"].work, ldwu=d, w_down=w["down"].work, ldwd=f,
                              y=o2, ldy=d)
        self.join2 = join(x1, o2, x2, n2, "post2", "scale2", "norm2", 2)
        self.head = P.linear_args(rows=rows, n_in=d, n_out=v, dtype=dt, x=n2, ldx=d, w=w["head"].work, ldw=d, y=self.logits, ldy=v)
        self.score = P.logp_args(rows=rows, vocab=v, dtype=dt, logits=self.logits, ldl=v, ids=self.targets, logp=self.logp, entropy=self.entropy)
        if top:
            self.score.top, self.score.top_ids, self.score.top_logp = top, self.top_ids.data_ptr(), self.top_logp.data_ptr()
        most = max(P.linear_workspace(self.mix_in), P.linear_workspace(self.mix_out), P.linear_workspace(self.head), P.scan_workspace(self.scan), P.logp_workspace(self.score))
        if train:
            put = lambda a, **kw: [setattr(a, k, t.data_ptr() if hasattr(t, "data_ptr") else t) for k, t in kw.items()]           # noqa: E731
            self.dlogp, self.dentropy, self.stats = new(rows, dtype=torch.float32), new(rows, dtype=torch.float32), new(rows, 2, dtype=torch.float32)
            grad = {k: t.grad for k, t in w.items()}
            dlogits, dn2, do2, dx1, dn1, do1, ds, dmix, dn0, dx0, dx2 = new(rows, v), *(new(rows, d) for _ in range(6)), new(rows, 3 * d), *(new(rows, d) for _ in range(3))
            put(self.score, stats=self.stats, dlogp=self.dlogp, dentropy=self.dentropy, dlogits=dlogits, lddl=v)
            put(self.head, dy=dlogits, lddy=v, dx=dn2, lddx=d, dw=grad["head"], accumulate=1)
            put(self.join2, dn=dn2, lddn=d, dx=dx1, lddx=d, db=do2, lddb=d, dgate=grad["scale2"], lddg=d, dpost_w=grad["post2"], dpre_w=grad["norm2"], accumulate=1, gate_accumulate=1)
            g, u = new(rows, f), new(rows, f)
            put(self.ffn, save=P.SAVE_FULL, gate=g, up=u, dy=do2, lddy=d, dx=dn1, lddx=d, dw_gate=grad["gate"], dw_up=grad["up"], dw_down=grad["down"], accumulate=1)
            put(self.join1, dy=dx1, lddy=d, dn=dn1, lddn=d, dx=dx0, lddx=d, db=do1, lddb=d, dgate=grad["scale1"], lddg=d, dpost_w=grad["post1"], dpre_w=grad["norm1"], accumulate=1,
                gate_accumulate=1)
            put(self.mix_out, dy=do1, lddy=d, dx=ds, lddx=d, dw=grad["mix_out"], accumulate=1)
            put(self.scan, dy=ds, lddy=d, df=dmix, lddf=3 * d, dx=dmix[:, d:], lddx=3 * d, dg=dmix[:, 2 * d:], lddg=3 * d)
            put(self.mix_in, dy=dmix, lddy=3 * d, dx=dn0, lddx=d, dw=grad["mix_in"], dbias=grad["mix_bias"], accumulate=1)
            put(self.join0, dy=dx0, lddy=d, dn=dn0, lddn=d, dx=dx2, lddx=d, dpre_w=grad["norm0"], accumulate=1)
            put(self.embed, dy=dx2, lddy=d, dtable=grad["table"], lddt=d, accumulate=1)
            most = max(most, P.ffn_workspace(self.ffn), P.ffn_workspace(self.ffn, True), P.linear_workspace(self.head, True), P.linear_workspace(self.mix_out, True),
                       P.linear_workspace(self.mix_in, True), P.scan_workspace(self.scan, True), P.embed_backward_workspace(self.embed),
                       *(P.join_workspace(j) for j in (self.join0, self.join1, self.join2)))
        else:
            most = max(most, P.ffn_workspace(self.ffn))
        ws = new(max(most, 1), dtype=torch.uint8)
        for a in (self.embed, self.join0, self.mix_in, self.scan, self.mix_out, self.join1, self.ffn, self.join2, self.head, self.score):
            a.ws, a.ws_bytes = ws.data_ptr(), ws.numel()

    def forward(self, stream):
        P.embed_forward(self.embed, stream)
        P.join_forward(self.join0, stream)
        P.linear_forward(self.mix_in, stream)
        P.scan_forward(self.scan, stream)
        P.linear_forward(self.mix_out, stream)
        P.join_forward(self.join1, stream)
        P.ffn_forward(self.ffn, stream)
        P.join_forward(self.join2, stream)
        P.linear_forward(self.head, stream)
        P.logp_forward(self.score, stream)

    def backward(self, stream):
        """of sum(dlogp * logp + dentropy * entropy); gradients are added to the weights'"""
        P.logp_backward(self.score, stream)
        P.linear_backward(self.head, stream)
        P.join_backward(self.join2, stream)
        P.ffn_backward(self.ffn, stream)
        P.join_backward(self.join1, stream)
        P.linear_backward(self.mix_out, stream)
        P.scan_backward(self.scan, stream)
        P.linear_backward(self.mix_in, stream)
        P.join_backward(self.join0, stream)
        P.embed_backward(self.embed, stream)


def batch(gen, vocab, starts):
    """(tokens, targets): the last target of a sequence is its first token, the others (-1) do not count"""
    n = starts[-1]
    ids = torch.randint(0, vocab, (n,), generator=gen, device="cuda", dtype=torch.int32)
    targets = torch.full((n,), -1, dtype=torch.int32, device="cuda")
    first = torch.tensor([a for a, b in zip(starts, starts[1:]) if b > a], device="cuda")
    last = torch.tensor([b - 1 for a, b in zip(starts, starts[1:]) if b > a], device="cuda")
    targets[last] = ids[first]
    return ids, targets


def train(steps=400, seqs=256, longest=8, lr=0.5, verbose=True):
    """-> (model, the losses)"""
    m = Model()
    gen = torch.Generator(device="cuda").manual_seed(2)
    starts = [0]
    for i in range(seqs):
        starts.append(starts[-1] + 2 + i % (longest - 1))
    r = Run(m, starts[-1], seqs, torch.tensor(starts, dtype=torch.int32, device="cuda"))
    stream, losses = torch.cuda.current_stream().cuda_stream, []
    r.dlogp.fill_(-1.0 / seqs)
    r.dentropy.zero_()
    for step in range(steps):
        ids, targets = batch(gen, m.vocab, starts)
        r.ids.copy_(ids)
        r.targets.copy_(targets)
        r.seed.fill_(step)
        r.forward(stream)
        r.backward(stream)
        for w in m.w.values():
            w.update(lr * (1 - step / steps))
        losses.append(-float(r.logp.sum()) / seqs)
        if verbose and step % 50 == 0:
            print(f"step {step}: loss {losses[-1]:.4f}", flush=True)
    return m, losses


def ask(m, prompts, top=3):
    """prompts [requests][tokens] -> (likeliest tokens behind each, their log probabilities): one token a step, the state stays in its place"""
    n, length = prompts.shape
    r = Run(m, n, n, train=False, top=top)
    r.targets.fill_(-1)
    stream = torch.cuda.current_stream().cuda_stream
    for t in range(length):
        r.ids.copy_(prompts[:, t])
        r.forward(stream)
    return r.top_ids, r.top_logp


if __name__ == "__main__":
    model, losses = train()
    prompts = torch.randint(0, model.vocab, (64, 6), device="cuda", dtype=torch.int32)
    ids, logp = ask(model, prompts)
    right = int((ids[:, 0] == prompts[:, 0]).sum())
    print(f"loss {losses[0]:.3f} -> {losses[-1]:.4f}; {right} of {len(prompts)} requests remembered, the likeliest with probability {float(logp[:, 0].exp().mean()):.3f}")
