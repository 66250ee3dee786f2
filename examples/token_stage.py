"""A token model trained as pipeline stages train: a table, gated feed-forward blocks and a head, two micro-batches in flight whose activations are
held in 8 bits, weight gradients accumulated in fp32, then one token at a time through the trained weights.

The task is a fixed permutation of the vocabulary (the token behind each token), so that a model without attention can learn it.

    python examples/token_stage.py            # needs an MI355X
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2110_02781_amd as P  # noqa: E402

BF = torch.bfloat16


def dev(*shape, dtype=BF):
    return torch.empty(*shape, dtype=dtype, device="cuda")


class Weight:
    """fp32 master, its accumulated gradient, and the bfloat16 copy that the products read"""

    def __init__(self, gen, rows, cols, std):
        self.master = torch.randn(rows, cols, generator=gen, device="cuda") * std
        self.grad = torch.zeros_like(self.master)
        self.velocity = torch.zeros_like(self.master)
        self.work = self.master.to(BF)

    def update(self, lr, momentum=0.9):
        self.velocity.mul_(momentum).add_(self.grad)
        self.master.add_(self.velocity, alpha=-lr)
        self.grad.zero_()
        self.work.copy_(self.master)


class Model:
    def __init__(self, vocab=512, width=256, hidden=704, blocks=2, seed=1):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.vocab, self.width, self.hidden = vocab, width, hidden
        self.table = Weight(gen, vocab, width, width ** -0.5)
        self.blocks = [dict(gate=Weight(gen, hidden, width, width ** -0.5), up=Weight(gen, hidden, width, width ** -0.5),
                            down=Weight(gen, width, hidden, hidden ** -0.5)) for _ in range(blocks)]
        self.head = Weight(gen, vocab, width, width ** -0.5)
        self.bias = torch.zeros(vocab, device="cuda")
        self.bias_grad = torch.zeros(vocab, device="cuda")

    def weights(self):
        return [self.table, self.head] + [w for b in self.blocks for w in b.values()]


class Slot:
    """One batch in flight: its buffers, its stash and the calls' records, made once."""

    def __init__(self, m, rows, train=True):
        d, f, v, self.rows = m.width, m.hidden, m.vocab, rows
        groups = lambda n: -(-n // 32)  # noqa: E731
        self.ids, self.labels = dev(rows, dtype=torch.int32), dev(rows, dtype=torch.int32)
        self.x = [dev(rows, d) for _ in range(len(m.blocks) + 1)]
        self.logits, self.loss = dev(rows, v), torch.zeros(1, device="cuda")
        keep = self.keep = []
        self.embed = P.embed_args(rows=rows, vocab=v, width=d, dtype=P.BF16, scale=d ** 0.5, ids=self.ids, table=m.table.work, ldt=d, out=self.x[0], ldo=d)
        self.ffn = []
        for i, b in enumerate(m.blocks):
            a = P.ffn_args(rows=rows, width=d, hidden=f, dtype=P.BF16, act=P.ACT_SILU, x=self.x[i], ldx=d, w_gate=b["gate"].work, ldwg=d, w_up=b["up"].work,
                           ldwu=d, w_down=b["down"].work, ldwd=f, residual=self.x[i], ldr=d, y=self.x[i + 1], ldy=d)
            if train:
                gate, up, gs, us = dev(rows, f, dtype=torch.uint8), dev(rows, f, dtype=torch.uint8), dev(rows, groups(f), dtype=torch.uint8), dev(rows, groups(f), dtype=torch.uint8)
                keep += [gate, up, gs, us]
                a.save, a.gate, a.up, a.gate_scales, a.up_scales = P.SAVE_ACT8, gate.data_ptr(), up.data_ptr(), gs.data_ptr(), us.data_ptr()
                a.dw_gate, a.dw_up, a.dw_down = (b[k].grad.data_ptr() for k in ("gate", "up", "down"))
                a.accumulate, a.dx_residual = 1, 1
            self.ffn.append(a)
        self.out = P.linear_args(rows=rows, n_in=d, n_out=v, dtype=P.BF16, x=self.x[-1], ldx=d, w=m.head.work, ldw=d, bias=m.bias, y=self.logits, ldy=v)
        ws = max([P.linear_workspace(self.out)] + [P.ffn_workspace(a) for a in self.ffn])
        if train:
            # what the forward leaves for the backward of a block besides gate and up is its input: held in 8 bits too, so that the bfloat16 rows can go
            self.pack = []
            for x in self.x[:-1]:
                q, s = dev(rows, d, dtype=torch.uint8), dev(rows, groups(d), dtype=torch.uint8)
                keep += [q, s]
                self.pack.append(P.act8_args(rows=rows, cols=d, dtype=P.BF16, x=x, ldx=d, q=q, ldq=d, scales=s, lds=groups(d)))
            self.dlogits, self.dx = dev(rows, v), [dev(rows, d) for _ in range(2)]
            o = self.out
            o.dy, o.lddy, o.dx, o.lddx, o.dw, o.dbias, o.accumulate = self.dlogits.data_ptr(), v, self.dx[0].data_ptr(), d, m.head.grad.data_ptr(), m.bias_grad.data_ptr(), 1
            ws = max([ws, P.linear_workspace(o, True)] + [P.ffn_workspace(self.backward_record(i), True) for i in range(len(self.ffn))])
            e = self.embed
            e.lddy, e.dy, e.dtable, e.lddt, e.accumulate = d, self.dx[len(self.ffn) % 2].data_ptr(), m.table.grad.data_ptr(), d, 1
            ws = max(ws, P.embed_backward_workspace(e))
        self.ws = dev(ws + 1, dtype=torch.uint8)
        for a in [self.embed, self.out, *self.ffn]:
            a.ws, a.ws_bytes = self.ws.data_ptr(), ws

    def backward_record(self, i):
        """the block's record with its input in 8 bits and the gradients' places"""
        a, p, d = type(self.ffn[i]).from_buffer_copy(self.ffn[i]), self.pack[i], self.x[0].shape[1]
        n = len(self.ffn) - 1 - i
        a.x, a.ldx, a.x_scales, a.ldxs = p.q, d, p.scales, p.lds
        a.dy, a.lddy, a.dx, a.lddx = self.dx[n % 2].data_ptr(), d, self.dx[(n + 1) % 2].data_ptr(), d
        return a

    def forward(self, stream, train=True):
        P.embed_forward(self.embed, stream)
        for i, a in enumerate(self.ffn):
            P.ffn_forward(a, stream)
            if train:
                P.act8_pack(self.pack[i], stream)
        P.linear_forward(self.out, stream)

    def backward(self, stream):
        P.softmax_ce_static(self.logits, self.labels, self.rows, self.logits.shape[1], P.BF16, self.dlogits, self.loss, stream)
        P.linear_backward(self.out, stream)
        for i in reversed(range(len(self.ffn))):
            P.ffn_backward(self.backward_record(i), stream)
        P.embed_backward(self.embed, stream)


def train(steps=60, rows=512, lr=0.2, verbose=True):
    """-> (model, the permutation, the losses): two micro-batches in flight per update, as a stage with a successor has"""
    m = Model()
    gen = torch.Generator(device="cuda").manual_seed(2)
    behind = torch.randperm(m.vocab, generator=gen, device="cuda").to(torch.int32)
    slots = [Slot(m, rows) for _ in range(2)]
    stream, losses = torch.cuda.current_stream().cuda_stream, []
    for step in range(steps):
        for s in slots:
            s.ids.copy_(torch.randint(0, m.vocab, (rows,), generator=gen, device="cuda"))
            s.labels.copy_(behind[s.ids.long()])
            s.forward(stream)
        for s in slots:
            s.backward(stream)
        for w in m.weights():
            w.update(lr / len(slots))
        m.bias.add_(m.bias_grad, alpha=-lr / len(slots))
        m.bias_grad.zero_()
        losses.append(float(sum(s.loss for s in slots)) / len(slots))
        if verbose and step % 10 == 0:
            print(f"step {step}: loss {losses[-1]:.4f}", flush=True)
    return m, behind, losses


def follow(m, first, n):
    """n tokens from `first` on, one at a time"""
    s = Slot(m, 1, train=False)
    stream, got = torch.cuda.current_stream().cuda_stream, []
    s.ids.fill_(first)
    for _ in range(n):
        s.forward(stream, train=False)
        s.ids.copy_(s.logits.argmax(1))
        got.append(int(s.ids))
    return got


if __name__ == "__main__":
    model, behind, losses = train()
    tokens = follow(model, 3, 32)
    want, t = [], 3
    for _ in tokens:
        t = int(behind[t])
        want.append(t)
    print(f"loss {losses[0]:.3f} -> {losses[-1]:.4f}; {sum(a == b for a, b in zip(tokens, want))} of {len(want)} tokens followed")
