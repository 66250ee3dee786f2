"""A token model trained as pipeline stages train: a table, gated feed-forward blocks and a head, two micro-batches in flight whose activations are
held in 8 bits, weight gradients accumulated in fp32, then one token at a time through the trained weights.

What a batch in flight holds between its forward and its backward is its ids, its logits, and in 8 bits every block's gate and up rows and input and the head's
input; the bfloat16 rows that go from unit to unit, their gradients and the workspace are the stage's, there once whichever batch is at work.

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


class Rows:
    """What passes from unit to unit, two buffers in turn: activations and (for training) their gradients."""

    def __init__(self, m, rows, train=True):
        self.x = [dev(rows, m.width) for _ in range(2)]
        self.dx = [dev(rows, m.width) for _ in range(2)] if train else []
        self.ws = None

    def space(self, n):
        """at least n bytes of workspace, the same for all calls: they follow one another on one stream"""
        if self.ws is None or self.ws.numel() < n:
            self.ws = dev(max(n, 1), dtype=torch.uint8)
        return self.ws


class Slot:
    """One batch in flight: its stash and the calls' records, made once."""

    def __init__(self, m, rows, between, train=True):
        d, f, v, n = m.width, m.hidden, m.vocab, len(m.blocks)
        groups = lambda k: -(-k // 32)  # noqa: E731
        self.rows, self.train = rows, train
        self.ids, self.labels = dev(rows, dtype=torch.int32), dev(rows, dtype=torch.int32)
        self.logits, self.loss = dev(rows, v), torch.zeros(1, device="cuda")
        self.keep = []

        def held(k):
            q, s = dev(rows, k, dtype=torch.uint8), dev(rows, groups(k), dtype=torch.uint8)
            self.keep += [q, s]
            return q.data_ptr(), s.data_ptr()
        x, dx = [between.x[i % 2] for i in range(n + 1)], between.dx
        self.embed = P.embed_args(rows=rows, vocab=v, width=d, dtype=P.BF16, scale=d ** 0.5, ids=self.ids, table=m.table.work, ldt=d, out=x[0], ldo=d)
        self.blocks = []
        for i, b in enumerate(m.blocks):
            a = P.ffn_args(rows=rows, width=d, hidden=f, dtype=P.BF16, act=P.ACT_SILU, x=x[i], ldx=d, w_gate=b["gate"].work, ldwg=d, w_up=b["up"].work, ldwu=d,
                           w_down=b["down"].work, ldwd=f, residual=x[i], ldr=d, y=x[i + 1], ldy=d)
            if train:
                a.save = P.SAVE_ACT8
                (a.gate, a.gate_scales), (a.up, a.up_scales) = held(f), held(f)
            self.blocks.append(a)
        self.head = P.linear_args(rows=rows, n_in=d, n_out=v, dtype=P.BF16, x=x[n], ldx=d, w=m.head.work, ldw=d, bias=m.bias, y=self.logits, ldy=v)
        calls, most = [self.embed, *self.blocks, self.head], max([P.linear_workspace(self.head)] + [P.ffn_workspace(a) for a in self.blocks])
        if train:
            # the inputs of the blocks and of the head, in 8 bits: the backward's records read these instead of the rows, which the next unit but one overwrites
            self.pack = []
            for rows_in in x:
                q, s = held(d)
                self.pack.append(P.act8_args(rows=rows, cols=d, dtype=P.BF16, x=rows_in, ldx=d, q=q, ldq=d, scales=s, lds=groups(d)))
            self.dlogits = dev(rows, v)
            self.head_back = self.from_stash(self.head, n, self.dlogits, v, dx[n % 2], dw=m.head.grad, dbias=m.bias_grad)
            self.blocks_back = [self.from_stash(a, i, dx[(i + 1) % 2], d, dx[i % 2], dx_residual=1, dw_gate=b["gate"].grad, dw_up=b["up"].grad, dw_down=b["down"].grad)
                                for i, (a, b) in enumerate(zip(self.blocks, m.blocks))]
            e = self.embed
            e.dy, e.lddy, e.dtable, e.lddt, e.accumulate = dx[0].data_ptr(), d, m.table.grad.data_ptr(), d, 1
            calls += [self.head_back, *self.blocks_back]
            most = max([most, P.linear_workspace(self.head_back, True), P.embed_backward_workspace(e)] + [P.ffn_workspace(a, True) for a in self.blocks_back])
        ws = between.space(most)
        self.keep.append(ws)
        for a in calls:
            a.ws, a.ws_bytes = ws.data_ptr(), ws.numel()

    def from_stash(self, record, unit, dy, lddy, dx, **gradients):
        """the backward's record of a unit: its input as the slot holds it, its gradients added to what is there"""
        a, p = type(record).from_buffer_copy(record), self.pack[unit]
        a.x, a.ldx, a.x_scales, a.ldxs = p.q, p.ldq, p.scales, p.lds
        a.dy, a.lddy, a.dx, a.lddx, a.accumulate = dy.data_ptr(), lddy, dx.data_ptr(), p.cols, 1
        for name, g in gradients.items():
            setattr(a, name, g.data_ptr() if hasattr(g, "data_ptr") else g)
        return a

    def forward(self, stream):
        P.embed_forward(self.embed, stream)
        for i, a in enumerate(self.blocks):
            if self.train:
                P.act8_pack(self.pack[i], stream)
            P.ffn_forward(a, stream)
        if self.train:
            P.act8_pack(self.pack[-1], stream)
        P.linear_forward(self.head, stream)

    def backward(self, stream):
        P.softmax_ce_static(self.logits, self.labels, self.rows, self.logits.shape[1], P.BF16, self.dlogits, self.loss, stream)
        P.linear_backward(self.head_back, stream)
        for a in reversed(self.blocks_back):
            P.ffn_backward(a, stream)
        P.embed_backward(self.embed, stream)


def train(steps=60, rows=512, lr=0.2, verbose=True):
    """-> (model, the permutation, the losses): two micro-batches in flight per update, as a stage with a successor has"""
    m = Model()
    gen = torch.Generator(device="cuda").manual_seed(2)
    behind = torch.randperm(m.vocab, generator=gen, device="cuda").to(torch.int32)
    between = Rows(m, rows)
    slots = [Slot(m, rows, between) for _ in range(2)]
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
    s = Slot(m, 1, Rows(m, 1, train=False), train=False)
    stream, got = torch.cuda.current_stream().cuda_stream, []
    s.ids.fill_(first)
    for _ in range(n):
        s.forward(stream)
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
