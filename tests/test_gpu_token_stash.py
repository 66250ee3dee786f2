"""The example's batches in flight: what a slot's backward reads is the slot's own, in 8 bits, whatever went through the stage since."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu


def test_a_batch_in_flight_is_held_in_8_bits():
    import torch
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    import token_stage as T
    rows, m = 96, T.Model()
    between = T.Rows(m, rows)
    a, b = (T.Slot(m, rows, between) for _ in range(2))
    stream = torch.cuda.current_stream().cuda_stream
    gen = torch.Generator(device="cuda").manual_seed(4)
    for s in (a, b):
        s.ids.copy_(torch.randint(0, m.vocab, (rows,), generator=gen, device="cuda"))
        s.labels.copy_(torch.randint(0, m.vocab, (rows,), generator=gen, device="cuda"))

    def gradients(other):
        for w in m.weights():
            w.grad.zero_()
        m.bias_grad.zero_()
        a.forward(stream)
        if other:
            b.forward(stream)
            for t in (*between.x, *between.dx, between.ws):      # nothing of the stage's own is read by the backward
                t.fill_(1)
        a.backward(stream)
        torch.cuda.synchronize()
        return [w.grad.clone() for w in m.weights()] + [m.bias_grad.clone()]
    first, second = gradients(False), gradients(True)
    assert all(bool(g.isfinite().all()) and bool(g.any()) for g in first)
    assert all(torch.equal(x, y) for x, y in zip(first, second))
    n, d, f = len(m.blocks), m.width, m.hidden
    stash = sum(t.numel() * t.element_size() for t in a.keep if t is not between.ws)
    assert stash == rows * (2 * n * (f + -(-f // 32)) + (n + 1) * (d + -(-d // 32)))             # a byte a value and one for 32 of them
