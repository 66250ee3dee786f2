"""The operators between the products run together, as a model uses them: gradients of a whole model against the formulas' in 64 bits and against differences, captured steps, two streams."""
import math
import os
import sys

import pytest

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def reference(torch, m, w, ids, targets, starts, keep, dlogp, dentropy):
    """the example's model in 64 bits from torch's elementary operations: (loss, logits)"""
    def norm(v, k):
        return v / ((v * v).mean(1, keepdim=True) + 1e-5).sqrt() * w[k]
    d = m.width
    x0 = w["table"][ids.long()] * math.sqrt(d)
    mix = norm(x0, "norm0") @ w["mix_in"].t() + w["mix_bias"]
    a = torch.sigmoid(mix[:, :d])
    u = (torch.sigmoid(-mix[:, :d]) * (1 + a)).sqrt() * mix[:, d:2 * d]
    rows = []
    for b, e in zip(starts, starts[1:]):
        h = torch.zeros(d, dtype=torch.float64, device="cuda")
        for t in range(b, e):
            h = a[t] * h + u[t]
            rows.append(h)
    s = torch.stack(rows) * torch.nn.functional.silu(mix[:, 2 * d:])
    x1 = x0 + 0.5 * w["scale1"] * keep[0] * norm(s @ w["mix_out"].t(), "post1")
    n1 = norm(x1, "norm1")
    h = torch.nn.functional.silu(n1 @ w["gate"].t()) * (n1 @ w["up"].t())
    x2 = x1 + 0.5 * w["scale2"] * keep[1] * norm(h @ w["down"].t(), "post2")
    logits = norm(x2, "norm2") @ w["head"].t()
    lp = torch.log_softmax(logits, 1)
    given = torch.where(targets >= 0, lp.gather(1, targets.long().clamp(min=0)[:, None])[:, 0], 0.0)
    entropy = -(lp.exp() * lp).sum(1)
    return (dlogp.double() * given + dentropy.double() * entropy).sum(), logits


def example(torch, T, B, lens, drop=0.2):
    m = T.Model(vocab=50, width=40, hidden=72, drop=drop, dtype="f32")
    starts = [0]
    for n in lens:
        starts.append(starts[-1] + n)
    r = T.Run(m, starts[-1], len(lens), torch.tensor(starts, dtype=torch.int32, device="cuda"))
    gen = torch.Generator(device="cuda").manual_seed(7)
    ids, targets = T.batch(gen, m.vocab, starts)
    r.ids.copy_(ids)
    r.targets.copy_(targets)
    r.targets[::3] = r.ids[::3]
    r.dlogp.copy_(torch.randn(starts[-1], generator=gen, device="cuda"))
    r.dentropy.copy_(torch.randn(starts[-1], generator=gen, device="cuda"))
    r.seed.fill_(11)
    keep = []
    for site in (1, 2):
        k, up = B.mask(starts[-1], m.width, drop, 11, site, 0)
        keep.append(k.double() * up)
    return m, r, starts, keep


def test_gradients_of_a_whole_model():
    """Every weight's gradient of a model in single precision against autograd's in 64 bits.  Tolerance: the chain has some 300 roundings of 2^-24 from an operand to a gradient (products of up to
    72 terms, sums over 175 rows, eleven operators forward and backward), whose errors are at most their sum, 300 * 2^-24 = 1.8e-5 of the gradient's own size where nothing cancels, ten times that
    where norms and the recurrence's sums do: 2e-4 of a gradient's largest."""
    import torch
    import between_ref as B
    import token_memory as T
    m, r, starts, keep = example(torch, T, B, [5, 40, 0, 1, 90, 39])
    stream = torch.cuda.current_stream().cuda_stream
    w = {k: t.master.double().requires_grad_(True) for k, t in m.w.items()}
    loss, logits = reference(torch, m, w, r.ids, r.targets, starts, keep, r.dlogp, r.dentropy)
    loss.backward()
    r.forward(stream)
    r.backward(stream)
    torch.cuda.synchronize()
    assert float((r.logits.double() - logits).abs().max()) <= 2e-4 * float(logits.abs().max())
    got = float((r.dlogp.double() * r.logp.double() + r.dentropy.double() * r.entropy.double()).sum())
    assert abs(got - float(loss)) <= 2e-4 * (float(r.dlogp.abs().sum()) * 5 + float(r.dentropy.abs().sum()) * 4)
    for k, t in w.items():
        off = (m.w[k].grad.double() - t.grad).abs().max()
        assert float(off) <= 2e-4 * float(t.grad.abs().max()), (k, float(off), float(t.grad.abs().max()))
    # and the formulas' against differences
    eps, gen = 1e-6, torch.Generator(device="cuda").manual_seed(3)
    with torch.no_grad():
        for k, t in w.items():
            v = torch.randn(t.shape, generator=gen, device="cuda", dtype=torch.float64)
            old = t.clone()
            sides = []
            for s in (1, -1):
                t.copy_(old + s * eps * v)
                sides.append(float(reference(torch, m, w, r.ids, r.targets, starts, keep, r.dlogp, r.dentropy)[0]))
            t.copy_(old)
            slope = float((t.grad * v).sum())
            # the differences' own error: the third derivative's eps^2, and 2^-53 of the sums (some 1e2) over eps, 1e-8
            assert abs((sides[0] - sides[1]) / (2 * eps) - slope) <= 1e-6 * (1 + abs(slope)), k


def test_a_captured_step_follows_its_inputs():
    """a training step in a graph, replayed with eager work between: the same bits as the eager step for the same tokens, masks by the seed in memory"""
    import torch
    import between_ref as B
    import token_memory as T
    m, r, starts, _ = example(torch, T, B, [5, 40, 0, 1, 90, 39])
    main = torch.cuda.current_stream().cuda_stream

    def eager(seed, shift):
        r.seed.fill_(seed)
        r.ids.copy_((r.ids + shift) % m.vocab)
        for t in m.w.values():
            t.grad.zero_()
        r.forward(main)
        r.backward(main)
        torch.cuda.synchronize()
        return [r.logp.clone(), r.entropy.clone()] + [t.grad.clone() for t in m.w.values()]
    r.forward(main)
    r.backward(main)
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        s = torch.cuda.current_stream().cuda_stream
        for t in m.w.values():
            t.grad.zero_()
        r.forward(s)
        r.backward(s)
    for seed, shift in ((3, 0), (4, 7), (3, 1), (9, 0)):
        want = eager(seed, shift)
        for t in m.w.values():
            t.grad.fill_(5.0)
        r.logp.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = [r.logp, r.entropy] + [t.grad for t in m.w.values()]
        for a, b in zip(got, want):
            assert torch.equal(a, b)
    assert not torch.equal(eager(3, 0)[0], eager(4, 0)[0])


def test_two_models_on_two_streams():
    """calls that overlap, each with its own workspace, give what they give alone"""
    import torch
    import between_ref as B
    import token_memory as T
    runs = [example(torch, T, B, lens, drop) for lens, drop in (([60, 3, 0, 200], 0.2), ([1] * 40 + [300], 0.4))]
    alone = []
    for m, r, _, _ in runs:
        s = torch.cuda.current_stream().cuda_stream
        r.forward(s)
        r.backward(s)
        torch.cuda.synchronize()
        alone.append([r.logp.clone()] + [t.grad.clone() for t in m.w.values()])
    streams = [torch.cuda.Stream() for _ in runs]
    for _ in range(3):
        for m, r, _, _ in runs:
            for t in m.w.values():
                t.grad.zero_()
        torch.cuda.synchronize()
        for (m, r, _, _), st in zip(runs, streams):
            r.forward(st.cuda_stream)
            r.backward(st.cuda_stream)
        torch.cuda.synchronize()
        for (m, r, _, _), want in zip(runs, alone):
            for a, b in zip([r.logp] + [t.grad for t in m.w.values()], want):
                assert torch.equal(a, b)


def test_token_by_token_is_the_whole_sequence():
    """the states that single tokens leave are those of a call over whole sequences, and so are the answers, in single precision within the recurrence's roundings (some 40 steps of a few 2^-24, through a head of
    40 columns: 1e-4)"""
    import torch
    import token_memory as T
    m = T.Model(vocab=50, width=40, hidden=72, drop=0.0, dtype="f32")
    n, length = 5, 40
    gen = torch.Generator(device="cuda").manual_seed(5)
    prompts = torch.randint(0, m.vocab, (n, length), generator=gen, device="cuda", dtype=torch.int32)
    s = torch.cuda.current_stream().cuda_stream
    whole = T.Run(m, n * length, n, torch.arange(0, n * length + 1, length, dtype=torch.int32, device="cuda"), train=False, top=3)
    whole.ids.copy_(prompts.reshape(-1))
    whole.targets.fill_(-1)
    whole.forward(s)
    ids, logp = T.ask(m, prompts)
    torch.cuda.synchronize()
    last = slice(length - 1, None, length)
    assert float((logp - whole.top_logp[last]).abs().max()) <= 1e-4
    gap = whole.top_logp[last][:, 0] - whole.top_logp[last][:, 1]
    sure = gap > 1e-3
    assert bool(sure.any()) and torch.equal(ids[sure, 0], whole.top_ids[last][sure, 0])


def test_the_example_runs():
    import torch
    import token_memory as T
    m, losses = T.train(steps=3, seqs=10, verbose=False)
    assert len(losses) == 3 and all(math.isfinite(v) for v in losses)
    ids, logp = T.ask(m, torch.zeros(4, 3, dtype=torch.int32, device="cuda"))
    assert ids.shape == (4, 3) and bool(((ids >= 0) & (ids < m.vocab)).all()) and bool((logp <= 0).all())
