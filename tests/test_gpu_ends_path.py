"""A word model's ends together with the vocabulary head: a training step from
words to gradients, and a search over scores from 4-bit weights."""
import importlib.util
import os

import pytest

from ends_util import captured, generator, matrix
from paper_1611_06172_amd import w2v

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
V, D, N, K = 3001, 40, 150, 12


class Model:
    """x = dropout(s E[words]); h = x + gelu(x W^T + b); scores = h E^T + c, the
    embedding and the output matrix being one."""

    def __init__(self, seed=1):
        import torch
        g = generator(seed)
        self.E, self.W = matrix(g, V, D, "float32", 0.3), matrix(g, D, D, "float32", 0.2)
        self.b, self.c = torch.randn(D, generator=g).cuda(), torch.randn(V, generator=g).cuda()

    def step(self, words, ids, values, offset):
        import torch
        drop = dict(p=0.2, seed=7, offset_dev=offset)
        x = w2v.dropout(w2v.embed(words, self.E, scale=D ** 0.5), **drop)
        pre = torch.empty_like(x)
        h = w2v.linear(x, self.W, self.b, activation="gelu", residual=x, pre=pre)
        z = w2v.linear(h, self.E, self.c)
        out = w2v.distill_loss(z, ids, values, temperature=2.0, want_grad=True)
        top = w2v.linear_backward(out["grad"], h, self.E)
        low = w2v.linear_backward(top["dx"], x, self.W, activation="gelu", pre=pre)
        dx = w2v.dropout(top["dx"] + low["dx"], **drop)
        w2v.embed_backward(dx, words, scale=D ** 0.5, grad=top["dw"], accumulate=True)
        return [out["loss"], top["dw"], top["db"], low["dw"], low["db"]]


def batch(g):
    import torch
    words = torch.randint(-1, V, (N,), generator=g, dtype=torch.int32)
    words[::3] = 17
    return (words.cuda(), torch.randint(0, V, (N, K), generator=g, dtype=torch.int32).cuda(),
            torch.randn((N, K), generator=g).cuda())


def test_gradients_of_a_step():
    """Against autograd in 64 bits. Every stage is a chain of fp32 sums of at most
    3,001 terms; 1e-4 of a tensor's largest element is 1,600 units of 2^-24 and
    sums that grow with the root of their length stay below a tenth of it."""
    import torch
    m = Model()
    words, ids, values = batch(generator(2))
    offset = torch.full((1,), 5, dtype=torch.int64, device="cuda")
    got = m.step(words, ids, values, offset)
    keep = (w2v.dropout(torch.ones((N, D), device="cuda"), 0.2, seed=7, offset=5) > 0).cpu()
    E, W, b, c = (t.cpu().double().requires_grad_() for t in (m.E, m.W, m.b, m.c))
    w = words.cpu().long()
    x = E[w.clamp(min=0)] * D ** 0.5 * (w >= 0)[:, None]
    x = x * keep / 0.8
    z = x + torch.nn.functional.gelu(x @ W.t() + b)
    z = z @ E.t() + c
    q = torch.softmax(values.cpu().double() / 2, 1)
    lp = torch.log_softmax(z / 2, 1)
    loss = 4 * (q * (torch.log(q) - torch.gather(lp, 1, ids.cpu().long()))).sum(1)
    loss.sum().backward()
    for have, want in zip(got, (loss.detach(), E.grad, c.grad, W.grad, b.grad)):
        assert (have.cpu().double() - want).abs().max() <= 1e-4 * want.abs().max()


def test_step_replayed_from_a_graph():
    import torch
    m = Model()
    g = generator(3)
    words, ids, values = batch(g)
    offset = torch.zeros(1, dtype=torch.int64, device="cuda")
    graph, held = captured(lambda: m.step(words, ids, values, offset))
    losses = []
    for i in range(4):
        for old, new in zip((words, ids, values), batch(g)):
            old.copy_(new)
        offset.add_(1)
        eager = m.step(words, ids, values, offset)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, eager))
        losses.append(held[0].clone())
    # another number a step: the same inputs lose other elements
    graph.replay()
    assert torch.equal(held[0], losses[-1])
    offset.add_(1)
    graph.replay()
    assert not torch.equal(held[0], losses[-1])


def search(m, scores_of, first, steps, beams, end):
    """Beam search for `steps` words after `first` (batch,): histories and scores."""
    import torch
    n = len(first)
    words = torch.full((n, beams), -1, dtype=torch.int32, device="cuda")
    words[:, 0] = first
    scores = torch.full((n, beams), float("-inf"), device="cuda")
    scores[:, 0] = 0.0
    finished = torch.zeros((n, beams), dtype=torch.uint8, device="cuda")
    hidden = w2v.embed(words.view(-1), m.E, scale=D ** 0.5)
    history = torch.full((n * beams, steps), -1, dtype=torch.int32, device="cuda")
    for i in range(steps):
        h = w2v.linear(hidden, m.W, m.b, activation="tanh")
        out = w2v.beam_step(scores_of(h), scores, finished=finished, end=end)
        hidden, history = w2v.beam_reorder([h, history], out["parents"])
        scores, finished = out["scores"], out["finished"]
        history[:, i] = out["words"].view(-1)
        hidden = w2v.linear(w2v.embed(out["words"].view(-1), m.E), m.W, residual=hidden)
    return history.view(n, beams, steps), scores


def test_search_over_scores_in_4_bits():
    """The beams' scores are the log-probabilities of their histories, followed
    one after the other in 64 bits with the matrix that the 4 bits stand for."""
    import torch
    from test_gpu_linear_q4 import unpacked
    m = Model(4)
    q = w2v.quantize_q4(m.E)
    first = torch.tensor([3, 17, 2999], dtype=torch.int32, device="cuda")
    steps, beams, end = 5, 4, 11
    history, scores = search(m, lambda h: w2v.linear_q4(h, q, m.c), first, steps, beams, end)
    code, scale = unpacked(q)
    Q = ((code.double() - 8) * torch.repeat_interleave(scale.double(), 32, dim=1))[:V, :D]
    E, W, b, c = (t.cpu().double() for t in (m.E, m.W, m.b, m.c))
    for e in range(3):
        assert len(set(tuple(h) for h in history[e].tolist())) == beams
        for k in range(beams):
            hidden, total, ended = E[int(first[e])] * D ** 0.5, 0.0, False
            for word in history[e, k].tolist():
                if ended:
                    assert word == end
                    continue
                h = torch.tanh(W @ hidden + b)
                total += float(torch.log_softmax(Q @ h + c, 0)[word])
                hidden = W @ E[word] + h
                ended = word == end
            # scores of up to some tens, each step's within about 1e-5
            assert abs(total - float(scores[e, k])) <= 1e-3


def test_search_replayed_from_a_graph():
    import torch
    m = Model(5)
    q = w2v.quantize_q4(m.E)
    first = torch.tensor([3, 17, 2999], dtype=torch.int32, device="cuda")
    graph, held = captured(lambda: search(m, lambda h: w2v.linear_q4(h, q, m.c), first, 3, 4, 11))
    for i in range(3):
        first.fill_(100 * i + 1)
        eager = search(m, lambda h: w2v.linear_q4(h, q, m.c), first, 3, 4, 11)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, eager))


def example():
    spec = importlib.util.spec_from_file_location(
        "next_words", os.path.join(ROOT, "examples", "next_words.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_example_runs():
    import torch
    losses, words, scores = example().main(V=500, topics=10, T=20_000, D=48, steps=12, batch=256,
                                           verbose=False)
    assert torch.isfinite(losses).all() and torch.isfinite(scores).all()
    assert words.shape == (4, 4, 6) and (words >= 0).all() and (words < 500).all()
    assert (scores <= 0).all() and (scores[:, 1:] <= scores[:, :-1]).all()


def test_example_gradients():
    """Against autograd in 64 bits, with the mask that the step draws; the bound as
    in test_gradients_of_a_step."""
    import torch
    model = example().Model(400, 40, p=0.3)
    g = generator(8)
    words = torch.randint(-1, 400, (90,), generator=g, dtype=torch.int32)
    labels = torch.randint(-1, 400, (90,), generator=g, dtype=torch.int32)
    model.b.copy_(torch.randn(40, generator=g))
    model.c.copy_(torch.randn(400, generator=g))
    loss, grads = model.gradients(words.cuda(), labels.cuda(), 17)
    keep = (w2v.dropout(torch.ones((90, 40), device="cuda"), 0.3, seed=3, offset=17) > 0).cpu()
    E, W, b, c = (t.cpu().double().requires_grad_() for t in (model.E, model.W, model.b, model.c))
    x = E[words.long().clamp(min=0)] * 40 ** 0.5 * (words >= 0)[:, None] * keep / 0.7
    lp = torch.log_softmax((x + torch.nn.functional.gelu(x @ W.t() + b)) @ E.t() + c, 1)
    want = -lp[torch.arange(90), labels.long().clamp(min=0)] * (labels >= 0)
    want.mean().backward()
    assert (loss.cpu().double() - want.detach()).abs().max() <= 1e-4 * want.max()
    for name, t in (("E", E), ("W", W), ("b", b), ("c", c)):
        assert (grads[name].cpu().double() - t.grad).abs().max() <= 1e-4 * t.grad.abs().max()
