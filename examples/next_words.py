"""A small model of the next word, trained, put into 4 bits and searched.

The words of a corpus of planted topics come in through an embedding with dropout,
one residual layer follows, and the scores are products with the same matrix:

    x = dropout(sqrt(D) E[words]); h = x + gelu(x W^T + b); scores = h E^T + c.

The loss is that of the true next word alone. The gradient of E has two parts, the
scores' matrix product and the rows of the words that came in, which are added to
it. At the end E is held in 4 bits and a beam search continues some words.

    python examples/next_words.py
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_1611_06172_amd import inputs, w2v  # noqa: E402


class Model:
    def __init__(self, V, D, p=0.1, seed=3):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        self.E = w2v.alloc_matrix(V, D, "cuda", torch.randn(
            (V, D), generator=g, device="cuda") * (0.5 / D ** 0.5))
        self.W = torch.randn((D, D), generator=g, device="cuda") / D ** 0.5
        self.b, self.c = torch.zeros(D, device="cuda"), torch.zeros(V, device="cuda")
        self.scale, self.p, self.seed = D ** 0.5, p, seed

    def hidden(self, words, step=None):
        """The layer before the scores of words int32 (n,); with a step's number,
        with its dropout."""
        x = w2v.embed(words, self.E, scale=self.scale)
        if step is not None:
            x = w2v.dropout(x, self.p, seed=self.seed, offset=step)
        pre = torch.empty_like(x)
        return w2v.linear(x, self.W, self.b, activation="gelu", residual=x, pre=pre), x, pre

    def gradients(self, words, labels, step):
        """Losses of the next words `labels` (-1: none), and the gradients of
        their mean."""
        h, x, pre = self.hidden(words, step)
        z = w2v.linear(h, self.E, self.c)
        n = len(words)
        none = torch.empty((n, 0), dtype=torch.int32, device="cuda")
        out = w2v.distill_loss(z, none, none.float(), labels=labels, soft=0.0, hard=1.0,
                               row_weight=torch.full((n,), 1.0 / n, device="cuda"), grad=z)
        top = w2v.linear_backward(out["grad"], h, self.E)
        low = w2v.linear_backward(top["dx"], x, self.W, activation="gelu", pre=pre)
        dx = w2v.dropout(top["dx"] + low["dx"], self.p, seed=self.seed, offset=step)
        w2v.embed_backward(dx, words, scale=self.scale, grad=top["dw"], accumulate=True)
        return out["loss"], {"E": top["dw"], "c": top["db"], "W": low["dw"], "b": low["db"]}

    def step(self, words, labels, step, rate):
        loss, grads = self.gradients(words, labels, step)
        for name, grad in grads.items():
            getattr(self, name).sub_(grad, alpha=rate)
        return loss

    def search(self, first, steps, beams=4, end=0):
        """The `beams` best continuations of words int32 (n,) by `steps` words, as
        far as a word `end`: words (n, beams, steps) and their log-probabilities."""
        packed = w2v.quantize_q4(self.E)
        n = len(first)
        scores = torch.full((n, beams), float("-inf"), device="cuda")
        scores[:, 0] = 0.0
        ended = torch.zeros((n, beams), dtype=torch.uint8, device="cuda")
        history = torch.full((n * beams, steps), -1, dtype=torch.int32, device="cuda")
        words = first.repeat_interleave(beams)
        for i in range(steps):
            z = w2v.linear_q4(self.hidden(words)[0], packed, self.c)
            out = w2v.beam_step(z, scores, finished=ended, end=end)
            scores, ended, words = out["scores"], out["finished"], out["words"].view(-1)
            history = w2v.beam_reorder(history, out["parents"])
            history[:, i] = words
        return history.view(n, beams, steps), scores


def main(V=20_000, topics=50, T=1_000_000, D=128, steps=400, batch=1_024, rate=1.0, verbose=True):
    corpus = torch.from_numpy(inputs.planted_topic_corpus(T, V, topics, 1.0, 0.05, 5)).cuda()
    model = Model(V, D)
    g = torch.Generator(device="cuda")
    g.manual_seed(11)
    losses = []
    for i in range(steps):
        at = torch.randint(0, T - 1, (batch,), generator=g, device="cuda")
        losses.append(model.step(corpus[at], corpus[at + 1], i, rate).mean())
        if verbose and i % 50 == 0:
            print(f"step {i}: loss {losses[-1].item():.4f}", flush=True)
    heads = (torch.arange(4, device="cuda") * (V // topics)).to(torch.int32) + 1
    words, scores = model.search(heads, steps=6)
    if verbose:
        for w, c, s in zip(heads.tolist(), words[:, 0].tolist(), scores[:, 0].tolist()):
            print(f"word {w}: {c} (log p {s:.2f})", flush=True)
    return torch.stack(losses), words, scores


if __name__ == "__main__":
    p = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    p.add_argument("--steps", type=int, default=400)
    main(steps=p.parse_args().steps)
