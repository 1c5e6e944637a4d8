"""A small model taught by a large one, and words drawn from it.

Trains word vectors on a corpus of planted topics (HogBatch), then distils
their distribution of context words, p(c | w) ~ exp(M_in[w] . M_out[c]) times
the unigram^0.75 that negatives are drawn with, into a model with a fraction
of the columns: an embedding, one residual layer and an output matrix. The
teacher answers with its top words only. At the end the small model draws
context words.

    python examples/smaller_vectors.py
"""
import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_1611_06172_amd import inputs, w2v  # noqa: E402


def train_teacher(V, topics, T, D, epochs, seed=5):
    """Word vectors of a planted-topic corpus, their corpus and word counts."""
    corpus = inputs.planted_topic_corpus(T, V, topics, 1.0, 0.05, seed)
    counts = inputs.word_counts(corpus, V)
    table, _ = w2v.build_tables(counts, 0.75, 0.0, 1_000_000, want_thresh=False)
    ids, table = torch.from_numpy(corpus).cuda(), torch.from_numpy(table).cuda()
    M_in = w2v.alloc_matrix(V, D, "cuda", torch.from_numpy(
        inputs.init_matrix(V, D, "uniform", 2)))
    M_out = w2v.alloc_matrix(V, D, "cuda")
    for e in range(epochs):
        w2v.train_epoch(ids, M_in, M_out, table, window=5, K=5, epoch=e, n_epochs=epochs,
                        seed=1)
    return M_in, M_out, ids, counts


class Teacher:
    """Scores of all words in the context of given ones, and the top of them."""

    def __init__(self, M_in, M_out, counts):
        self.M_in, self.M_out = M_in, M_out
        self.bias = torch.from_numpy(0.75 * np.log(np.maximum(counts, 1))).float().cuda()

    def top(self, words, K):
        scores = w2v.linear(self.M_in[words], self.M_out, self.bias)
        values, ids = torch.topk(scores, K, dim=1)
        return ids.to(torch.int32), values


class Student:
    """x = E[words]; h = x + gelu(x W^T + b); scores = h O^T + c."""

    def __init__(self, V, D, bias, seed=3):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        self.E = torch.randn((V, D), generator=g, device="cuda") / D ** 0.5
        self.W = torch.randn((D, D), generator=g, device="cuda") / D ** 0.5
        self.b = torch.zeros(D, device="cuda")
        self.O = w2v.alloc_matrix(V, D, "cuda", torch.randn(
            (V, D), generator=g, device="cuda") / D ** 0.5)
        self.c = bias - bias.mean()

    def scores(self, words):
        x = self.E[words]
        pre = torch.empty_like(x)
        h = w2v.linear(x, self.W, self.b, activation="gelu", residual=x, pre=pre)
        return w2v.linear(h, self.O, self.c), (x, pre, h)

    def step(self, words, ids, values, labels, rate, temperature=2.0):
        """One step on the mean loss; returns the rows' losses."""
        z, (x, pre, h) = self.scores(words)
        n = len(words)
        weight = torch.full((n,), 1.0 / n, device="cuda")
        out = w2v.distill_loss(z, ids, values, temperature=temperature, labels=labels,
                               soft=0.9, hard=0.1, row_weight=weight, grad=z)
        top = w2v.linear_backward(out["grad"], h, self.O)
        low = w2v.linear_backward(top["dx"], x, self.W, activation="gelu", pre=pre)
        dx = top["dx"] + low["dx"]  # the layer's and its residual's
        self.O -= rate * top["dw"]
        self.c -= rate * top["db"]
        self.W -= rate * low["dw"]
        self.b -= rate * low["db"]
        self.E.index_add_(0, words, dx, alpha=-rate)
        return out["loss"]


def main(V=20_000, topics=50, T=2_000_000, D=200, d=64, K=64, epochs=3, steps=500, batch=2_048,
         rate=10.0, verbose=True):
    M_in, M_out, corpus, counts = train_teacher(V, topics, T, D, epochs)
    teacher = Teacher(M_in, M_out, counts)
    student = Student(V, d, teacher.bias)
    g = torch.Generator(device="cuda")
    g.manual_seed(11)
    losses = []
    for i in range(steps):
        at = torch.randint(0, T - 1, (batch,), generator=g, device="cuda")
        words = corpus[at].long()
        ids, values = teacher.top(words, K)
        losses.append(student.step(words, ids, values, corpus[at + 1], rate).mean())
        if verbose and i % 50 == 0:
            print(f"step {i}: loss {losses[-1].item():.4f}", flush=True)
    # context words of the most frequent word of each of a few topics
    heads = torch.arange(4, device="cuda") * (V // topics)
    scores, _ = student.scores(heads)
    u = torch.rand((len(heads), V), generator=g, device="cuda")
    drawn = w2v.sample_words(scores, u, temperature=0.8, top_k=50, top_p=0.95)
    if verbose:
        for w, c, p in zip(heads.tolist(), drawn["ids"].tolist(), drawn["logprob"].tolist()):
            print(f"word {w}: drew {c} (log p {p:.2f})", flush=True)
    return torch.stack(losses), heads, drawn


if __name__ == "__main__":
    p = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    p.add_argument("--steps", type=int, default=500)
    main(steps=p.parse_args().steps)
