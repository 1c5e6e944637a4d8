"""w2v_sample_words against the definition in 64 bits, row by row, and against
the probabilities that it draws with.

A drawn word has to be the 64-bit one. Where two words' race scores are closer
than fp32 can tell (2^-24 of |x| + |g| in each of a few steps: 16 u (|x| + |g|
+ 1) is allowed, fixed beforehand), or a word is within that of where a filter
ends, either is right; the test then asks that the drawn word is allowed by
the filters widened by 1e-6 and that its score is that close to the best."""
import math

import numpy as np
import pytest

from gpu_util import expect_device_flag
from paper_1611_06172_amd import w2v

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


def draw64(z, u, T, k, p, least, slack=0.0):
    """(kept indices, their race scores, log-probabilities of all) of a row."""
    z = z.astype(np.float64)
    order = np.argsort(-z, kind="stable")
    n = int((z > -np.inf).sum())
    order = order[:n]
    x = (z[order] - z[order[0]]) / T
    w = np.exp(x)
    lp = x - np.log(w.sum())
    if 0 < k < len(z):
        n = min(n, k)
    if p < 1:
        c = np.cumsum(w[:n])
        before = np.concatenate([[0.0], c[:-1]])
        n = max(1, int((before < p * c[-1] * (1 + slack)).sum()))
    if least > 0:
        n = max(1, min(n, int((w >= least * (1 - slack)).sum())))
    with np.errstate(divide="ignore"):
        g = -np.log(-np.log(u[order[:n]].astype(np.float64)))
    return order[:n], x[:n] + g, dict(zip(order.tolist(), lp.tolist())), np.abs(x[:n]) + np.abs(g)


def check(z, u, out, T, k, p, least):
    zc, uc = z.float().cpu().numpy(), u.cpu().numpy()
    ids, logprob = out["ids"].cpu().numpy(), out["logprob"].cpu().numpy()

    def of(v, r):
        return v[r].item() if hasattr(v, "cpu") else v

    close = 0
    for r in range(len(ids)):
        args = of(T, r), of(k, r), of(p, r), of(least, r)
        kept, score, lp, size = draw64(zc[r], uc[r], *args)
        best = score.max()
        want = kept[score == best].min()
        got = int(ids[r])
        if got != want:
            wide, s2, _, m2 = draw64(zc[r], uc[r], *args, slack=1e-6)
            assert got in wide, (r, got, want)
            at = int(np.nonzero(wide == got)[0][0])
            assert best - s2[at] <= 16 * U * (m2[at] + 1) + (1e-5 if len(wide) != len(kept)
                                                            else 0), (r, got, want)
            close += 1
        bound = U * (512 + 8 * abs(lp[got]))
        assert abs(logprob[r] - lp[got]) <= bound, (r, logprob[r], lp[got])
    assert close <= max(1, len(ids) // 100), close


def scores(rows, V, name, seed, scale=3.0, zipf=1.0, masked=0.05):
    import torch
    g = torch.Generator()
    g.manual_seed(seed)
    z = torch.randn((rows, V), generator=g) * scale - zipf * torch.log(
        torch.arange(1, V + 1).float())
    if V > 1:
        z[torch.rand((rows, V), generator=g) < masked] = float("-inf")
        z[:, 0] = 0.25  # something is left
    u = torch.rand((rows, V), generator=g)
    return z.to(getattr(torch, name)).cuda(), u.cuda()


FILTERS = [(0, 1.0, 0.0), (1, 1.0, 0.0), (5, 1.0, 0.0), (40, 0.95, 0.0), (1000, 0.9, 0.01),
           (0, 0.9, 0.0), (0, 0.3, 0.0), (0, 1.0, 0.1), (0, 0.999, 0.05), (1024, 1.0, 0.0),
           (3, 0.5, 0.9)]


@pytest.mark.parametrize("name", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("rows,V", [(1, 1), (3, 2), (5, 7), (40, 1000), (7, 4097), (3, 71_290),
                                    (2, 250_007)])
def test_against_64_bits(rows, V, name):
    for i, (k, p, least) in enumerate(FILTERS):
        T = (0.7, 1.0, 1.5)[i % 3]
        z, u = scores(rows, V, name, 100 * i + rows)
        out = w2v.sample_words(z, u, temperature=T, top_k=k, top_p=p, min_p=least)
        check(z, u, out, T, k, p, least)


@pytest.mark.parametrize("rows,V,name", [(700, 1000, "float32"), (300, 5001, "bfloat16"),
                                         (1100, 333, "float16")])
def test_many_rows(rows, V, name):
    for k, p, least in ((0, 1.0, 0.0), (50, 0.9, 0.0), (0, 0.8, 0.02)):
        z, u = scores(rows, V, name, rows)
        out = w2v.sample_words(z, u, temperature=0.9, top_k=k, top_p=p, min_p=least)
        check(z, u, out, 0.9, k, p, least)


def test_flat_and_steep_scores():
    """Nearly equal scores (a prefix of many thousand words, and a bin that
    holds most words), and scores whose weights underflow."""
    for scale in (1e-3, 0.05, 60.0, 3000.0):
        for name in ("float32", "bfloat16"):
            z, u = scores(2, 60_000, name, 7, scale=scale, zipf=0.0)
            for k, p, least in ((0, 0.5, 0.0), (500, 0.7, 0.0), (0, 1.0, 0.5),
                                (1000, 1.0, 0.0)):
                for T in (0.5, 1.0):
                    out = w2v.sample_words(z, u, temperature=T, top_k=k, top_p=p,
                                           min_p=least)
                    check(z, u, out, T, k, p, least)


@pytest.mark.parametrize("V", [8, 900, 5000, 50_000])
def test_equal_scores_are_ranked_by_index(V):
    """All words equal: the kept ones are the first, exactly."""
    import torch
    z = torch.full((4, V), 1.5, device="cuda")
    half = V // 2
    for kw, n in ((dict(top_k=5), 5), (dict(top_p=0.5), half),
                  (dict(top_k=8, top_p=0.25), 2), (dict(top_p=1e-9), 1), (dict(), V)):
        u = torch.full((4, V), 0.3, device="cuda")
        u[0, n - 1] = 0.99  # the last kept word
        if n < V:
            u[1, n] = 0.99  # the first one left out: the others tie
            u[2, n:] = 1.0
        u[3] = 0.5  # all tie
        ids = w2v.sample_words(z, u, **kw)["ids"].tolist()
        assert ids[0] == n - 1
        assert ids[1:] == [0, 0, 0], (kw, ids)


@pytest.mark.parametrize("name", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("rows,V", [(40, 300), (16, 20_000), (3, 100_003), (130, 66_000)])
def test_log_probability_of_a_nearly_certain_word(rows, V, name):
    """A word that has all but 1e-2 to 1e-9 of the weight: its log-probability
    is -log(1 + the others' weight), to within that weight's own error: 128
    additions, arguments of exp of two roundings, |x| up to 60, and a logarithm
    of a few units: 300 units of 2^-24."""
    import torch
    g = torch.Generator()
    g.manual_seed(V)
    z = torch.randn((rows, V), generator=g) - 9 - math.log(V) - 10 * torch.rand(
        (rows, 1), generator=g)
    z[:, V // 3] = 0.75
    z = z.to(getattr(torch, name))
    u = torch.rand((rows, V), generator=g).cuda()
    for T in (1.0, 0.8):
        x = (z.double() - 0.75) / T
        x[:, V // 3] = float("-inf")
        exact = -torch.log1p(torch.exp(x).sum(dim=1))
        for kw in (dict(top_k=1), dict(top_p=0.5), dict(min_p=0.9)):
            out = w2v.sample_words(z.cuda(), u, temperature=T, **kw)
            assert (out["ids"] == V // 3).all()
            got = out["logprob"].double().cpu()
            assert ((got - exact).abs() <= 300 * U * exact.abs()).all(), \
                ((got - exact) / exact).abs().max() / U


def test_temperature_zero_takes_the_best():
    import torch
    z, u = scores(9, 20_000, "bfloat16", 3)
    out = w2v.sample_words(z, temperature=0)
    top = z.float().max(dim=1).values
    want = [int(torch.nonzero(z[r].float() == top[r])[0]) for r in range(9)]
    assert out["ids"].tolist() == want and (out["logprob"] == 0).all()
    t = torch.tensor([0.0, 1.0] * 4 + [0.0], device="cuda")
    mixed = w2v.sample_words(z, u, temperature=t, top_k=20)
    ones = w2v.sample_words(z, u, temperature=1.0, top_k=20)
    for r in range(9):
        assert mixed["ids"][r] == (want[r] if r % 2 == 0 else ones["ids"][r])


@pytest.mark.parametrize("rows,V", [(3, 700), (2, 20_000), (2, 100_000)])
def test_smallest_temperatures_take_the_best(rows, V):
    """Temperatures down to the least number above 0 leave the best word's
    weight alone, whose log-probability is 0."""
    import torch
    z, u = scores(rows, V, "float32", V)
    want = torch.argmax(z, dim=1).tolist()
    for T in (1e-30, 1.2e-38, 5e-39, 1e-39, 1e-45):
        for kw in (dict(), dict(top_k=9), dict(top_p=0.9), dict(min_p=0.5)):
            for t in (T, torch.full((rows,), T, device="cuda")):
                out = w2v.sample_words(z, u, temperature=t, **kw)
                assert out["ids"].tolist() == want, (T, kw)
                assert (out["logprob"] == 0).all()


def test_settings_of_each_row():
    import torch
    z, u = scores(len(FILTERS), 30_000, "float32", 17)
    k, p, least = (list(v) for v in zip(*FILTERS))
    T = [0.5 + 0.1 * i for i in range(len(FILTERS))]
    t32 = dict(dtype=torch.float32, device="cuda")
    T, p, least = torch.tensor(T, **t32), torch.tensor(p, **t32), torch.tensor(least, **t32)
    k = torch.tensor(k, dtype=torch.int32, device="cuda")
    out = w2v.sample_words(z, u, temperature=T, top_k=k, top_p=p, min_p=least)
    check(z, u, out, T, k, p, least)
    k[:] = 0
    out = w2v.sample_words(z, u, temperature=0.8, top_k=k, top_p=p, min_p=0.01)
    check(z, u, out, 0.8, k, p, 0.01)


@pytest.mark.parametrize("V", [6, 40_000])
def test_frequencies(V):
    """20,000 draws from one row: each kept word's share is within 5 standard
    deviations of its probability over the kept words'."""
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(12)
    n, base = 20_000, 1000
    row = torch.full((V,), -30.0, device="cuda")
    row[[5, 1, 3, 0]] = torch.tensor([2.0, 1.5, 0.5, -1.0], device="cuda")
    counts = torch.zeros(V)
    for _ in range(n // base):
        z = row.repeat(base, 1)
        u = torch.rand((base, V), generator=g, device="cuda")
        ids = w2v.sample_words(z, u, temperature=0.9, top_k=3)["ids"]
        counts += torch.bincount(ids.cpu(), minlength=V)
    p = torch.softmax(torch.tensor([2.0, 1.5, 0.5], dtype=torch.float64) / 0.9, 0)
    for i, w in enumerate((5, 1, 3)):
        sd = math.sqrt(n * float(p[i]) * (1 - float(p[i])))
        assert abs(float(counts[w]) - n * float(p[i])) <= 5 * sd
    assert counts.sum() == n and counts[[5, 1, 3]].sum() == n


def test_rows_without_a_word():
    import torch
    for V in (50, 30_000):
        z, u = scores(6, V, "float32", V)
        clean = w2v.sample_words(z, u, top_p=0.9)
        z[1] = float("-inf")
        z[2, V - 1] = float("nan")
        z[3, 4] = float("inf")
        z[4, 1:] = float("-inf")
        z[5] = torch.finfo(torch.float32).min
        for kw in (dict(top_p=0.9), dict(top_k=7), dict(), dict(min_p=0.1)):
            out = w2v.sample_words(z, u, **kw)
            ids = out["ids"].tolist()
            assert ids[1] == -1 and ids[2] == -1 and torch.isnan(out["logprob"][1:3]).all()
            assert ids[3] == 4 and ids[4] == 0 and out["logprob"][3] == 0
            assert 0 <= ids[5] < V
            if kw == dict(top_p=0.9):
                assert ids[0] == clean["ids"][0]
        assert w2v.sample_words(z, temperature=0)["ids"].tolist()[1:3] == [-1, -1]


def test_random_numbers_at_the_edges():
    import torch
    z = torch.zeros((4, 100), device="cuda")
    u = torch.full((4, 100), 0.5, device="cuda")
    u[0] = 0.0
    u[0, 60] = 1e-30  # loses against nobody but is above 0
    u[1, 7] = 1.0
    u[2, 3] = float("nan")
    u[3] = 0.0
    ids = w2v.sample_words(z, u)["ids"].tolist()
    assert ids == [60, 7, 0, 0]


def test_settings_out_of_range_skip_the_row():
    import torch
    z, u = scores(6, 5000, "float32", 9)
    clean = w2v.sample_words(z, u, top_k=10, top_p=0.9, min_p=0.01)["ids"].tolist()
    ok = dict(temperature=1.0, top_k=10, top_p=0.9, min_p=0.01)
    bad = dict(temperature=[-1.0, float("inf"), float("nan")], top_k=[-1, 1025, 4999],
               top_p=[0.0, -0.5, float("nan")], min_p=[-0.1, 1.5, float("nan")])
    for key, values in bad.items():
        t = torch.full((6,), ok[key], device="cuda",
                       dtype=torch.int32 if key == "top_k" else torch.float32)
        t[:3] = torch.tensor(values, dtype=t.dtype)
        out = w2v.sample_words(z, u, **dict(ok, **{key: t}))
        expect_device_flag()
        assert out["ids"].tolist() == [-1, -1, -1] + clean[3:], key


def test_strides_streams_and_long_offsets():
    import torch
    z, u = scores(4, 3001, "bfloat16", 31)
    want = w2v.sample_words(z, u, top_p=0.9, temperature=0.8)
    far = torch.empty(3 * (1 << 30) + 4096, dtype=torch.bfloat16, device="cuda")
    zz = far.as_strided((4, 3001), (1 << 30, 1))
    zz.copy_(z)
    uu = torch.full((4, 4000), float("nan"), device="cuda")[:, 3:3004]
    uu.copy_(u)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = w2v.sample_words(zz, uu, top_p=0.9, temperature=0.8, stream=s)
    s.synchronize()
    assert torch.equal(got["ids"], want["ids"]) and torch.equal(got["logprob"],
                                                                want["logprob"])
    del far, zz
    torch.cuda.empty_cache()


def test_no_rows_and_refusals():
    import torch
    z, u = torch.zeros((3, 2000), device="cuda"), torch.rand((3, 2000), device="cuda")
    assert w2v.sample_words(z[:0], u[:0])["ids"].shape == (0,)
    for kw in (dict(temperature=-1.0), dict(top_k=-1), dict(top_p=0.0), dict(min_p=1.5),
               dict(top_k=1500), dict(top_p=float("nan"))):
        with pytest.raises(w2v.W2VError):
            w2v.sample_words(z, u, **kw)
    with pytest.raises(w2v.W2VError):
        w2v.sample_words(z)
    with pytest.raises(ValueError):
        w2v.sample_words(z, u[:, :1000])
    with pytest.raises(TypeError):
        w2v.sample_words(z, u.half())
    with pytest.raises(ValueError):
        w2v.sample_words(z, u, temperature=torch.ones(2, device="cuda"))
    assert w2v.sample_words(z, u, top_k=2000)["ids"].min() >= 0  # V and more: off
