"""w2v_dropout: the mask bit for bit against Philox4x32-10 in Python integers, and
the values against the definition in 64 bits (one fp32 rounding of the factor, one
of the product with the sum, one to the type)."""
import math

import numpy as np
import pytest

from ends_util import EPS, TINY, captured, dtype_of, generator, guarded, matrix
from paper_1611_06172_amd import w2v

pytestmark = pytest.mark.gpu

MASK = 0xFFFFFFFF


def philox(c, k):
    """One block of Philox4x32-10, from its published definition."""
    c, k = list(c), list(k)
    for _ in range(10):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [(b >> 32) ^ c[1] ^ k[0], b & MASK, (a >> 32) ^ c[3] ^ k[1], a & MASK]
        k = [(k[0] + 0x9E3779B9) & MASK, (k[1] + 0xBB67AE85) & MASK]
    return c


def number(i, seed, offset):
    b, j = i // 8, i % 8

    def half(stream):
        w = philox([b & MASK, (b >> 32) | stream << 31, offset & MASK, offset >> 32],
                   [seed & MASK, seed >> 32])
        return (w[j // 2] >> 16 * (j % 2)) & 0xFFFF

    return half(0) << 16 | half(1)


def numbers(n, seed, offset):
    """number() of 0..n - 1 in 64-bit arrays."""
    x = np.zeros((2, 4, (n + 7) // 8), dtype=np.uint64)
    x[:, 0] = np.arange(x.shape[2])
    x[1, 1] = 1 << 31
    x[:, 2], x[:, 3] = offset & MASK, offset >> 32
    k = [seed & MASK, seed >> 32]
    low, up = np.uint64(MASK), np.uint64(32)
    for _ in range(10):
        a, b = x[:, 0] * np.uint64(0xD2511F53), x[:, 2] * np.uint64(0xCD9E8D57)
        x = np.stack([(b >> up) ^ x[:, 1] ^ np.uint64(k[0]), b & low,
                      (a >> up) ^ x[:, 3] ^ np.uint64(k[1]), a & low], axis=1)
        k = [(k[0] + 0x9E3779B9) & MASK, (k[1] + 0xBB67AE85) & MASK]
    halves = np.stack([x & np.uint64(0xFFFF), x >> np.uint64(16)], axis=2)  # [s][word][half][b]
    halves = halves.transpose(0, 3, 1, 2).reshape(2, -1)[:, :n]
    return (halves[0] << np.uint64(16)) | halves[1]


def test_generator_of_this_test():
    """The known answers published with the generator, and the array form."""
    assert philox([0] * 4, [0] * 2) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    assert philox([0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344],
                  [0xA4093822, 0x299F31D0]) == [0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1]
    got = numbers(45, 0x123456789ABCDEF0, 0xFEDCBA9876543210)
    assert [int(v) for v in got] == [number(i, 0x123456789ABCDEF0, 0xFEDCBA9876543210)
                                     for i in range(45)]


def check(x, p, seed, offset, out, residual=None):
    import torch
    below = math.floor(p * 2.0 ** 32 + 0.5)
    rows, cols = x.shape
    keep = torch.from_numpy(numbers(rows * cols, seed, offset) >= np.uint64(below)).view(rows, cols)
    name = str(x.dtype).split(".")[1]
    factor = 2.0 ** 32 / (2.0 ** 32 - below) if below < 2 ** 32 else 0.0
    want = torch.where(keep, x.cpu().double() * factor, 0.0)
    size = want.abs()
    if residual is not None:
        want = want + residual.cpu().double()
    bound = 2.0 ** -24 * (size + want.abs()) + EPS[name] * want.abs() * (1 + 2.0 ** -7) + TINY[name]
    got = out.cpu().double()
    assert ((got - want).abs() <= bound).all()
    if residual is None:
        assert (got[~keep] == 0).all()
    else:
        assert (got[~keep] == residual.cpu().double()[~keep]).all()
    return keep


@pytest.mark.parametrize("name", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("with_residual", [False, True])
@pytest.mark.parametrize("rows,cols,pad", [(1, 1, 0), (1, 7, 0), (5, 3, 2), (3, 8, 0), (64, 300, 0),
                                           (33, 300, 20), (17, 641, 1), (200, 5, 3), (9, 2500, 4),
                                           (4000, 1, 1), (700, 33, 0)])
def test_values(name, with_residual, rows, cols, pad):
    g = generator(rows + cols)
    x = matrix(g, rows, cols, name, pad=pad)
    r = matrix(g, rows, cols, name, pad=pad + 1) if with_residual else None
    for p, seed, offset in ((0.1, 5, 0), (0.5, 2**64 - 1, 2**63 + 12345), (0.937, 1 << 40, 1 << 32)):
        out = w2v.dropout(x, p, seed=seed, offset=offset, residual=r)
        check(x, p, seed, offset, out, r)
    view, untouched = guarded(rows, cols, name)
    w2v.dropout(x, 0.3, seed=9, offset=4, residual=r, out=view)
    check(x, 0.3, 9, 4, view, r)
    assert untouched()


def test_lower_halves_decide():
    """Thresholds that equal an element's upper half: its lower half is compared."""
    import torch
    x = torch.ones((1, 4096), device="cuda")
    r = numbers(4096, 3, 1)
    for i in (0, 5, 1001, 4095):
        for step in (0, 1):  # kept at its own number, dropped one above
            p = (int(r[i]) + step) / 2.0 ** 32
            keep = check(x, p, 3, 1, w2v.dropout(x, p, seed=3, offset=1))
            assert bool(keep[0, i]) == (step == 0)


def test_all_and_nothing():
    import torch
    for name in ("float32", "bfloat16", "float16"):
        x = matrix(generator(2), 50, 70, name)
        assert torch.equal(w2v.dropout(x, 0.0, seed=1), x)
        assert (w2v.dropout(x, 1.0, seed=1) == 0).all()
        assert torch.equal(w2v.dropout(x, 1.0, seed=1, residual=x), x)
    assert w2v.dropout(x[:0], 0.5, seed=1).shape == (0, 70)


def test_share_of_dropped():
    """Of n elements a share of p is dropped, within five deviations."""
    import torch
    n = 1 << 22
    x = torch.ones((1, n), dtype=torch.bfloat16, device="cuda")
    for p in (0.01, 0.1, 0.5, 0.9):
        gone = int((w2v.dropout(x, p, seed=77, offset=3) == 0).sum())
        assert abs(gone - n * p) <= 5 * math.sqrt(n * p * (1 - p))


def test_mask_does_not_follow_from_the_layout_or_the_type():
    import torch
    one = torch.ones((40, 300), device="cuda")
    wide = torch.ones((40, 320), device="cuda")[:, :300]
    want = w2v.dropout(one, 0.4, seed=8, offset=2) > 0
    assert torch.equal(w2v.dropout(wide, 0.4, seed=8, offset=2) > 0, want)
    assert torch.equal(w2v.dropout(one.view(1, -1), 0.4, seed=8, offset=2).view(40, 300) > 0, want)
    assert torch.equal(w2v.dropout(one.half(), 0.4, seed=8, offset=2) > 0, want)
    assert not torch.equal(w2v.dropout(one, 0.4, seed=8, offset=3) > 0, want)
    assert not torch.equal(w2v.dropout(one, 0.4, seed=9, offset=2) > 0, want)
    # the binding takes both modulo 2^64
    assert torch.equal(w2v.dropout(one, 0.4, seed=8 + 2**64, offset=2 - 2**64) > 0, want)


def test_dropped_values_stay_out():
    import torch
    x = torch.ones((3, 900), device="cuda")
    keep = check(x, 0.5, 6, 0, w2v.dropout(x, 0.5, seed=6))
    x[~keep.cuda()] = float("nan")
    x[0][~keep[0].cuda()] = float("inf")
    out = w2v.dropout(x, 0.5, seed=6)
    assert torch.equal(out, torch.where(keep.cuda(), 2.0, 0.0))


@pytest.mark.parametrize("pad", [0, 11])
def test_in_place(pad):
    g = generator(4)
    x, r = matrix(g, 60, 301, "bfloat16", pad=pad), matrix(g, 60, 301, "bfloat16", pad=pad)
    want = w2v.dropout(x, 0.2, seed=1, offset=9, residual=r)
    y = x.as_strided(x.size(), x.stride())
    own = r.clone() if pad == 0 else r
    w2v.dropout(x, 0.2, seed=1, offset=9, residual=own, out=own)
    assert (own == want).all()
    plain = w2v.dropout(x, 0.2, seed=1, offset=9)
    w2v.dropout(x, 0.2, seed=1, offset=9, out=y)
    assert (y == plain).all()


def test_gradient_is_the_same_call():
    """y is linear in x: differences of sum(c y) are dropout(c), and the
    residual's gradient is c itself."""
    import torch
    g = generator(6)
    x, c, r = (matrix(g, 20, 30, "float32") for _ in range(3))
    grad = w2v.dropout(c, 0.3, seed=2, offset=1).double()
    size = 8 * c.double().abs().sum()
    for i, j in ((0, 0), (7, 13), (19, 29), (4, 4)):
        step = torch.zeros_like(x)
        step[i, j] = 0.5
        for a, b, want in ((step, 0 * step, grad[i, j]), (0 * step, step, c[i, j].double())):
            up = w2v.dropout(x + a, 0.3, seed=2, offset=1, residual=r + b).double()
            low = w2v.dropout(x - a, 0.3, seed=2, offset=1, residual=r - b).double()
            assert abs(((up - low) * c.double()).sum() - want) <= 4 * 2.0 ** -24 * size


def test_elements_beyond_32_bits():
    """Element numbers past 2^32: the block's counter goes on."""
    import torch
    n = 2**32 + 4096
    x = torch.ones((4096, n // 4096), dtype=torch.bfloat16, device="cuda")
    out = w2v.dropout(x, 0.5, seed=12, offset=1)
    for first in (0, 2**31 - 64, 2**32 - 512, n - 1024):
        part = out.view(-1)[first:first + 512].cpu()
        want = [number(i, 12, 1) >= 2**31 for i in range(first, first + 512)]
        assert (part > 0).tolist() == want
    # and with gaps between the rows
    cols = n // 4096 - 1
    out = w2v.dropout(x[:, :cols], 0.5, seed=12, offset=1)
    want = [number(4095 * cols + j, 12, 1) >= 2**31 for j in range(cols - 512, cols)]
    assert (out[4095, cols - 512:].cpu() > 0).tolist() == want


def test_replayed_with_a_counter_on_the_gpu():
    import torch
    g = generator(7)
    x = matrix(g, 100, 333, "float16")
    step = torch.zeros(1, dtype=torch.int64, device="cuda")
    graph, held = captured(lambda: w2v.dropout(x, 0.25, seed=3, offset=40, offset_dev=step))
    seen = []
    for i in range(4):
        step.fill_(i * (2**61 - 1))
        graph.replay()
        torch.cuda.synchronize()
        want = w2v.dropout(x, 0.25, seed=3, offset=40 + i * (2**61 - 1))
        assert torch.equal(held, want)
        assert all(not torch.equal(held, other) for other in seen)
        seen.append(held.clone())
    step.fill_(-1)
    graph.replay()
    assert torch.equal(held, w2v.dropout(x, 0.25, seed=3, offset=39))


def test_another_stream():
    import torch
    x = matrix(generator(3), 500, 300, "float32")
    want = w2v.dropout(x, 0.1, seed=5)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    out = w2v.dropout(x, 0.1, seed=5, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(out, want)


def test_refused_arguments():
    import torch
    x = torch.zeros((4, 8), device="cuda")
    for call in (lambda: w2v.dropout(x.double(), 0.1, seed=1),
                 lambda: w2v.dropout(x, 0.1, seed=1, residual=x.half()),
                 lambda: w2v.dropout(x, 0.1, seed=1, out=x.half()),
                 lambda: w2v.dropout(x, 0.1, seed=1, offset_dev=torch.zeros(1, device="cuda"))):
        with pytest.raises(TypeError):
            call()
    for call in (lambda: w2v.dropout(x.t(), 0.1, seed=1), lambda: w2v.dropout(x[0], 0.1, seed=1),
                 lambda: w2v.dropout(x, 0.1, seed=1, residual=x[:3])):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(w2v.W2VError):
        w2v.dropout(x, 1.01, seed=1)
