"""w2v_quantize_q4 against its definition, bit for bit, and w2v_linear_q4 against
products in 64 bits with the matrix that the codes and scales stand for.

Tolerance, fixed beforehand: a group's sum is one of x (q + 16) and of -24 sum(x),
itself a sum of the group's x, all in fp32: (3 group + 4) 2^-24 of sum |x| (q +
16 + 24) in any order; times the scale and added up over G groups, (G + 2) 2^-24
of the same; an output is rounded once."""
import pytest

from ends_util import EPS, TINY, captured, dtype_of, generator, guarded, matrix
from paper_1611_06172_amd import w2v

pytestmark = pytest.mark.gpu


def quantised64(w, group):
    """Codes and scales of a matrix, from the definition (on the CPU)."""
    import torch
    N, K = w.shape
    G = (K + group - 1) // group
    full = torch.zeros((N, G * group))
    full[:, :K] = w.cpu().float()
    full = full.view(N, G, group)
    scale = (full.abs().amax(dim=2) / 7).bfloat16()
    s = scale.float()[:, :, None]
    code = torch.where(s > 0, torch.round(full / s), torch.zeros_like(full)).clamp(-8, 7)
    return code.view(N, -1).to(torch.int64) + 8, scale


def unpacked(q):
    """Codes [tiles * 16][B * 32] and scales [tiles * 16][G] of a packed matrix,
    word by word from the header's description."""
    import numpy as np
    import torch
    (N, K), group = q["shape"], q["group"]
    tiles, G = (N + 15) // 16, (K + group - 1) // group
    B = G * group // 32
    words = q["packed"].cpu().numpy().view(np.uint32).reshape(tiles, B * 64)
    raw = q["scales"].cpu().view(torch.int16).numpy().reshape(tiles, G * 16)
    codes = np.zeros((tiles * 16, B * 32), dtype=np.int64)
    scales = np.zeros((tiles * 16, G), dtype=np.int16)
    for b in range(B):
        i, j, R = b // 4, b % 4, B % 4
        for c in range(4):
            for r in range(16):
                lane = 16 * c + r
                at = 256 * i + 4 * lane + j if i < B // 4 else 256 * (B // 4) + R * lane + j
                for k in range(8):
                    bit = 2 * k if k % 2 == 0 else 2 * k + 14
                    codes[r::16, 32 * b + 8 * c + k] = (words[:, at] >> np.uint32(bit)) & 15
    for g in range(G):
        i, j, R = g // 4, g % 4, G % 4
        for r in range(16):
            at = 64 * i + 4 * r + j if i < G // 4 else 64 * (G // 4) + R * r + j
            scales[r::16, g] = raw[:, at]
    return torch.from_numpy(codes), torch.from_numpy(scales).view(torch.bfloat16)


@pytest.mark.parametrize("name", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("N,K,pad", [(1, 1, 0), (15, 31, 2), (16, 32, 0), (17, 33, 1), (100, 300, 20),
                                     (33, 129, 0), (50, 641, 7), (16, 224, 0)])
def test_codes(name, group, N, K, pad):
    import torch
    w = matrix(generator(N + K), N, K, name, scale=0.3, pad=pad)
    q = w2v.quantize_q4(w, group=group)
    code, scale = quantised64(w, group)
    got, got_scale = unpacked(q)
    assert torch.equal(got[:N, :code.shape[1]], code)
    assert torch.equal(got_scale[:N].view(torch.int16), scale.view(torch.int16))
    assert (got[N:] == 8).all() and (got_scale[N:].float() == 0).all()
    assert (got[:, K:] == 8).all()


def test_groups_without_a_range():
    """Zeros, one value, the smallest magnitudes, NaN and infinities."""
    import torch
    w = torch.zeros((9, 64))
    w[1, :] = -3.5
    w[2, 40] = 1e-40
    w[3, 5] = float("nan")
    w[4, 33] = float("inf")
    w[5, 63] = -float("inf")
    w[6, :] = 3.38e38
    w[7, ::2] = 1e-39
    q = w2v.quantize_q4(w.cuda())
    code, scale = unpacked(q)
    want, want_scale = quantised64(w, 32)
    for r in (0, 1, 2, 6, 7, 8):
        assert torch.equal(code[r], want[r])
        assert torch.equal(scale[r].view(torch.int16), want_scale[r].view(torch.int16))
    for r, bad in ((3, 0), (4, 1), (5, 1)):
        assert torch.isnan(scale[r, bad].float()) and scale[r, 1 - bad] == 0
    y = w2v.linear_q4(torch.ones((1, 64), device="cuda"), q)[0].tolist()
    assert [v != v for v in y] == [False, False, False, True, True, True, False, False, False]


def random_q4(g, N, K, group, device="cuda"):
    """A matrix in 4 bits with codes and scales of every size."""
    import torch
    w = matrix(g, N, K, "float32", scale=0.2)
    w *= torch.exp2(torch.randint(-6, 6, (N, 1), generator=g).float()).cuda()
    return w2v.quantize_q4(w, group=group)


def check(x, q, out, bias=None):
    import torch
    (N, K), group = q["shape"], q["group"]
    code, scale = unpacked(q)
    full = torch.repeat_interleave(scale.double(), group, dim=1)[:N, :K]
    code = code[:N, :K].double()
    x64 = x.cpu().double()
    want = x64 @ ((code - 8) * full).t()
    G = scale.shape[1]
    bound = (3 * min(group, K) + G + 6) * 2.0 ** -24 * (x64.abs() @ ((code + 40) * full).t())
    if bias is not None:
        want = want + bias.cpu().double()
        bound = bound + 2.0 ** -24 * want.abs()
    name = str(out.dtype).split(".")[1]
    error = (out.cpu().double() - want).abs()
    assert (error <= bound + EPS[name] * (want.abs() + bound) + TINY[name]).all()


@pytest.mark.parametrize("name", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("M,N,K", [(1, 1, 1), (1, 1000, 300), (3, 17, 33), (16, 130, 64), (17, 300, 129),
                                   (33, 500, 224), (64, 257, 300), (65, 31, 600), (130, 90, 40),
                                   (2, 48, 2000)])
def test_products(name, group, M, N, K):
    import torch
    g = generator(M + N + K)
    q = random_q4(g, N, K, group)
    x = matrix(g, M, K, name, pad=3)
    bias = torch.randn(N, generator=g).cuda()
    check(x, q, w2v.linear_q4(x, q, bias), bias)
    check(x, q, w2v.linear_q4(x, q, out_dtype=torch.float32))
    view, untouched = guarded(M, N, name)
    w2v.linear_q4(x, q, bias, out=view)
    check(x, q, view, bias)
    assert untouched()


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("name,M,K", [("float32", 5, 9001), ("bfloat16", 40, 9001),
                                      ("float16", 64, 4500), ("float32", 20, 4500),
                                      ("float32", 40, 700), ("bfloat16", 64, 1100),
                                      ("float16", 20, 2100), ("float32", 3, 1000)])
def test_long_sums(name, M, K, group):
    """More columns than LDS holds of x at once, or of all of its rows."""
    g = generator(K)
    q = random_q4(g, 70, K, group)
    x = matrix(g, M, K, name)
    check(x, q, w2v.linear_q4(x, q))


@pytest.mark.parametrize("M", [1, 16, 64])
def test_many_rows_of_the_matrix(M):
    """More tiles than the blocks of a launch."""
    import torch
    g = generator(M)
    N, K = 150_001, 40
    q = random_q4(g, N, K, 32)
    x = matrix(g, M, K, "bfloat16")
    out = w2v.linear_q4(x, q, out_dtype=torch.float32)
    # rows in reverse order of tiles give the same sums, by tile
    tiles = (N + 15) // 16
    turned = dict(q, packed=q["packed"].view(tiles, -1).flip(0).reshape(-1).contiguous(),
                  scales=q["scales"].view(tiles, -1).flip(0).reshape(-1).contiguous(),
                  shape=(tiles * 16, K))
    back = w2v.linear_q4(x, turned, out_dtype=torch.float32)
    back = back.view(M, tiles, 16).flip(1).reshape(M, -1)[:, :N]
    assert torch.equal(out, back)
    for first in (0, 70_000 // 16 * 16, (N - 33) // 16 * 16):
        part = dict(q, shape=(min(64, N - first), K))
        for key, per in (("packed", 2 * 256), ("scales", 2 * 16)):
            part[key] = q[key][first // 16 * per:][:(part["shape"][0] + 15) // 16 * per].clone()
        check(x, part, out[:, first:first + 64])


@pytest.mark.parametrize("name,M,N,K,group", [
    ("float32", 32, 400, 700, 32), ("float32", 64, 400, 1000, 64), ("float16", 20, 410, 2100, 32),
    ("float32", 40, 50_000, 700, 64), ("bfloat16", 64, 100_003, 1100, 32),
    ("float16", 61, 50_001, 2100, 64), ("float32", 16, 100_003, 1400, 128)])
def test_rows_in_parts(name, M, N, K, group):
    """All rows of x against W at once, a part of their columns at a time, over one
    and several rounds of tiles."""
    import torch
    g = generator(N + K)
    q = random_q4(g, N, K, group)
    x = matrix(g, M, K, name, pad=1)
    bias = torch.randn(N, generator=g).cuda()
    out = w2v.linear_q4(x, q, bias)
    G = (K + group - 1) // group
    blocks = G * group // 32
    for first in (0, N // 3 // 16 * 16, 2 * N // 3 // 16 * 16, (N - 33) // 16 * 16):
        part = dict(q, shape=(min(512, N - first), K))
        tiles = (part["shape"][0] + 15) // 16
        for key, per in (("packed", blocks * 256), ("scales", G * 16)):
            per //= q[key].element_size() if key == "packed" else 1
            part[key] = q[key][first // 16 * per:][:tiles * per].clone()
        check(x, part, out[:, first:first + 512], bias[first:first + 512])


@pytest.mark.parametrize("M", [1, 20])
@pytest.mark.parametrize("group", [32, 64, 128])
def test_correction_is_not_rounded(M, group):
    """x of 16 bits in [1, 2), scales of 2^-3: in multiples of 2^-15, 24 sum(x) takes more
    than 24 bits, but the result fewer, and those of its first pieces, and so does every
    sum on the way as it is documented: nothing is rounded."""
    import torch
    g = generator(group)
    K, N = 2 * group, 200
    w = torch.randint(-7, 8, (N, K), generator=g).float()
    w[:, ::group] = 7.0
    x = 1.0 + torch.randint(0, 1 << 15, (M, K), generator=g).float() / (1 << 15)
    want = x.double() @ (w.double() / 8).t()
    fits = want.abs() < 32  # with 31 |x| 2^-7 of the others' products: 9 bits before the point
    for half in (w[:, :group], w[:, group:]):
        fits &= (x[:, :group].double() @ half.double().t()).abs() < 256
        fits &= (x[:, group:].double() @ half.double().t()).abs() < 256
    assert fits.float().mean() > 0.5
    q = w2v.quantize_q4((w / 8).cuda(), group=group)
    y = w2v.linear_q4(x.cuda(), q).cpu().double()
    assert torch.equal(y[fits], want[fits])


def test_pieces_of_float32():
    """Three bfloat16 pieces hold all bits of x: an identity returns it."""
    import torch
    g = generator(2)
    N = K = 96
    # 7 (scale 1 / 7, rounded) on the diagonal
    q = w2v.quantize_q4(torch.eye(N, device="cuda"))
    scale = float(unpacked(q)[1][0, 0])
    x = torch.randn((16, K), generator=g).cuda() * torch.exp2(
        torch.randint(-60, 60, (16, 1), generator=g).float()).cuda()
    check(x, q, w2v.linear_q4(x, q))
    # a column on its own has no other terms
    alone = torch.zeros((16, K), device="cuda")
    alone[:, 5] = x[:, 5]
    got = w2v.linear_q4(alone, q)[:, 5].double()
    want = alone[:, 5].double() * 7 * scale
    assert ((got - want).abs() <= 16 * 2.0 ** -24 * want.abs()).all()


def test_values_that_are_not_finite():
    import torch
    g = generator(3)
    q = random_q4(g, 40, 70, 32)
    for name in ("float32", "bfloat16", "float16"):
        x = matrix(g, 5, 70, name)
        want = w2v.linear_q4(x, q)
        for bad in (float("nan"), float("inf"), -float("inf")):
            y = x.clone()
            y[2, 69] = bad
            out = w2v.linear_q4(y, q)
            assert torch.isnan(out[2]).all()
            rest = [0, 1, 3, 4]
            assert torch.equal(out[rest], want[rest])


def test_close_to_the_matrix_itself():
    """The product with the matrix in 4 bits is that with the matrix, but for
    half a code in each of its weights."""
    import torch
    g = generator(4)
    w, x = matrix(g, 200, 300, "float32", scale=0.1), matrix(g, 8, 300, "float32")
    q = w2v.quantize_q4(w)
    scale = torch.repeat_interleave(unpacked(q)[1].double(), 32, dim=1)[:200, :300].cuda()
    # codes end at 7: a scale that was rounded down leaves up to 7 2^-8 of it
    bound = x.double().abs() @ ((0.5 + 7 * 2.0 ** -8) * scale).t()
    diff = (w2v.linear_q4(x, q).double() - x.double() @ w.double().t()).abs()
    assert (diff <= bound * 1.001).all()


def test_same_bits_streams_and_graphs():
    import torch
    g = generator(6)
    q, x = random_q4(g, 3000, 300, 64), matrix(g, 9, 300, "bfloat16")
    want = w2v.linear_q4(x, q)
    assert torch.equal(w2v.linear_q4(x, q), want)
    assert torch.equal(w2v.linear_q4(x[4:5], q), want[4:5])
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    out = w2v.linear_q4(x, q, stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(out, want)
    w = matrix(g, 3000, 300, "bfloat16")

    def call():
        new = w2v.quantize_q4(w, group=64)
        return [new["packed"], new["scales"], w2v.linear_q4(x, new)]

    graph, held = captured(call)
    for _ in range(3):
        x.copy_(torch.randn(x.shape, generator=g))
        w.copy_(torch.randn(w.shape, generator=g))
        eager = call()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, eager))


def test_refused_arguments():
    import torch
    w = torch.zeros((5, 40), device="cuda")
    q = w2v.quantize_q4(w)
    x = torch.zeros((2, 40), device="cuda")
    assert w2v.linear_q4(x[:0], q).shape == (0, 5)
    for call in (lambda: w2v.linear_q4(x.double(), q), lambda: w2v.quantize_q4(w.double()),
                 lambda: w2v.linear_q4(x, q, out_dtype=torch.float16),
                 lambda: w2v.linear_q4(x, q, torch.zeros(5, device="cuda").half()),
                 lambda: w2v.linear_q4(x, dict(q, packed=q["packed"].view(torch.int32)))):
        with pytest.raises(TypeError):
            call()
    for call in (lambda: w2v.linear_q4(x[:, :39], q), lambda: w2v.quantize_q4(w.t()),
                 lambda: w2v.linear_q4(x, q, torch.zeros(4, device="cuda")),
                 lambda: w2v.linear_q4(x, dict(q, scales=q["scales"][1:])),
                 lambda: w2v.linear_q4(x, dict(q, shape=(17, 40))),
                 lambda: w2v.linear_q4(x, q, out=torch.zeros((2, 6), device="cuda"))):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: w2v.quantize_q4(w, group=48), lambda: w2v.quantize_q4(w[:0])):
        with pytest.raises(w2v.W2VError):
            call()


def test_calls_of_two_threads():
    """Calls of one kernel with more and with less LDS, side by side."""
    import threading

    import torch
    g = generator(12)
    jobs, done = [], []
    for K in (1000, 600):
        q, x = random_q4(g, 200, K, 32), matrix(g, 60, K, "float16")
        jobs.append((q, x, w2v.linear_q4(x, q)))

    def work(q, x, want):
        s = torch.cuda.Stream()
        out = [w2v.linear_q4(x, q, stream=s) for _ in range(200)]
        s.synchronize()
        done.append(all(torch.equal(o, want) for o in out))

    torch.cuda.synchronize()
    threads = [threading.Thread(target=work, args=job) for job in jobs]
    for t in threads:
        t.start()
    for t in threads:
        t.join(60)
    assert done == [True, True]


def test_much_of_lds_in_a_graph():
    import torch
    g = generator(13)
    q, x = random_q4(g, 200, 1000, 32), matrix(g, 60, 1000, "float16")
    graph, held = captured(lambda: w2v.linear_q4(x, q))
    for _ in range(3):
        x.copy_(torch.randn(x.shape, generator=g))
        eager = w2v.linear_q4(x, q)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(held, eager)
