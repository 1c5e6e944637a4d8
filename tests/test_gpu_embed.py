"""w2v_embed and w2v_embed_backward against the definitions in 64 bits.

Tolerances, fixed beforehand: a looked-up element is one fp32 product and one
rounding to the output's type. A word's sum of c rows in fp32 is within (c + 2)
2^-24 of the sum of magnitudes in any order (2 for the scale and the old
value), and is rounded once."""
import pytest

from ends_util import EPS, TINY, captured, dtype_of, generator, guarded, matrix
from gpu_util import expect_device_flag
from paper_1611_06172_amd import w2v

pytestmark = pytest.mark.gpu

NAMES = ["float32", "bfloat16", "float16"]


def words(g, n, V, absent=0.1, skew=3.0):
    """Words of which low ones are frequent; some absent."""
    import torch
    ids = torch.floor(torch.rand(n, generator=g, dtype=torch.float64) ** skew * V).to(torch.int32)
    ids[torch.rand(n, generator=g) < absent] = -1
    return ids


def check_embed(ids, w, out, scale):
    import torch
    i = ids.cpu().long()
    want = w.cpu().double()[i.clamp(min=0)] * scale
    want[i < 0] = 0
    name = str(out.dtype).split(".")[1]
    bound = want.abs() * (EPS[name] + 2 * 2.0 ** -24) + TINY[name]
    assert ((out.cpu().double() - want).abs() <= bound).all()


@pytest.mark.parametrize("name", NAMES)
@pytest.mark.parametrize("out", NAMES)
@pytest.mark.parametrize("n,V,D,pad", [(1, 1, 1, 0), (7, 5, 3, 2), (64, 1000, 8, 0),
                                       (33, 77, 9, 1), (1000, 300, 300, 20), (129, 50, 641, 0)])
def test_lookup(name, out, n, V, D, pad):
    g = generator(n + D)
    ids, w = words(g, n, V).cuda(), matrix(g, V, D, name, pad=pad)
    scale = 1.0 if D % 2 else 17.25
    check_embed(ids, w, w2v.embed(ids, w, scale=scale, out_dtype=dtype_of(out)), scale)
    view, untouched = guarded(n, D, out)
    assert w2v.embed(ids, w, scale=scale, out=view) is view
    check_embed(ids, w, view, scale)
    assert untouched()


def test_lookup_of_wide_rows_and_none():
    import torch
    g = generator(1)
    w = matrix(g, 9, 20_011, "float32", pad=5)
    ids = words(g, 23, 9).cuda()
    check_embed(ids, w, w2v.embed(ids, w), 1.0)
    assert w2v.embed(ids[:0], w).shape == (0, 20_011)
    gone = torch.full((4,), -1, dtype=torch.int32, device="cuda")
    assert (w2v.embed(gone, w) == 0).all()


def test_absent_words_read_nothing_of_their_own():
    """Rows of NaN stay out of an absent word's row."""
    import torch
    w = torch.full((3, 40), float("nan"), device="cuda")
    w[1] = 2.0
    ids = torch.tensor([-1, 1, -1], dtype=torch.int32, device="cuda")
    assert w2v.embed(ids, w).tolist() == [[0.0] * 40, [2.0] * 40, [0.0] * 40]


def test_gradient_of_more_chunks_than_a_launch_has_threads():
    """72 GB cleared by blocks of 1,024 beside the sort: 4.5 x 10^9 chunks."""
    import torch
    if torch.cuda.mem_get_info()[0] < 100 << 30:
        pytest.skip("needs 100 GiB of GPU memory")
    V, D = 60_000_000, 300
    grad = torch.ones((V, D), device="cuda")
    ids = torch.tensor([V - 1, 5, 5, 31_234_567], dtype=torch.int32, device="cuda")
    dy = torch.full((4, D), 2.0, device="cuda")
    w2v.embed_backward(dy, ids, grad=grad)
    for row, want in ((V - 1, 2.0), (5, 4.0), (31_234_567, 2.0)):
        assert (grad[row] == want).all()
        grad[row] = 0
    for first in range(0, V, 1_000_000):
        assert not grad[first:first + 1_000_000].any()
    del grad
    torch.cuda.empty_cache()


def test_rows_beyond_32_bit_offsets():
    """Offsets past 2^32 elements in the matrix and past 2^31 bytes in y."""
    import torch
    V, D = 9_000_000, 512
    w = torch.empty((V, D), dtype=torch.bfloat16, device="cuda")
    at = [0, 4_194_303, 4_194_304, 8_388_607, 8_388_608, V - 1]
    for j, v in enumerate(at):
        w[v] = float(j + 1)
    ids = torch.tensor(at, dtype=torch.int32, device="cuda").repeat(400_000)
    y = w2v.embed(ids, w)
    assert torch.equal(y[:, 0].float(), torch.arange(1, 7, device="cuda").float().repeat(400_000))
    assert torch.equal(y[:, -1], y[:, 0])
    del y
    # its gradient: one row of each kind adds one to itself
    dy = torch.ones((6, D), dtype=torch.bfloat16, device="cuda")
    w2v.embed_backward(dy, ids[:6], grad=w, accumulate=True)
    assert [w[v, 0].item() for v in at] == [2.0, 3.0, 4.0, 5.0, 6.0, 7.0]
    assert [w[v, -1].item() for v in at] == [2.0, 3.0, 4.0, 5.0, 6.0, 7.0]


def test_out_of_range_words_are_reported():
    import torch
    w = torch.ones((5, 16), device="cuda")
    w2v.device_status()
    for bad in (5, -2, 2**31 - 1, -2**31):
        ids = torch.tensor([0, bad, 4], dtype=torch.int32, device="cuda")
        y = w2v.embed(ids, w)
        assert y[:, 0].tolist() == [1.0, 0.0, 1.0]
        expect_device_flag()
        grad = w2v.embed_backward(torch.ones((3, 16), device="cuda"), ids, 5)
        assert grad[:, 3].tolist() == [1.0, 0.0, 0.0, 0.0, 1.0]
        expect_device_flag()
    many = torch.full((9000,), 3, dtype=torch.int32, device="cuda")
    many[8191] = 5
    grad = w2v.embed_backward(torch.ones((9000, 16), device="cuda"), many, 5)
    assert grad[:, 3].tolist() == [0.0, 0.0, 0.0, 8999.0, 0.0]
    expect_device_flag()


def sums64(dy, ids, V, scale):
    """Sums by word, sums of magnitudes and counts."""
    import torch
    i = ids.cpu().long()
    at = i >= 0
    rows = dy.cpu().double()[at] * scale
    total = torch.zeros((V, dy.shape[1]), dtype=torch.float64)
    size = torch.zeros_like(total)
    total.index_add_(0, i[at], rows)
    size.index_add_(0, i[at], rows.abs())
    return total, size, torch.bincount(i[at], minlength=V)[:, None]


def check_back(dy, ids, out, V, scale, old=None):
    total, size, count = sums64(dy, ids, V, scale)
    if old is not None:
        total, size = total + old, size + old.abs()
    name = str(out.dtype).split(".")[1]
    bound = (count + 2) * 2.0 ** -24 * size + EPS[name] * total.abs() + TINY[name]
    got = out.cpu().double()
    assert ((got - total).abs() <= bound).all()
    if old is not None:  # rows that do not occur keep their bits
        assert (got[count[:, 0] == 0] == old[count[:, 0] == 0]).all()


@pytest.mark.parametrize("name", NAMES)
@pytest.mark.parametrize("grad", NAMES)
@pytest.mark.parametrize("n,V,D,pad", [
    (1, 1, 1, 0), (1, 1000, 300, 0), (9, 4, 7, 3), (70, 1, 64, 0), (500, 30, 9, 1),
    (3000, 700, 300, 20), (8192, 5, 16, 0), (8193, 5, 16, 0), (20_000, 3000, 33, 0),
    (600, 40, 513, 0), (300, 70, 1100, 7), (3000, 50, 100, 0), (2500, 700, 128, 1),
    (9001, 90, 200, 0), (2500, 9, 256, 0), (2500, 9, 257, 3), (70_001, 60_000, 72, 0)])
def test_gradient(name, grad, n, V, D, pad):
    g = generator(3 * n + D)
    ids, dy = words(g, n, V).cuda(), matrix(g, n, D, name, pad=pad)
    scale = -0.75
    out = w2v.embed_backward(dy, ids, V, scale=scale, dtype=dtype_of(grad))
    check_back(dy, ids, out, V, scale)
    again = w2v.embed_backward(dy, ids, V, scale=scale, dtype=dtype_of(grad))
    assert (out == again).all()
    view, untouched = guarded(V, D, grad)
    w2v.embed_backward(dy, ids, V, scale=scale, grad=view)
    assert (view == out).all() and untouched()
    view.copy_(matrix(g, V, D, grad))
    old = view.cpu().double()
    w2v.embed_backward(dy, ids, scale=scale, grad=view, accumulate=True)
    check_back(dy, ids, view, V, scale, old)
    assert untouched()


@pytest.mark.parametrize("n,V", [(40_000, 1), (300_000, 2), (300_000, 1_000_000),
                                 (100_003, 65_536), (66_000, 63), (65_536, 1_500_000),
                                 (65_537, 3), (9_000, 1_048_576), (1_200_000, 70_000)])
def test_long_runs_of_one_word(n, V):
    """A word over many chunks, words whose runs end at a chunk's end, and a
    vocabulary of several digits."""
    import torch
    g = generator(n)
    D = 24
    ids = words(g, n, V, skew=6.0)
    ids[: n // 3] = 0
    ids[n // 2: n // 2 + 64] = V - 1
    dy = matrix(g, n, D, "float32")
    check_back(dy, ids.cuda(), w2v.embed_backward(dy, ids.cuda(), V), V, 1.0)
    # counts are exact
    one = torch.ones((n, 3), dtype=torch.bfloat16, device="cuda")
    out = w2v.embed_backward(one, ids.cuda(), V, dtype=torch.float32)
    want = torch.bincount(ids[ids >= 0].long(), minlength=V).float()
    assert torch.equal(out.cpu(), want[:, None].expand(V, 3))


@pytest.mark.parametrize("run", [1, 7, 8, 9, 16, 63, 64, 65, 200])
@pytest.mark.parametrize("n", [50, 640, 70_000])
def test_equal_runs(run, n):
    """Runs of one length, whose ends meet the chunks' in every way."""
    import torch
    ids = (torch.arange(n) // run).to(torch.int32)
    V = int(ids[-1]) + 3
    ids = ids[torch.randperm(n, generator=generator(run))].cuda()
    dy = (torch.arange(n, device="cuda") % 5 + 1.0)[:, None].expand(n, 9).contiguous()
    out = w2v.embed_backward(dy, ids, V)
    want = torch.zeros(V, dtype=torch.float64).index_add_(0, ids.cpu().long(),
                                                          dy[:, 0].cpu().double())
    assert torch.equal(out.cpu().double(), want[:, None].expand(V, 9))


def test_nothing_to_add():
    import torch
    empty = torch.empty((0, 12), device="cuda")
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    assert (w2v.embed_backward(empty, none, 7) == 0).all()
    gone = torch.full((5000,), -1, dtype=torch.int32, device="cuda")
    dy = torch.full((5000, 12), float("nan"), device="cuda")
    assert (w2v.embed_backward(dy, gone, 7) == 0).all()
    old = torch.full((7, 12), 3.0, device="cuda")
    w2v.embed_backward(dy, gone, grad=old, accumulate=True)
    w2v.embed_backward(empty, none, grad=old, accumulate=True)
    assert (old == 3.0).all()


def test_nan_stays_with_its_word():
    import torch
    dy = torch.ones((200, 20), device="cuda")
    ids = (torch.arange(200, device="cuda") % 4).to(torch.int32)
    dy[6, 3] = float("nan")
    dy[7, 5] = float("inf")
    out = w2v.embed_backward(dy, ids, 4)
    assert torch.isnan(out[2, 3]) and torch.isinf(out[3, 5])
    out[2, 3] = out[3, 5] = 50.0
    assert (out == 50.0).all()


def test_gradient_against_differences():
    """The loss sum(c y) is linear in W: its difference over a step is the
    gradient, to fp32's rounding of y and of the sum."""
    import torch
    g = generator(5)
    V, D, n = 11, 20, 64
    w, c = matrix(g, V, D, "float32"), matrix(g, n, D, "float32")
    ids = words(g, n, V).cuda()
    grad = w2v.embed_backward(c, ids, V, scale=1.5).double()
    for v, d in ((0, 0), (0, 19), (3, 7), (10, 11)):
        step = torch.zeros_like(w)
        step[v, d] = 0.5
        up = (w2v.embed(ids, w + step, scale=1.5).double() * c.double()).sum()
        low = (w2v.embed(ids, w - step, scale=1.5).double() * c.double()).sum()
        size = (c.double().abs() * 6).sum()
        assert abs((up - low) - grad[v, d]) <= 4 * 2.0 ** -24 * size


def test_another_stream_and_shared_workspace():
    import torch
    g = generator(8)
    n, V, D = 20_000, 500, 40
    dy, ids = matrix(g, n, D, "bfloat16"), words(g, n, V).cuda()
    want = w2v.embed_backward(dy, ids, V)
    ws = torch.empty(w2v.embed_backward_workspace_bytes(n, V, D), dtype=torch.uint8,
                     device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    first = w2v.embed_backward(dy, ids, V, workspace=ws, stream=s)
    second = w2v.embed_backward(dy, ids, V, workspace=ws, stream=s)
    y = w2v.embed(ids, dy[:V], stream=s)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(first, want) and torch.equal(second, want)
    assert torch.equal(y, w2v.embed(ids, dy[:V]))


@pytest.mark.parametrize("n", [100, 12_000])
def test_replayed_from_a_graph(n):
    import torch
    g = generator(9)
    V, D = 900, 50
    w, dy = matrix(g, V, D, "float32"), matrix(g, n, D, "float32")
    ids = words(g, n, V).cuda()

    def call():
        return [w2v.embed(ids, w), w2v.embed_backward(dy, ids, V)]

    graph, held = captured(call)
    for i in range(4):
        ids.copy_(words(g, n, V))
        dy.copy_(torch.randn((n, D), generator=g))
        eager = call()
        graph.replay()
        torch.cuda.synchronize()
        for got, want in zip(held, eager):
            assert torch.equal(got, want)


def test_refused_arguments():
    import torch
    w = torch.zeros((5, 8), device="cuda")
    ids = torch.zeros(3, dtype=torch.int32, device="cuda")
    for call in (lambda: w2v.embed(ids.long(), w), lambda: w2v.embed(ids, w.double()),
                 lambda: w2v.embed(ids, w, out_dtype=torch.int32),
                 lambda: w2v.embed(ids, w, out=w[:3], out_dtype=torch.float16),
                 lambda: w2v.embed_backward(w[:3].double(), ids, 5),
                 lambda: w2v.embed_backward(w[:3], ids, 5, dtype=torch.float64)):
        with pytest.raises(TypeError):
            call()
    for call in (lambda: w2v.embed(ids, w.t()), lambda: w2v.embed(ids.view(3, 1), w),
                 lambda: w2v.embed(ids, w, out=torch.zeros((4, 8), device="cuda")),
                 lambda: w2v.embed_backward(w, ids, 5), lambda: w2v.embed_backward(w[:3], ids),
                 lambda: w2v.embed_backward(w[:3], ids, 5, accumulate=True),
                 lambda: w2v.embed_backward(w[:3], ids, 4, grad=w),
                 lambda: w2v.embed_backward(w[:3], ids, grad=torch.zeros((5, 9), device="cuda"))):
        with pytest.raises(ValueError):
            call()


@pytest.mark.parametrize("n,V", [(20_000, 700), (20_000, 5_000), (300_000, 5_000),
                                 (300_000, 2_000_000)])
def test_words_that_change_during_the_call(n, V):
    """Every row is added to one of the words that stood in its place, once, whatever
    another stream writes there meanwhile: the sums are of whole numbers below 2^24, so
    nothing is rounded."""
    import torch
    g = generator(n + V)
    a = torch.randint(0, V, (n,), generator=g, dtype=torch.int32).cuda()
    b = (V - 1 - a).contiguous()
    dy = torch.randint(-3, 4, (n, 8), generator=g).float().cuda()
    want = dy.double().sum(0)
    ids = a.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(10):
        with torch.cuda.stream(side):
            for _ in range(20):
                ids.copy_(b)
                ids.copy_(a)
        grad = w2v.embed_backward(dy, ids, V)
        assert torch.equal(grad.double().sum(0), want)
    side.synchronize()
    check = torch.zeros((V, 8), dtype=torch.float64, device="cuda")
    check.index_add_(0, a.long(), dy.double())
    assert torch.equal(w2v.embed_backward(dy, ids, V).double(), check)
