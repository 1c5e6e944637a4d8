"""How far w2v_linear_q4's sums are rounded: no farther than a product in fp32, whatever
the mean of x, as behind a relu or a residual, and of its columns.

Tolerance, fixed beforehand, from independent roundings, each of the same share of the
sum it is made of. A product in fp32 that rounds behind each of K columns makes K of
them. The kernel rounds a group's sum at most once for every 4 columns, and twice more
for the scale and the row's sum: K / 4 + 2 G in all, G the groups. Where the matrix
instruction cuts a product's bits off instead of rounding it, the error is twice as
large: 2 root((K / 4 + 2 G) / K) of the other error."""
import pytest

from ends_util import generator
from paper_1611_06172_amd import w2v
from test_gpu_linear_q4 import random_q4, unpacked

pytestmark = pytest.mark.gpu


def weights64(q):
    import torch
    (N, K), group = q["shape"], q["group"]
    code, scale = unpacked(q)
    return ((code.double() - 8) * torch.repeat_interleave(scale.double(), group, dim=1))[:N, :K]


def column_by_column(x, w):
    """x w^T in fp32, rounded behind each column."""
    import torch
    y = torch.zeros((x.shape[0], w.shape[0]))
    for k in range(x.shape[1]):
        y = (y.double() + x[:, k, None].double() * w[None, :, k]).float()
    return y


def inputs(kind, M, K, g):
    import torch
    x = torch.randn((M, K), generator=g)
    if kind == "relu":
        return x.clamp(min=0)
    if kind == "turns":  # means of neighbouring columns have opposite signs
        return x + torch.tensor([2.0, -2.0]).repeat(K // 2)
    if kind == "outlier":
        x[:, 7] *= 100
        return x
    return x + kind


@pytest.mark.parametrize("kind", [0.0, 1.0, -3.0, "relu", "turns", "outlier"])
@pytest.mark.parametrize("name", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("M", [1, 9, 20, 40])
def test_sums_are_as_exact_as_those_of_fp32(M, group, name, kind):
    import torch
    g = generator(M + group)
    N, K = 500, 384
    q = w2v.quantize_q4((torch.randn((N, K), generator=g) * 0.05).cuda(), group=group)
    x = inputs(kind, M, K, g).to(getattr(torch, name))
    w = weights64(q)
    want = x.double() @ w.t()
    got = w2v.linear_q4(x.cuda(), q, out_dtype=torch.float32).cpu().double()

    def rms(t):
        return float((t.double() - want).square().mean().sqrt())

    roundings = K / 4 + 2 * K / group
    assert rms(got) <= rms(column_by_column(x, w)) * 2 * (roundings / K) ** 0.5


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("M,K", [(1, 300), (16, 96), (20, 300), (40, 300), (3, 3001), (40, 1401),
                                 (20, 4500)])
def test_every_bit_of_float32(M, K, group):
    """A column on its own, of 24 bits, in every kernel: the products of its three pieces
    are exact, two sums of them and the scale's product are rounded, each to 2^-23 where
    bits are cut off, and the zeros of other groups are added."""
    import torch
    g = generator(M + K)
    N = 70
    q = random_q4(g, N, K, group)
    w = weights64(q)
    for column in {0, K // 2 + 1, K - 1}:
        x = torch.zeros((M, K))
        x[:, column] = torch.randn(M, generator=g) * 2.0 ** torch.randint(
            -40, 40, (M,), generator=g).float()
        got = w2v.linear_q4(x.cuda(), q).cpu().double()
        want = x.double() @ w.t()
        assert ((got - want).abs() <= 6 * 2.0 ** -24 * want.abs()).all()


def test_many_rows_of_x():
    """More than a hundred tiles of rows, the last with a remainder."""
    import torch
    g = generator(8)
    M, N, K = 5_001, 40, 33
    q = random_q4(g, N, K, 32)
    for name in ("float32", "bfloat16"):
        x = torch.randn((M, K), generator=g).to(getattr(torch, name))
        got = w2v.linear_q4(x.cuda(), q, out_dtype=torch.float32).cpu().double()
        w = weights64(q)
        want = x.double() @ w.t()
        # K products and G = 2 scales, each rounded to 2^-23 at most
        bound = 2 * (K + 4) * 2.0 ** -24 * (x.double().abs() @ w.abs().t())
        assert ((got - want).abs() <= bound).all()


@pytest.mark.parametrize("name", ["float32", "bfloat16", "float16"])
def test_an_infinity_in_any_column(name):
    """Its row is NaN, also where it meets a weight of 0; others are as they were."""
    import torch
    g = generator(9)
    K = 37
    q = random_q4(g, 20, K, 32)
    x = torch.randn((K + 1, K), generator=g).to(getattr(torch, name)).cuda()
    want = w2v.linear_q4(x, q)
    for bad in (float("inf"), -float("inf"), float("nan")):
        y = x.clone()
        y[torch.arange(K), torch.arange(K)] = bad
        got = w2v.linear_q4(y, q)
        assert torch.isnan(got[:K]).all() and torch.equal(got[K], want[K])


def test_large_numbers_do_not_overflow():
    """Sums are of |x (q - 8)|: x of 2^120 whose result fits stay finite."""
    import torch
    w = torch.zeros((3, 64))
    w[0, :2], w[1, 40], w[2, :] = torch.tensor([7.0, -7.0]), 7.0, 7.0
    q = w2v.quantize_q4((w / 1024).cuda())
    for name in ("float32", "bfloat16"):
        x = torch.full((1, 64), 2.0 ** 120).to(getattr(torch, name))
        got = w2v.linear_q4(x.cuda(), q, out_dtype=torch.float32).cpu().double()
        want = x.double() @ weights64(q).t()
        assert ((got - want).abs() <= 66 * 2.0 ** -23 * want.abs()).all() and got[0, 0] == 0
