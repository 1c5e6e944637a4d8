"""Products that are large enough for the widest tiles, for copies with aligned
rows and for splits of those tiles, against products in 64 bits. Which shape
takes which kernel is in head_shapes.py. Tolerances as in test_gpu_linear.py;
sums of more than 100 products meet in a tree of tiles and blocks, so sqrt(K) of
the any-order bound is used for them, as there."""
import math

import pytest

import head_shapes as shapes
from paper_1611_06172_amd import w2v
from test_gpu_linear import EPS, act64, check, dtype_of, generator, matrix, slope64

pytestmark = pytest.mark.gpu


def terms(K):
    return K if K <= 100 else 2 * math.sqrt(K)


def mm64(a, b):
    """The product in 64 bits and that of absolute values."""
    import torch
    a, b = a.double(), b.double().contiguous()
    return torch.mm(a, b).cpu(), torch.mm(a.abs(), b.abs()).cpu()


def aligned(t):
    """The same values in rows on 64-byte lines."""
    import torch
    cols = (t.shape[1] + 31) // 32 * 32
    out = torch.empty((t.shape[0], cols), dtype=t.dtype, device=t.device)[:, :t.shape[1]]
    out.copy_(t)
    return out


@pytest.mark.parametrize("M,N,K,name", list(shapes.FORWARD))
def test_forward(M, N, K, name):
    import torch
    g = generator(M + N + K)
    x, w = matrix(g, M, K, name, pad=3), matrix(g, N, K, name, K ** -0.5, pad=1)
    b = torch.randn(N, generator=g).cuda()
    got = w2v.linear(x, w, b)
    z, sums = mm64(x, w.t())
    z, sums = z + b.double().cpu(), sums + b.abs().double().cpu()
    check(got, z, sums, terms(K), name)
    # rows that need no copy: the same sums
    assert torch.equal(w2v.linear(aligned(x), aligned(w), b), got)
    assert torch.equal(w2v.linear(x, w, b), got)
    if name != shapes.F32:
        check(w2v.linear(x, w, b, out_dtype=torch.float32), z, sums, terms(K), "float32")


@pytest.mark.parametrize("activation", ["gelu", "silu", "none"])
@pytest.mark.parametrize("M,N,K,name", list(shapes.FORWARD))
def test_whole_epilogue(M, N, K, name, activation):
    import torch
    g = generator(M + N + K + 1)
    x, w = matrix(g, M, K, name, pad=1), matrix(g, N, K, name, 2 * K ** -0.5, pad=2)
    b = torch.randn(N, generator=g).cuda()
    r = matrix(g, M, N, name, pad=5)
    pre = torch.full((M, N + 3), 9.0, dtype=dtype_of(name), device="cuda")
    buf = torch.full((M, N + 1), 7.0, dtype=dtype_of(name), device="cuda")
    got = w2v.linear(x, w, b, activation=activation, residual=r, out=buf[:, :N],
                     pre=pre[:, :N])
    z, sums = mm64(x, w.t())
    z, sums = z + b.double().cpu(), sums + b.abs().double().cpu()
    check(pre[:, :N], z, sums, terms(K), name)
    R = r.double().cpu()
    check(got, act64(z, activation) + R, sums + R.abs(), terms(K), name)
    assert (buf[:, N] == 7.0).all() and (pre[:, N:] == 9.0).all()
    again = w2v.linear(x, w, b, activation=activation, residual=r, out=r)
    assert torch.equal(again, got)


@pytest.mark.parametrize("activation", ["none", "silu"])
@pytest.mark.parametrize("M,N,K,name", list(shapes.BACKWARD))
def test_backward(M, N, K, name, activation):
    import torch
    g = generator(M + N + K + 2)
    x, w = matrix(g, M, K, name, pad=1), matrix(g, N, K, name, N ** -0.5, pad=3)
    dy, pre = matrix(g, M, N, name, pad=2), matrix(g, M, N, name, 2.0, pad=1)
    kw = {} if activation == "none" else {"activation": activation, "pre": pre}
    out = w2v.linear_backward(dy, x, w, **kw)
    dz = dy.double() * slope64(pre.double(), activation)
    # dz is rounded once where there is an activation, its slope within 8 units
    # of 2^-24 of 1.1
    eps = 0.0 if activation == "none" else EPS[name] + 9 * 2.0 ** -24
    low = 0.0 if activation == "none" else 2.0 ** -24
    want, sums = mm64(dz, w)
    check(out["dx"], want, sums, terms(N), name,
          eps * sums + low * w.double().abs().sum(dim=0).cpu())
    want, sums = mm64(dz.t().contiguous(), x)
    check(out["dw"], want, sums, terms(M), name,
          eps * sums + low * x.double().abs().sum(dim=0).cpu())
    ab = dy.double().abs().sum(dim=0).cpu()
    check(out["db"], dz.sum(dim=0).cpu(), ab, terms(M), "float32",
          0.0 if activation == "none" else 9 * 2.0 ** -24 * 1.13 * ab)
    again = w2v.linear_backward(dy, x, w, **kw)
    assert all(torch.equal(out[k], again[k]) for k in out)


@pytest.mark.parametrize("M,N,K,name", [(4_099, 4_001, 72, "bfloat16"),
                                        (3_300, 3_203, 40, "float16"),
                                        (600, 30_001, 513, "bfloat16"),
                                        (40, 70, 20_000, "float32")])
def test_what_the_workspace_held_does_not_matter(M, N, K, name):
    import torch
    g = generator(M)
    x, w = matrix(g, M, K, name, pad=1), matrix(g, N, K, name, K ** -0.5, pad=1)
    dy, pre = matrix(g, M, N, name, 0.1), matrix(g, M, N, name)
    y = w2v.linear(x, w)
    d = w2v.linear_backward(dy, x, w, activation="gelu", pre=pre)
    n = max(w2v.linear_workspace_bytes(M, N, K, x.dtype),
            w2v.linear_backward_workspace_bytes(M, N, K, x.dtype, "gelu"))
    for byte in (255, 0):  # NaN in every type, zeros
        ws = torch.full((n + 256,), byte, dtype=torch.uint8, device="cuda")
        assert torch.equal(w2v.linear(x, w, workspace=ws), y)
        assert (ws[w2v.linear_workspace_bytes(M, N, K, x.dtype):] == byte).all()
        ws.fill_(byte)
        got = w2v.linear_backward(dy, x, w, activation="gelu", pre=pre, workspace=ws)
        assert all(torch.equal(got[k], d[k]) for k in d)
        used = w2v.linear_backward_workspace_bytes(M, N, K, x.dtype, "gelu")
        assert (ws[used:] == byte).all()
