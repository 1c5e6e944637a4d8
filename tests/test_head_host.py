"""Refusals of the vocabulary head's entry points, which come before any HIP
call, and its workspace sizes (host only)."""
import pytest

from paper_1611_06172_amd import w2v

FAKE = 0x100000  # never dereferenced: validation fails first


def refused(entry, args, needle, code=w2v.EINVAL):
    assert entry(*args.values()) == code
    assert needle in w2v.lib().w2v_last_error().decode()


def linear_args(**over):
    args = dict(x=FAKE, ldx=8, w=FAKE, ldw=8, bias=None, r=None, ldr=5, y=FAKE, ldy=5,
                pre=None, ldp=5, M=4, N=5, K=8, dtype=0, out=0, act=0, ws=None, ws_bytes=0,
                stream=None)
    args.update(over)
    return args


@pytest.mark.parametrize("over,needle", [
    (dict(M=-1), "M"), (dict(N=0), "N"), (dict(K=0), "K"), (dict(dtype=3), "dtype"),
    (dict(dtype=-1), "dtype"), (dict(out=1), "out_dtype"), (dict(dtype=1, out=2), "out_dtype"),
    (dict(act=6), "activation"), (dict(act=-1), "activation"), (dict(x=None), "x"),
    (dict(w=None), "w"), (dict(y=None), "y"), (dict(ldx=7), "x: the row stride"),
    (dict(ldw=7), "w: the row stride"), (dict(ldy=4), "y: the row stride"),
    (dict(r=FAKE, ldr=4), "residual"), (dict(pre=FAKE, ldp=4), "pre"),
    (dict(x=FAKE + 2), "x must be aligned"), (dict(bias=FAKE + 1), "bias"),
    (dict(ldx=1 << 62), "out of range"),
    (dict(M=40, K=20_000, ldx=20_000, ldw=20_000), "workspace must hold"),
    (dict(M=40, K=20_000, ldx=20_000, ldw=20_000, ws=FAKE + 64, ws_bytes=1 << 40), "aligned"),
])
def test_linear_rejects(over, needle):
    refused(w2v.lib().w2v_linear, linear_args(**over), needle)


def test_linear_residual_in_the_output_has_its_stride():
    """Another stride over the same memory would read rows that are written."""
    refused(w2v.lib().w2v_linear, linear_args(r=FAKE, ldr=6, ldy=5), "stride")
    # as it is, the call gets as far as its workspace
    refused(w2v.lib().w2v_linear, linear_args(r=FAKE, ldr=6, ldy=6, M=40, K=20_000,
                                              ldx=20_000, ldw=20_000), "workspace must hold")


def test_linear_blocks_fit_a_grid():
    """More blocks than a grid's 2^32 threads hold are refused, not launched;
    a large output of 128 x 128 tiles is not among them."""
    refused(w2v.lib().w2v_linear, linear_args(M=1, N=2**30 + 1, K=1, ldr=2**30 + 1,
                                              ldy=2**30 + 1, ldp=2**30 + 1), "launch",
            w2v.EUNSUPPORTED)
    refused(w2v.lib().w2v_linear_backward, backward_args(M=2**31 - 64, N=5, K=3), "launch",
            w2v.EUNSUPPORTED)
    import torch
    assert w2v.linear_workspace_bytes(1_000_000, 100_000, 300, torch.bfloat16) > 0


def test_linear_too_many_tiles():
    big = 2**31 - 1
    refused(w2v.lib().w2v_linear, linear_args(M=big, N=big, ldr=big, ldy=big, ldp=big),
            "tiles", w2v.EUNSUPPORTED)


def backward_args(**over):
    args = dict(dy=FAKE, lddy=5, x=FAKE, ldx=8, w=FAKE, ldw=8, pre=None, ldp=5, dx=FAKE,
                lddx=8, dw=FAKE, lddw=8, db=FAKE, M=4, N=5, K=8, dtype=0, act=0, ws=None,
                ws_bytes=0, stream=None)
    args.update(over)
    return args


@pytest.mark.parametrize("over,needle", [
    (dict(M=-1), "M"), (dict(N=0), "N"), (dict(K=0), "K"), (dict(dtype=9), "dtype"),
    (dict(act=7), "activation"), (dict(dy=None), "dy"), (dict(x=None), "x"),
    (dict(w=None), "w"), (dict(lddy=4), "dy"), (dict(ldx=7), "x"), (dict(ldw=7), "w"),
    (dict(lddx=7), "dx"), (dict(lddw=7), "dw"), (dict(db=FAKE + 2), "db"),
    (dict(act=1), "pre is NULL"), (dict(act=1, pre=FAKE, ldp=4), "pre"),
    (dict(act=1, pre=FAKE), "workspace must hold"),
])
def test_linear_backward_rejects(over, needle):
    refused(w2v.lib().w2v_linear_backward, backward_args(**over), needle)


def test_linear_workspaces():
    import torch
    assert w2v.linear_workspace_bytes(512, 1_000_000, 300, torch.float32) == 0
    # copies of x and W with rows on 64-byte lines
    assert w2v.linear_workspace_bytes(4_096, 71_290, 300, torch.bfloat16) >= \
        (4_096 + 71_290) * 320 * 2
    assert w2v.linear_workspace_bytes(1, 1_000_000, 300, torch.float32) == 0
    n = w2v.linear_backward_workspace_bytes(64, 71_290, 300, torch.bfloat16)
    assert n > 0 and n % 256 == 0
    # an activation adds its dz
    assert w2v.linear_backward_workspace_bytes(
        64, 71_290, 300, torch.bfloat16, "silu") >= n + 64 * 71_290 * 2
    assert w2v.lib().w2v_linear_workspace_bytes(-1, 5, 5, 0) == 0
    assert w2v.lib().w2v_linear_workspace_bytes(1, 5, 5, 7) == 0


def distill_args(**over):
    args = dict(logits=FAKE, ld=100, rows=4, V=100, dtype=0, ids=FAKE, teacher=FAKE, K=8,
                tdtype=0, labels=None, T=2.0, soft=1.0, hard=0.0, weight=None, loss=FAKE,
                stats=FAKE, grad=FAKE, ldg=100, ws=FAKE, ws_bytes=1 << 30, stream=None)
    args.update(over)
    return args


@pytest.mark.parametrize("over,needle", [
    (dict(rows=-1), "rows"), (dict(V=0), "V"), (dict(dtype=3), "dtype"),
    (dict(tdtype=-1), "teacher_dtype"), (dict(K=-1), "K"), (dict(K=1025), "K"),
    (dict(T=0.0), "temperature"), (dict(T=float("nan")), "temperature"),
    (dict(T=2.0**21), "temperature"), (dict(soft=float("inf")), "soft"),
    (dict(hard=float("nan")), "hard"), (dict(ids=None), "ids"),
    (dict(teacher=None), "teacher"), (dict(ids=FAKE + 2), "ids"),
    (dict(logits=None), "logits"), (dict(ld=99), "logits"), (dict(loss=None), "loss"),
    (dict(stats=None), "stats"), (dict(ldg=99), "grad"), (dict(labels=FAKE + 1), "labels"),
    (dict(weight=FAKE + 1), "row_weight"), (dict(ws=None), "workspace"),
    (dict(ws=FAKE + 8), "aligned"), (dict(ld=120, ldg=110, grad=FAKE), "stride"),
])
def test_distill_rejects(over, needle):
    refused(w2v.lib().w2v_distill_loss, distill_args(**over), needle)


@pytest.mark.parametrize("over,needle", [
    (dict(rows=-1), "rows"), (dict(K=1025), "K"), (dict(T=-1.0), "temperature"),
    (dict(dloss=None), "dloss"), (dict(stats=None), "stats"), (dict(grad=None), "grad"),
    (dict(grad=FAKE, ldg=101), "stride"), (dict(logits=None), "logits"),
])
def test_distill_backward_rejects(over, needle):
    args = dict(dloss=FAKE, logits=FAKE, ld=100, rows=4, V=100, dtype=0, ids=FAKE,
                teacher=FAKE, K=8, tdtype=0, labels=None, T=2.0, soft=1.0, hard=0.0,
                stats=FAKE, grad=FAKE, ldg=100, stream=None)
    args.update(over)
    refused(w2v.lib().w2v_distill_backward, args, needle)


@pytest.mark.parametrize("over,needle,code", [
    (dict(rows=-1), "rows", -1), (dict(V=0), "V", -1), (dict(dtype=5), "dtype", -1),
    (dict(z=None), "logits", -1), (dict(ld=199_999), "logits", -1), (dict(u=None), "uniforms", -1),
    (dict(ldu=199_999), "uniforms", -1), (dict(T=-1.0), "temperature", -1),
    (dict(T=float("inf")), "temperature", -1), (dict(k=-1), "top_k", -1),
    (dict(V=5000, ld=5000, ldu=5000, k=1025), "top_k", -4), (dict(p=0.0), "top_p", -1),
    (dict(p=float("nan")), "top_p", -1), (dict(least=-0.1), "min_p", -1),
    (dict(least=1.1), "min_p", -1), (dict(ids=None), "ids", -1), (dict(ts=FAKE + 1),
                                                                "temperatures", -1),
    (dict(lp=FAKE + 2), "logprob", -1), (dict(ws=None), "workspace", -1),
    (dict(ws_bytes=10), "workspace", -1), (dict(ws=FAKE + 8), "aligned", -1),
])
def test_sample_rejects(over, needle, code):
    args = dict(z=FAKE, ld=200_000, u=FAKE, ldu=200_000, rows=4, V=200_000, dtype=0, ts=None, T=1.0,
                ks=None, k=0, ps=None, p=1.0, ms=None, least=0.0, ids=FAKE, lp=None, ws=FAKE,
                ws_bytes=1 << 30, stream=None)
    args.update(over)
    refused(w2v.lib().w2v_sample_words, args, needle, code)


def test_sample_workspace():
    """Short rows, and enough rows, are a block's each and need none."""
    assert w2v.sample_workspace_bytes(4, 1000) == 0
    assert w2v.sample_workspace_bytes(65_536, 1_000_000) == 0
    assert w2v.sample_workspace_bytes(4, 1_000_000) % 256 == 0
    assert w2v.sample_workspace_bytes(4, 1_000_000) > 0
    assert w2v.sample_workspace_bytes(-1, 10) == 0
