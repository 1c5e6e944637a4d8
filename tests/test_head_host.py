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
    assert w2v.linear_workspace_bytes(4_096, 71_290, 300, torch.bfloat16) == 0
    assert w2v.linear_workspace_bytes(1, 1_000_000, 300, torch.float32) == 0
    n = w2v.linear_backward_workspace_bytes(64, 71_290, 300, torch.bfloat16)
    assert n > 0 and n % 256 == 0
    # an activation adds its dz
    assert w2v.linear_backward_workspace_bytes(
        64, 71_290, 300, torch.bfloat16, "silu") >= n + 64 * 71_290 * 2
    assert w2v.lib().w2v_linear_workspace_bytes(-1, 5, 5, 0) == 0
    assert w2v.lib().w2v_linear_workspace_bytes(1, 5, 5, 7) == 0
