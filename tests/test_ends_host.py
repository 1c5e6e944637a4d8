"""Refusals of the entry points of a word model's ends (embedding, dropout, 4-bit
products, beam search), which come before any HIP call, and their sizes (host
only)."""
import ctypes

import pytest

from paper_1611_06172_amd import w2v

FAKE = 0x100000  # never dereferenced: validation fails first


def refused(entry, args, needle, code=w2v.EINVAL):
    assert entry(*args.values()) == code
    assert needle in w2v.lib().w2v_last_error().decode()


@pytest.mark.parametrize("over,needle", [
    (dict(n=-1), "n must"), (dict(V=0), "V"), (dict(D=0), "D"), (dict(dtype=3), "dtype"),
    (dict(out=-1), "out_dtype"), (dict(scale=float("inf")), "scale"),
    (dict(scale=float("nan")), "scale"), (dict(ids=None), "ids"), (dict(ids=FAKE + 2), "ids"),
    (dict(w=None), "weight"), (dict(ldw=7), "weight: the row stride"), (dict(w=FAKE + 2), "weight"),
    (dict(y=None), "y"), (dict(ldy=7), "y: the row stride"), (dict(y=FAKE + 1, out=1), "y"),
    (dict(ldw=1 << 62), "out of range"),
])
def test_embed_rejects(over, needle):
    args = dict(ids=FAKE, n=4, w=FAKE, ldw=8, V=10, D=8, dtype=0, scale=1.0, y=FAKE, ldy=8,
                out=0, stream=None)
    args.update(over)
    refused(w2v.lib().w2v_embed, args, needle)


@pytest.mark.parametrize("over,needle", [
    (dict(n=-1), "n must"), (dict(V=0), "V"), (dict(D=0), "D"), (dict(dtype=3), "dtype"),
    (dict(gdtype=7), "grad_dtype"), (dict(scale=float("nan")), "scale"), (dict(ids=None), "ids"),
    (dict(dy=None), "dy"), (dict(lddy=7), "dy"), (dict(grad=None), "grad"), (dict(ldg=7), "grad"),
    (dict(add=2), "accumulate"), (dict(add=-1), "accumulate"), (dict(ws=None), "workspace must"),
    (dict(ws_bytes=10), "workspace must"), (dict(ws=FAKE + 8), "aligned"),
])
def test_embed_backward_rejects(over, needle):
    args = dict(dy=FAKE, lddy=8, ids=FAKE, n=4, dtype=0, scale=1.0, grad=FAKE, ldg=8, V=10, D=8,
                gdtype=0, add=0, ws=FAKE, ws_bytes=1 << 30, stream=None)
    args.update(over)
    refused(w2v.lib().w2v_embed_backward, args, needle)


def test_embed_wide_rows():
    args = dict(ids=FAKE, n=4, w=FAKE, ldw=1 << 25, V=10, D=(1 << 24) + 1, dtype=0, scale=1.0,
                y=FAKE, ldy=1 << 25, out=0, stream=None)
    refused(w2v.lib().w2v_embed, args, "D must be at most", w2v.EUNSUPPORTED)
    assert w2v.embed_backward_workspace_bytes(0, 10, 8) == 0
    assert w2v.embed_backward_workspace_bytes(-1, 10, 8) == 0
    assert w2v.embed_backward_workspace_bytes(5, 10, 8) % 256 == 0
    assert w2v.embed_backward_workspace_bytes(5, 10, 8) > 0


@pytest.mark.parametrize("over,needle,code", [
    (dict(rows=-1), "rows", -1), (dict(cols=0), "cols", -1),
    (dict(cols=(1 << 30) + 1, ldx=1 << 31, ldy=1 << 31), "cols", -4), (dict(dtype=9), "dtype", -1),
    (dict(p=-0.1), "p must", -1), (dict(p=1.5), "p must", -1), (dict(p=float("nan")), "p must", -1),
    (dict(x=None), "x is NULL", -1), (dict(ldx=7), "x: the row", -1), (dict(y=None), "y", -1),
    (dict(ldy=7), "y: the row", -1), (dict(r=FAKE, ldr=7), "residual", -1),
    (dict(x=FAKE, y=FAKE, ldx=9, ldy=8), "stride", -1),
    (dict(r=FAKE + 64, y=FAKE + 64, ldr=9), "stride", -1), (dict(dev=FAKE + 4), "offset_dev", -1),
    (dict(x=FAKE + 2), "x must be aligned", -1),
])
def test_dropout_rejects(over, needle, code):
    args = dict(x=FAKE, ldx=8, r=None, ldr=8, y=FAKE + 64, ldy=8, rows=4, cols=8, dtype=0, p=0.1,
                seed=1, offset=2, dev=None, stream=None)
    args.update(over)
    refused(w2v.lib().w2v_dropout, args, needle, code)


@pytest.mark.parametrize("over,needle", [
    (dict(N=0), "N"), (dict(K=0), "K"), (dict(group=16), "group"), (dict(group=0), "group"),
    (dict(dtype=3), "dtype"), (dict(w=None), "w is NULL"), (dict(ldw=7), "w: the row"),
    (dict(packed=None), "packed"), (dict(packed=FAKE + 8), "packed"), (dict(scales=None), "scales"),
    (dict(scales=FAKE + 1), "scales"), (dict(scales=FAKE + 2), "16-byte"),
])
def test_quantize_rejects(over, needle):
    args = dict(w=FAKE, ldw=8, N=4, K=8, dtype=0, group=32, packed=FAKE, scales=FAKE, stream=None)
    args.update(over)
    refused(w2v.lib().w2v_quantize_q4, args, needle)


@pytest.mark.parametrize("over,needle,code", [
    (dict(M=-1), "M", -1), (dict(M=(1 << 20) + 1), "M must be at most", -4), (dict(N=0), "N", -1),
    (dict(K=0), "K", -1), (dict(group=96), "group", -1), (dict(dtype=3), "dtype", -1),
    (dict(out=1), "out_dtype", -1), (dict(dtype=1, out=2), "out_dtype", -1),
    (dict(x=None), "x", -1), (dict(ldx=7), "x: the row", -1), (dict(packed=None), "packed", -1),
    (dict(scales=FAKE + 2), "scales", -1), (dict(y=None), "y", -1), (dict(ldy=4), "y: the row", -1),
    (dict(bias=FAKE + 2), "bias", -1), (dict(K=(1 << 24) + 1, ldx=1 << 25), "K must", -4),
])
def test_linear_q4_rejects(over, needle, code):
    args = dict(x=FAKE, ldx=8, packed=FAKE, scales=FAKE, bias=None, y=FAKE, ldy=5, M=4, N=5, K=8,
                group=32, dtype=0, out=0, stream=None)
    args.update(over)
    refused(w2v.lib().w2v_linear_q4, args, needle, code)


@pytest.mark.parametrize("N,K,group,blocks,groups", [
    (16, 32, 32, 1, 1), (17, 33, 32, 2, 2), (1, 300, 32, 10, 10), (1, 300, 64, 10, 5),
    (1, 300, 128, 12, 3), (71_290, 600, 64, 20, 10),
])
def test_q4_sizes(N, K, group, blocks, groups):
    tiles = (N + 15) // 16
    assert w2v.lib().w2v_q4_packed_bytes(N, K, group) == tiles * blocks * 256
    assert w2v.lib().w2v_q4_scale_count(N, K, group) == tiles * groups * 16
    assert w2v.lib().w2v_q4_packed_bytes(N, K, 48) == 0
    assert w2v.lib().w2v_q4_scale_count(0, K, group) == 0


def beam_args(**over):
    args = dict(z=FAKE, ld=100, batch=2, beams=3, V=100, dtype=0, scores=FAKE, finished=None,
                end=-1, width=4, words=FAKE, parents=FAKE, new=FAKE + 64, ended=None, ws=FAKE,
                ws_bytes=1 << 30, stream=None)
    args.update(over)
    return args


@pytest.mark.parametrize("over,needle", [
    (dict(batch=-1), "batch"), (dict(beams=0), "beams"), (dict(beams=65), "beams"),
    (dict(width=0), "width"), (dict(width=65), "width"), (dict(V=0), "V"), (dict(dtype=3), "dtype"),
    (dict(end=-2), "end"), (dict(end=100), "end"), (dict(finished=FAKE), "finished needs"),
    (dict(z=None), "logits"), (dict(ld=99), "logits"), (dict(scores=None), "scores"),
    (dict(words=None), "words"), (dict(parents=None), "parents"), (dict(new=None), "new_scores"),
    (dict(new=FAKE), "in place"), (dict(finished=FAKE, ended=FAKE, end=1), "in place"),
    (dict(ws=None), "workspace must"), (dict(ws_bytes=8), "workspace must"),
    (dict(ws=FAKE + 8), "aligned"), (dict(scores=FAKE + 2), "scores"),
])
def test_beam_step_rejects(over, needle):
    refused(w2v.lib().w2v_beam_step, beam_args(**over), needle)


def test_beam_batches_beyond_31_bits():
    refused(w2v.lib().w2v_beam_step, beam_args(batch=1 << 26), "batch must be at most",
            w2v.EUNSUPPORTED)
    assert w2v.lib().w2v_beam_step_workspace_bytes(0, 3, 3, 100, 0) == 0
    assert w2v.lib().w2v_beam_step_workspace_bytes(2, 65, 3, 100, 0) == 0
    assert w2v.lib().w2v_beam_step_workspace_bytes(2, 3, 3, 100, 0) % 256 == 0


@pytest.mark.parametrize("places", [((0, 1), (1, 0)), ((0, 2), (1, 2)), ((0, 2), (1, 0))])
def test_beam_reorder_rejects_states_that_change_places(places):
    table = (w2v._BeamState * 2)(*(
        w2v._BeamState(src=FAKE + 4096 * src, src_stride=8, dst=FAKE + 4096 * dst, dst_stride=8,
                       row_bytes=8) for src, dst in places))
    refused(w2v.lib().w2v_beam_reorder,
            dict(states=table, count=2, parents=FAKE, batch=2, beams=3, width=3, stream=None),
            "in place")


@pytest.mark.parametrize("over,needle,code", [
    (dict(count=-1), "count", -1), (dict(count=17), "count", -1), (dict(states=None), "states", -1),
    (dict(parents=None), "parents", -1), (dict(beams=0), "beams", -1), (dict(width=65), "width", -1),
    (dict(state=dict(row_bytes=0)), "row_bytes", -1),
    (dict(state=dict(row_bytes=(1 << 34) + 1)), "too many bytes", -4),
    (dict(state=dict(src_stride=7)), "strides", -1), (dict(state=dict(dst_stride=7)), "strides", -1),
    (dict(state=dict(src=None)), "NULL", -1), (dict(state=dict(dst=None)), "NULL", -1),
    (dict(state=dict(dst=FAKE)), "in place", -1),
    (dict(state=dict(src_stride=1 << 62)), "out of range", -1),
])
def test_beam_reorder_rejects(over, needle, code):
    state = dict(src=FAKE, src_stride=8, dst=FAKE + 4096, dst_stride=8, row_bytes=8)
    state.update(over.pop("state", {}))
    table = (w2v._BeamState * 1)(w2v._BeamState(**state))
    args = dict(states=table, count=1, parents=FAKE, batch=2, beams=3, width=3, stream=None)
    args.update(over)
    if args["states"] is None:
        args["states"] = ctypes.cast(None, ctypes.POINTER(w2v._BeamState))
    refused(w2v.lib().w2v_beam_reorder, args, needle, code)


def test_binding_rejects():
    """What the binding itself refuses, with CPU tensors."""
    import torch
    ids, w = torch.zeros(3, dtype=torch.int32), torch.zeros((4, 8))
    for call in (lambda: w2v.embed(ids, w), lambda: w2v.embed_backward(w, ids, 5),
                 lambda: w2v.dropout(w, 0.1, seed=1), lambda: w2v.quantize_q4(w),
                 lambda: w2v.beam_step(w, torch.zeros((2, 2))),
                 lambda: w2v.beam_reorder(w, ids.view(1, 3))):
        with pytest.raises(TypeError):
            call()


@pytest.mark.parametrize("group", [32, 64, 128])
def test_sizes_of_a_matrix_in_4_bits(group):
    """What the binding expects of a dict's arrays without asking the library."""
    for N in (1, 16, 17, 71_290):
        for K in (1, 31, 33, 300, 1000):
            tiles, groups = (N + 15) // 16, (K + group - 1) // group
            assert w2v.lib().w2v_q4_packed_bytes(N, K, group) == tiles * groups * group * 8
            assert w2v.lib().w2v_q4_scale_count(N, K, group) == tiles * groups * 16


def test_most_rows_of_a_4_bit_product():
    """W2V_MAX_Q4_ROWS is 524,288, in the header and in the check."""
    args = dict(x=FAKE, ldx=8, packed=FAKE, scales=FAKE, bias=None, y=FAKE, ldy=5, M=524_289, N=5,
                K=8, group=32, dtype=0, out=0, stream=None)
    refused(w2v.lib().w2v_linear_q4, args, "M must be at most 524288", w2v.EUNSUPPORTED)
    # as many as that pass it: the next check is another argument's
    refused(w2v.lib().w2v_linear_q4, dict(args, M=524_288, x=None), "x is NULL")
