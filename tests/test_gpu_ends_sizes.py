"""Sizes that the library's 32-bit numbers do not hold are refused, not cut off."""
import pytest

from paper_1611_06172_amd import w2v

pytestmark = pytest.mark.gpu

MANY = 2 ** 32 + 8


def test_sizes_beyond_31_bits_are_refused():
    """What ctypes would make 8 rows or columns of. Nothing of the memory is touched."""
    import torch
    row = torch.empty((1, MANY), dtype=torch.float16, device="cuda")
    column = row.view(MANY, 1)
    ids = torch.zeros(4, dtype=torch.int32, device="cuda")
    one = torch.ones((4, 1), dtype=torch.float16, device="cuda")
    score = torch.zeros((1, 1), device="cuda")
    for call in (lambda: w2v.dropout(row, 0.5, seed=1), lambda: w2v.dropout(column, 0.5, seed=1),
                 lambda: w2v.embed(ids, column), lambda: w2v.embed(ids, row),
                 lambda: w2v.embed_backward(one, ids, MANY),
                 lambda: w2v.embed_backward(one, ids, grad=column, accumulate=True),
                 lambda: w2v.quantize_q4(row), lambda: w2v.beam_step(row, score),
                 lambda: w2v.linear(column, one[:1]),
                 lambda: w2v.sample_words(row, torch.empty((1, MANY), device="cuda"))):
        with pytest.raises(ValueError, match="less than 2\\^31"):
            call()


def test_states_beyond_31_bits_are_refused():
    import torch
    state = torch.empty((MANY, 1), dtype=torch.uint8, device="cuda")
    parents = torch.zeros((1, 4), dtype=torch.int32, device="cuda")
    with pytest.raises(ValueError, match="less than 2\\^31"):
        w2v.beam_reorder(state, parents)
