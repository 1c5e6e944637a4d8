"""Distillation of rows that no block's registers hold, enough of them to be a
block's each: the end of a row is kept, the rest read twice. A block keeps 14
turns of 1,024 packs of 16 bytes and takes rows of more than 9,216 packs, so the
lengths here are just past that, just past what is kept, and ones with 1, 2, 3
and 5 whole turns before it, of no whole number of packs. Formulas and bounds as in
test_gpu_distill.py, for all rows at once."""
import pytest

from paper_1611_06172_amd import w2v
from test_gpu_distill import EPS, U, case

pytestmark = pytest.mark.gpu

LENGTHS = {"float32": [36_865, 57_344, 57_345, 65_533, 69_631, 77_821],
           "bfloat16": [73_729, 114_688, 114_689, 131_069, 139_259, 155_643],
           "float16": [73_735, 114_695, 155_641]}


def whole(c, T, soft, hard):
    """(loss, its bound, gradient, its bound) in 64 bits for all rows."""
    import torch
    z = c["logits"].double()
    rows, V = z.shape
    none = (z == float("-inf")).all(dim=1, keepdim=True)
    s = torch.where(none, torch.zeros_like(z), z)
    x = s - s.amax(dim=1, keepdim=True)
    ids, w = c["ids"].long(), c["weight"].double()[:, None]
    there, at = (ids >= 0) & ~none, ids.clamp(min=0)
    some = there.any(dim=1, keepdim=True)
    t = torch.where(there, c["teacher"].double() / T, torch.full_like(at, 0).double() - 1e300)
    lq = torch.log_softmax(t, dim=1)
    q = torch.where(there, lq.exp(), torch.zeros_like(lq))
    lq = torch.where(there, lq, torch.zeros_like(lq))
    lp = torch.log_softmax(x / T, dim=1)
    part = torch.where(there, q * (lq - torch.gather(lp, 1, at)), torch.zeros_like(q))
    loss = soft * T * T * part.sum(dim=1)
    big = torch.where(there, (c["teacher"].double() / T).abs(), torch.zeros_like(lq))
    far = torch.where(there, torch.gather(x, 1, at).abs() / T, torch.zeros_like(lq))
    lb = soft * T * T * U * (512 + 8 * (q * (far + lq.abs() + big.amax(
        dim=1, keepdim=True))).sum(dim=1))
    p = lp.exp() * some
    grad = w * soft * T * p
    gb = grad * U * (300 + 4 * (x / T).abs().clamp(max=1e4))
    grad.scatter_add_(1, at, -w * soft * T * q)
    gb.scatter_add_(1, at, w * soft * T * q * U * 300)
    if c["labels"] is not None:
        y = c["labels"].long()[:, None]
        has = ((y >= 0) & ~none).double()
        y = y.clamp(min=0)
        l1 = torch.log_softmax(x, dim=1)
        loss -= hard * (has * torch.where(has > 0, torch.gather(l1, 1, y), 0.0))[:, 0]
        lb += hard * U * (512 + 8 * (has * torch.gather(x.abs().clamp(max=1e30), 1, y))[:, 0])
        p = l1.exp() * has
        grad += w * hard * p
        gb += w * hard * p * U * (300 + 8 * x.abs().clamp(max=1e4))
        grad.scatter_add_(1, y, -w * hard * has)
        gb.scatter_add_(1, y, w * hard * has * U * 8)
    live = (~none).double()
    return loss * live[:, 0], lb, grad * live, gb


@pytest.mark.parametrize("name,V", [(n, v) for n in LENGTHS for v in LENGTHS[n]])
def test_long_rows(name, V):
    import torch
    rows = 257
    T, labels = [(1.0, True), (2.0, True), (4.0, True), (3.0, True), (2.0, False),
                 (0.5, False)][LENGTHS[name].index(V)]
    c = case(rows, V, 20, name, V, labels=labels, pad=V % 4)
    soft, hard = (0.7, 0.3) if labels else (1.0, 0.0)
    kw = dict(temperature=T, labels=c["labels"], soft=soft, hard=hard)
    out = w2v.distill_loss(c["logits"], c["ids"], c["teacher"], row_weight=c["weight"],
                           want_grad=True, **kw)
    loss, lb, grad, gb = whole(c, T, soft, hard)
    assert ((out["loss"].double() - loss).abs() <= lb + U * loss.abs()).all()
    bound = gb + EPS[name] * 1.01 * grad.abs() + 2.0 ** -25
    assert ((out["grad"].double() - grad).abs() <= bound).all()
    alone = w2v.distill_loss(c["logits"], c["ids"], c["teacher"], **kw)
    assert torch.equal(alone["loss"], out["loss"]) and torch.equal(alone["stats"], out["stats"])
    back = w2v.distill_backward(c["weight"], c["logits"], c["ids"], c["teacher"], out["stats"],
                                **kw)
    assert ((back.double() - grad).abs() <= bound).all()
    keep = c["logits"].clone()
    w2v.distill_loss(c["logits"], c["ids"], c["teacher"], row_weight=c["weight"],
                     grad=c["logits"], **kw)
    assert torch.equal(c["logits"], out["grad"])
    c["logits"].copy_(keep)
    w2v.distill_backward(c["weight"], c["logits"], c["ids"], c["teacher"], out["stats"],
                         grad=c["logits"], **kw)
    assert torch.equal(c["logits"], back)


@pytest.mark.parametrize("where", [0, 4_000, 12_345, 60_000, 77_820])
def test_nan_and_infinity_anywhere_in_a_long_row(where):
    """In the part that is read twice and in the part that is kept."""
    import torch
    c = case(256, 77_821, 8, "float32", 3, masked=False)
    c["teacher"] = torch.nan_to_num(c["teacher"], nan=0.0)
    kw = dict(labels=c["labels"], hard=0.5, temperature=2.0, want_grad=True)
    clean = w2v.distill_loss(c["logits"], c["ids"], c["teacher"], **kw)
    z = c["logits"].clone()
    z[5, where], z[2, where] = float("nan"), float("inf")
    out = w2v.distill_loss(z, c["ids"], c["teacher"], **kw)
    bad = [2, 5]
    good = [r for r in range(256) if r not in bad]
    assert torch.isnan(out["loss"][bad]).all() and torch.isnan(out["grad"][bad]).all()
    for key in ("loss", "grad"):
        assert torch.equal(out[key][good], clean[key][good])
