"""w2v_distill_loss and w2v_distill_backward against the formulas in 64 bits,
row by row; the gradient also against differences.

Tolerances, fixed beforehand, in units of u = 2^-24. An exponential's argument
has two roundings, so it is within (2 |x| + 4) u of exp(x) relatively; x exp(x)
<= 1 bounds what that adds to a sum whose largest term is 1; a sum is added up
in partial sums of at most 128 terms. So log-sums are within 256 u absolutely,
log-probabilities within 256 u + 8 u (|x| + |log q|), and a probability within
(300 + 4 |x|) u of itself. A gradient of p bits is rounded once, 2^-p of its
value, plus half of float16's smallest step."""
import math

import pytest

from gpu_util import expect_device_flag
from paper_1611_06172_amd import w2v

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
EPS = {"float32": U, "bfloat16": 2.0 ** -8, "float16": 2.0 ** -11}


def case(rows, V, K, name, seed, labels=True, masked=True, pad=0, scale=3.0):
    """Scores, teacher's list with absent entries and empty rows, labels."""
    import torch
    g = torch.Generator()
    g.manual_seed(seed)
    t = getattr(torch, name)
    buf = torch.full((rows, V + pad), float("nan"), dtype=t)
    buf[:, :V] = (torch.randn((rows, V), generator=g) * scale).to(t)
    if masked and V > 4:
        buf[:, :V][torch.rand((rows, V), generator=g) < 0.1] = float("-inf")
        buf[0, 1:V] = torch.finfo(t).min
    ids = torch.stack([torch.randperm(V, generator=g)[:K] if V >= K else
                       torch.randint(0, V, (K,), generator=g) for _ in range(rows)]) \
        if K else torch.empty((rows, 0), dtype=torch.int64)
    # listed words are not masked: their loss would be infinite
    z = buf[:, :V]
    at = torch.gather(z.float(), 1, ids)
    teacher = torch.randn((rows, K), generator=g) * 2 + 1
    z.scatter_(1, ids, torch.where(torch.isinf(at) | (at < -1e4), torch.ones_like(at),
                                   at).to(t))
    gone = torch.rand((rows, K), generator=g) < 0.2
    if rows > 2:
        gone[2] = True
    ids = torch.where(gone, torch.full_like(ids, -1), ids)
    teacher = torch.where(gone, torch.full_like(teacher, float("nan")), teacher).to(t)
    y = torch.randint(0, V, (rows,), generator=g)
    r = torch.arange(rows)
    bad = torch.isinf(z[r, y].float()) | (z[r, y].float() < -1e4)
    z[r[bad], y[bad]] = 0.5
    y[1::4] = -1
    if rows > 3:
        z[3] = float("-inf")  # nothing is left of the row
    w = torch.rand(rows, generator=g) + 0.5
    return dict(logits=buf.cuda()[:, :V], ids=ids.to(torch.int32).cuda(),
                teacher=teacher.cuda(), labels=y.to(torch.int32).cuda() if labels else None,
                weight=w.cuda())


def exact(c, T, soft, hard):
    """Loss, gradient and their bounds in 64 bits, by plain loops over rows."""
    import torch
    z = c["logits"].double().cpu()
    rows, V = z.shape
    loss, lb = torch.zeros(rows, dtype=torch.float64), torch.zeros(rows, dtype=torch.float64)
    grad, gb = torch.zeros_like(z), torch.zeros_like(z)
    for r in range(rows):
        s = z[r]
        if (s == float("-inf")).all():
            continue
        w = float(c["weight"][r])
        lp = torch.log_softmax(s / T, 0)
        x = (s - s.max()) / T
        ids = c["ids"][r].long().cpu()
        t = c["teacher"][r].double().cpu()[ids >= 0]
        ids = ids[ids >= 0]
        if len(ids):
            lq = torch.log_softmax(t / T, 0)
            q = lq.exp()
            loss[r] += soft * T * T * (q * (lq - lp[ids])).sum()
            lb[r] += soft * T * T * U * (
                512 + 8 * (q * (x[ids].abs() + lq.abs() + (t / T).abs().max())).sum())
            p = lp.exp()
            grad[r] += w * soft * T * p
            gb[r] += w * soft * T * p * U * (300 + 4 * x.abs().clamp(max=1e4))
            grad[r].index_add_(0, ids, -w * soft * T * q)
            gb[r].index_add_(0, ids, w * soft * T * q * U * 300)
        y = -1 if c["labels"] is None else int(c["labels"][r])
        if y >= 0:
            l1 = torch.log_softmax(s, 0)
            d = (s - s.max()).abs()
            loss[r] -= hard * l1[y]
            lb[r] += hard * U * (512 + 8 * d[y])
            p = l1.exp()
            grad[r] += w * hard * p
            # squaring exp(x / T) doubles its relative error each time
            gb[r] += w * hard * p * U * (300 + 8 * d.clamp(max=1e4))
            grad[r, y] -= w * hard
            gb[r, y] += w * hard * U * 8
    return loss, lb, grad, gb


def compare(c, name, T, soft, hard):
    import torch
    kw = dict(temperature=T, labels=c["labels"], soft=soft, hard=hard)
    out = w2v.distill_loss(c["logits"], c["ids"], c["teacher"], row_weight=c["weight"],
                           want_grad=True, **kw)
    loss, lb, grad, gb = exact(c, T, soft, hard)
    got = out["loss"].double().cpu()
    assert ((got - loss).abs() <= lb + U * loss.abs()).all(), ((got - loss).abs() / lb).max()
    got = out["grad"].double().cpu()
    bound = gb + EPS[name] * 1.01 * grad.abs() + 2.0 ** -25
    assert ((got - grad).abs() <= bound).all(), ((got - grad).abs() / bound).max()
    # the loss alone, the gradient from the statistics, and in place
    alone = w2v.distill_loss(c["logits"], c["ids"], c["teacher"], **kw)
    assert alone["grad"] is None and torch.equal(alone["loss"], out["loss"])
    assert torch.equal(alone["stats"], out["stats"])
    back = w2v.distill_backward(c["weight"], c["logits"], c["ids"], c["teacher"],
                                out["stats"], **kw)
    got = back.double().cpu()
    assert ((got - grad).abs() <= bound).all()
    keep = c["logits"].clone()
    for call in (lambda: w2v.distill_loss(
            c["logits"], c["ids"], c["teacher"], row_weight=c["weight"],
            grad=c["logits"], **kw)["grad"],
            lambda: w2v.distill_backward(c["weight"], c["logits"], c["ids"], c["teacher"],
                                         out["stats"], grad=c["logits"], **kw)):
        there = call()
        assert there.data_ptr() == c["logits"].data_ptr()
        got = there.double().cpu()
        assert ((got - grad).abs() <= bound).all()
        c["logits"].copy_(keep)
    return out


@pytest.mark.parametrize("name", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("rows,V,K,T", [
    (1, 1, 1, 1.0), (2, 2, 1, 2.0), (5, 7, 3, 0.5), (4, 63, 64, 1.0), (9, 1000, 16, 2.0),
    (6, 1001, 100, 4.0), (5, 4099, 1, 3.0), (4, 9_999, 1024, 2.0), (6, 20_011, 33, 1.0),
    (4, 71_290, 64, 2.0), (5, 131_071, 20, 2.5), (2, 300_001, 256, 4.0)])
def test_loss_and_gradient(rows, V, K, T, name):
    c = case(rows, V, K, name, rows + V + K, pad=V % 4)
    compare(c, name, T, 0.7, 0.3)


@pytest.mark.parametrize("name", ["float32", "bfloat16"])
@pytest.mark.parametrize("rows,V,K,T", [(7, 300, 5, 1.0), (5, 30_000, 50, 2.0),
                                        (1500, 130, 8, 2.0), (1100, 9_001, 3, 3.0)])
def test_without_labels(rows, V, K, T, name):
    compare(case(rows, V, K, name, V, labels=False), name, T, 1.0, 0.0)


def test_labels_alone():
    """No teacher's list at all: the cross entropy of the labels."""
    compare(case(6, 5000, 0, "float32", 3), "float32", 2.0, 1.0, 1.0)


def test_words_listed_twice_add_up():
    import torch
    c = case(4, 50, 8, "float32", 11, masked=False)
    c["ids"][:, 4:] = c["ids"][:, :4]
    c["ids"][0] = 7
    c["teacher"] = torch.nan_to_num(c["teacher"], nan=0.5)
    compare(c, "float32", 2.0, 1.0, 0.5)


def test_gradient_against_differences():
    """Central differences of the 64-bit loss along a random direction."""
    import torch
    c = case(5, 400, 12, "float32", 21, masked=False)
    c["weight"].fill_(1.0)
    out = w2v.distill_loss(c["logits"], c["ids"], c["teacher"], temperature=2.0,
                           labels=c["labels"], soft=0.7, hard=0.3, want_grad=True)
    g = torch.Generator()
    g.manual_seed(1)
    v = torch.randn((5, 400), generator=g, dtype=torch.float64)
    v[3] = 0
    h = 1e-5
    base = c["logits"].double()
    values = []
    for sign in (1, -1):
        moved = dict(c, logits=base + sign * h * v.cuda())
        values.append(exact(moved, 2.0, 0.7, 0.3)[0].sum())
    slope = (values[0] - values[1]) / (2 * h)
    got = (out["grad"].double().cpu() * v).sum()
    assert abs(got - slope) <= 1e-5 * (out["grad"].double().cpu().abs() * v.abs()).sum()


def test_gradient_of_a_row_sums_to_zero():
    import torch
    c = case(64, 2000, 10, "float32", 5, masked=False)
    out = w2v.distill_loss(c["logits"], c["ids"], c["teacher"], temperature=2.0,
                           labels=c["labels"], soft=0.5, hard=0.5, want_grad=True)
    sums = out["grad"].double().sum(dim=1).abs().max().item()
    assert sums <= 600 * U * 2


def test_large_scores_are_in_range():
    """Scores near a type's limits, spread out far beyond exp's range."""
    import torch
    z = torch.full((3, 500), -3.0e38, device="cuda")
    z[0, 7], z[1, :] = 3.0e38, 1e30
    z[2] = torch.linspace(-1e6, 1e6, 500)
    ids = torch.tensor([[7, -1], [3, 4], [499, -1]], dtype=torch.int32, device="cuda")
    t = torch.zeros((3, 2), device="cuda")
    out = w2v.distill_loss(z, ids, t, temperature=0.5, want_grad=True)
    assert torch.isfinite(out["loss"]).all() and torch.isfinite(out["grad"]).all()
    assert out["loss"][0] == 0 and out["loss"][2] == 0
    assert abs(out["loss"][1].item() - 0.25 * math.log(250)) <= 600 * U
    assert (out["grad"][0] == 0).all()


def test_nan_and_infinity_show_in_their_row():
    import torch
    for V in (600, 20_000, 100_000):
        c = case(8, V, 5, "float32", V, masked=False, labels=False)
        c["ids"].clamp_(min=0)
        c["teacher"] = torch.nan_to_num(c["teacher"], nan=0.0)
        kw = dict(temperature=2.0, want_grad=True)
        clean = w2v.distill_loss(c["logits"], c["ids"], c["teacher"], **kw)
        z, t = c["logits"].clone(), c["teacher"].clone()
        z[0, V - 1] = float("nan")
        z[1] = float("nan")
        z[2, 3] = float("inf")
        t[4, 1] = float("nan")
        out = w2v.distill_loss(z, c["ids"], t, **kw)
        bad = [0, 1, 2, 4]
        good = [5, 6, 7]
        assert torch.isnan(out["loss"][bad]).all()
        for key in ("loss", "grad"):
            assert torch.equal(out[key][good], clean[key][good])
        assert torch.isnan(out["grad"][[0, 1]]).all()
        # a masked word that the teacher lists costs infinitely much
        z = c["logits"].clone()
        z[6, c["ids"][6, 0].long()] = float("-inf")
        out = w2v.distill_loss(z, c["ids"], c["teacher"], temperature=2.0)
        assert out["loss"][6] == float("inf") and torch.isfinite(out["loss"][7])


@pytest.mark.parametrize("name", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("V", [5, 500, 30_000, 100_000, 200_001])
def test_list_of_masked_words_alone_is_no_list(V, name):
    """A row whose present teacher logits are all -inf has nothing to learn
    from: no soft term in its loss or its gradient, like a row of absent
    entries; one entry above -inf is a list of that entry."""
    import torch
    c = case(6, V, 4, name, V, masked=False)
    ids = c["ids"]
    ids[:] = torch.randint(0, V, ids.shape)
    c["teacher"].fill_(float("-inf"))
    c["teacher"][4, 2] = 1.0
    ids[5, 3] = -1
    c["labels"][0] = ids[0, 1]
    c["labels"][5] = 3
    absent = dict(c, ids=ids.clone())
    absent["ids"][[0, 1, 2, 3, 5]] = -1
    for labels in (True, False):
        kw = dict(temperature=2.0, soft=0.7, hard=0.3)
        one = dict(absent, labels=c["labels"] if labels else None)
        kw["labels"] = one["labels"]
        loss, lb, grad, gb = exact(
            dict(one, ids=torch.where(one["teacher"] > -1, one["ids"],
                                      torch.full_like(one["ids"], -1))), 2.0, 0.7, 0.3)
        want = w2v.distill_loss(one["logits"], one["ids"], one["teacher"], want_grad=True, **kw)
        got = w2v.distill_loss(c["logits"], ids, c["teacher"], want_grad=True, **kw)
        assert torch.isfinite(got["loss"]).all() and torch.isfinite(got["grad"]).all()
        assert ((got["loss"].double().cpu() - loss).abs() <= lb + U * loss.abs()).all()
        assert torch.equal(got["loss"], want["loss"])
        assert torch.equal(got["grad"], want["grad"])
        back = w2v.distill_backward(torch.ones(6, device="cuda"), c["logits"], ids,
                                    c["teacher"], got["stats"], **kw)
        there = w2v.distill_backward(torch.ones(6, device="cuda"), one["logits"], one["ids"],
                                     one["teacher"], want["stats"], **kw)
        assert torch.isfinite(back).all() and torch.equal(back, there)


@pytest.mark.parametrize("rows,V", [(12, 7), (12, 600), (12, 20_000), (12, 60_000),
                                    (12, 100_000), (260, 40_001)])
@pytest.mark.parametrize("T", [1.0, 2.0, 3.0])
def test_nan_and_infinity_show_without_a_list(rows, V, T):
    """A score of NaN or +inf makes its row's loss and gradient NaN whatever
    terms the row has: a label alone, a list alone, both or neither."""
    import torch
    c = case(rows, V, 5, "float32", V, masked=False)
    c["teacher"] = torch.nan_to_num(c["teacher"], nan=0.0)
    c["ids"].clamp_(min=0)
    c["ids"][:8] = -1  # rows 0 to 7: no list
    c["labels"][:] = 1
    c["labels"][4:10] = -1  # rows 4 to 9: no label
    z = c["logits"]
    z[3] = 0.25
    bad = [0, 1, 4, 5, 8, 10]
    for r in bad:
        z[r, V - 1 if r % 2 else 3] = float("inf" if r in (1, 5, 10) else "nan")
    good = [r for r in range(rows) if r not in bad]
    clean = z.clone()
    clean[bad] = 0.0
    one = torch.ones(rows, device="cuda")
    for ids, teacher in ((c["ids"], c["teacher"]),
                         (c["ids"][:, :0].contiguous(), c["teacher"][:, :0].contiguous())):
        kw = dict(temperature=T, labels=c["labels"], hard=0.5)
        out = w2v.distill_loss(z, ids, teacher, want_grad=True, **kw)
        want = w2v.distill_loss(clean, ids, teacher, want_grad=True, **kw)
        back = w2v.distill_backward(one, z, ids, teacher, out["stats"], **kw)
        assert torch.isnan(out["loss"][bad]).all()
        assert torch.isnan(out["grad"][bad]).all() and torch.isnan(back[bad]).all()
        for key in ("loss", "grad"):
            assert torch.equal(out[key][good], want[key][good])
        assert torch.isfinite(back[good]).all()

@pytest.mark.parametrize("V", [40, 9_000, 100_000])
def test_term_without_weight_is_left_out(V):
    """soft = 0 or hard = 0 takes the term out, also where it would be
    infinite: a masked word that the teacher lists, a masked label."""
    import torch
    c = case(8, V, 5, "float32", V, masked=False)
    z, ids = c["logits"], c["ids"]
    z[3] = 0.5
    ids[0, 0], ids[4, 1] = 2, 2
    c["labels"][[0, 6]] = 2
    z[[0, 4, 6], 2] = float("-inf")
    kw = dict(temperature=2.0, want_grad=True)
    none = torch.full_like(ids, -1)
    a = w2v.distill_loss(z, ids, c["teacher"], labels=c["labels"], soft=0.0, hard=0.5, **kw)
    b = w2v.distill_loss(z, none, c["teacher"], labels=c["labels"], soft=0.0, hard=0.5, **kw)
    assert torch.equal(a["loss"], b["loss"]) and a["loss"][6] == float("inf")
    keep = [r for r in range(8) if r != 6 and r != 0]
    assert torch.isfinite(a["loss"][keep]).all() and torch.isfinite(a["grad"]).all()
    a = w2v.distill_loss(z, ids, c["teacher"], labels=c["labels"], soft=0.7, hard=0.0, **kw)
    b = w2v.distill_loss(z, ids, c["teacher"], soft=0.7, **kw)
    # (row 0's word may be listed with a NaN)
    assert torch.equal(a["loss"][1:], b["loss"][1:]) and torch.isfinite(a["grad"][1:]).all()
    assert torch.isfinite(a["loss"][[1, 2, 3, 5, 6, 7]]).all()


@pytest.mark.parametrize("V", [100, 30_000, 90_000])
def test_ids_outside_the_vocabulary_skip_the_row(V):
    import torch
    c = case(6, V, 4, "bfloat16", 7, masked=False)
    clean = w2v.distill_loss(c["logits"], c["ids"], c["teacher"], labels=c["labels"],
                             hard=0.5, want_grad=True)
    w2v.device_status()
    for row, where in ((0, "ids"), (4, "ids"), (5, "labels")):
        ids, labels = c["ids"].clone(), c["labels"].clone()
        if where == "ids":
            ids[row, 1] = V if row == 0 else -2
        else:
            labels[row] = V
        out = w2v.distill_loss(c["logits"], ids, c["teacher"], labels=labels, hard=0.5,
                               want_grad=True)
        expect_device_flag()
        assert out["loss"][row] == 0 and (out["grad"][row] == 0).all()
        keep = [r for r in range(6) if r != row]
        assert torch.equal(out["loss"][keep], clean["loss"][keep])
        assert torch.equal(out["grad"][keep], clean["grad"][keep])
        w2v.distill_backward(c["weight"], c["logits"], ids, c["teacher"], clean["stats"],
                             labels=labels, hard=0.5)
        expect_device_flag()


def test_rows_far_apart():
    """Row offsets past 2^31 elements."""
    import torch
    far = torch.empty(3 * (1 << 30) + 2048, dtype=torch.bfloat16, device="cuda")
    z = far.as_strided((4, 1500), (1 << 30, 1))
    c = case(4, 1500, 9, "bfloat16", 2, masked=False)
    z.copy_(c["logits"])
    kw = dict(labels=c["labels"], hard=0.5)
    a = w2v.distill_loss(c["logits"], c["ids"], c["teacher"], want_grad=True, **kw)
    b = w2v.distill_loss(z, c["ids"], c["teacher"], grad=z, **kw)
    assert torch.equal(a["loss"], b["loss"]) and torch.equal(a["grad"], b["grad"])
    del z, far, b
    torch.cuda.empty_cache()


def test_same_bits_and_another_stream():
    import torch
    c = case(40, 50_000, 30, "float32", 4)
    kw = dict(labels=c["labels"], hard=0.5, want_grad=True, temperature=3.0)
    a = w2v.distill_loss(c["logits"], c["ids"], c["teacher"], **kw)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    b = w2v.distill_loss(c["logits"], c["ids"], c["teacher"], stream=s, **kw)
    s.synchronize()
    assert all(torch.equal(a[k].nan_to_num(nan=5.0), b[k].nan_to_num(nan=5.0)) for k in a)


def test_no_rows():
    import torch
    z = torch.empty((0, 30), device="cuda")
    ids = torch.empty((0, 4), dtype=torch.int32, device="cuda")
    out = w2v.distill_loss(z, ids, torch.empty((0, 4), device="cuda"), want_grad=True)
    assert out["loss"].shape == (0,) and out["grad"].shape == (0, 30)


def test_binding_refuses():
    import torch
    z = torch.zeros((3, 20), device="cuda")
    ids = torch.zeros((3, 4), dtype=torch.int32, device="cuda")
    t = torch.zeros((3, 4), device="cuda")
    with pytest.raises(TypeError):
        w2v.distill_loss(z.double(), ids, t)
    with pytest.raises(TypeError):
        w2v.distill_loss(z, ids.long(), t)
    with pytest.raises(ValueError):
        w2v.distill_loss(z, ids[:2], t)
    with pytest.raises(ValueError):
        w2v.distill_loss(z, ids, t[:, :3].contiguous())
    with pytest.raises(ValueError):
        w2v.distill_loss(z, ids, t, labels=torch.zeros(2, dtype=torch.int32, device="cuda"))
    with pytest.raises(w2v.W2VError):
        w2v.distill_loss(z, ids, t, temperature=0.0)
    with pytest.raises(ValueError):
        w2v.distill_backward(torch.ones(3, device="cuda"), z, ids, t,
                             torch.zeros((3, 2), device="cuda"))
