"""Cases of the vocabulary head: the operators that a trained model is asked
for its distribution over the vocabulary with, each in a plain form of
elementary torch operations in 32 bits and, where `own` is true, through
paper_1611_06172_amd.w2v as a program calls it.

  linear    y = act(x W^T + b) + residual: scores of a batch of contexts
            against every row of M_out, and a hidden layer between
  back      its backward pass: dx, dW and db
  distill   distillation from a teacher's top logits: the loss of each row
            ("loss"), loss and gradient of a training step ("step"), or the
            gradient from the saved statistics ("backward")
  sample    words drawn with temperature, top-k, top-p and min-p from given
            uniform random numbers

Vocabulary sizes and dimensions are those of paper_1611_06172_amd.configs
(1,000, 71,290, 100,000 and 10^6 words; 64 to 600 columns); rows are the
contexts that are in hand at once, from one to the kernel test's 65,536.
Scores follow a Zipf law, as a model's with a unigram bias do.
"""
import math

import torch

own = False

_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_ACTIVATIONS = ["none", "relu", "gelu", "silu", "tanh", "sigmoid"]


def _linear(name, M, N, K, dtype, **over):
    c = {"name": name, "kind": "linear", "M": M, "N": N, "K": K, "dtype": dtype,
         "out": dtype, "activation": "none", "bias": True, "residual": False,
         "padded": False}
    c.update(over)
    return c


def _distill(name, rows, V, K, dtype, **over):
    c = {"name": name, "kind": "distill", "rows": rows, "V": V, "K": K, "dtype": dtype,
         "mode": "step", "temperature": 2.0, "labels": False, "padded": False}
    c.update(over)
    return c


def _sample(name, rows, V, dtype, **over):
    c = {"name": name, "kind": "sample", "rows": rows, "V": V, "dtype": dtype,
         "temperature": 1.0, "top_k": 0, "top_p": 1.0, "min_p": 0.0, "per_row": False}
    c.update(over)
    return c


def listed():
    return [
        # One context against the planted model's M_out, as it was trained:
        # what a query answers with. Latency and one pass over the matrix.
        _linear("scores_1_f32", 1, 71_290, 200, "f32"),
        # A hidden layer of a student over the kernel test's batch, whole
        # epilogue: bias, gelu and the input added back.
        _linear("hidden_gelu_bf16", 65_536, 300, 300, "bf16", activation="gelu",
                residual=True),
        # Scores of an ordinary training batch: the output is what moves.
        _linear("scores_4096_bf16", 4_096, 71_290, 300, "bf16"),
        # Scores over the throughput workload's vocabulary from fp32 matrices
        # with rows on 128-byte lines, as the trainer holds them.
        _linear("scores_512_f32", 512, 1_000_000, 300, "f32", padded=True),
        # Backward pass of the scores, over a batch that no tile divides: a
        # long sum over the vocabulary for dx, a large matrix for dW.
        _linear("back_scores_bf16", 8_191, 71_290, 300, "bf16", kind="back"),
        # Backward pass of a hidden layer through its activation.
        _linear("back_hidden_f32", 4_096, 600, 600, "f32", kind="back",
                activation="silu"),
        # The tiny model's vocabulary, a few rows: launches are all there is.
        _distill("distill_8x1000_f32", 8, 1_000, 16, "f32"),
        # A training step of a student on the planted vocabulary.
        _distill("distill_4096_bf16", 4_096, 71_290, 64, "bf16"),
        # A step over 10^6 words with the true next word mixed in.
        _distill("distill_2048x1e6_bf16", 2_048, 1_000_000, 256, "bf16", labels=True),
        # One answer: the usual filters on one row.
        _sample("sample_1_f32", 1, 71_290, "f32", temperature=0.8, top_k=40, top_p=0.95),
        # A batch of requests, each with its own settings.
        _sample("sample_257_f16", 257, 100_000, "f16", temperature=0.9, top_k=50,
                top_p=0.9, min_p=0.02, per_row=True),
        # The nucleus of a vocabulary of 10^6 words.
        _sample("sample_64x1e6_bf16", 64, 1_000_000, "bf16", top_p=0.9),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    kind = rng.choice(["linear", "back", "distill", "sample"])
    dtype = rng.choice(["f32", "bf16", "bf16", "f16"])
    if kind in ("linear", "back"):
        K = _log(rng, 24, 640)
        N = _log(rng, 100, 1_000_000 if kind == "linear" else 200_000)
        M = _log(rng, 1, min(65_536, 1.5e11 / (float(N) * K), 4e8 / N))
        wide = N > 2_000
        c = _linear("", M, N, K, dtype, kind=kind,
                    activation="none" if wide else rng.choice(_ACTIVATIONS),
                    bias=rng.random() < 0.7,
                    residual=kind == "linear" and not wide and rng.random() < 0.5,
                    padded=rng.random() < 0.5)
        if kind == "linear" and rng.random() < 0.3:
            c["out"] = "f32"
    elif kind == "distill":
        V = _log(rng, 1_000, 1_000_000)
        c = _distill("", _log(rng, 1, min(65_536, 1e9 / V)), V, _log(rng, 1, 512), dtype,
                     mode=rng.choice(["step", "step", "loss", "backward"]),
                     temperature=rng.choice([1.0, 2.0, 4.0]),
                     labels=rng.random() < 0.5, padded=rng.random() < 0.5)
    else:
        V = _log(rng, 1_000, 1_000_000)
        c = _sample("", _log(rng, 1, min(512, 6e7 / V)), V, dtype,
                    temperature=rng.choice([0.0, 0.6, 0.8, 1.0, 1.3]),
                    top_k=rng.choice([0, 0, 1, 20, 50, 200, 1000]),
                    top_p=rng.choice([1.0, 1.0, 0.5, 0.9, 0.95]),
                    min_p=rng.choice([0.0, 0.0, 0.02, 0.1]),
                    per_row=rng.random() < 0.3)
    del c["name"]
    return c


# ------------------------------------------------------------------ inputs --

def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _normal(g, rows, cols, scale, dtype, padded=False):
    """rows x cols normal values; padded: a view whose rows start on 128-byte
    lines, as w2v.alloc_matrix lays them out."""
    wide = cols if not padded else (cols + 63) // 64 * 64
    out = torch.empty((rows, wide), dtype=dtype, device="cuda")[:, :cols]
    step = max(1, (1 << 28) // max(1, cols))
    for b in range(0, rows, step):
        e = min(rows, b + step)
        out[b:e] = torch.randn((e - b, cols), generator=g, device="cuda") * scale
    return out


def _scores(g, rows, V, dtype, padded=False):
    """Scores of a model with a unigram bias: Zipf's law and what the
    contexts add."""
    out = _normal(g, rows, V, 2.0, dtype, padded)
    rank = torch.arange(1, V + 1, device="cuda", dtype=torch.float32)
    prior = (-1.07 * torch.log(rank)).to(dtype)
    step = max(1, (1 << 28) // V)
    for b in range(0, rows, step):
        out[b:b + step] += prior
    return out


def _prepare_linear(c, seed):
    g = _generator(seed)
    M, N, K, t = c["M"], c["N"], c["K"], _TYPES[c["dtype"]]
    s = {"case": c, "x": _normal(g, M, K, 1.0, t, c["padded"]),
         "w": _normal(g, N, K, 1.0 / math.sqrt(K), t, c["padded"]),
         "b": torch.randn(N, generator=g, device="cuda") if c["bias"] else None,
         "r": None, "pre": None, "dy": None}
    if c["kind"] == "linear":
        if c["residual"]:
            s["r"] = _normal(g, M, N, 1.0, _TYPES[c["out"]])
    else:
        s["dy"] = _normal(g, M, N, 1.0, t)
        if c["activation"] != "none":
            s["pre"] = _normal(g, M, N, 1.0, t)
    return s


def _prepare_distill(c, seed):
    g = _generator(seed)
    rows, V, K, t = c["rows"], c["V"], min(c["K"], c["V"]), _TYPES[c["dtype"]]
    logits = _scores(g, rows, V, t, c["padded"])
    # A teacher's top words are mostly frequent ones: one word from each of K
    # ranges of ids that widen towards the rare words.
    edge = torch.arange(K + 1, device="cuda", dtype=torch.float64) / K
    edge = torch.arange(K + 1, device="cuda") + torch.floor((V - K) * edge ** 3).long()
    u = torch.rand((rows, K), generator=g, device="cuda", dtype=torch.float64)
    ids = (edge[:-1] + torch.floor(u * (edge[1:] - edge[:-1]))).long()
    teacher = torch.gather(logits, 1, ids).float() + torch.randn(
        (rows, K), generator=g, device="cuda") + 2.0
    teacher = teacher.to(t)
    # One row in sixteen has no teacher, the others list at least half of K.
    there = torch.arange(K, device="cuda")[None, :] < torch.randint(
        (K + 1) // 2, K + 1, (rows, 1), generator=g, device="cuda")
    there &= torch.rand((rows, 1), generator=g, device="cuda") >= 1.0 / 16.0
    ids = torch.where(there, ids, torch.full_like(ids, -1)).to(torch.int32)
    s = {"case": c, "logits": logits, "ids": ids, "teacher": teacher, "labels": None,
         "weight": torch.rand(rows, generator=g, device="cuda") + 0.5,
         "soft": 1.0, "hard": 0.0, "stats": None}
    if c["labels"]:
        y = torch.rand(rows, generator=g, device="cuda", dtype=torch.float64)
        s["labels"] = torch.floor((V - 1) * y ** 4).to(torch.int32)
        s["labels"][3::16] = -1
        s["soft"], s["hard"] = 0.7, 0.3
    if c["mode"] == "backward":
        s["stats"] = torch.empty((rows, 3), device="cuda")
        step = max(1, (1 << 27) // V)
        for b in range(0, rows, step):
            z = logits[b:b + step].double()
            m = z.amax(dim=1)
            z = z - m[:, None]
            s["stats"][b:b + step, 0] = m
            s["stats"][b:b + step, 1] = torch.exp(z / c["temperature"]).sum(dim=1).log()
            s["stats"][b:b + step, 2] = torch.exp(z).sum(dim=1).log()
    return s


def _prepare_sample(c, seed):
    g = _generator(seed)
    rows, V = c["rows"], c["V"]
    s = {"case": c, "logits": _scores(g, rows, V, _TYPES[c["dtype"]]),
         "uniforms": torch.rand((rows, V), generator=g, device="cuda"),
         "temperature": c["temperature"], "top_k": c["top_k"], "top_p": c["top_p"],
         "min_p": c["min_p"]}
    # A word in 32 is not allowed in the row.
    gone = torch.rand((rows, (V + 31) // 32), generator=g, device="cuda")
    gone = torch.floor(gone * min(32, V)).long() + 32 * torch.arange(
        gone.shape[1], device="cuda")
    s["logits"].scatter_(1, gone.clamp(max=V - 1), float("-inf"))
    if c["per_row"]:
        v = torch.rand((4, rows), generator=g, device="cuda")
        s["temperature"] = c["temperature"] * (0.75 + 0.5 * v[0])
        s["top_k"] = torch.ceil(c["top_k"] * (0.5 + 0.5 * v[1])).to(torch.int32)
        s["top_p"] = 1.0 - (1.0 - c["top_p"]) * (0.5 + v[2])
        s["min_p"] = c["min_p"] * (0.5 + v[3])
    return s


def prepare(case, seed):
    return {"linear": _prepare_linear, "back": _prepare_linear,
            "distill": _prepare_distill, "sample": _prepare_sample}[case["kind"]](
                case, int(seed))


# ------------------------------------------------------------- plain forms --

def _activate(z, name):
    if name == "relu":
        return torch.clamp(z, min=0)
    if name == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    if name == "silu":
        return z / (1.0 + torch.exp(-z))
    if name == "tanh":
        return torch.tanh(z)
    if name == "sigmoid":
        return 1.0 / (1.0 + torch.exp(-z))
    return z


def _slope(z, name):
    if name == "relu":
        return (z > 0).to(z.dtype)
    if name == "gelu":
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + \
            z * torch.exp(-0.5 * z * z) * (1.0 / math.sqrt(2.0 * math.pi))
    if name == "silu":
        p = 1.0 / (1.0 + torch.exp(-z))
        return p * (1.0 + z * (1.0 - p))
    if name == "tanh":
        return 1.0 - torch.tanh(z) ** 2
    if name == "sigmoid":
        p = 1.0 / (1.0 + torch.exp(-z))
        return p * (1.0 - p)
    return torch.ones_like(z)


def _plain_linear(s):
    c = s["case"]
    z = s["x"].float() @ s["w"].float().t()
    if s["b"] is not None:
        z = z + s["b"]
    y = _activate(z, c["activation"])
    if s["r"] is not None:
        y = y + s["r"].float()
    return y.to(_TYPES[c["out"]])


def _plain_back(s):
    c = s["case"]
    t = _TYPES[c["dtype"]]
    dz = s["dy"].float()
    if c["activation"] != "none":
        dz = dz * _slope(s["pre"].float(), c["activation"])
    out = {"dx": (dz @ s["w"].float()).to(t), "dw": (dz.t() @ s["x"].float()).to(t)}
    if c["bias"]:
        out["db"] = dz.sum(dim=0)
    return out


def _teacher(ids, teacher, T):
    """Probabilities of the listed words (0 where absent), their logarithms,
    and whether the row lists any."""
    there = ids >= 0
    t = torch.where(there, teacher / T, torch.full_like(teacher, float("-inf")))
    m = t.amax(dim=1, keepdim=True)
    m = torch.where(m == float("-inf"), torch.zeros_like(m), m)
    e = torch.exp(t - m)
    total = e.sum(dim=1, keepdim=True)
    some = total > 0
    safe = torch.where(some, total, torch.ones_like(total))
    q = e / safe
    logq = torch.where(q > 0, t - m - torch.log(safe), torch.zeros_like(t))
    return q, logq, some


def _plain_distill(s):
    c, T = s["case"], s["case"]["temperature"]
    z = s["logits"].float()
    ids = s["ids"].long()
    at = ids.clamp(min=0)
    q, logq, some = _teacher(ids, s["teacher"].float(), T)
    if s["stats"] is None:
        m = z.amax(dim=1, keepdim=True)
        log_t = torch.log(torch.exp((z - m) / T).sum(dim=1, keepdim=True))
        log_1 = torch.log(torch.exp(z - m).sum(dim=1, keepdim=True))
    else:
        m, log_t, log_1 = s["stats"][:, 0:1], s["stats"][:, 1:2], s["stats"][:, 2:3]
    out = {}
    has = None
    if s["labels"] is not None:
        y = s["labels"].long()[:, None]
        has = (y >= 0).float()
        y = y.clamp(min=0)
    if c["mode"] != "backward":
        x = (torch.gather(z, 1, at) - m) / T - log_t
        loss = s["soft"] * T * T * (q * (logq - x)).sum(dim=1)
        if has is not None:
            loss = loss + s["hard"] * (has * (log_1 - (torch.gather(z, 1, y) - m)))[:, 0]
        out["loss"] = loss
    if c["mode"] != "loss":
        w = s["weight"][:, None]
        g = torch.exp((z - m) / T - log_t) * (w * some.float() * (s["soft"] * T))
        g.scatter_add_(1, at, -(w * (s["soft"] * T)) * q)
        if has is not None:
            g += torch.exp(z - m - log_1) * (w * has * s["hard"])
            g.scatter_add_(1, y, -(w * has * s["hard"]))
        out["grad"] = g.to(s["logits"].dtype)
    return out


def _column(v, like):
    if isinstance(v, torch.Tensor):
        return v[:, None].to(like.dtype if v.is_floating_point() else v.dtype)
    return v


def _filtered(s, z):
    """Words drawn from the scores z [rows, V], in z's type."""
    c = s["case"]
    V = c["V"]
    u = s["uniforms"].to(z.dtype)
    T = _column(s["temperature"], z)
    m, first = z.max(dim=1, keepdim=True)
    if c["temperature"] == 0:
        first = torch.where(z == m, torch.arange(V, device=z.device), V).amin(dim=1)
        return first.to(torch.int32), torch.zeros_like(m[:, 0])
    x = (z - m) / T
    e = torch.exp(x)
    total = e.sum(dim=1, keepdim=True)
    keep = x > float("-inf")
    k, p, least = s["top_k"], s["top_p"], s["min_p"]
    if c["top_k"] > 0 or c["top_p"] < 1:
        ranked, order = torch.sort(z, dim=1, descending=True, stable=True)
        w = torch.exp((ranked - m) / T)
        inside = ranked > float("-inf")
        if c["top_k"] > 0:
            k = _column(k, z) if isinstance(k, torch.Tensor) else k
            inside &= torch.arange(V, device=z.device)[None, :] < k
        if c["top_p"] < 1:
            w = torch.where(inside, w, torch.zeros_like(w))
            before = torch.cumsum(w, dim=1) - w
            inside &= before < _column(p, z) * w.sum(dim=1, keepdim=True)
            inside[:, 0] = True
        keep &= torch.zeros_like(keep).scatter_(1, order, inside)
    if c["min_p"] > 0:
        keep &= e >= _column(least, z)
    race = x - torch.log(-torch.log(u))
    race = torch.where(keep, race, torch.full_like(race, float("-inf")))
    best = race.amax(dim=1, keepdim=True)
    at = torch.where(keep & (race == best), torch.arange(V, device=z.device), V)
    at = at.amin(dim=1, keepdim=True)
    logprob = torch.gather(x, 1, at) - torch.log(total)
    return at[:, 0].to(torch.int32), logprob[:, 0]


def _plain_sample(s):
    ids, logprob = _filtered(s, s["logits"].float())
    return {"ids": ids, "logprob": logprob}


# -------------------------------------------------------------------- run --

def _own(s):
    from paper_1611_06172_amd import w2v

    c = s["case"]
    if c["kind"] == "linear":
        return w2v.linear(s["x"], s["w"], s["b"], activation=c["activation"],
                          residual=s["r"], out_dtype=_TYPES[c["out"]])
    if c["kind"] == "back":
        out = w2v.linear_backward(s["dy"], s["x"], s["w"], activation=c["activation"],
                                  pre=s["pre"], want_db=c["bias"])
        return {k: v for k, v in out.items() if v is not None}
    if c["kind"] == "sample":
        return w2v.sample_words(s["logits"], s["uniforms"], temperature=s["temperature"],
                                top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"])
    kw = dict(temperature=c["temperature"], labels=s["labels"], soft=s["soft"],
              hard=s["hard"])
    if c["mode"] == "backward":
        return {"grad": w2v.distill_backward(s["weight"], s["logits"], s["ids"],
                                             s["teacher"], s["stats"], **kw)}
    out = w2v.distill_loss(s["logits"], s["ids"], s["teacher"],
                           row_weight=s["weight"] if c["mode"] == "step" else None,
                           want_grad=c["mode"] == "step", **kw)
    return {k: out[k] for k in ("loss", "grad") if out[k] is not None}


def run(state):
    if own:
        return _own(state)
    return {"linear": _plain_linear, "back": _plain_back, "distill": _plain_distill,
            "sample": _plain_sample}[state["case"]["kind"]](state)


# -------------------------------------------------------- work and 64 bits --

def work(case):
    c = case
    size = 4.0 if c["dtype"] == "f32" else 2.0
    if c["kind"] in ("linear", "back"):
        M, N, K = float(c["M"]), float(c["N"]), float(c["K"])
        out = 4.0 if c["out"] == "f32" else 2.0
        if c["kind"] == "linear":
            return {"bytes": size * (M + N) * K + out * M * N * (2 if c["residual"] else 1)
                    + (4.0 * N if c["bias"] else 0.0),
                    "flops": 2.0 * M * N * K}
        return {"bytes": 2.0 * size * (M + N) * K + size * M * N *
                (1 if c["activation"] == "none" else 2) + (4.0 * N if c["bias"] else 0.0),
                "flops": 4.0 * M * N * K}
    rows, V = float(c["rows"]), float(c["V"])
    if c["kind"] == "distill":
        K = min(c["K"], c["V"])
        return {"bytes": size * rows * V * (1 if c["mode"] == "loss" else 2)
                + rows * K * (4.0 + size) + 8.0 * rows,
                "flops": rows * V * (4.0 if c["mode"] == "loss" else 8.0)}
    # without a filter every word has its random number read
    drawn = V if c["top_k"] == 0 and c["top_p"] >= 1 and c["min_p"] == 0 else \
        (c["top_k"] or 64)
    if c["temperature"] == 0:
        drawn = 0
    return {"bytes": size * rows * V + 4.0 * rows * min(V, drawn) + 8.0 * rows,
            "flops": 4.0 * rows * V}


def _exact_linear(s):
    c = s["case"]
    z = torch.mm(s["x"].double(), s["w"].double().t().contiguous())
    if s["b"] is not None:
        z += s["b"].double()
    if c["activation"] == "gelu":
        y = 0.5 * z * torch.special.erfc(-z / math.sqrt(2.0))
    elif c["activation"] == "silu":
        y = z * torch.sigmoid(z)
    elif c["activation"] == "relu":
        y = torch.relu(z)
    elif c["activation"] in ("tanh", "sigmoid"):
        y = getattr(torch, c["activation"])(z)
    else:
        y = z
    return y if s["r"] is None else y + s["r"].double()


def _exact_back(s):
    c = s["case"]
    dz = s["dy"].double()
    if c["activation"] != "none":
        z = s["pre"].double()
        p = torch.sigmoid(z)
        dz *= {"relu": lambda: torch.where(z > 0, 1.0, 0.0),
               "gelu": lambda: 0.5 * torch.special.erfc(-z / math.sqrt(2.0))
               + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi),
               "silu": lambda: p + z * p * (1 - p),
               "tanh": lambda: 1.0 / torch.cosh(z) ** 2,
               "sigmoid": lambda: p * (1 - p)}[c["activation"]]()
    out = {"dx": torch.mm(dz, s["w"].double()),
           "dw": torch.mm(dz.t().contiguous(), s["x"].double())}
    if c["bias"]:
        out["db"] = dz.sum(dim=0)
    return out


def _exact_distill(s):
    """Row by row in blocks, the gradient formed as a dense target's."""
    c, T, V = s["case"], s["case"]["temperature"], s["case"]["V"]
    rows = c["rows"]
    loss = torch.zeros(rows, dtype=torch.float64, device="cuda")
    whole = c["mode"] != "loss"
    grad = torch.empty((rows, V), dtype=torch.float64, device="cuda") if whole else None
    step = max(1, (1 << 26) // V)
    for b in range(0, rows, step):
        z = s["logits"][b:b + step].double()
        ids = s["ids"][b:b + step].long()
        there = ids >= 0
        t = s["teacher"][b:b + step].double() / T
        t = t.masked_fill(~there, float("-inf"))
        any_ = there.any(dim=1)
        q = torch.softmax(t[any_], dim=1)
        target = torch.zeros((z.shape[0], V), dtype=torch.float64, device="cuda")
        filled = torch.zeros((int(any_.sum()), V), dtype=torch.float64, device="cuda")
        filled.scatter_add_(1, ids[any_].clamp(min=0), q)
        target[any_] = filled
        lp = torch.log_softmax(z / T, dim=1)
        entropy = torch.where(q > 0, q * torch.log(q.clamp(min=1e-300)), 0.0).sum(dim=1)
        part = torch.zeros(z.shape[0], dtype=torch.float64, device="cuda")
        part[any_] = entropy
        cross = torch.where(target > 0, target * lp, 0.0).sum(dim=1)
        part = (part - cross) * (s["soft"] * T * T)
        g = None
        if grad is not None:
            g = (torch.exp(lp) * any_[:, None] - target) * (s["soft"] * T)
        if s["labels"] is not None:
            y = s["labels"][b:b + step].long()
            r = torch.nonzero(y >= 0)[:, 0]
            lq = torch.log_softmax(z, dim=1)
            part[r] -= s["hard"] * lq[r, y[r]]
            if g is not None:
                g[r] += s["hard"] * torch.exp(lq[r])
                g[r, y[r]] -= s["hard"]
        loss[b:b + step] = part
        if g is not None:
            grad[b:b + step] = g * s["weight"][b:b + step].double()[:, None]
    out = {}
    if c["mode"] != "backward":
        out["loss"] = loss
    if whole:
        out["grad"] = grad
    return out


def _exact_sample(s):
    """One row after the other, over the words in order of their scores."""
    c = s["case"]
    ids = torch.empty(c["rows"], dtype=torch.int32, device="cuda")
    logprob = torch.zeros(c["rows"], dtype=torch.float64, device="cuda")

    def of(v, r):
        return float(v[r]) if isinstance(v, torch.Tensor) else float(v)

    for r in range(c["rows"]):
        z, order = torch.sort(s["logits"][r].double(), descending=True, stable=True)
        T = of(s["temperature"], r)
        if T == 0:
            ids[r] = order[0]
            continue
        z = (z - z[0]) / T
        w = torch.exp(z)
        n = int((z > float("-inf")).sum())
        if c["top_k"] > 0:
            n = min(n, int(of(s["top_k"], r)))
        if c["top_p"] < 1:
            c_w = torch.cumsum(w[:n], dim=0)
            n = 1 + int((c_w[:-1] < of(s["top_p"], r) * c_w[-1]).sum())
        if c["min_p"] > 0:
            n = int((w[:n] >= of(s["min_p"], r)).sum())
        at = order[:n]
        race = z[:n] - torch.log(-torch.log(s["uniforms"][r].double()[at]))
        best = race.max()
        win = at[race == best].min()
        ids[r] = win
        logprob[r] = z[torch.nonzero(order == win)[0, 0]] - torch.log(w.sum())
    return {"ids": ids, "logprob": logprob}


def exact(case, seed):
    """What run() returns for these inputs, from the definitions in 64 bits."""
    s = prepare(case, seed)
    return {"linear": _exact_linear, "back": _exact_back, "distill": _exact_distill,
            "sample": _exact_sample}[case["kind"]](s)
