"""The dense operators on both sides of the mixture of experts: embed, linear, sample.

embed     token ids -> scaled rows of a table; backward -> gradient of the table
linear    y = act(x W^T + bias) + residual; backward -> gradients of x, W and the bias (the residual's is grad_y itself)
sample    logits -> the next token of every row: temperature, top-k, min-p, top-p, one given random number per row

`run` computes a case in its plain form (elementary torch operations) or, with `own`, through the library's calls.
`exact` restates the definitions in 64 bits.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}
PAD = 0  # the token id that gets no gradient where a case pads its batch


# ---------------------------------------------------------------------------------------------------------- cases
def _linear(rows, n, k, dtype, act="none", bias=True, residual=False, out="same", backward=False, wide=False, name=None):
    """wide: the bias and the gradients of W and of the bias are fp32"""
    c = {"op": "linear", "rows": rows, "n": n, "k": k, "dtype": dtype, "act": act, "bias": bias, "residual": residual, "out": out,
         "backward": backward, "wide": wide}
    return {"name": name, **c} if name else c


def _sample(rows, vocab, dtype, filters, name=None):
    """filters: none | top_k | top_p | all (every row its own temperature, top-k, top-p and min-p)"""
    c = {"op": "sample", "rows": rows, "vocab": vocab, "dtype": dtype, "filters": filters}
    return {"name": name, **c} if name else c


def _embed(tokens, vocab, d, dtype, backward, pad=0.0, wide=False, name=None):
    """wide: the table's gradient is fp32"""
    c = {"op": "embed", "tokens": tokens, "vocab": vocab, "d": d, "dtype": dtype, "backward": backward, "pad": pad, "wide": wide}
    return {"name": name, **c} if name else c


def listed():
    return [
        # one token of one request through a dense layer back into the residual stream: latency
        _linear(1, 2048, 1024, "bf16", residual=True, name="linear_one_token"),
        # a decoding step of 48 requests: the vocabulary's logits, bound by the weights
        _linear(48, 128000, 2048, "bf16", bias=False, out="f32", name="linear_logits_decode"),
        # a prompt of odd length through a layer's second product
        _linear(1021, 2048, 5632, "bf16", residual=True, name="linear_prompt"),
        # the router of the routing batch: 65536 tokens, 128 experts, fp32 logits
        _linear(65536, 128, 2048, "bf16", bias=False, out="f32", name="linear_router"),
        # a small training step with ragged widths
        _linear(777, 1003, 520, "f16", act="gelu", residual=True, backward=True, name="linear_train_ragged"),
        # an ordinary training step of a layer's first product, fp32 gradients for the optimiser
        _linear(16384, 8192, 2048, "bf16", act="silu", backward=True, wide=True, name="linear_train_large"),
        # the next token of one request
        _sample(1, 50021, "f32", "all", name="sample_one"),
        # a decoding step of 48 requests without filters, 16-bit logits
        _sample(48, 128000, "bf16", "none", name="sample_plain"),
        # a large decoding step, every request with settings of its own
        _sample(256, 128000, "f32", "all", name="sample_batch"),
        # a decoding step of 48 requests
        _embed(48, 128000, 2048, "bf16", False, name="embed_decode"),
        # a small training step, a tenth of it padding
        _embed(4093, 50021, 1000, "f16", True, pad=0.1, name="embed_train_ragged"),
        # a training step of the routing batch, fp32 gradient
        _embed(65536, 128000, 2048, "bf16", True, wide=True, name="embed_train_large"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["linear", "linear", "sample", "embed"])
    if op == "sample":
        while True:
            rows, vocab = _log_int(rng, 1, 512), _log_int(rng, 16, 262144)
            if rows * vocab <= 256 * 128000:
                return _sample(rows, vocab, rng.choice(["f32", "f32", "bf16", "f16"]), rng.choice(["none", "top_k", "top_p", "all", "all"]))
    if op == "embed":
        while True:
            tokens, vocab, d = _log_int(rng, 1, 65536), _log_int(rng, 64, 131072), _log_int(rng, 32, 4096)
            d = rng.choice([d, 8 * (d // 8), 8 * (d // 8)])
            if vocab * d <= 128000 * 2048 and tokens * d <= 65536 * 2048:
                return _embed(tokens, vocab, d, rng.choice(["bf16", "bf16", "f16", "f32"]), rng.random() < 0.6,
                              pad=rng.choice([0.0, 0.1]), wide=rng.random() < 0.3)
    while True:
        rows, n, k = _log_int(rng, 1, 65536), _log_int(rng, 8, 65536), 8 * _log_int(rng, 8, 1024)
        n = rng.choice([n, 8 * (n // 8)])
        backward = rng.random() < 0.5
        if max(rows * n * k * (3 if backward else 1) // 2048, rows * n, rows * k, n * k // 2) <= 16384 * 8192:
            return _linear(rows, n, k, rng.choice(["bf16", "bf16", "f16"]), act=rng.choice(["none", "none", "relu", "silu", "gelu", "gelu_tanh"]),
                           bias=rng.random() < 0.6, residual=rng.random() < 0.4, out=rng.choice(["same", "same", "f32"]), backward=backward,
                           wide=rng.random() < 0.3)


# --------------------------------------------------------------------------------------------------------- inputs
def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = {"case": c}
    {"linear": _prepare_linear, "sample": _prepare_sample, "embed": _prepare_embed}[c["op"]](c, s, gen)
    if own:
        {"linear": _own_linear, "sample": _own_sample, "embed": _own_embed}[c["op"]](c, s)
    return s


def _prepare_linear(c, s, gen):
    """activations with channels of different size, weights that keep their scale"""
    dt, (M, N, K) = DTYPES[c["dtype"]], (c[n] for n in ("rows", "n", "k"))
    out = torch.float32 if c["out"] == "f32" else dt
    channel = torch.exp(0.3 * torch.randn(K, device="cuda", generator=gen))
    s["x"] = (torch.randn(M, K, device="cuda", generator=gen) * channel).to(dt)
    s["w"] = torch.empty(N, K, device="cuda", dtype=dt).normal_(0, K ** -0.5, generator=gen)
    s["bias"] = (0.2 * torch.randn(N, device="cuda", generator=gen)).to(torch.float32 if c["wide"] else dt) if c["bias"] else None
    s["residual"] = torch.randn(M, N, device="cuda", generator=gen).to(out) if c["residual"] else None
    if c["backward"]:
        s["grad_y"] = torch.randn(M, N, device="cuda", generator=gen).to(out)


def _prepare_sample(c, s, gen):
    """a language model's logits: most tokens far behind, a few that matter, some excluded; per-row settings as requests bring them"""
    R, V = c["rows"], c["vocab"]
    x = torch.randn(R, V, device="cuda", generator=gen)
    x.mul_(2.0).add_(torch.randn(V, device="cuda", generator=gen))
    n = min(V, 40)
    at = torch.randint(0, V, (R, n), device="cuda", generator=gen)
    x.scatter_reduce_(1, at, 6 + 3 * torch.randn(R, n, device="cuda", generator=gen), "amax")  # where two meet, the same one every time
    x[torch.rand(R, V, device="cuda", generator=gen) < 0.001] = -math.inf
    x[:, 0] = 0.0  # something to choose in every row
    s["logits"] = x.to(DTYPES[c["dtype"]])
    s["u"] = torch.rand(R, device="cuda", generator=gen)

    def pick(values):
        return torch.tensor(values, device="cuda")[torch.randint(0, len(values), (R,), device="cuda", generator=gen)]

    every = c["filters"] == "all"
    s["temperature"] = pick([0.0, 0.3, 0.7, 1.0, 1.0, 1.3]) if every else torch.full((R,), 0.8, device="cuda")
    s["top_k"] = pick([0, 0, 1, 20, 50, 1000]).to(torch.int32) if every else \
        torch.full((R,), 40 if c["filters"] == "top_k" else 0, device="cuda", dtype=torch.int32)
    s["top_p"] = pick([1.0, 0.95, 0.9, 0.5]) if every else torch.full((R,), 0.9 if c["filters"] == "top_p" else 1.0, device="cuda")
    s["min_p"] = pick([0.0, 0.0, 0.02, 0.1]) if every else torch.zeros(R, device="cuda")


def _prepare_embed(c, s, gen):
    """words by Zipf's law over a shuffled vocabulary"""
    n, V, D, dt = c["tokens"], c["vocab"], c["d"], DTYPES[c["dtype"]]
    rank = (((V + 2.7) / 2.7) ** torch.rand(n, device="cuda", generator=gen, dtype=torch.float64) * 2.7 - 2.7).long().clamp_(0, V - 1)
    ids = torch.randperm(V, device="cuda", generator=gen)[rank]
    if c["pad"]:
        ids[torch.rand(n, device="cuda", generator=gen) < c["pad"]] = PAD
    s["ids"] = ids.to(torch.int32)
    s["scale"] = D ** 0.5
    s["table"] = torch.empty(V, D, device="cuda", dtype=dt).normal_(0, D ** -0.5, generator=gen)
    if c["backward"]:
        s["grad_y"] = torch.randn(n, D, device="cuda", generator=gen).to(dt)


def _own_linear(c, s):
    """what a program keeps: workspace, outputs, the saved pre-activation"""
    import paper_2608_06912_b200 as L

    dt, M = DTYPES[c["dtype"]], c["rows"]
    out = torch.float32 if c["out"] == "f32" else dt
    s["ws"] = L.LinearWorkspace(M, c["n"], c["k"], activation=L.ACTIVATIONS[c["act"]], io_dtype=L.IO_OF[dt], out_dtype=L.IO_OF[out],
                                training=c["backward"])
    s["y"] = torch.empty(M, c["n"], device="cuda", dtype=out)
    if c["backward"]:
        s["pre"] = s["ws"].new_pre()
        wide = torch.float32 if c["wide"] else dt
        s["grads"] = (torch.empty_like(s["x"]), torch.empty_like(s["w"], dtype=wide),
                      torch.empty(c["n"], device="cuda", dtype=wide) if c["bias"] else None)


def _own_sample(c, s):
    import paper_2608_06912_b200 as L

    R = c["rows"]
    s["params"] = L.sample_params(io_dtype=L.IO_OF[DTYPES[c["dtype"]]])
    s["out"] = (torch.empty(R, device="cuda", dtype=torch.int32), torch.empty(R, device="cuda"),
                torch.empty(R, device="cuda", dtype=torch.int32))


def _own_embed(c, s):
    import paper_2608_06912_b200 as L

    n, V, D, dt = c["tokens"], c["vocab"], c["d"], DTYPES[c["dtype"]]
    s["y"] = torch.empty(n, D, device="cuda", dtype=dt)
    if c["backward"]:
        s["ws"] = L.EmbedWorkspace(n, V, D)
        s["grad_table"] = torch.empty(V, D, device="cuda", dtype=torch.float32 if c["wide"] else dt)


# ------------------------------------------------------------------------------------------------------ one pass
def run(state):
    c = state["case"]
    if own:
        return {"linear": _linear_own, "sample": _sample_own, "embed": _embed_own}[c["op"]](c, state)
    return {"linear": _linear_plain, "sample": _sample_plain, "embed": _embed_plain}[c["op"]](c, state)


def _linear_own(c, s):
    import paper_2608_06912_b200 as L

    L.lapsum_linear_forward(s["x"], s["w"], s["bias"], s["residual"], s["y"], s["ws"], pre=s.get("pre"))
    if not c["backward"]:
        return s["y"]
    gx, gw, gb = s["grads"]
    L.lapsum_linear_backward(s["grad_y"], s["x"], s["w"], s["pre"], gx, gw, gb, s["ws"])
    return (s["y"], gx, gw, gb) if c["bias"] else (s["y"], gx, gw)


def _sample_own(c, s):
    import paper_2608_06912_b200 as L

    token, logprob, kept = s["out"]
    L.lapsum_sample(s["logits"], s["u"], s["params"], token, logprob, kept, temperature=s["temperature"], top_k=s["top_k"],
                    top_p=s["top_p"], min_p=s["min_p"])
    return token, logprob, kept


def _embed_own(c, s):
    import paper_2608_06912_b200 as L

    L.lapsum_embed_forward(s["ids"], s["table"], s["y"], scale=s["scale"])
    if not c["backward"]:
        return s["y"]
    L.lapsum_embed_backward(s["grad_y"], s["ids"], s["grad_table"], s["ws"], scale=s["scale"], skip=PAD if c["pad"] else -1)
    return s["y"], s["grad_table"]


def _act(name, p):
    """the activation and its slope"""
    if name == "none":
        return p, None
    if name == "relu":
        return p * (p > 0), (p > 0).to(p.dtype)
    if name == "silu":
        g = 1 / (1 + torch.exp(-p))
        return p * g, g * (1 + p * (1 - g))
    if name == "gelu":
        half = 0.5 * (1 + torch.erf(p * 0.5 ** 0.5))
        return p * half, half + p * torch.exp(-0.5 * p * p) * (2 * math.pi) ** -0.5
    a, b = (2 / math.pi) ** 0.5, 0.044715
    t = torch.tanh(a * (p + b * p * p * p))
    return 0.5 * p * (1 + t), 0.5 * (1 + t) + 0.5 * p * (1 - t * t) * a * (1 + 3 * b * p * p)


def _linear_plain(c, s):
    x, w, dt = s["x"].float(), s["w"].float(), s["x"].dtype
    out = torch.float32 if c["out"] == "f32" else dt
    p = x @ w.t()
    if c["bias"]:
        p = p + s["bias"].float()
    y, slope = _act(c["act"], p)
    if c["residual"]:
        y = y + s["residual"].float()
    y = y.to(out)
    if not c["backward"]:
        return y
    gp = s["grad_y"].float()
    if slope is not None:
        gp = gp * slope
    wide = torch.float32 if c["wide"] else dt
    grads = [(gp @ w).to(dt), (gp.t() @ x).to(wide)]
    if c["bias"]:
        grads.append(gp.sum(0).to(wide))
    return (y, *grads)


def _sample_plain(c, s):
    """in 64 bits: which token wins hangs on sums next to a border.  A row of temperature 0 keeps its largest logit."""
    x = s["logits"].double()
    V = x.shape[1]
    t = s["temperature"].double()[:, None]
    order = x.sort(dim=1, descending=True, stable=True)
    top = order.values[:, :1]
    e = torch.exp((order.values - top) / torch.where(t > 0, t, 1.0))
    rank = torch.arange(V, device="cuda")[None]
    k = s["top_k"].long()[:, None]
    keep = (e >= s["min_p"].double()[:, None]) & (order.values > -math.inf) & ((k <= 0) | (rank < k))
    e = e * keep
    run_sum = e.cumsum(1)
    p = s["top_p"].double()[:, None]
    keep &= (p >= 1) | (run_sum - e < p * run_sum[:, -1:])
    keep = torch.where(t > 0, keep, rank == 0)
    e = e * keep
    by_index = torch.zeros_like(e).scatter_(1, order.indices, e)
    run_sum = by_index.cumsum(1)
    total = run_sum[:, -1:]
    token = (run_sum <= s["u"].double()[:, None] * total).sum(1, keepdim=True).clamp_(max=V - 1)
    logprob = torch.log(by_index.gather(1, token) / total)
    return token[:, 0].to(torch.int32), logprob[:, 0].float(), keep.sum(1).to(torch.int32)


def _embed_plain(c, s):
    ids, dt = s["ids"].long(), s["table"].dtype
    y = (s["table"][ids].float() * s["scale"]).to(dt)
    if not c["backward"]:
        return y
    g = s["grad_y"].float() * s["scale"]
    if c["pad"]:
        g = g * (ids != PAD)[:, None]
    grad = torch.zeros(c["vocab"], c["d"], device="cuda").index_add_(0, ids, g)
    return y, grad if c["wide"] else grad.to(dt)


# --------------------------------------------------------------------------------------------- the work of a pass
def work(case):
    c = case
    b = BYTES[c["dtype"]]
    if c["op"] == "linear":
        M, N, K = c["rows"], c["n"], c["k"]
        o, wide = 4 if c["out"] == "f32" else b, 4 if c["wide"] else b
        n = M * K * b + N * K * b + M * N * o * (2 if c["residual"] else 1) + (N * wide if c["bias"] else 0)
        if c["backward"]:
            n += M * N * o + M * K * b + N * K * wide + (N * wide if c["bias"] else 0)
        return {"bytes": n, "flops": 2 * M * N * K * (3 if c["backward"] else 1)}
    if c["op"] == "sample":
        return {"bytes": c["rows"] * (c["vocab"] * b + 32), "flops": c["rows"] * c["vocab"] * 4}
    n, V, D = c["tokens"], c["vocab"], c["d"]
    used = sum(1 - (1 - p) ** n for p in _zipf(V))
    total = n * 4 + used * D * b + n * D * b
    if c["backward"]:
        total += n * D * b + V * D * (4 if c["wide"] else b)
    return {"bytes": int(total), "flops": n * D * (2 if c["backward"] else 1)}


def _zipf(V):
    """probabilities of the ranks as the inputs draw them"""
    full = math.log((V + 2.7) / 2.7)
    return [math.log((r + 3.7) / (r + 2.7)) / full for r in range(V)]


# -------------------------------------------------------------------------------------------------------- 64 bits
def exact(case, seed):
    c = case
    keep_own = globals()["own"]
    globals()["own"] = False
    try:
        s = prepare(c, seed)
    finally:
        globals()["own"] = keep_own
    return {"linear": _linear_exact, "sample": _sample_exact, "embed": _embed_exact}[c["op"]](c, s)


def _linear_exact(c, s):
    """the definition with automatic differentiation"""
    back = c["backward"]
    x, w = s["x"].double().requires_grad_(back), s["w"].double().requires_grad_(back)
    b = s["bias"].double().requires_grad_(back) if c["bias"] else None
    F = torch.nn.functional
    act = {"none": lambda t: t, "relu": F.relu, "silu": F.silu, "gelu": F.gelu, "gelu_tanh": lambda t: F.gelu(t, approximate="tanh")}[c["act"]]
    y = act(F.linear(x, w, b))
    if c["residual"]:
        y = y + s["residual"].double()
    if not back:
        return y
    leaves = [x, w] + ([b] if c["bias"] else [])
    return (y.detach(), *torch.autograd.grad(y, leaves, s["grad_y"].double()))


def _sample_exact(c, s):
    """request by request in numpy, the filters one after the other as sets of tokens"""
    import numpy as np

    logits = s["logits"].double().cpu().numpy()
    u, t, k, p, m = (s[n].double().cpu().numpy() for n in ("u", "temperature", "top_k", "top_p", "min_p"))
    tokens, logprobs, counts = [], [], []
    for r in range(c["rows"]):
        x = logits[r]
        order = np.argsort(-x, kind="stable")
        order = order[x[order] > -np.inf]
        if t[r] == 0:
            order = order[:1]
            weight = np.ones(1)
        else:
            if k[r] > 0:
                order = order[:int(k[r])]
            weight = np.exp((x[order] - x[order[0]]) / t[r])
            order, weight = order[weight >= m[r]], weight[weight >= m[r]]
            if p[r] < 1:
                reached = np.cumsum(weight) >= p[r] * np.sum(weight)
                n = int(np.argmax(reached)) + 1
                order, weight = order[:n], weight[:n]
        by_index = np.argsort(order, kind="stable")
        order, weight = order[by_index], weight[by_index]
        total = np.cumsum(weight)
        at = min(int(np.searchsorted(total, u[r] * total[-1], side="right")), len(order) - 1)
        tokens.append(int(order[at]))
        logprobs.append(math.log(weight[at] / total[-1]))
        counts.append(len(order))
    return (torch.tensor(tokens, dtype=torch.int32), torch.tensor(logprobs, dtype=torch.float64), torch.tensor(counts, dtype=torch.int32))


def _embed_exact(c, s):
    ids = s["ids"].long()
    y = torch.nn.functional.embedding(ids, s["table"]).double() * s["scale"]
    if not c["backward"]:
        return y
    rows = s["grad_y"].double() * s["scale"]
    if c["pad"]:
        real = ids != PAD
        ids, rows = ids[real], rows[real]
    grad = torch.zeros(c["vocab"], c["d"], device="cuda", dtype=torch.float64)
    return y, grad.index_put_((ids,), rows, accumulate=True)
