"""The mixture-of-experts operators next to the soft top-k: routing, dispatch and the experts' products.

route     logits -> the k chosen experts of every token and their weights; backward -> gradient of the logits
dispatch  chosen experts -> the tokens of every expert side by side (counts, offsets, both directions of the map)
experts   y_t = sum_j w_tj W_down[e] (silu(g) * u), [g; u] = W_gate_up[e] x_t, e = idx_tj; backward -> every gradient

`run` computes a case in its plain form (elementary torch operations in 32 bits) or, with `own`, through the
library's calls.  `exact` restates the definitions in 64 bits.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}
MARGIN = 4e-6  # choices closer than this are redrawn: which expert wins must not hang on the last bits of an exponential


# ---------------------------------------------------------------------------------------------------------- cases
def _route(tokens, experts, k, score, dtype, backward, bias=False, groups=1, kept=1, top=2, renorm=True, scale=1.0, name=None):
    c = {"op": "route", "tokens": tokens, "experts": experts, "k": k, "score": score, "dtype": dtype, "backward": backward,
         "bias": bias, "groups": groups, "kept": kept, "top": top, "renorm": renorm, "scale": scale}
    return {"name": name, **c} if name else c


def _dispatch(tokens, experts, k, tile_rows, drop=0.0, name=None):
    c = {"op": "dispatch", "tokens": tokens, "experts": experts, "k": k, "tile_rows": tile_rows, "drop": drop}
    return {"name": name, **c} if name else c


def _experts(tokens, experts, k, d, f, dtype, backward, drop=0.0, name=None):
    c = {"op": "experts", "tokens": tokens, "experts": experts, "k": k, "d": d, "f": f, "dtype": dtype, "backward": backward,
         "drop": drop}
    return {"name": name, **c} if name else c


def listed():
    return [
        # one token of one request: nothing but latency
        _route(1, 128, 8, "softmax", "f32", False, name="route_one_token"),
        # the routing batch of the soft top-k's own benchmark: 65536 tokens, 128 experts, 8 chosen; a training step
        _route(65536, 128, 8, "softmax", "f32", True, name="route_batch"),
        # balance by a bias on sigmoid scores, experts in 8 groups of which 4 stay; 16-bit logits, an odd number of tokens
        _route(16381, 256, 8, "sigmoid", "bf16", True, bias=True, groups=8, kept=4, scale=2.5, name="route_groups"),
        # a decoding step of 32 requests
        _dispatch(32, 128, 8, 16, name="dispatch_decode"),
        # a training batch; one entry in fifty dropped (padding, capacity)
        _dispatch(65536, 128, 8, 128, drop=0.02, name="dispatch_batch"),
        # one token of one request: eight experts' weights are read once
        _experts(1, 64, 8, 2048, 1024, "bf16", False, name="experts_one_token"),
        # a decoding step of 48 requests: nearly every expert is needed, for a few tokens each
        _experts(48, 128, 8, 2048, 768, "f16", False, name="experts_decode"),
        # a prompt of odd length
        _experts(1021, 64, 6, 2048, 1408, "bf16", False, name="experts_prompt"),
        # a batch of prompts
        _experts(16384, 64, 8, 2048, 1024, "bf16", False, name="experts_batch"),
        # a small training step with ragged widths, few experts and dropped entries
        _experts(777, 24, 2, 1000, 520, "f16", True, drop=0.1, name="experts_train_ragged"),
        # ordinary training steps
        _experts(8192, 32, 4, 2048, 1024, "bf16", True, name="experts_train"),
        _experts(16384, 64, 8, 2048, 1024, "bf16", True, name="experts_train_large"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["route", "dispatch", "experts", "experts"])
    if op == "route":
        experts = rng.choice([8, 16, 60, 64, 100, 128, 160, 256, 384, 512])
        tokens = _log_int(rng, 1, 65536 * 128 // max(experts, 128))
        score = rng.choice(["softmax", "sigmoid", "given"])
        groups, kept = 1, 1
        if score == "sigmoid" and rng.random() < 0.5:
            groups = rng.choice([g for g in (2, 4, 8) if experts % g == 0 and experts // g >= 2])
            kept = rng.randint(1, groups)
        k = rng.randint(1, min(10, experts // groups * kept))
        return _route(tokens, experts, k, score, rng.choice(["f32", "f32", "bf16", "f16"]), rng.random() < 0.6,
                      bias=score != "softmax" and rng.random() < 0.5, groups=groups, kept=kept, top=rng.choice([1, 2]),
                      renorm=rng.random() < 0.7, scale=rng.choice([1.0, 1.0, 2.5]))
    if op == "dispatch":
        experts = rng.choice([4, 8, 60, 64, 128, 160, 256, 512])
        return _dispatch(_log_int(rng, 1, 65536), experts, rng.randint(1, min(8, experts)), rng.choice([16, 32, 64, 128]),
                         drop=rng.choice([0.0, 0.05]))
    while True:
        d, f = 8 * rng.randint(32, 256), 8 * rng.randint(16, 176)
        experts = rng.choice([8, 16, 60, 64, 100, 128])
        k, tokens = rng.randint(1, 8), _log_int(rng, 1, 16384)
        backward = rng.random() < 0.5
        c = _experts(tokens, experts, k, d, f, rng.choice(["bf16", "bf16", "f16"]), backward, drop=rng.choice([0.0, 0.0, 0.05]))
        if tokens * k * d * f <= 16384 * 8 * 2048 * 1024 // 2 and experts * d * f <= 64 * 2048 * 1024:
            return c


# --------------------------------------------------------------------------------------------------------- inputs
def _choice_keys(c, logits, bias):
    """what the experts are compared by, in 64 bits"""
    x = logits.double()
    if c["score"] == "sigmoid" and (bias is not None or c["groups"] > 1):
        x = torch.sigmoid(x)
    return x if bias is None else x + bias.double()


def _unclear(c, logits, bias):
    """rows in which two keys that matter differ by less than the margin (equal keys are clear: the lower index wins)"""
    if bias is None and c["groups"] == 1:
        return torch.zeros(logits.shape[0], dtype=torch.bool, device=logits.device)  # compared as they stand
    keys, bad = _choice_keys(c, logits, bias), None
    if c["groups"] > 1:
        grp = keys.view(keys.shape[0], c["groups"], -1)
        s = grp.topk(min(c["top"], grp.shape[2]), 2).values.sum(2).sort(dim=1, descending=True)
        if c["kept"] < c["groups"]:
            bad = s.values[:, c["kept"] - 1] - s.values[:, c["kept"]] < MARGIN
        keep = torch.zeros_like(s.values, dtype=torch.bool).scatter_(1, s.indices[:, :c["kept"]], True)
        keys = torch.where(keep[:, :, None], grp, float("-inf")).reshape(keys.shape)
    top = keys.topk(min(c["k"] + 1, keys.shape[1]), 1).values
    gap = top[:, :-1] - top[:, 1:]
    near = ((gap > 0) & (gap < MARGIN)).any(1)
    return near if bad is None else bad | near


def _logits(c, gen):
    """router outputs: N(0, 1.5) with a popularity offset per expert; `given` scores lie in (0, 1) like a soft mask"""
    dt, T, E = DTYPES[c["dtype"]], c["tokens"], c["experts"]
    offset = 0.5 * torch.randn(E, device="cuda", generator=gen)
    bias = 0.02 * torch.randn(E, device="cuda", generator=gen) if c["bias"] else None

    def rows(n):
        x = 1.5 * torch.randn(n, E, device="cuda", generator=gen) + offset
        return (torch.sigmoid(2 * x - 4) if c["score"] == "given" else x).to(dt)

    x = rows(T)
    for _ in range(20):
        bad = _unclear(c, x, bias).nonzero()[:, 0]
        if bad.numel() == 0:
            break
        x[bad] = rows(bad.numel())
    return x, bias


def _chosen(c, gen):
    """k different experts per token, some experts far more popular than others; dropped entries are -1"""
    T, E, k = c["tokens"], c["experts"], c["k"]
    noise = -torch.log(-torch.log(torch.rand(T, E, device="cuda", generator=gen).clamp_(1e-9, 1 - 1e-7)))
    idx = (noise + 0.6 * torch.randn(E, device="cuda", generator=gen)).topk(k, 1).indices.to(torch.int32)
    if c["drop"]:
        idx[torch.rand(T, k, device="cuda", generator=gen) < c["drop"]] = -1
    return idx


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = {"case": c}
    if c["op"] == "route":
        s["logits"], s["bias"] = _logits(c, gen)
        s["grad_w"] = torch.randn(c["tokens"], c["k"], device="cuda", generator=gen)
    elif c["op"] == "dispatch":
        s["idx"] = _chosen(c, gen)
    else:
        dt, (T, E, D, F) = DTYPES[c["dtype"]], (c[n] for n in ("tokens", "experts", "d", "f"))
        channel = torch.exp(0.3 * torch.randn(D, device="cuda", generator=gen))
        s["x"] = (torch.randn(T, D, device="cuda", generator=gen) * channel).to(dt)
        s["w_gate_up"] = torch.empty(E, 2 * F, D, device="cuda", dtype=dt).normal_(0, D ** -0.5, generator=gen)
        s["w_down"] = torch.empty(E, D, F, device="cuda", dtype=dt).normal_(0, F ** -0.5, generator=gen)
        s["idx"] = _chosen(c, gen)
        s["w"] = torch.softmax(torch.randn(T, c["k"], device="cuda", generator=gen), 1)
        if c["backward"]:
            s["grad_y"] = torch.randn(T, D, device="cuda", generator=gen).to(dt)
    if own:
        _prepare_own(c, s)
    return s


def _prepare_own(c, s):
    """what a program keeps: output buffers, the dispatch tables, the experts' workspace and saved activations"""
    import paper_2608_06912_b200 as L

    T, E, k = c["tokens"], c["experts"], c["k"]
    if c["op"] == "route":
        s["params"] = L.route_params(k=k, score=L.ROUTE_SCORES[c["score"]], groups=c["groups"], groups_kept=c["kept"],
                                     group_top=c["top"], renormalise=int(c["renorm"]), scale=c["scale"],
                                     io_dtype=L.IO_OF[DTYPES[c["dtype"]]])
        s["idx"] = torch.empty(T, k, device="cuda", dtype=torch.int32)
        s["w"] = torch.empty(T, k, device="cuda")
        s["grad_logits"] = torch.empty_like(s["logits"])
        return
    if c["op"] == "dispatch":
        s["dispatch"] = L.Dispatch(T, k, E, tile_rows=c["tile_rows"])
        return
    s["dispatch"] = L.Dispatch(T, k, E, tile_rows=L.dispatch_tile_rows(T, k, E, training=c["backward"]))
    s["experts"] = L.ExpertsWorkspace(s["dispatch"], c["d"], c["f"], io_dtype=L.IO_OF[DTYPES[c["dtype"]]], training=c["backward"])
    s["y"] = torch.empty_like(s["x"])
    if c["backward"]:
        s["saved"] = s["experts"].new_saved()
        s["out"] = {"grad_x": torch.empty_like(s["x"]), "grad_w_gate_up": torch.empty_like(s["w_gate_up"]),
                    "grad_w_down": torch.empty_like(s["w_down"]), "grad_w": torch.empty_like(s["w"], dtype=DTYPES[c["dtype"]])}


# ------------------------------------------------------------------------------------------------------ one pass
def run(state):
    c = state["case"]
    if own:
        return {"route": _route_own, "dispatch": _dispatch_own, "experts": _experts_own}[c["op"]](c, state)
    return {"route": _route_plain, "dispatch": _dispatch_plain, "experts": _experts_plain}[c["op"]](c, state)


def _route_own(c, s):
    import paper_2608_06912_b200 as L

    L.lapsum_route_forward(s["logits"], s["bias"], s["params"], s["idx"], s["w"])
    if not c["backward"]:
        return s["idx"], s["w"]
    L.lapsum_route_backward(s["grad_w"], s["logits"], s["idx"], s["w"], s["params"], s["grad_logits"])
    return s["idx"], s["w"], s["grad_logits"]


def _dispatch_own(c, s):
    import paper_2608_06912_b200 as L

    p = s["dispatch"]
    L.lapsum_dispatch(s["idx"], p)
    return p.counts, p.offsets, p.slot_of, p.entry_of


def _experts_own(c, s):
    import paper_2608_06912_b200 as L

    L.lapsum_dispatch(s["idx"], s["dispatch"])
    L.lapsum_experts_forward(s["x"], s["w_gate_up"], s["w_down"], s["w"], s["dispatch"], s["y"], s["experts"],
                             saved=s.get("saved"))
    if not c["backward"]:
        return s["y"]
    o = s["out"]
    L.lapsum_experts_backward(s["grad_y"], s["x"], s["w_gate_up"], s["w_down"], s["w"], s["dispatch"], s["saved"],
                              o["grad_x"], o["grad_w_gate_up"], o["grad_w_down"], o["grad_w"], s["experts"])
    return s["y"], o["grad_x"], o["grad_w_gate_up"], o["grad_w_down"], o["grad_w"]


def _route_plain(c, s):
    """scores, the choice by score plus bias inside the best groups, weights from the scores alone"""
    x, bias, k = s["logits"].float(), s["bias"], c["k"]
    if c["score"] == "softmax":
        e = torch.exp(x - x.max(1, keepdim=True).values)
        score = e / e.sum(1, keepdim=True)
    elif c["score"] == "sigmoid":
        score = 1 / (1 + torch.exp(-x))
    else:
        score = x
    if bias is not None:
        keys = score + bias
    else:
        keys = score if c["groups"] > 1 else x  # both scores rise with the logit: without a bias the logits decide
    if c["groups"] > 1:
        grp = keys.view(keys.shape[0], c["groups"], -1)
        best = grp.sort(dim=2, descending=True).values[:, :, :min(c["top"], grp.shape[2])].sum(2)
        at = best.sort(dim=1, descending=True, stable=True).indices[:, :c["kept"]]
        keep = torch.zeros_like(best, dtype=torch.bool).scatter_(1, at, True)
        keys = torch.where(keep[:, :, None], grp, float("-inf")).reshape(keys.shape)
    idx = keys.sort(dim=1, descending=True, stable=True).indices[:, :k]
    picked = score.gather(1, idx)
    total = picked.sum(1, keepdim=True)
    w = c["scale"] * (picked / total if c["renorm"] else picked)
    if not c["backward"]:
        return idx.to(torch.int32), w
    gw = s["grad_w"]
    if c["renorm"]:
        gp = (c["scale"] * gw - (gw * w).sum(1, keepdim=True)) / total  # gradient of the chosen scores
    else:
        gp = c["scale"] * gw
    gs = torch.zeros_like(score).scatter_(1, idx, gp)
    if c["score"] == "softmax":
        gx = score * (gs - (gs * score).sum(1, keepdim=True))
    elif c["score"] == "sigmoid":
        gx = gs * score * (1 - score)
    else:
        gx = gs
    return idx.to(torch.int32), w, gx.to(s["logits"].dtype)


def _capacity(c):
    n, rows = c["tokens"] * c["k"], c["tile_rows"]
    return (n + min(n, c["experts"]) * (rows - 1)) // rows * rows


def _dispatch_plain(c, s):
    """entries sorted by expert (stable), every expert's rows starting at a multiple of tile_rows; holes hold -1"""
    idx, E, rows = s["idx"], c["experts"], c["tile_rows"]
    flat = idx.reshape(-1).long()
    key = torch.where(flat < 0, E, flat)
    order = key.sort(dim=0, stable=True).indices
    counts = (torch.zeros(E + 1, dtype=torch.int64, device="cuda")).index_add_(0, key, torch.ones_like(key))[:E]
    offsets = torch.zeros(E + 1, dtype=torch.int64, device="cuda")
    offsets[1:] = ((counts + rows - 1) // rows * rows).cumsum(0)
    first = counts.cumsum(0) - counts
    sorted_key = key[order]
    e = sorted_key.clamp(max=E - 1)
    pos = torch.arange(flat.numel(), device="cuda") - first[e] + offsets[e]
    pos = torch.where(sorted_key < E, pos, -1)
    slot_of = torch.empty_like(flat)
    slot_of[order] = pos
    entry_of = torch.full((_capacity(c) + 1,), -1, dtype=torch.int64, device="cuda")
    entry_of[torch.where(pos < 0, _capacity(c), pos)] = order
    i32 = torch.int32
    return counts.to(i32), offsets.to(i32), slot_of.view(idx.shape).to(i32), entry_of[:-1].to(i32)


def _experts_plain(c, s):
    """short batches: the experts in use as one padded batch; long ones: expert by expert; all in 32 bits"""
    idx, wgu, wd = s["idx"], s["w_gate_up"], s["w_down"]
    T, E, k, D = c["tokens"], c["experts"], c["k"], c["d"]
    flat = idx.reshape(-1).long()
    key = torch.where(flat < 0, E, flat)
    order = key.sort(dim=0, stable=True).indices
    counts = torch.zeros(E + 1, dtype=torch.int64, device="cuda").index_add_(0, key, torch.ones_like(key))[:E]
    first = counts.cumsum(0) - counts
    dt, back = s["x"].dtype, c["backward"]
    x = s["x"].float()
    out = torch.zeros(T * k, D, device="cuda")
    grads = None
    if back:
        grads = (s["grad_y"].float(), torch.zeros(T * k, D, device="cuda"), torch.zeros_like(wgu), torch.zeros_like(wd),
                 torch.zeros(T * k, device="cuda"))
    if T <= 1024:
        used, most = counts.nonzero()[:, 0], int(counts.max())
        at = torch.arange(most, device="cuda")
        real = at < counts[used, None]
        rows = order[torch.where(real, first[used, None] + at, 0)]
        _experts_part(c, s, x, used, rows, real, out, grads)
    else:
        begin = 0
        for e, n in enumerate(counts.tolist()):
            if n:
                _experts_part(c, s, x, slice(e, e + 1), order[None, begin:begin + n], None, out, grads)
            begin += n
    y = out.view(T, k, D).sum(1).to(dt)
    if not back:
        return y
    return y, grads[1].view(T, k, D).sum(1).to(dt), grads[2], grads[3], grads[4].view(T, k).to(dt)


def _experts_part(c, s, x, used, rows, real, out, grads):
    """some experts' products on their tokens (rows: an expert's entries, padded where `real` says no)"""
    k, F, dt = c["k"], c["f"], s["x"].dtype
    a, b = s["w_gate_up"][used].float(), s["w_down"][used].float()
    xe, we = x[rows // k], s["w"].reshape(-1)[rows]
    if real is not None:
        xe, we = xe * real[:, :, None], we * real
    to = rows[0] if real is None else rows[real]
    gu = xe @ a.transpose(1, 2)
    g, u = gu[:, :, :F], gu[:, :, F:]
    sg = 1 / (1 + torch.exp(-g))
    h = g * sg * u
    o = h @ b.transpose(1, 2)
    out[to] = _flat(o * we[:, :, None], real)
    if grads is None:
        return
    gy, gx, ggu, gd, gw = grads
    dy = gy[rows // k]
    gw[to] = _flat((dy * o).sum(2), real)
    dy = dy * we[:, :, None]
    gd[used] = (dy.transpose(1, 2) @ h).to(dt)
    dh = dy @ b
    dgu = torch.cat([dh * u * sg * (1 + g * (1 - sg)), dh * g * sg], 2)
    ggu[used] = (dgu.transpose(1, 2) @ xe).to(dt)
    gx[to] = _flat(dgu @ a, real)


def _flat(v, real):
    return v[0] if real is None else v[real]


# --------------------------------------------------------------------------------------------- the work of a pass
def work(case):
    c = case
    T, E, k = c["tokens"], c["experts"], c["k"]
    if c["op"] == "route":
        b = BYTES[c["dtype"]]
        n = T * E * b + T * k * 8 + (E * 4 if c["bias"] else 0)
        if c["backward"]:
            n += T * k * 4 + T * E * b
        return {"bytes": n, "flops": T * E * (8 if c["backward"] else 4)}
    if c["op"] == "dispatch":
        return {"bytes": T * k * 8 + _capacity(c) * 4 + E * 8 + 4, "flops": T * k}
    b, D, F = BYTES[c["dtype"]], c["d"], c["f"]
    n = T * k * (1 - c["drop"])
    active = E * (1 - (1 - k * (1 - c["drop"]) / E) ** T) if k < E else E
    weights = 3 * D * F * b
    total = 2 * T * D * b + T * k * 8 + active * weights
    if c["backward"]:
        total += 2 * T * D * b + T * k * b + E * weights  # grad_y, grad_x, grad_w; every expert's gradient is written
    return {"bytes": int(total), "flops": int(6 * n * D * F * (3 if c["backward"] else 1))}


# -------------------------------------------------------------------------------------------------------- 64 bits
def exact(case, seed):
    c = case
    keep_own = globals()["own"]
    globals()["own"] = False
    try:
        s = prepare(c, seed)
    finally:
        globals()["own"] = keep_own
    if c["op"] == "route":
        return _route_exact(c, s)
    if c["op"] == "dispatch":
        return _dispatch_exact(c, s)
    return _experts_exact(c, s)


def _route_exact(c, s):
    """the definition with automatic differentiation"""
    x = s["logits"].double().requires_grad_(c["backward"])
    score = {"softmax": lambda t: torch.softmax(t, 1), "sigmoid": torch.sigmoid, "given": lambda t: t}[c["score"]](x)
    keys = _choice_keys(c, s["logits"], s["bias"])
    T, E = keys.shape
    if c["groups"] > 1:
        per = E // c["groups"]
        members = keys.view(T, c["groups"], per)
        strength = members.topk(min(c["top"], per), 2).values.sum(2)
        rank = strength.argsort(dim=1, descending=True, stable=True).argsort(1)
        keys = keys.masked_fill((rank >= c["kept"]).repeat_interleave(per, 1), -math.inf)
    idx = keys.argsort(dim=1, descending=True, stable=True)[:, :c["k"]]
    w = score.gather(1, idx)
    if c["renorm"]:
        w = w / w.sum(1, keepdim=True)
    w = w * c["scale"]
    if not c["backward"]:
        return idx.to(torch.int32), w
    (gx,) = torch.autograd.grad(w, x, s["grad_w"].double())
    return idx.to(torch.int32), w.detach(), gx


def _dispatch_exact(c, s):
    """by counting in plain Python and numpy"""
    import numpy as np

    idx = s["idx"].cpu().numpy()
    flat, rows = idx.reshape(-1), c["tile_rows"]
    counts, offsets = np.zeros(c["experts"], np.int32), np.zeros(c["experts"] + 1, np.int32)
    slot_of, entry_of = np.full(flat.size, -1, np.int32), np.full(_capacity(c), -1, np.int32)
    base = 0
    for e in range(c["experts"]):
        mine = np.flatnonzero(flat == e)
        counts[e], offsets[e] = mine.size, base
        slot_of[mine] = base + np.arange(mine.size)
        entry_of[base:base + mine.size] = mine
        base += -(-mine.size // rows) * rows
    offsets[-1] = base
    return tuple(torch.from_numpy(a) for a in (counts, offsets, slot_of.reshape(idx.shape), entry_of))


def _experts_exact(c, s):
    """token by choice in 64 bits, expert by expert, gradients by automatic differentiation of each expert's part"""
    F, E, back = c["f"], c["experts"], c["backward"]
    x, w = s["x"].double(), s["w"].double()
    y = torch.zeros_like(x)
    if back:
        gy, gx, gw = s["grad_y"].double(), torch.zeros_like(x), torch.zeros_like(w)
        ggu = torch.zeros(s["w_gate_up"].shape, device="cuda", dtype=torch.float64)
        gd = torch.zeros(s["w_down"].shape, device="cuda", dtype=torch.float64)
    for e in range(E):
        t, j = (s["idx"] == e).nonzero(as_tuple=True)
        if t.numel() == 0:
            continue
        xe, we = x[t].requires_grad_(back), w[t, j].requires_grad_(back)
        a, b = s["w_gate_up"][e].double().requires_grad_(back), s["w_down"][e].double().requires_grad_(back)
        gate, up = torch.split(torch.nn.functional.linear(xe, a), F, dim=1)
        part = torch.nn.functional.linear(torch.nn.functional.silu(gate) * up, b) * we[:, None]
        y.index_add_(0, t, part.detach())
        if back:
            gxe, gwe, ggu[e], gd[e] = torch.autograd.grad(part, (xe, we, a, b), gy[t])
            gx.index_add_(0, t, gxe)
            gw[t, j] = gwe
    return (y, gx, ggu, gd, gw) if back else y
