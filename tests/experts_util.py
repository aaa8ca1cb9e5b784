"""64-bit references of the mixture-of-experts operators, with the error bounds that the GPU tests use.

Bounds.  U is half a unit in the last place of the 16-bit type relative to 1 (half its epsilon: bf16 2^-8, fp16
2^-11), the largest relative error of one rounding.  The kernels round
w h, g, u, dg, du, the per-slot results and the outputs once each; sums are fp32 (their error, below 2^-20 of the terms'
size, disappears in U).  An output is a sum of many terms with independent rounding errors, each at most E in size
(standard deviation E / sqrt 3), so its error is compared with 6 sqrt(sum E^2) (more than ten deviations), plus U |value|
for the output's own rounding, or half the type's smallest subnormal where that is more:
    y        E = U |w h W_down| per term, and U |w o| per slot
    grad_w   E = U |dh| (1.1 |g u| + |silu(g) u|)          (g and u are rounded; |silu'| < 1.1)
    dg       E = U (2 |dg| + 0.6 |w dh u|)                 (|g silu''(g)| < 0.6)       du  E = U (|du| + 1.1 |w dh g|)
    grad_x, grad_w_gate_up: the sums of dg's and du's E through the product; grad_w_down: E = U |dy w h|
"""
import torch

U = {t: torch.finfo(t).eps / 2 for t in (torch.bfloat16, torch.float16)}


def route_reference(logits, bias, k, score="softmax", groups=1, kept=1, top=2, renorm=True, scale=1.0, grad_w=None):
    """(idx, w, grad_logits or None) in 64 bits on the CPU, token by token"""
    x = logits.double().cpu()
    T, E = x.shape
    b = None if bias is None else bias.double().cpu()
    idx, w = torch.full((T, k), -1, dtype=torch.int64), torch.zeros(T, k, dtype=torch.float64)
    grad = torch.zeros(T, E, dtype=torch.float64)
    for t in range(T):
        l = x[t].clone()
        usable = l > float("-inf")  # false for -inf and NaN
        l[~usable] = float("-inf")
        if not usable.any():
            continue
        s = {"softmax": lambda v: torch.softmax(v, 0), "sigmoid": torch.sigmoid, "given": lambda v: v}[score](l)
        strength_keys = s if b is None else s + b
        keys = l if b is None else strength_keys
        alive = usable & (keys > float("-inf"))
        if groups > 1:
            per, strength = E // groups, []
            for g in range(groups):
                v = sorted(strength_keys[g * per:(g + 1) * per][alive[g * per:(g + 1) * per]].tolist(), reverse=True)[:top]
                strength.append(sum(v) if v else float("-inf"))
            order = sorted((g for g in range(groups) if strength[g] > float("-inf")), key=lambda g: (-strength[g], g))[:kept]
            inside = torch.zeros(E, dtype=torch.bool)
            for g in order:
                inside[g * per:(g + 1) * per] = True
            alive = alive & inside
        chosen = sorted(torch.nonzero(alive)[:, 0].tolist(), key=lambda e: (-float(keys[e]), e))[:k]
        n = len(chosen)
        if n == 0:
            continue
        lt = l.clone().requires_grad_(True)
        st = {"softmax": lambda v: torch.log_softmax(v, 0), "sigmoid": torch.nn.functional.logsigmoid, "given": lambda v: v}[score](lt)[chosen]
        if score == "given":
            wt = (st / st.sum() if float(st.detach().sum()) != 0 else st * 0) if renorm else st
        else:
            wt = torch.softmax(st, 0) if renorm else torch.exp(st)
        wt = scale * wt
        idx[t, :n], w[t, :n] = torch.tensor(chosen), wt.detach()
        if grad_w is not None:
            (g,) = torch.autograd.grad((wt * grad_w[t, :n].double().cpu()).sum(), lt)
            grad[t] = torch.nan_to_num(g, nan=0.0)  # -inf entries: the derivative of softmax there is 0
    return idx, w, grad


def dispatch_reference(idx, experts, rows):
    """counts, offsets, slot_of, entry_of (up to the last offset) by plain counting"""
    flat = idx.reshape(-1).tolist()
    lists = [[] for _ in range(experts)]
    for i, e in enumerate(flat):
        if 0 <= e < experts:
            lists[e].append(i)
    counts, offsets, slot_of, entry_of = [len(v) for v in lists], [0], [-1] * len(flat), []
    for v in lists:
        for j, i in enumerate(v):
            slot_of[i] = offsets[-1] + j
        entry_of += v + [-1] * (-len(v) % rows)
        offsets.append(len(entry_of))
    return counts, offsets, slot_of, entry_of


def experts_reference(x, w_gate_up, w_down, idx, w, grad_y=None):
    """{name: (value, error bound)} in 64 bits for y and, with grad_y, every gradient"""
    u = U[x.dtype]
    x64, a64, b64, w64 = x.double(), w_gate_up.double(), w_down.double(), w.double()
    E, F2, D = a64.shape
    F = F2 // 2
    T, k = idx.shape
    y, ey = torch.zeros(T, D, dtype=torch.float64, device=x.device), torch.zeros(T, D, dtype=torch.float64, device=x.device)
    if grad_y is not None:
        gy = grad_y.double()
        gx, egx = torch.zeros_like(y), torch.zeros_like(y)
        gw, egw = torch.zeros_like(w64), torch.zeros_like(w64)
        ga, ega = torch.zeros_like(a64), torch.zeros_like(a64)
        gb, egb = torch.zeros_like(b64), torch.zeros_like(b64)
    for e in range(E):
        t, j = (idx == e).nonzero(as_tuple=True)
        if t.numel() == 0:
            continue
        a, b, we = a64[e], b64[e], w64[t, j][:, None]
        g, up = (x64[t] @ a.T).split(F, dim=1)
        sg = torch.sigmoid(g)
        act = g * sg
        h = act * up
        o = h @ b.T
        y.index_add_(0, t, we * o)
        ey.index_add_(0, t, (we * h) ** 2 @ b.T ** 2 + (we * o) ** 2)
        if grad_y is None:
            continue
        dy = gy[t]
        dh = dy @ b
        gw[t, j] = (dh * h).sum(1)
        egw[t, j] = ((dh * (1.1 * (g * up).abs() + h.abs())) ** 2).sum(1)
        dg, du = we * dh * up * (sg + act * (1 - sg)), we * dh * act
        eg, eu = 2 * dg.abs() + 0.6 * (we * dh * up).abs(), du.abs() + 1.1 * (we * dh * g).abs()
        d, ed = torch.cat([dg, du], 1), torch.cat([eg, eu], 1)
        s = d @ a
        gx.index_add_(0, t, s)
        egx.index_add_(0, t, ed ** 2 @ a ** 2 + s ** 2)
        ga[e], ega[e] = d.T @ x64[t], (ed ** 2).T @ x64[t] ** 2
        gb[e], egb[e] = dy.T @ (we * h), (dy ** 2).T @ (we * h) ** 2

    def bound(v, e2):
        return (u * v.abs()).clamp(min=torch.finfo(x.dtype).smallest_normal * u) + 6 * u * e2.sqrt()

    out = {"y": (y, bound(y, ey))}
    if grad_y is not None:
        out.update(grad_x=(gx, bound(gx, egx)), grad_w=(gw, bound(gw, egw)), grad_w_gate_up=(ga, bound(ga, ega)),
                   grad_w_down=(gb, bound(gb, egb)))
    return out


def chosen(T, E, k, gen, drop=0.0, skew=0.7, device="cuda"):
    """k different experts per token (int32), some experts far more popular; dropped entries are -1"""
    pop = skew * torch.randn(E, generator=gen, device=device)
    noise = -torch.log(-torch.log(torch.rand(T, E, generator=gen, device=device).clamp(1e-9, 1 - 1e-7)))
    idx = (pop + noise).topk(k, 1).indices.to(torch.int32) if T else torch.zeros(0, k, dtype=torch.int32, device=device)
    if drop:
        idx[torch.rand(T, k, generator=gen, device=device) < drop] = -1
    return idx
