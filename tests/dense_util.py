"""64-bit references of the dense operators (linear, sample, embed), with the error bounds that the GPU tests use.

Linear.  U is the largest relative error of one rounding to the 16-bit type (half its epsilon).  A product of two 16-bit values is exact in
fp32; the tensor core adds them sixteen at a time, each addition off by at most 2^-22 of the partial sum, and the partial sums of terms t
with random signs stay below 3 sqrt(sum t^2):  |dP| <= B(P) = 3 (K / 16 + 2) 2^-22 sqrt(sum t^2).
    y       1.13 B(P) (the largest slope) + 2^-19 (|act| + 1) (its evaluation) + one rounding of y
    dP      is rounded (U |dP|, or U^2 |dP| where grad_w is fp32) and its slope is taken at a P rounded to pre's type (U_P):
            |act''| <= 1.2, so E = U |dP| + 1.2 |dy| (U_P |P| + B(P)) + 2^-19 |dy| (the slope's evaluation)
    grad_x, grad_w: sums of many terms with independent errors of at most E |w| (E |x|): 6 sqrt(sum of squares), plus the sum's own error B
            and one rounding.    grad_bias sums the unrounded dP: E without U |dP|, additions off by 2^-24 of partial sums below 3 sqrt(sum dP^2)
relu's slope jumps at 0, where P's own error decides the side: there |dP| <= |dy| is off by as much, so E = |dy| where |P| <= B(P).
"""
import numpy as np
import torch

U = {torch.bfloat16: torch.finfo(torch.bfloat16).eps / 2, torch.float16: torch.finfo(torch.float16).eps / 2, torch.float32: 2.0 ** -24}


def act64(name, p):
    F = torch.nn.functional
    return {"none": lambda t: t, "relu": F.relu, "silu": F.silu, "gelu": F.gelu, "gelu_tanh": lambda t: F.gelu(t, approximate="tanh")}[name](p)


def one_rounding(v, dtype):
    """largest error of rounding v to dtype, the smallest subnormals included"""
    return (U[dtype] * v.abs()).clamp(min=torch.finfo(dtype).smallest_normal * U[dtype])


def linear_reference(x, w, bias, residual, act, out_dtype, grad_y=None, grad_w_dtype=None, grad_bias_dtype=None, pre_dtype=torch.float32):
    """{name: (value, error bound)} in 64 bits"""
    u = U[x.dtype]
    x64, w64 = x.double(), w.double()
    b64 = 0 if bias is None else bias.double()
    rows, k = x.shape
    n = w.shape[0]

    def sums(a, b, terms):  # a @ b and the bound of its summation
        return a @ b, 3 * (terms / 16 + 2) * 2.0 ** -22 * (a ** 2 @ b ** 2).sqrt()

    p, bp = sums(x64, w64.t(), k)
    p = p + b64
    bp = bp + 2.0 ** -23 * p.abs()
    leaf = p.clone().requires_grad_()
    a = act64(act, leaf)
    y = a.detach() + (0 if residual is None else residual.double())
    out = {"y": (y, 1.13 * bp + (0 if act == "none" else 2.0 ** -19 * (a.detach().abs() + 1)) + 2.0 ** -23 * y.abs() + one_rounding(y, out_dtype))}
    if grad_y is None:
        return out
    gy = grad_y.double()
    (slope,) = torch.autograd.grad(a.sum(), leaf) if act != "none" else (torch.ones_like(p),)
    gp = gy * slope
    off = torch.zeros_like(gp) if act == "none" else 1.2 * gy.abs() * (U[pre_dtype] * p.abs() + bp) + 2.0 ** -19 * gy.abs()
    if act == "relu":
        off = torch.where(p.abs() <= bp, gy.abs(), torch.zeros_like(gp))
    e = off + u * gp.abs()
    wide = off + (u * u if grad_w_dtype == torch.float32 else u) * gp.abs()  # the remainder of the rounding is rounded in its turn
    gx, bx = sums(gp, w64, n)
    out["grad_x"] = (gx, 6 * (e ** 2 @ w64 ** 2).sqrt() + bx + one_rounding(gx, x.dtype))
    gw, bw = sums(gp.t(), x64, rows)
    out["grad_w"] = (gw, 6 * ((wide ** 2).t() @ x64 ** 2).sqrt() + bw + one_rounding(gw, grad_w_dtype or x.dtype))
    if bias is not None:
        gb = gp.sum(0)
        out["grad_bias"] = (gb, 6 * (off ** 2).sum(0).sqrt() + 3 * (rows + 2) * 2.0 ** -24 * (gp ** 2).sum(0).sqrt()
                            + one_rounding(gb, grad_bias_dtype or x.dtype))
    return out


def sample_reference(logits, u, temperature, top_k, top_p, min_p):
    """(token, logprob, kept) of every row in 64 bits; the settings are one per row.  Rows one by one, sets of tokens."""
    x_all = logits.double().cpu().numpy()
    tokens, logprobs, counts = [], [], []
    for r in range(x_all.shape[0]):
        x, t, k, p, m, ur = x_all[r], float(temperature[r]), int(top_k[r]), float(top_p[r]), float(min_p[r]), float(u[r])
        if not (0 <= t < np.inf and p > 0 and 0 <= m <= 1 and 0 <= ur < 1):
            tokens.append(-1), logprobs.append(np.nan), counts.append(0)
            continue
        usable = np.flatnonzero(x > -np.inf)
        if usable.size == 0:
            tokens.append(-1), logprobs.append(-np.inf), counts.append(0)
            continue
        if x[usable].max() == np.inf:
            usable = usable[x[usable] == np.inf]
        order = usable[np.argsort(-x[usable], kind="stable")]
        top = x[order[0]]
        if t == 0:
            order, weight = order[:1], np.ones(1)
        else:
            weight = np.ones(len(order)) if top == np.inf else np.exp((x[order] - top) / t)
            n = int((weight >= m).sum())
            if k > 0:
                n = min(n, k)
            order, weight = order[:n], weight[:n]
            if p < 1:
                n = int(np.argmax(np.cumsum(weight) >= p * weight.sum())) + 1
                order, weight = order[:n], weight[:n]
        by = np.argsort(order, kind="stable")
        order, weight = order[by], weight[by]
        run = np.cumsum(weight)
        at = min(int(np.searchsorted(run, ur * run[-1], side="right")), len(order) - 1)
        tokens.append(int(order[at])), logprobs.append(float(np.log(weight[at] / run[-1]))), counts.append(len(order))
    return np.array(tokens), np.array(logprobs), np.array(counts)


def embed_reference(ids, grad, vocab, scale, skip, out_dtype):
    """the table's gradient in 64 bits and its error bound: each of the n terms' additions is off by at most 2^-24 of a partial sum"""
    g = grad.double()
    real = (ids >= 0) & (ids < vocab) & (ids != skip)
    at = ids[real].long()
    value = torch.zeros(vocab, grad.shape[1], dtype=torch.float64, device=grad.device).index_put_((at,), g[real] * scale, accumulate=True)
    total = torch.zeros_like(value).index_put_((at,), (g[real] * scale).abs(), accumulate=True)
    n = torch.bincount(at, minlength=vocab).double()[:, None]
    return value, (n + 2) * 2.0 ** -24 * total + one_rounding(value, out_dtype)
