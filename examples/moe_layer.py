"""A mixture-of-experts layer routed by the exact-budget soft top-k, trained for a few steps and then asked for single tokens.

    logits --lapsum_forward--> soft mask p (sum p = k) --route--> k experts and weights --dispatch--> tables --experts--> y

The backward runs the same chain the other way: the experts' gradients, the weights' gradient through the route to the mask, and
lapsum_backward from the mask to the router's logits.

    python examples/moe_layer.py [--tokens 512] [--steps 30]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2608_06912_b200 as L  # noqa: E402


class MoeLayer:
    """Weights and buffers of one layer for batches of one size (bf16 experts, fp32 router)."""

    def __init__(self, tokens, experts=16, k=4, d=256, f=512, alpha=-0.25, training=True, weights=None, seed=0):
        self.tokens, self.experts, self.k, self.alpha, self.training = tokens, experts, k, alpha, training
        gen = torch.Generator(device="cuda").manual_seed(seed)

        def rand(*shape, scale, dtype=torch.bfloat16):
            return (scale * torch.randn(*shape, device="cuda", generator=gen)).to(dtype)

        self.router, self.w_gate_up, self.w_down = weights if weights is not None else (
            rand(experts, d, scale=d ** -0.5, dtype=torch.float32), rand(experts, 2 * f, d, scale=d ** -0.5),
            rand(experts, d, f, scale=f ** -0.5))
        self.mask_ws = L.Workspace(tokens, experts)
        self.params = L.route_params(k=k, score=L.ROUTE_GIVEN, grad_w_dtype=L.IO_BF16)
        self.tables = L.Dispatch(tokens, k, experts, training=training)
        self.ws = L.ExpertsWorkspace(self.tables, d, f, io_dtype=L.IO_BF16, training=training)
        self.saved = self.ws.new_saved() if training else None
        self.mask, self.b = torch.empty(tokens, experts, device="cuda"), torch.empty(tokens, device="cuda")
        self.idx, self.w = torch.empty(tokens, k, device="cuda", dtype=torch.int32), torch.empty(tokens, k, device="cuda")
        self.y = torch.empty(tokens, d, device="cuda", dtype=torch.bfloat16)

    def forward(self, x):
        self.logits = x.float() @ self.router.t()
        L.lapsum_forward(self.logits, float(self.k), self.alpha, self.mask, self.b, self.mask_ws)
        L.lapsum_route_forward(self.mask, None, self.params, self.idx, self.w)
        L.lapsum_dispatch(self.idx, self.tables)
        L.lapsum_experts_forward(x, self.w_gate_up, self.w_down, self.w, self.tables, self.y, self.ws, saved=self.saved)
        return self.y

    def backward(self, x, grad_y):
        """gradients of x, the router and the experts' weights"""
        gx, ga, gb = torch.empty_like(x), torch.empty_like(self.w_gate_up), torch.empty_like(self.w_down)
        gw = torch.empty_like(self.w, dtype=torch.bfloat16)
        L.lapsum_experts_backward(grad_y, x, self.w_gate_up, self.w_down, self.w, self.tables, self.saved, gx, ga, gb, gw, self.ws)
        grad_mask, grad_logits = torch.empty_like(self.mask), torch.empty_like(self.mask)
        L.lapsum_route_backward(gw, self.mask, self.idx, self.w, self.params, grad_mask)
        L.lapsum_backward(grad_mask, self.logits, self.b, float(self.k), self.alpha, grad_logits, self.mask_ws)
        gx += (grad_logits @ self.router).to(gx.dtype)
        return gx, grad_logits.t() @ x.float(), ga, gb


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--tokens", type=int, default=512)
    ap.add_argument("--steps", type=int, default=30)
    a = ap.parse_args(argv)
    d = 256
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(a.tokens, d, device="cuda", generator=gen).to(torch.bfloat16)
    target = (x.float() @ torch.randn(d, d, device="cuda", generator=gen) * d ** -0.5).tanh()  # what the layer shall learn
    layer = MoeLayer(a.tokens, d=d)
    masters = [t.float() for t in (layer.router, layer.w_gate_up, layer.w_down)]  # fp32 copies that the steps go to
    losses = []
    for step in range(a.steps):
        y = layer.forward(x)
        diff = y.float() - target
        losses.append(diff.square().mean().item())
        _, *grads = layer.backward(x, (2 * diff / a.tokens).to(torch.bfloat16))
        for own, master, g in zip((layer.router, layer.w_gate_up, layer.w_down), masters, grads):
            master -= 0.5 * g.float()
            own.copy_(master)
        if step % 10 == 0 or step == a.steps - 1:
            print(f"step {step}: loss {losses[-1]:.4f}, tokens per expert {layer.tables.counts.tolist()}")
    one = MoeLayer(1, d=d, training=False, weights=(layer.router, layer.w_gate_up, layer.w_down))  # the same weights, one token at a time
    layer.forward(x)
    apart = max((one.forward(x[t:t + 1])[0].float() - layer.y[t].float()).abs().max().item() for t in range(min(8, a.tokens)))
    print(f"single tokens against the batch: largest difference {apart:.4f} (values up to {layer.y.abs().max().item():.2f})")
    if layer.ws.status() or one.ws.status():
        raise RuntimeError("a kernel gave up waiting")
    return losses, apart


if __name__ == "__main__":
    main()
