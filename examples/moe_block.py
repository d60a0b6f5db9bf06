"""An MoE block with the library's operators, as a program runs them: one boundary between blocks (norm after the last block, gate, residual
sum, norm before this one), routing, plan, dispatch, the experts' products, combine; and the gradients of all of it.

    python examples/moe_block.py            decode, prefill and a training step on cuda:0, checked against plain torch
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2512_22036_amd as fusco  # noqa: E402


def _empty(*shape, like=None, dtype=torch.bfloat16):
    return torch.empty(shape, dtype=like.dtype if like is not None else dtype, device="cuda")


class MoEBlock:
    """Weights and calls of one block: H columns, E experts of I units each, k per token, D devices, groups = devices."""

    def __init__(self, H, I, E, k, D, keep_groups, seed=0):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        normal = lambda *s, std: torch.randn(s, generator=gen, device="cuda").mul_(std)
        self.H, self.I, self.E, self.k, self.D, self.keep = H, I, E, k, D, keep_groups
        self.gain, self.before = 1 + normal(H, std=0.1), 1 + normal(H, std=0.1)
        self.gate = 0.5 + normal(H, std=0.1)
        self.router, self.bias = normal(E, H, std=H ** -0.5), normal(E, std=0.02)
        self.w_in, self.w_out = normal(E, 2 * I, H, std=H ** -0.5).bfloat16(), normal(E, H, I, std=I ** -0.5).bfloat16()

    def forward(self, r, y, keep=False):
        """The stream r before, and the output y of, the last block -> (stream, this block's output); with keep also what
        backward needs."""
        N = r.shape[0]
        s, x = _empty(N, self.H, like=r), _empty(N, self.H)
        fusco.fusco_norm_after(r, y, self.gain, s, gate=self.gate, scale=0.5, next_gain=self.before, next_out=x)
        logits = x.float() @ self.router.t()
        idx, w = _empty(N, self.k, dtype=torch.int32), _empty(N, self.k, dtype=torch.float32)
        fusco.fusco_route(logits, idx, w, bias=self.bias, score=fusco.SCORE_SIGMOID, groups=self.D, keep_groups=self.keep, group_best=2)
        L = fusco.Layout(N, self.k, self.E, self.D)
        rows = _empty(L.P, self.H)
        if N <= 2048 // self.k:
            fusco.fusco_plan_dispatch(L, idx, x, rows)
        else:
            fusco.fusco_plan(L, idx)
            fusco.fusco_dispatch(L, x, rows)
        h, out_rows, out = _empty(L.P, self.I), _empty(L.P, self.H), _empty(N, self.H)
        pre = _empty(L.P, 2 * self.I) if keep else None
        fusco.fusco_experts_gated(L, rows, self.w_in, h, pre)
        fusco.fusco_experts_linear(L, h, self.w_out, out_rows)
        fusco.fusco_combine(L, out_rows, w, out)
        return (s, out, (r, y, s, x, logits, idx, w, L, rows, pre, h, out_rows)) if keep else (s, out)

    def backward(self, kept, ds, dout):
        """Gradients of the stream s (past this block) and of the block's output -> gradients of r, y and all weights."""
        r, y, s, x, logits, idx, w, L, rows, pre, h, out_rows = kept
        N, ones = r.shape[0], torch.ones_like(w)
        d_rows, dw = torch.empty_like(out_rows), torch.empty_like(w)
        fusco.fusco_combine_backward(L, out_rows, w, dout, d_rows, dw)
        dpre, dw_out = torch.empty_like(pre), torch.empty_like(self.w_out)
        fusco.fusco_experts_input_grad(L, d_rows, self.w_out, dpre, pre=pre)
        fusco.fusco_experts_weight_grad(L, d_rows, h, dw_out)
        dx_rows, dw_in = torch.empty_like(rows), torch.empty_like(self.w_in)
        fusco.fusco_experts_input_grad(L, dpre, self.w_in, dx_rows)
        fusco.fusco_experts_weight_grad(L, dpre, rows, dw_in)
        dx = _empty(N, self.H, dtype=torch.float32)
        fusco.fusco_combine(L, dx_rows, ones, dx)               # the dispatch's gradient
        dlogits = torch.empty_like(logits)
        fusco.fusco_route_backward(logits, idx, dw, dlogits, score=fusco.SCORE_SIGMOID)
        d_router = dlogits.t() @ x.float()
        dx = (dx + dlogits @ self.router).bfloat16()
        dr, dy = torch.empty_like(r), torch.empty_like(y)
        d_gain, d_gate, d_before = torch.empty_like(self.gain), torch.empty_like(self.gate), torch.empty_like(self.before)
        fusco.fusco_norm_after_backward(ds, y, self.gain, dr, dy, d_gain, gate=self.gate, dgate=d_gate, scale=0.5, dnext=dx, out=s, next_gain=self.before, dnext_gain=d_before)
        return dict(r=dr, y=dy, gain=d_gain, gate=d_gate, before=d_before, router=d_router, w_in=dw_in, w_out=dw_out)

    def plain(self, r, y, idx, p):
        """The same block in plain torch with the experts given, differentiable in p (weights by name, with r and y)."""
        unit = lambda v: v / (v.square().mean(dim=1, keepdim=True) + 1e-6).sqrt()
        s = p["r"] + 0.5 * p["gate"] * unit(p["y"]) * p["gain"]
        x = unit(s) * p["before"]
        score = torch.sigmoid(x @ p["router"].t()).gather(1, idx.long())
        w = score / score.sum(dim=1, keepdim=True)
        out = torch.zeros_like(x)
        for e in range(self.E):
            t, j = (idx == e).nonzero(as_tuple=True)
            g, u = (x[t] @ p["w_in"][e].t()).split(self.I, dim=1)
            out = out.index_add(0, t, w[t, j][:, None] * ((g * torch.sigmoid(g) * u) @ p["w_out"][e].t()))
        return s, out


def timed(f, n=20):
    for _ in range(3):
        f()
    a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    a.record()
    for _ in range(n):
        f()
    b.record()
    torch.cuda.synchronize()
    return a.elapsed_time(b) / n * 1e3


def check(N=96, H=256, I=128, E=16, k=4, D=4, keep_groups=2):
    """Forward and backward of a small block against plain torch in 64 bits: relative errors by tensor."""
    block = MoEBlock(H, I, E, k, D, keep_groups)
    gen = torch.Generator(device="cuda").manual_seed(1)
    normal = lambda *s: torch.randn(s, generator=gen, device="cuda")
    r, y, ds, dout = normal(N, H), normal(N, H).bfloat16(), normal(N, H), normal(N, H).bfloat16()
    s, out, kept = block.forward(r, y, keep=True)
    got = dict(block.backward(kept, ds, dout), s=s, out=out)
    p = {n: t.detach().double().requires_grad_() for n, t in dict(r=r, y=y, gain=block.gain, gate=block.gate, before=block.before, router=block.router, w_in=block.w_in, w_out=block.w_out).items()}
    want_s, want_out = block.plain(r, y, kept[5], p)
    grads = torch.autograd.grad([want_s, want_out], list(p.values()), [ds.double(), dout.double()])
    want = dict(zip(p, grads), s=want_s.detach(), out=want_out.detach())
    return {n: float((got[n].double() - want[n]).norm() / want[n].norm()) for n in want}


def main():
    fusco.load_library()
    torch.cuda.set_device(0)
    far = check()
    print("relative error against 64 bits: " + ", ".join("%s %.1e" % (n, v) for n, v in far.items()))
    assert max(far.values()) < 0.02
    block = MoEBlock(H=4096, I=1280, E=128, k=8, D=16, keep_groups=8)
    for N in (1, 128, 16384):
        r, y = torch.randn((N, 4096), device="cuda").bfloat16(), torch.randn((N, 4096), device="cuda").bfloat16()
        us = timed(lambda: block.forward(r, y))
        print("forward of %5d tokens: %.1f us" % (N, us))
    r, y = torch.randn((8192, 4096), device="cuda"), torch.randn((8192, 4096), device="cuda").bfloat16()
    s, out, kept = block.forward(r, y, keep=True)
    ds, dout = torch.randn_like(s), torch.randn_like(out)
    print("backward of %5d tokens: %.1f us" % (8192, timed(lambda: block.backward(kept, ds, dout), 5)))


if __name__ == "__main__":
    main()
