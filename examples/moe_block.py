"""An MoE block with the library's operators, as a program runs them: one boundary between blocks (norm after the last block, gate, residual
sum, norm before this one), routing, plan, dispatch, the experts' products, combine; and the gradients of all of it.  MoEBlock holds its weights
and rows in bf16, EightBlock in e4m3.

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

    def before_experts(self, r, y):
        """-> stream, rows for the experts, logits, experts and weights of every token"""
        N = r.shape[0]
        s, x = _empty(N, self.H, like=r), _empty(N, self.H)
        fusco.fusco_norm_after(r, y, self.gain, s, gate=self.gate, scale=0.5, next_gain=self.before, next_out=x)
        logits = x.float() @ self.router.t()
        idx, w = _empty(N, self.k, dtype=torch.int32), _empty(N, self.k, dtype=torch.float32)
        fusco.fusco_route(logits, idx, w, bias=self.bias, score=fusco.SCORE_SIGMOID, groups=self.D, keep_groups=self.keep, group_best=2)
        return s, x, logits, idx, w

    def forward(self, r, y, keep=False):
        """The stream r before, and the output y of, the last block -> (stream, this block's output); with keep also what
        backward needs."""
        N = r.shape[0]
        s, x, logits, idx, w = self.before_experts(r, y)
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
        dx_rows, dw_in, dw_out = self.through_experts(L, d_rows, rows, pre, h)
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

    def through_experts(self, L, d_rows, rows, pre, h):
        dpre, dw_out = torch.empty_like(pre), torch.empty_like(self.w_out)
        fusco.fusco_experts_input_grad(L, d_rows, self.w_out, dpre, pre=pre)
        fusco.fusco_experts_weight_grad(L, d_rows, h, dw_out)
        dx_rows, dw_in = torch.empty_like(rows), torch.empty_like(self.w_in)
        fusco.fusco_experts_input_grad(L, dpre, self.w_in, dx_rows)
        fusco.fusco_experts_weight_grad(L, dpre, rows, dw_in)
        return dx_rows, dw_in, dw_out

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


def to_eight(x):
    """Rows, or matrices, in e4m3 with their scales; rows of scales have whole units of 16 bytes, as a dispatch takes them"""
    blocks = lambda n, unit=128: -(-n // unit)
    shape = (x.shape[0], blocks(x.shape[1], 512) * 4) if x.dim() == 2 else (x.shape[0], blocks(x.shape[1]), blocks(x.shape[2]))
    q, scale = _empty(*x.shape, dtype=torch.float8_e4m3fn), _empty(*shape, dtype=torch.float32)
    fusco.fusco_to_fp8(x, q, scale)
    return q, scale


def from_eight(q, scale):
    """Their values, which bf16 holds exactly as long as the scales are powers of two"""
    x = _empty(*q.shape)
    fusco.fusco_from_fp8(q, scale, x)
    return x


class EightBlock(MoEBlock):
    """The block with weights of e4m3, rows sent and multiplied in e4m3, and in e4m3 what backward needs of them.  Gradients are those of the
    products as they were computed: roundings to e4m3 count as constants (w_in and w_out are here the rounded weights).

    FEW: tokens up to which the layer for a few tokens is taken, which needs no rows in e4m3 but passes over an expert's weights again for every few of its tokens.  Experts alone,
    that way / scaling, plan, dispatch, products and combine, us: 128 experts of 4096 x 1280, 8 per token: 1 token 36 / 55, 8 159 / 162, 16 264 / 258, 64 479 / 382; 32 such
    experts, 8 tokens 99 / 98, 64 285 / 138; 64 of 2048 x 1408, 6 per token, 8 tokens 67 / 70, 64 181 / 126; 64 of 7168 x 2048, 8 per token, 1 token 80 / 85, 8 347 / 314."""
    FEW = 8

    def __init__(self, *sizes, **named):
        super().__init__(*sizes, **named)
        q, scale = to_eight(self.w_in.view(self.E * 2, self.I, self.H))     # gate and up rows begin blocks of their own
        self.in8 = q.view(self.E, 2 * self.I, self.H), scale.view(self.E, -1, scale.shape[2])
        self.out8 = to_eight(self.w_out)
        self.w_in, self.w_out = from_eight(q, scale).view_as(self.w_in), from_eight(*self.out8)

    def forward(self, r, y, keep=False):
        N = r.shape[0]
        s, x, logits, idx, w = self.before_experts(r, y)
        if N <= self.FEW and not keep:
            return s, self.few(x, idx, w)
        out = _empty(N, self.H)
        x8, x_scale = to_eight(x)
        L = fusco.Layout(N, self.k, self.E, self.D)
        rows, rows_scale = _empty(L.P, self.H, like=x8), _empty(L.P, x_scale.shape[1], like=x_scale)
        fusco.fusco_plan(L, idx)
        fusco.fusco_dispatch(L, x8, rows, x_aux=x_scale, expert_aux=rows_scale)
        h, out_rows = _empty(L.P, self.I), _empty(L.P, self.H)
        pre = _empty(L.P, 2 * self.I) if keep else None
        fusco.fusco_experts_gated_fp8(L, rows, rows_scale, *self.in8, h, pre=pre)
        h = to_eight(h)
        fusco.fusco_experts_linear_fp8(L, *h, *self.out8, out_rows)
        fusco.fusco_combine(L, out_rows, w, out)
        return (s, out, (r, y, s, x, logits, idx, w, L, (rows, rows_scale), to_eight(pre), h, out_rows)) if keep else (s, out)

    def few(self, x, idx, w):
        out = _empty(*x.shape)
        fusco.fusco_moe_few(x, idx, w, self.in8[0], self.out8[0], out, w_in_scale=self.in8[1], w_out_scale=self.out8[1])
        return out

    def through_experts(self, L, d_rows, rows, pre, h):
        dpre, dw_out = _empty(L.P, 2 * self.I), torch.empty_like(self.w_out)
        fusco.fusco_experts_input_grad(L, d_rows, self.w_out, dpre, pre=pre[0], pre_scale=pre[1])
        fusco.fusco_experts_weight_grad(L, d_rows, h[0], dw_out, x_scale=h[1])
        dx_rows, dw_in = _empty(L.P, self.H), torch.empty_like(self.w_in)
        fusco.fusco_experts_input_grad(L, dpre, self.w_in, dx_rows)
        fusco.fusco_experts_weight_grad(L, dpre, rows[0], dw_in, x_scale=rows[1])
        return dx_rows, dw_in, dw_out

    def plain_experts(self, kept, dout):
        """From the values that were kept, in 64 bits: pre-activations, activations, the block's output; gradients of the router's weights, of x, of w_in and w_out"""
        r, y, s, x, logits, idx, w, L, rows, pre, h, out_rows = kept
        x8, pre8, h8 = (from_eight(*t).double() for t in (rows, pre, h))
        w_in, w_out, w, dout = self.w_in.double(), self.w_out.double(), w.double(), dout.double()
        bounds, slot = L.array("exp_off").tolist(), L.array("pair_slot").long().view_as(idx)
        token = torch.empty(L.P, dtype=torch.long, device="cuda")
        token[slot.flatten()] = torch.arange(idx.numel(), device="cuda") // self.k
        weight = torch.empty(L.P, dtype=torch.float64, device="cuda")
        weight[slot.flatten()] = w.flatten()
        d_rows = weight[:, None] * dout[token]
        act, y8, dx, dw_in, dw_out = torch.zeros_like(h8), torch.zeros_like(d_rows), torch.zeros_like(d_rows), torch.zeros_like(w_in), torch.zeros_like(w_out)
        both = torch.zeros_like(pre8)
        for e in range(self.E):
            rs = slice(bounds[e], bounds[e + 1])
            both[rs] = x8[rs] @ w_in[e].t()
            y8[rs] = h8[rs] @ w_out[e].t()
            g, u = pre8[rs].split(self.I, dim=1)
            q, dh = torch.sigmoid(g), d_rows[rs] @ w_out[e]
            dpre = torch.cat([dh * u * (q + g * q * (1 - q)), dh * g * q], dim=1)
            dx[rs], dw_in[e], dw_out[e] = dpre @ w_in[e], dpre.t() @ x8[rs], d_rows[rs].t() @ h8[rs]
        g, u = both.split(self.I, dim=1)
        sums = lambda v: torch.zeros_like(dout).index_add(0, token, v)
        dw = (y8[slot] * dout[:, None]).sum(dim=2)
        return dict(pre=both, h=g * torch.sigmoid(g) * u, out=sums(weight[:, None] * y8)), dw, sums(dx), dict(w_in=dw_in, w_out=dw_out)


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


def check_eight(N=96, H=256, I=128, E=16, k=4, D=4, keep_groups=2):
    """The same of the block in e4m3, against 64 bits from the values that it kept -> (errors of results and gradients, errors of what is kept in e4m3)."""
    block = EightBlock(H, I, E, k, D, keep_groups)
    gen = torch.Generator(device="cuda").manual_seed(1)
    normal = lambda *s: torch.randn(s, generator=gen, device="cuda")
    r, y, ds, dout = normal(N, H), normal(N, H).bfloat16(), normal(N, H), normal(N, H).bfloat16()
    s, out, kept = block.forward(r, y, keep=True)
    got = dict(block.backward(kept, ds, dout), s=s, out=out)
    results, dw, dx, want = block.plain_experts(kept, dout)
    p = {n: t.detach().double().requires_grad_() for n, t in dict(r=r, y=y, gain=block.gain, gate=block.gate, before=block.before, router=block.router).items()}
    unit = lambda v: v / (v.square().mean(dim=1, keepdim=True) + 1e-6).sqrt()
    want_s = p["r"] + 0.5 * p["gate"] * unit(p["y"]) * p["gain"]
    x = unit(want_s) * p["before"]
    score = torch.sigmoid(x @ p["router"].t()).gather(1, kept[5].long())
    want.update(zip(p, torch.autograd.grad([want_s, x, score / score.sum(dim=1, keepdim=True)], list(p.values()), [ds.double(), dx, dw])))
    want.update(s=want_s.detach(), out=results["out"])
    if N <= 64:   # the layer for a few tokens: rows and activations as they are
        got["few"] = block.few(kept[3], kept[5], kept[6])
        rows = torch.zeros_like(want["out"])
        for e in range(E):
            t, j = (kept[5] == e).nonzero(as_tuple=True)
            g, u = (kept[3][t].double() @ block.w_in[e].double().t()).split(I, dim=1)
            rows.index_add_(0, t, kept[6][t, j].double()[:, None] * ((g * torch.sigmoid(g) * u) @ block.w_out[e].double().t()))
        want["few"] = rows
    far = lambda a, b: float((a.double() - b).norm() / b.norm())
    return {n: far(got[n], want[n]) for n in want}, {n: far(from_eight(*t), v) for n, t, v in (("x", to_eight(kept[3]), kept[3].double()), ("pre", kept[9], results["pre"]), ("h", kept[10], results["h"]))}


def main():
    fusco.load_library()
    torch.cuda.set_device(0)
    far = check()
    print("relative error against 64 bits: " + ", ".join("%s %.1e" % (n, v) for n, v in far.items()))
    assert max(far.values()) < 0.02
    far, eight = check_eight()
    print("in e4m3, against 64 bits from what is kept: " + ", ".join("%s %.1e" % (n, v) for n, v in far.items()) + "; kept " + ", ".join("%s %.1e" % (n, v) for n, v in eight.items()))
    assert max(far.values()) < 0.02 and max(eight.values()) < 2.0 ** -4 + 0.02
    for name, kind in (("bf16", MoEBlock), ("e4m3", EightBlock)):
        block = kind(H=4096, I=1280, E=128, k=8, D=16, keep_groups=8)
        for N in (1, 128, 16384):
            r, y = torch.randn((N, 4096), device="cuda").bfloat16(), torch.randn((N, 4096), device="cuda").bfloat16()
            us = timed(lambda: block.forward(r, y))
            print("%s: forward of %5d tokens: %.1f us" % (name, N, us))
        r, y = torch.randn((8192, 4096), device="cuda"), torch.randn((8192, 4096), device="cuda").bfloat16()
        s, out, kept = block.forward(r, y, keep=True)
        ds, dout = torch.randn_like(s), torch.randn_like(out)
        print("%s: backward of %5d tokens: %.1f us" % (name, 8192, timed(lambda: block.backward(kept, ds, dout), 5)))
        del kept


if __name__ == "__main__":
    main()
