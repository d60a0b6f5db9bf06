"""The operators on e4m3 with tensors of more than 2^32 bytes: rows at both ends against the same rows in small tensors, bit by bit.  Factors are whole numbers and halves
with scales of 1, so that every sum is exact in fp32 and its order does not count; the rows between are zeros."""
import pytest
import torch

import test_gpu_fp8 as fp8
from test_gpu_experts import bf16, fusco

pytestmark = pytest.mark.gpu
FP8 = torch.float8_e4m3fn
ROWS, COLUMNS, ENDS = 280_000, 16384, 300      # 4.6e9 bytes of e4m3


def exact(gen, *shape):
    return fp8.eight(gen, *shape, scales=(1,), std=1.0, whole=True)[0]


def ends(t, rows):
    """A large tensor of zeros with t's first half of rows at its beginning and the second at its end."""
    large = torch.zeros((rows,) + tuple(t.shape[1:]), dtype=torch.uint8, device="cuda").view(t.dtype) if t.dtype == FP8 else torch.zeros((rows,) + tuple(t.shape[1:]), dtype=t.dtype, device="cuda")
    large.view(torch.uint8)[:ENDS], large.view(torch.uint8)[-ENDS:] = t.view(torch.uint8)[:ENDS], t.view(torch.uint8)[-ENDS:]
    return large


def layouts():
    """Half of the rows go to the first expert, half to the second; a row per token, in order."""
    f = fusco()
    pair = []
    for rows in (ROWS, 2 * ENDS):
        L = f.Layout(rows, 1, 2, 1)
        f.fusco_plan(L, (torch.arange(rows, device="cuda") >= rows // 2).int().view(rows, 1))
        pair.append(L)
    return pair


def same_ends(large, small, zeros_between=True):
    assert torch.equal(large[:ENDS], small[:ENDS]) and torch.equal(large[-ENDS:], small[-ENDS:])
    if zeros_between:
        for part in large[ENDS:-ENDS].split(20_000):
            assert not bool(part.float().any())


@pytest.fixture()
def gen():
    torch.cuda.empty_cache()
    yield torch.Generator(device="cuda").manual_seed(51)
    torch.cuda.empty_cache()


def test_there_and_back(gen):
    f = fusco()
    x = bf16(gen, 2 * ENDS, COLUMNS)
    large = ends(x, ROWS)
    out = []
    for t in (large, x):
        q, scale, back = torch.empty(t.shape, dtype=torch.uint8, device="cuda").fill_(1).view(FP8), torch.zeros((t.shape[0], COLUMNS // 128), device="cuda"), torch.ones_like(t)
        f.fusco_to_fp8(t, q, scale)
        f.fusco_from_fp8(q, scale, back)
        out.append((q.view(torch.uint8), scale, back))
    for a, b in zip(*out):
        same_ends(a, b, zeros_between=a.dtype != torch.float32)
    assert bool((out[0][1][ENDS:-ENDS] == 1).all())


def test_products(gen):
    f = fusco()
    pair = layouts()
    x, w = exact(gen, 2 * ENDS, COLUMNS), exact(gen, 2, 32, COLUMNS)
    scales = torch.ones((2, 2, COLUMNS // 128), device="cuda")
    out = []
    for L, rows in zip(pair, (ends(x, ROWS), x)):
        y, h, pre = (torch.ones((L.P, n), dtype=torch.bfloat16, device="cuda") for n in (32, 16, 32))
        row_scale = torch.ones((L.P, COLUMNS // 128), device="cuda")
        f.fusco_experts_linear_fp8(L, rows, row_scale, w, scales[:, :1].contiguous(), y)
        f.fusco_experts_gated_fp8(L, rows, row_scale, w, scales, h, pre)
        out.append((y, h, pre))
    for a, b in zip(*out):
        same_ends(a, b)


def test_wide_results(gen):
    """Results past 2^32 bytes, from short sums."""
    f = fusco()
    pair = layouts()
    x, w = exact(gen, 2 * ENDS, 128), exact(gen, 2, COLUMNS, 128)
    out = []
    for L, rows in zip(pair, (ends(x, ROWS), x)):
        y, h, pre = (torch.ones((L.P, n), dtype=torch.bfloat16, device="cuda") for n in (COLUMNS, COLUMNS // 2, COLUMNS))
        row_scale = torch.ones((L.P, 1), device="cuda")
        f.fusco_experts_linear_fp8(L, rows, row_scale, w, torch.ones((2, COLUMNS // 128, 1), device="cuda"), y)
        f.fusco_experts_gated_fp8(L, rows, row_scale, w, torch.ones((2, COLUMNS // 128, 1), device="cuda"), h, pre)
        out.append((y, h, pre))
    for a, b in zip(*out):
        same_ends(a, b)


def test_kept(gen):
    f = fusco()
    pair = layouts()
    x, dy, w = exact(gen, 2 * ENDS, COLUMNS), exact(gen, 2 * ENDS, 16).float().bfloat16(), exact(gen, 2, 16, COLUMNS // 2).float().bfloat16()
    out = []
    for L, rows, grads in zip(pair, (ends(x, ROWS), x), (ends(dy, ROWS), dy)):
        scale = torch.ones((L.P, COLUMNS // 128), device="cuda")
        dw, dpre = torch.ones((2, 16, COLUMNS), device="cuda"), torch.ones((L.P, COLUMNS), dtype=torch.bfloat16, device="cuda")
        f.fusco_experts_weight_grad(L, grads, rows, dw, x_scale=scale)
        f.fusco_experts_input_grad(L, grads, w, dpre, pre=rows, pre_scale=scale)
        out.append((dw, dpre))
    assert torch.equal(out[0][0], out[1][0])
    same_ends(out[0][1], out[1][1])


@pytest.mark.parametrize("eights", [True, False])
def test_far_weights(gen, eights):
    """The last of many experts, past 2^32 bytes of weights, as if it were the only one."""
    f = fusco()
    E, H, I, N = 600, 2048, 2048, 24
    type_ = FP8 if eights else torch.bfloat16
    x = exact(gen, N, H).float().bfloat16()
    w_in, w_out = exact(gen, 1, 2 * I, H).float().to(type_), torch.eye(H, I, device="cuda").view(1, H, I).to(type_)   # an output is a unit's h: nothing to add up
    out = []
    for experts in (E, 1):
        wide_in, wide_out = torch.zeros((experts, 2 * I, H), dtype=torch.uint8 if eights else type_, device="cuda"), torch.zeros((experts, H, I), dtype=torch.uint8 if eights else type_, device="cuda")
        assert experts == 1 or wide_out.numel() * wide_out.element_size() > 2 * 10 ** 9 and wide_in.numel() * wide_in.element_size() > 2 ** 32
        wide_in, wide_out = wide_in.view(type_), wide_out.view(type_)
        wide_in.view(torch.uint8)[-1], wide_out.view(torch.uint8)[-1] = w_in.view(torch.uint8)[0], w_out.view(torch.uint8)[0]
        chosen, weight = torch.full((N, 1), experts - 1, dtype=torch.int32, device="cuda"), torch.ones((N, 1), device="cuda")
        scales = [torch.zeros((experts, rows, 16), device="cuda") for rows in (32, 16)]
        for s in scales:
            s[-1] = 1.0
        few, got = torch.zeros((N, H), device="cuda"), []
        f.fusco_moe_few(x, chosen, weight, wide_in, wide_out, few, **(dict(w_in_scale=scales[0], w_out_scale=scales[1]) if eights else {}))
        if eights:
            L = f.Layout(N, 1, experts, 1)
            f.fusco_plan(L, chosen)
            h, y = torch.zeros((N, I), dtype=torch.bfloat16, device="cuda"), torch.zeros((N, H), dtype=torch.bfloat16, device="cuda")
            f.fusco_experts_gated_fp8(L, x.float().to(FP8), torch.ones((N, 16), device="cuda"), wide_in, scales[0], h)
            f.fusco_experts_linear_fp8(L, x.float().to(FP8), torch.ones((N, 16), device="cuda"), wide_out, scales[1], y)
            got = [h, y]
        out.append([few] + got)
    assert bool(out[0][0].any())
    for a, b in zip(*out):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("E,M,C", [(300, 520, 1040), (40, 1408, 2064)])     # e4m3 of more and of less than half of what the caches hold
def test_matrices_by_one(gen, E, M, C, dtype):
    f = fusco()
    x = torch.randn((E, M, C), generator=gen, device="cuda").mul_(torch.rand((E, 1, 1), generator=gen, device="cuda")).to(dtype)
    shape = (E, fp8.blocks(M), fp8.blocks(C))
    q, scale, one, its = torch.zeros((E, M, C), dtype=torch.uint8, device="cuda"), torch.zeros(shape, device="cuda"), torch.zeros((1, M, C), dtype=torch.uint8, device="cuda"), torch.zeros((1,) + shape[1:], device="cuda")
    f.fusco_to_fp8(x, q.view(FP8), scale)
    for e in range(E):
        f.fusco_to_fp8(x[e:e + 1], one.view(FP8), its)
        assert torch.equal(q[e:e + 1], one) and torch.equal(scale[e:e + 1], its)
