"""The products on e4m3 and the gradients from kept rows where workgroups take several tiles one after the other, each of several turns through LDS: tiles of
64, 128 and 256 rows of every product, with ragged ends of rows, outputs and sums.  What is compared, and how closely, is as for the small sizes."""
import pytest
import torch

import test_gpu_fp8 as fp8
import test_gpu_fp8_kept as kept
from test_gpu_experts import bf16, fusco, make
from test_gpu_experts_many_tiles import SIZES, WORKGROUPS, holds

pytestmark = pytest.mark.gpu

# products summed per output: a part of a block (one turn), a block and a bit, several turns with and without a ragged end; and, for tiles of 64 rows, turns of three stages, whole and filled up
SUMS = [(80, "normal"), (144, "skewed"), (912, "skewed"), (912, "invalid"), (1024, "normal"), (304, "normal"), (1040, "invalid"), (1408, "skewed"), (2896, "normal")]


@pytest.mark.parametrize("total,routing", SUMS)
@pytest.mark.parametrize("N,k,E,outputs,rows", SIZES)
def test_linear(N, k, E, outputs, rows, total, routing):
    holds(fusco().PRODUCT_LINEAR, N, k, E, outputs, total // 2, rows)
    fp8.test_linear(N, k, E, total, outputs, routing, True)


@pytest.mark.parametrize("keep_pre", [False, True])
@pytest.mark.parametrize("total,routing", SUMS)
@pytest.mark.parametrize("N,k,E,outputs,rows", [(640, 4, 160, 264, 64), (450, 8, 160, 136, 64), (1600, 4, 64, 520, 128), (3100, 2, 64, 1032, 128), (1300, 5, 40, 1032, 256), (4100, 2, 8, 1288, 256)])
def test_gated(N, k, E, outputs, rows, total, routing, keep_pre):
    holds(fusco().PRODUCT_GATED, N, k, E, outputs, total // 2, rows)
    fp8.test_gated(N, k, E, total, outputs, routing, keep_pre, True)


@pytest.mark.parametrize("any_scale", [False, True])
@pytest.mark.parametrize("total,routing", [(72, "normal"), (456, "skewed"), (456, "invalid"), (1024, "normal")])
@pytest.mark.parametrize("N,k,E,outputs,rows", [(640, 4, 160, 528, 64), (450, 8, 160, 272, 64), (1600, 4, 64, 1040, 128), (3100, 2, 64, 1040, 128), (1300, 5, 40, 2064, 256), (4100, 2, 8, 2320, 256)])
def test_input_grad(N, k, E, outputs, rows, total, routing, any_scale):
    holds(fusco().PRODUCT_INPUT_GRAD_ACTIVATION, N, k, E, outputs, total, rows)
    kept.test_input_grad(N, k, E, outputs, total, routing, any_scale)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("N,k,E,C,M,routing", [(1300, 5, 40, 784, 520, "normal"), (4600, 4, 30, 784, 776, "skewed"), (1700, 3, 30, 528, 776, "invalid"), (9000, 2, 6, 2064, 1544, "normal")])
def test_weight_grad(N, k, E, C, M, routing, dtype):
    assert E * ((C + 255) // 256) * ((M + 255) // 256) > WORKGROUPS
    kept.test_weight_grad(N, k, E, C, M, routing, dtype, True)


@pytest.mark.parametrize("routing", ["normal", "skewed"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("N,k,E,C,M", [(8192, 4, 64, 2048, 2816), (2000, 2, 16, 2048, 4096)])
def test_weight_grad_same_as_from_bf16(N, k, E, C, M, dtype, routing):
    """Large tensors that no cache holds, kept rows against the bf16 rows of the same values, bit by bit, the first call included."""
    f = fusco()
    L, gen, bounds = make(N, k, E, 41, routing)
    dy = bf16(gen, L.P, M)
    x, scale = kept.kept(gen, L.P, C, False)
    wide = torch.empty((L.P, C), dtype=torch.bfloat16, device="cuda")
    f.fusco_from_fp8(x, scale, wide)
    want, got = torch.empty((E, M, C), dtype=dtype, device="cuda"), torch.empty((E, M, C), dtype=dtype, device="cuda")
    f.fusco_experts_weight_grad(L, dy, wide, want)
    for _ in range(3):
        torch.empty(1 << 29, dtype=torch.uint8, device="cuda").zero_()     # past what the caches hold
        got.fill_(7.0)
        f.fusco_experts_weight_grad(L, dy, x, got, x_scale=scale)
        assert torch.equal(got, want)


@pytest.mark.parametrize("N,rows", [(10000, 128), (20000, 256)])
def test_an_experts_values_stay_its_own(N, rows):
    f = fusco()
    L = f.Layout(N, 2, 4, 1)
    assert f.fusco_probe_experts_tile_rows(L, f.PRODUCT_LINEAR, 136, 104) == rows
    fp8.test_an_experts_values_stay_its_own(N)


@pytest.mark.parametrize("C", [128, 384, 640])     # an odd number of stages, so that one of a tile's is filled up
@pytest.mark.parametrize("N,E", [(10000, 16), (20000, 8)])
def test_scales_of_a_tile_stay_its_own(N, E, C):
    """Every other expert's weight scales are NaN: workgroups go from such tiles to others and back."""
    f = fusco()
    L, gen, bounds = make(N, 2, E, 14, "normal")
    M = 520
    assert f.fusco_probe_experts_tile_rows(L, f.PRODUCT_LINEAR, M, C) == 256
    x, xs = fp8.eight(gen, L.P, C, scales=(L.P, fp8.blocks(C)), std=1.0)
    w, ws = fp8.eight(gen, L.E, M, C, scales=(L.E, fp8.blocks(M), fp8.blocks(C)), std=1.0)
    ws[::2] = float("nan")
    y = torch.empty((L.P, M), dtype=torch.bfloat16, device="cuda")
    for _ in range(3):
        f.fusco_experts_linear_fp8(L, x, xs, w, ws, y)
        for e in range(L.E):
            part = y[bounds[e]:bounds[e + 1]]
            assert bool(part.isnan().all() if e % 2 == 0 else part.isfinite().all()), e


@pytest.mark.parametrize("N,k,E,I,M,routing", [(2400, 2, 120, 256, 1040, "skewed"), (300, 2, 16, 528, 1040, "normal"), (64, 1, 60, 272, 72, "invalid"), (9, 2, 8, 2048, 64, "normal"), (5808, 1, 88, 256, 336, "round")])
def test_input_grad_of_few_tiles(monkeypatch, N, k, E, I, M, routing):
    """Tiles of 128 outputs, up to as many as there are workgroups by the mean of the rows; with 66 rows for every expert there are more."""
    if routing == "round":
        f, gen = fusco(), torch.Generator(device="cuda").manual_seed(16)
        L = f.Layout(N, k, E, 1)
        f.fusco_plan(L, torch.arange(N, device="cuda").remainder(E).int().view(N, 1))
        bounds = L.array("exp_off").tolist()
        assert sum((b - a + 63) // 64 for a, b in zip(bounds, bounds[1:])) * 2 > WORKGROUPS
        monkeypatch.setattr(kept, "make", lambda *a: (L, gen, bounds))
    assert max(E, N * k / 64 + 0.4 * E) * ((I + 127) // 128) <= WORKGROUPS
    kept.test_input_grad(N, k, E, I, M, routing, True)
