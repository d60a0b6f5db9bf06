"""The experts' products where workgroups take several tiles one after the other, each of several turns through LDS: tiles of 64, 128 and 256 rows of
every product, with ragged ends of rows, outputs and sums.  What is compared, and how closely, is as for the small sizes."""
import pytest
import test_gpu_experts as small

pytestmark = pytest.mark.gpu

WORKGROUPS = 256

# N, k, E, outputs per row, rows per tile: more tiles than workgroups
SIZES = [(640, 4, 160, 520, 64), (450, 8, 160, 264, 64), (1600, 4, 64, 1032, 128), (3100, 2, 64, 1032, 128), (1300, 5, 40, 2056, 256), (4100, 2, 8, 2312, 256)]
# products summed per output: two stages and a bit (one turn), several turns with and without a ragged end
SUMS = [(72, "normal"), (456, "skewed"), (456, "invalid"), (1024, "normal")]


def holds(which, N, k, E, outputs, total, rows):
    f = small.fusco()
    units = 128 if which == f.PRODUCT_GATED else 256
    assert max(E, N * k // rows) * ((outputs + units - 1) // units) > WORKGROUPS
    assert f.fusco_probe_experts_tile_rows(f.Layout(N, k, E, 1), which, outputs, total) == rows


@pytest.mark.parametrize("total,routing", SUMS)
@pytest.mark.parametrize("N,k,E,outputs,rows", SIZES)
def test_linear(N, k, E, outputs, rows, total, routing):
    holds(small.fusco().PRODUCT_LINEAR, N, k, E, outputs, total, rows)
    small.test_linear(N, k, E, total, outputs, routing)


@pytest.mark.parametrize("keep_pre", [False, True])
@pytest.mark.parametrize("total,routing", SUMS)
@pytest.mark.parametrize("N,k,E,outputs,rows", [(640, 4, 160, 264, 64), (450, 8, 160, 136, 64), (1600, 4, 64, 520, 128), (3100, 2, 64, 1032, 128), (1300, 5, 40, 1032, 256), (4100, 2, 8, 1288, 256)])
def test_gated(N, k, E, outputs, rows, total, routing, keep_pre):
    holds(small.fusco().PRODUCT_GATED, N, k, E, outputs, total, rows)
    small.test_gated(N, k, E, total, outputs, routing, keep_pre)


@pytest.mark.parametrize("total,routing", SUMS)
@pytest.mark.parametrize("N,k,E,outputs,rows", SIZES)
def test_input_grad(N, k, E, outputs, rows, total, routing):
    holds(small.fusco().PRODUCT_INPUT_GRAD, N, k, E, outputs, total, rows)
    small.test_input_grad(N, k, E, outputs, total, routing)


@pytest.mark.parametrize("total,routing", SUMS)
@pytest.mark.parametrize("N,k,E,outputs,rows", SIZES)
def test_input_grad_through_the_activation(N, k, E, outputs, rows, total, routing):
    holds(small.fusco().PRODUCT_INPUT_GRAD_ACTIVATION, N, k, E, outputs, total, rows)
    small.test_input_grad_through_the_activation(N, k, E, outputs, total, routing)


@pytest.mark.parametrize("dtype", [small.torch.bfloat16, small.torch.float32])
@pytest.mark.parametrize("N,k,E,C,M,routing", [(1300, 5, 40, 776, 520, "normal"), (4600, 4, 30, 776, 776, "skewed"), (1700, 3, 30, 520, 776, "invalid"), (9000, 2, 6, 2056, 1544, "normal")])
def test_weight_grad(N, k, E, C, M, routing, dtype):
    assert E * ((C + 255) // 256) * ((M + 255) // 256) > WORKGROUPS
    small.test_weight_grad(N, k, E, C, M, routing, dtype)


@pytest.mark.parametrize("N,rows", [(10000, 128), (20000, 256)])
def test_an_experts_values_stay_its_own(N, rows):
    f = small.fusco()
    L = f.Layout(N, 2, 4, 1)
    assert f.fusco_probe_experts_tile_rows(L, f.PRODUCT_LINEAR, 136, 200) == f.fusco_probe_experts_tile_rows(L, f.PRODUCT_INPUT_GRAD, 200, 136) == rows
    small.test_an_experts_values_stay_its_own(N)


def test_few_rows_of_very_many_outputs():
    """7.8 rows per expert, 352512 outputs of 8 products each: more threads than one launch of the kernel for few rows may have."""
    f = small.fusco()
    torch = small.torch
    N, k, E, C, M = 1000, 8, 1024, 8, 352512
    L, gen, bounds = small.make(N, k, E, 12, "normal")
    assert f.fusco_probe_experts_tile_rows(L, f.PRODUCT_LINEAR, M, C) == 64
    x, w = small.bf16(gen, L.P, C), torch.empty((E, M, C), dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    y = torch.full((L.P, M), 7.0, dtype=torch.bfloat16, device="cuda")
    f.fusco_experts_linear(L, x, w, y)
    for e, rows in small.segments(bounds, x):
        if e % 64 in (0, 63):
            want, err = small.product(x[rows], w[e])
            small.within(y[rows], want, err + small.BF16 * (want.abs() + err) + small.TINY)
    assert not bool((y[:, ::4099] == 7.0).all(dim=1).any())
