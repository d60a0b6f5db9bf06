"""How many of an expert's rows a tile of the experts' products holds, as the library's host-only query tells it from the sizes.  No GPU is needed."""
import ctypes
import os

import pytest


@pytest.fixture(scope="module")
def rows():
    from paper_2512_22036_amd import binding
    if not os.path.exists(binding.library_path()):
        from paper_2512_22036_amd.build import build_library
        build_library()
    lib = binding.load_library()

    def ask(N, k, E, which, outputs, total):
        L = binding._CLayout()
        assert lib.fusco_layout_bind(ctypes.byref(L), N, k, E, 1, 0x10000000, lib.fusco_layout_bytes(N, k, E, 1)) == 0
        return lib.fusco_probe_experts_tile_rows(ctypes.byref(L), which, outputs, total)

    return ask


GATED, LINEAR, INPUT_GRAD, ACTIVATION = 0, 1, 2, 3


def test_constants():
    import paper_2512_22036_amd as f
    assert (f.PRODUCT_GATED, f.PRODUCT_LINEAR, f.PRODUCT_INPUT_GRAD, f.PRODUCT_INPUT_GRAD_ACTIVATION) == (GATED, LINEAR, INPUT_GRAD, ACTIVATION)


def test_few_rows(rows):
    for which in (GATED, LINEAR):
        assert [rows(N, 8, 128, which, 1280, 4096) for N in (1, 32, 127)] == [16, 16, 16]
        assert rows(128, 8, 128, which, 1280, 4096) == 64            # eight rows per expert
    assert rows(1, 8, 128, INPUT_GRAD, 1280, 4096) == 64             # the gradients have no kernel of their own for few rows


def test_few_rows_of_very_many_outputs(rows):
    """A launch has fewer than 2^32 threads: what would exceed that with a workgroup per 16 rows and 32 outputs goes by tiles of more rows."""
    assert rows(1000, 8, 1024, LINEAR, 32768, 8) == 16
    assert rows(1000, 8, 1024, LINEAR, 352512, 8) == 64            # 1524 tiles of rows, 11016 blocks of outputs, 256 threads: 4.30e9
    assert rows(1000, 8, 1024, LINEAR, 352000, 8) == 16            # 4.29e9
    assert rows(1000, 8, 1024, GATED, 176256, 8) == 64 and rows(1000, 8, 1024, GATED, 176000, 8) == 16
    assert rows(127, 8, 128, LINEAR, 1 << 18, 2048) == 16


def test_rounds_of_tiles(rows):
    """The sizes that the rule's comment gives measured times for: the fastest height, or one within 15 us of it."""
    assert [rows(N, 8, 128, GATED, 1280, 4096) for N in (128, 1024, 2048, 16384)] == [64, 128, 256, 256]
    assert rows(230 * 2, 8, 16, GATED, 1280, 4096) == 256
    assert rows(230 * 2, 8, 16, ACTIVATION, 1280, 4096) == 128
    assert rows(128 * 2, 8, 16, ACTIVATION, 1408, 2048) == 64


def test_bad_sizes(rows):
    for which, outputs, total in ((-1, 64, 64), (4, 64, 64), (GATED, 0, 64), (GATED, 64, 12), (GATED, 1 << 19, 8), (ACTIVATION, 1 << 19, 8), (LINEAR, (1 << 19) + 8, 8), (LINEAR, 1 << 16, 1 << 15)):
        assert rows(16, 2, 8, which, outputs, total) == -1, (which, outputs, total)
