"""Argument checks of the calls for e4m3 without a GPU: bad sizes, types and pointers are refused before anything is launched, and the
ctypes struct lies in memory as the header's does."""
import ctypes
import os
import subprocess

import pytest

from test_block_boundary_host import BUF, ROOT, layout, lib  # noqa: F401


def test_struct_lies_as_in_the_header(tmp_path):
    from paper_2512_22036_amd.binding import _CFp8
    names = [f for f, _ in _CFp8._fields_]
    lines = ["#include <stdio.h>", "#include <stddef.h>", '#include "fusco.h"', "int main(void) {"]
    lines += ['printf("%%zu\\n", offsetof(fusco_fp8, %s));' % f for f in names] + ['printf("%zu\\n", sizeof(fusco_fp8));', "return 0; }"]
    (tmp_path / "a.c").write_text("\n".join(lines))
    subprocess.check_call(["gcc", "-I", os.path.join(ROOT, "include"), "-o", str(tmp_path / "a"), str(tmp_path / "a.c")])
    said = [int(v) for v in subprocess.check_output([str(tmp_path / "a")]).split()]
    assert said == [getattr(_CFp8, f).offset for f in names] + [ctypes.sizeof(_CFp8)]


def fp8(**kw):
    from paper_2512_22036_amd.binding import _CFp8
    return _CFp8(**{**dict(rows=64, columns=256, dtype=0, matrix_rows=0, scale_stride=2), **kw})


@pytest.mark.parametrize("name", ["fusco_to_fp8", "fusco_from_fp8"])
def test_there_and_back(lib, name):  # noqa: F811
    call = lambda f, *a: getattr(lib, name)(ctypes.byref(f), *a)
    for bad in (dict(rows=-1), dict(columns=0), dict(columns=-16), dict(columns=8), dict(columns=24), dict(columns=(1 << 20) + 16), dict(matrix_rows=-1), dict(scale_stride=1), dict(scale_stride=-1),
                dict(scale_stride=65537), dict(matrix_rows=60), dict(matrix_rows=32, scale_stride=3), dict(rows=1 << 31), dict(rows=1 << 30, columns=512, scale_stride=4),
                dict(rows=1 << 62), dict(rows=1 << 29, columns=16, scale_stride=1), dict(rows=1 << 23, matrix_rows=1, columns=16, scale_stride=1),
                dict(rows=1 << 27, matrix_rows=1 << 7, columns=2048, scale_stride=16)):   # more threads than a launch has
        assert call(fp8(**bad), BUF, BUF, BUF, None) == -1, bad
    for bad in (dict(dtype=2), dict(dtype=-1)):
        assert call(fp8(**bad), BUF, BUF, BUF, None) == -3, bad
    for i in range(3):
        assert call(fp8(), *[None if j == i else BUF for j in range(3)], None) == -1
        assert call(fp8(), *[BUF + 8 if j == i else BUF for j in range(3)], None) == -1
    assert getattr(lib, name)(None, BUF, BUF, BUF, None) == -1
    assert call(fp8(rows=0), None, None, None, None) == 0
    assert call(fp8(rows=0, columns=8), None, None, None, None) == -1


@pytest.mark.parametrize("name", ["fusco_to_fp8", "fusco_from_fp8"])
def test_whole_workgroups_of_a_launch(lib, name):  # noqa: F811
    """A workgroup has 32 blocks of rows and 256 threads: with 2^29 - 31 blocks the launch would come to 2^32 threads."""
    for size in (dict(rows=(1 << 29) - 1, columns=16, scale_stride=1), dict(rows=(1 << 29) - 31, columns=16, scale_stride=1), dict(rows=(1 << 28) - 1, columns=256, scale_stride=2),
                 dict(rows=(1 << 29) - 16, columns=16, scale_stride=1, matrix_rows=(1 << 29) - 16)):
        assert getattr(lib, name)(ctypes.byref(fp8(**size)), BUF, BUF, BUF, None) == -1, size


def test_products(lib):  # noqa: F811
    L, empty = layout(lib), layout(lib, N=0)
    g = lambda *a: lib.fusco_experts_gated_fp8(ctypes.byref(L), *a)
    good = [BUF, BUF, 1, BUF, BUF, BUF, None, 64, 64, None]
    for i in (0, 1, 3, 4, 5):
        assert g(*[None if j == i else v for j, v in enumerate(good)]) == -1, i
        assert g(*[BUF + 4 if j == i else v for j, v in enumerate(good)]) == -1, i
    assert g(*[BUF + 2 if j == 6 else v for j, v in enumerate(good)]) == -1
    for H, I, stride in ((0, 64, 1), (64, 0, 1), (24, 64, 1), (64, 4, 1), (-16, 64, 1), ((1 << 20) + 16, 64, 8193), (64, 1 << 19, 1), (1 << 16, 1 << 15, 512), (256, 64, 1), (64, 64, 65537)):
        assert g(BUF, BUF, stride, BUF, BUF, BUF, None, H, I, None) == -1, (H, I, stride)
    assert lib.fusco_experts_gated_fp8(None, *good) == -1
    assert lib.fusco_experts_gated_fp8(ctypes.byref(empty), None, None, 1, None, None, None, None, 64, 64, None) == 0
    assert lib.fusco_experts_gated_fp8(ctypes.byref(empty), None, None, 1, None, None, None, None, 72, 64, None) == -1
    y = lambda *a: lib.fusco_experts_linear_fp8(ctypes.byref(L), *a)
    good = [BUF, BUF, 1, BUF, BUF, BUF, 64, 64, None]
    for i in (0, 1, 3, 4, 5):
        assert y(*[None if j == i else v for j, v in enumerate(good)]) == -1, i
    for C, M, stride in ((8, 64, 1), (64, 6, 1), (0, 64, 1), (144, 64, 1), (1 << 20, 1 << 11, 8192)):
        assert y(BUF, BUF, stride, BUF, BUF, BUF, C, M, None) == -1, (C, M, stride)
    assert lib.fusco_experts_linear_fp8(ctypes.byref(empty), None, None, 1, None, None, None, 64, 64, None) == 0


def test_gradients(lib):  # noqa: F811
    L, empty = layout(lib), layout(lib, N=0)
    i = lambda *a: lib.fusco_experts_input_grad_fp8(ctypes.byref(L), *a)
    good = [BUF, BUF, BUF, BUF, BUF, 1, 64, 64, None]
    for n in range(5):
        assert i(*[None if j == n else v for j, v in enumerate(good)]) == -1, n
        assert i(*[BUF + 8 if j == n else v for j, v in enumerate(good)]) == -1, n
    for stride, M, C in ((1, 64, 72), (1, 64, 128), (1, 4, 64), (0, 64, 64), (8192, 64, 1 << 19), (65537, 64, 64)):
        assert i(BUF, BUF, BUF, BUF, BUF, stride, M, C, None) == -1, (stride, M, C)
    assert lib.fusco_experts_input_grad_fp8(ctypes.byref(empty), None, None, None, None, None, 1, 64, 64, None) == 0
    w = lambda *a: lib.fusco_experts_weight_grad_fp8(ctypes.byref(L), *a)
    good = [BUF, BUF, BUF, 1, BUF, 0, 64, 64, None]
    for n in (0, 1, 2, 4):
        assert w(*[None if j == n else v for j, v in enumerate(good)]) == -1, n
        assert w(*[BUF + 8 if j == n else v for j, v in enumerate(good)]) == -1, n
    assert w(BUF, BUF, BUF, 1, BUF, 2, 64, 64, None) == -3
    for stride, M, C in ((1, 64, 72), (1, 64, 144), (1, 4, 64), (1, 64, 0), (4096, 64, (1 << 19) + 16)):
        assert w(BUF, BUF, BUF, stride, BUF, 0, M, C, None) == -1, (stride, M, C)
    assert lib.fusco_experts_weight_grad_fp8(ctypes.byref(empty), None, None, None, 1, None, 0, 64, 64, None) == -1   # dw is written even then


def few(**kw):
    from paper_2512_22036_amd.binding import _CFew
    return _CFew(**{**dict(N=4, E=8, k=2, H=64, I=32, weight_dtype=0, out_dtype=0), **kw})


def test_few_struct_lies_as_in_the_header(tmp_path):
    from paper_2512_22036_amd.binding import _CFew
    names = [f for f, _ in _CFew._fields_]
    lines = ["#include <stdio.h>", "#include <stddef.h>", '#include "fusco.h"', "int main(void) {"]
    lines += ['printf("%%zu\\n", offsetof(fusco_few, %s));' % f for f in names] + ['printf("%zu\\n", sizeof(fusco_few));', "return 0; }"]
    (tmp_path / "a.c").write_text("\n".join(lines))
    subprocess.check_call(["gcc", "-I", os.path.join(ROOT, "include"), "-o", str(tmp_path / "a"), str(tmp_path / "a.c")])
    said = [int(v) for v in subprocess.check_output([str(tmp_path / "a")]).split()]
    assert said == [getattr(_CFew, f).offset for f in names] + [ctypes.sizeof(_CFew)]


def test_few(lib):  # noqa: F811
    need = lib.fusco_moe_few_scratch_bytes(4, 2, 32)
    assert need >= 4 * 2 * 32 * 4 and lib.fusco_moe_few_scratch_bytes(65, 2, 32) == lib.fusco_moe_few_scratch_bytes(-1, 2, 32) == lib.fusco_moe_few_scratch_bytes(4, 65, 32) == 0
    call = lambda f, *a: lib.fusco_moe_few(ctypes.byref(f), *a)
    good = [BUF, BUF, BUF, BUF, None, BUF, None, BUF, BUF, need, None]
    for bad in (dict(N=-1), dict(N=65), dict(E=0), dict(E=1025), dict(k=0), dict(k=65), dict(H=0), dict(H=12), dict(I=4), dict(I=-8), dict(H=1 << 20), dict(H=1 << 15, I=1 << 15), dict(N=64, k=64, E=256, H=8, I=1 << 19)):
        assert call(few(**bad), *good[:9], 1 << 40, None) == -1, bad
    for bad in (dict(weight_dtype=1), dict(weight_dtype=3), dict(out_dtype=2), dict(out_dtype=-1)):
        assert call(few(**bad), *good) == -3, bad
    for i in (0, 1, 2, 3, 5, 7, 8):
        assert call(few(), *[None if j == i else v for j, v in enumerate(good)]) == -1, i
        assert call(few(), *[BUF + 8 if j == i else v for j, v in enumerate(good)]) == -1, i
    assert call(few(), *good[:9], need - 1, None) == -2
    eight = [BUF, BUF, BUF, BUF, BUF, BUF, BUF, BUF, BUF, need, None]
    for i in (4, 6):
        assert call(few(weight_dtype=2), *[None if j == i else v for j, v in enumerate(eight)]) == -1, i
    for bad in (dict(H=72), dict(I=40)):
        assert call(few(weight_dtype=2, **bad), *eight[:9], 1 << 20, None) == -1, bad
    assert lib.fusco_moe_few(None, *good) == -1
    assert call(few(N=0), None, None, None, None, None, None, None, None, None, 0, None) == 0
