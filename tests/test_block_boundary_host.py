"""Argument checks of the operators around the shuffle, without a GPU: bad sizes, types and pointers are refused before anything is
launched, and the ctypes structs lie in memory as the header's do."""
import ctypes
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
BUF = 0x20000000   # never dereferenced


@pytest.fixture(scope="module")
def lib():
    from paper_2512_22036_amd import binding
    if not os.path.exists(binding.library_path()):
        from paper_2512_22036_amd.build import build_library
        build_library()
    return binding.load_library()


def layout(lib, N=64, k=2, E=8, D=4):
    from paper_2512_22036_amd.binding import _CLayout
    L = _CLayout()
    assert lib.fusco_layout_bind(ctypes.byref(L), N, k, E, D, 0x10000000, lib.fusco_layout_bytes(N, k, E, D)) == 0
    return L


def test_structs_lie_as_in_the_header(tmp_path):
    from paper_2512_22036_amd.binding import _CNorm, _CRouter
    lines = ["#include <stdio.h>", "#include <stddef.h>", '#include "fusco.h"', "int main(void) {"]
    for name, struct in (("fusco_router", _CRouter), ("fusco_norm", _CNorm)):
        lines += ['printf("%%zu\\n", offsetof(%s, %s));' % (name, f) for f, _ in struct._fields_] + ['printf("%%zu\\n", sizeof(%s));' % name]
    (tmp_path / "a.c").write_text("\n".join(lines + ["return 0; }"]))
    subprocess.check_call(["gcc", "-I", os.path.join(ROOT, "include"), "-o", str(tmp_path / "a"), str(tmp_path / "a.c")])
    said = [int(v) for v in subprocess.check_output([str(tmp_path / "a")]).split()]
    want = []
    for struct in (_CRouter, _CNorm):
        want += [getattr(struct, f).offset for f, _ in struct._fields_] + [ctypes.sizeof(struct)]
    assert said == want


def test_experts(lib):
    L, empty = layout(lib), layout(lib, N=0)
    g = lambda *a: lib.fusco_experts_gated(ctypes.byref(L), *a)
    assert g(None, BUF, BUF, None, 64, 64, None) == -1
    assert g(BUF, None, BUF, None, 64, 64, None) == -1
    assert g(BUF, BUF, None, None, 64, 64, None) == -1
    assert g(BUF + 8, BUF, BUF, None, 64, 64, None) == -1
    assert g(BUF, BUF, BUF, BUF + 2, 64, 64, None) == -1
    for H, I in ((0, 64), (64, 0), (12, 64), (64, 4), (-8, 64), ((1 << 19) + 8, 64), (64, 1 << 19), (1 << 15, 1 << 15)):
        assert g(BUF, BUF, BUF, None, H, I, None) == -1, (H, I)      # row sizes; the last: an expert's weights are 4 GiB
    assert lib.fusco_experts_gated(None, BUF, BUF, BUF, None, 64, 64, None) == -1
    assert lib.fusco_experts_gated(ctypes.byref(empty), None, None, None, None, 64, 64, None) == 0
    assert lib.fusco_experts_gated(ctypes.byref(empty), None, None, None, None, 60, 64, None) == -1
    for call in (lib.fusco_experts_linear, ):
        assert call(ctypes.byref(L), BUF, BUF, None, 64, 64, None) == -1
        assert call(ctypes.byref(L), BUF, BUF, BUF, 6, 64, None) == -1
        assert call(ctypes.byref(empty), None, None, None, 64, 64, None) == 0
    i = lambda *a: lib.fusco_experts_input_grad(ctypes.byref(L), *a)
    assert i(BUF, BUF, None, None, 64, 64, None) == -1
    assert i(BUF, BUF, BUF, BUF + 4, 64, 64, None) == -1
    assert i(BUF, BUF, BUF, BUF, 64, 1 << 19, None) == -1            # rows of both factors are too long
    w = lambda *a: lib.fusco_experts_weight_grad(ctypes.byref(L), *a)
    assert w(BUF, BUF, BUF, 2, 64, 64, None) == -3
    assert w(BUF, BUF, None, 0, 64, 64, None) == -1
    assert w(None, BUF, BUF, 0, 64, 64, None) == -1
    assert w(BUF, BUF, BUF, 0, 64, 65, None) == -1
    assert lib.fusco_experts_weight_grad(ctypes.byref(empty), None, None, None, 0, 64, 64, None) == -1   # dw is written even then


def router(**kw):
    from paper_2512_22036_amd.binding import _CRouter
    return _CRouter(**{**dict(N=16, E=32, k=4, score=0, groups=1, keep_groups=1, group_best=1, renorm=1, logits_dtype=1, scale=1.0, logits_stride=32), **kw})


def test_route(lib):
    r = lambda R, *a: lib.fusco_route(ctypes.byref(R), *a)
    good = (BUF, None, BUF, BUF, None)
    for bad in (dict(N=-1), dict(E=0), dict(E=1025, logits_stride=1025), dict(k=0), dict(k=65), dict(k=33), dict(groups=0), dict(groups=65), dict(groups=5), dict(groups=4, keep_groups=5),
                dict(groups=4, keep_groups=0), dict(groups=16, keep_groups=1), dict(group_best=0), dict(group_best=3), dict(groups=32, keep_groups=8, group_best=2), dict(logits_stride=31),
                dict(scale=float("inf")), dict(N=1 << 30, k=4)):
        assert r(router(**bad), *good) == -1, bad
    for bad in (dict(score=2), dict(renorm=2), dict(logits_dtype=2)):
        assert r(router(**bad), *good) == -3, bad
    assert r(router(), None, None, BUF, BUF, None) == -1
    assert r(router(), BUF + 2, None, BUF, BUF, None) == -1          # fp32 logits at an odd place
    assert r(router(), BUF, BUF + 2, BUF, BUF, None) == -1
    assert r(router(), BUF, None, BUF + 4, BUF, None) == -1
    assert r(router(), BUF, None, BUF, None, None) == -1
    assert lib.fusco_route(None, *good) == -1
    assert r(router(N=0), None, None, None, None, None) == 0
    b = lambda R, *a: lib.fusco_route_backward(ctypes.byref(R), *a)
    assert b(router(), BUF, BUF, BUF, None, None) == -1
    assert b(router(), BUF, None, BUF, BUF, None) == -1
    assert b(router(), BUF, BUF, BUF + 8, BUF, None) == -1
    assert b(router(N=0), None, None, None, None, None) == 0


def norm(**kw):
    from paper_2512_22036_amd.binding import _CNorm
    return _CNorm(**{**dict(N=16, H=64, stream_dtype=1, block_dtype=0, gain_dtype=1, gate_kind=0, scale=1.0, eps=1e-6), **kw})


def test_norms(lib):
    before = lambda n, *a: lib.fusco_norm_before(ctypes.byref(n), *a)
    for bad in (dict(N=-1), dict(H=0), dict(H=12), dict(H=32776), dict(eps=0.0), dict(eps=-1.0), dict(eps=float("nan"))):
        assert before(norm(**bad), BUF, BUF, BUF, None) == -1, bad
    for bad in (dict(stream_dtype=2), dict(block_dtype=-1), dict(gain_dtype=7), dict(stream_dtype=0, block_dtype=1)):
        assert before(norm(**bad), BUF, BUF, BUF, None) == -3, bad
    assert before(norm(), None, BUF, BUF, None) == -1 and before(norm(), BUF, None, BUF, None) == -1 and before(norm(), BUF, BUF, BUF + 8, None) == -1
    assert before(norm(N=0), None, BUF, None, None) == 0
    after = lambda n, *a: lib.fusco_norm_after(ctypes.byref(n), *a)
    good = [BUF, BUF, BUF, None, BUF, None, None, None]
    for i in (0, 1, 2, 4):
        assert after(norm(), *[None if j == i else v for j, v in enumerate(good)]) == -1, i
    assert after(norm(gate_kind=1), *good) == -1                     # a gate without a tensor
    assert after(norm(gate_kind=3), *good) == -3
    assert after(norm(scale=float("inf")), *good) == -1
    assert after(norm(), BUF, BUF, BUF, None, BUF, None, BUF, None) == -1   # next without its gain
    assert after(norm(N=0, gate_kind=2), None, None, BUF, None, None, None, None, None) == 0
    assert lib.fusco_norm_scratch_bytes(16, 64) == 16 * 3 * 64 * 4
    assert lib.fusco_norm_scratch_bytes(-1, 64) == lib.fusco_norm_scratch_bytes(16, 60) == lib.fusco_norm_scratch_bytes(16, 32776) == 0
    need = lib.fusco_norm_scratch_bytes(16, 64)
    bb = lambda n, *a: lib.fusco_norm_before_backward(ctypes.byref(n), *a)
    assert bb(norm(), BUF, BUF, BUF, None, BUF, BUF, BUF, need - 1, None) == -2
    assert bb(norm(), BUF, BUF, BUF, None, BUF, BUF, None, need, None) == -1
    assert bb(norm(), BUF, BUF, BUF, BUF + 4, BUF, BUF, BUF, need, None) == -1
    ab = lambda n, *a: lib.fusco_norm_after_backward(ctypes.byref(n), *a)
    assert ab(norm(), None, None, BUF, None, BUF, None, None, BUF, BUF, BUF, None, None, BUF, need, None) == -1    # no gradient at all
    assert ab(norm(), BUF, BUF, BUF, None, BUF, None, BUF, BUF, BUF, BUF, None, BUF, BUF, need, None) == -1        # dnext without out
    assert ab(norm(gate_kind=2), BUF, None, BUF, None, BUF, BUF, None, BUF, BUF, BUF, None, None, BUF, need, None) == -1   # no dgate
    assert ab(norm(), BUF, None, BUF, None, BUF, None, None, BUF, BUF, BUF, None, None, BUF, need - 4, None) == -2


def test_combine_backward(lib):
    L, empty = layout(lib), layout(lib, N=0)
    c = lambda *a: lib.fusco_combine_backward(ctypes.byref(L), *a)
    good = [BUF, 0, BUF, BUF, 0, BUF, BUF, 64, None]
    for i in (0, 2, 3, 5, 6):
        assert c(*[None if j == i else v for j, v in enumerate(good)]) == -1, i
        assert c(*[BUF + 4 if j == i else v for j, v in enumerate(good)]) == -1, i
    for H in (0, 12, 32776):
        assert c(*good[:7], H, None) == -1
    assert c(BUF, 2, *good[2:]) == -3 and c(*good[:4], 5, *good[5:]) == -3
    assert lib.fusco_combine_backward(ctypes.byref(empty), None, 0, None, None, 0, None, None, 64, None) == 0
