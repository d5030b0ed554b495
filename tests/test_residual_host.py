"""Refusals and size queries of the operators of a residual stage: everything is decided on the host, without a GPU."""
import ctypes
import re

import pytest

GOOD = 0x10000  # never dereferenced on the host


@pytest.fixture(scope="module")
def A():
    from paper_2311_05827_b200 import build
    build.build()
    import paper_2311_05827_b200 as pkg
    return pkg


@pytest.fixture(scope="module")
def lib(A):
    from paper_2311_05827_b200 import binding
    return binding.lib()


def test_structs_match_the_header(A):
    from paper_2311_05827_b200 import binding as b
    assert ctypes.sizeof(b.CDropoutParams) == 64 and b.CDropoutParams.p.offset == 48 and b.CDropoutParams.reserved.offset == 60
    assert ctypes.sizeof(b.CRmsNormParams) == 72 and b.CRmsNormParams.eps.offset == 48 and b.CRmsNormParams.format.offset == 68
    assert ctypes.sizeof(b.CMicroParams) == 56 and b.CMicroParams.dtype.offset == 40 and b.CMicroParams.block.offset == 48
    assert ctypes.sizeof(b.CMicroMatmulParams) == 40 and b.CMicroMatmulParams.accumulate.offset == 36


def test_header_declares_what_the_binding_exports(A):
    from paper_2311_05827_b200 import binding as b
    import os
    with open(os.path.join(os.path.dirname(b._HERE), "include", "accept.h")) as f:
        declared = set(re.findall(r"\b(accept_\w+)\(const accept_(?:dropout|rms_norm|micro)\w*_params", f.read()))
    assert declared == {n for n in b.EXPORTS if re.match("accept_(dropout|rms_norm|micro)", n)}


def test_dropout_params(A):
    P, check = A.DropoutParams, A.accept_dropout_check_params
    assert check(P(3, 5, 0.0)) == 0 and check(P(0, 5, 1.0)) == 0 and check(P(3, 0, 0.5)) == 0
    for rate in (-0.1, 1.1, float("nan"), float("inf"), -float("inf")):
        assert check(P(3, 5, rate)) == 9
    assert check(P(3, 5, 0.1, ld_x=4)) == 9 and check(P(3, 5, 0.1, ld_y=4)) == 9
    assert check(P(1 << 41, 1, 0.1)) == 9 and check(P(1, 1 << 41, 0.1)) == 9 and check(P(1 << 30, 1 << 31, 0.1)) == 9
    assert check(P(3, 5, 0.1, dtype_x=3)) == 4 and check(P(3, 5, 0.1, dtype_y=-1)) == 4


def test_dropout_refusals(A, lib):
    before = A.accept_launch_count()
    c, f = ctypes.byref(A.DropoutParams(10, 100, 0.1, A.DTYPE_BF16, A.DTYPE_F32).c()), lib.accept_dropout
    assert f(None, GOOD, GOOD, GOOD, None) == 1
    assert f(c, None, GOOD, GOOD, None) == 1 and f(c, GOOD, GOOD, None, None) == 1
    assert f(c, GOOD + 1, GOOD, GOOD, None) == 10 and f(c, GOOD, GOOD + 2, GOOD, None) == 10 and f(c, GOOD, GOOD, GOOD + 2, None) == 10
    assert f(ctypes.byref(A.DropoutParams(10, 100, 2.0).c()), GOOD, GOOD, GOOD, None) == 9
    assert A.accept_launch_count() == before


def test_rms_norm_params(A):
    P, check = A.RmsNormParams, A.accept_rms_norm_check_params
    assert check(P(3, 5)) == 0 and check(P(0, 5)) == 0 and check(P(3, 5, 0.0, p=1.0)) == 0
    assert check(P(3, 0)) == 9 and check(P(3, 1 << 31)) == 9 and check(P(3, 5, ld_x=4)) == 9 and check(P(3, 5, ld_y=4)) == 9 and check(P(1 << 40, 1 << 30)) == 9
    for eps in (-1.0, float("nan"), float("inf")):
        assert check(P(3, 5, eps)) == 9
    for rate in (-0.1, 1.5, float("nan")):
        assert check(P(3, 5, p=rate)) == 9
    for name in ("dtype_x", "dtype_y", "dtype_w"):
        assert check(P(3, 5, **{name: 3})) == 4 and check(P(3, 5, **{name: -1})) == 4
    assert check(P(3, 5, format=2)) == 4
    assert A.accept_rms_norm_workspace_size(P(3, 0)) == 0 and A.accept_rms_norm_workspace_size(P(3, 5)) >= 16
    assert A.accept_rms_norm_workspace_size(P(16384, 4096)) == 16 + 148 * 4 * 4096


def test_rms_norm_refusals(A, lib):
    before = A.accept_launch_count()
    p = A.RmsNormParams(10, 100, dtype_x=A.DTYPE_BF16)
    c, size = ctypes.byref(p.c()), A.accept_rms_norm_workspace_size(p)
    f, b = lib.accept_rms_norm_forward, lib.accept_rms_norm_backward
    args = [GOOD] * 9  # x, branch, gamma, sum, y, q, scale, rstd, workspace

    def but(values, **more):
        return [more.get("_%d" % i, v) for i, v in enumerate(values)]

    assert f(None, *args, 16, None) == 1
    assert f(c, *but(args, _0=None), 16, None) == 1
    assert f(c, *but(args, _5=None), 16, None) == 1 and f(c, *but(args, _6=None), 16, None) == 1 and f(c, *but(args, _8=None), 16, None) == 1
    assert f(c, GOOD, GOOD, GOOD, None, None, None, None, None, None, 0, None) == 1  # nothing asked for
    assert f(c, *args, 15, None) == 5
    for i, by in ((0, 1), (1, 2), (2, 2), (3, 1), (4, 2), (5, 8), (6, 8), (7, 2), (8, 2)):
        assert f(c, *but(args, **{"_%d" % i: GOOD + by}), 16, None) == 10, i
    assert f(ctypes.byref(A.RmsNormParams(1 << 31, 1).c()), *args, 16, None) == 9  # codes of too many rows
    assert f(ctypes.byref(A.RmsNormParams(3, 5, dtype_w=9).c()), *args, 16, None) == 4
    # dy, s, gamma, rstd, dsum, dx, dbranch, dgamma, workspace
    assert b(None, *args, size, None) == 1
    assert b(c, *args, size - 1, None) == 5
    for i in (0, 1, 3, 8):
        assert b(c, *but(args, **{"_%d" % i: None}), size, None) == 1
    assert b(c, *but(args, _5=None, _6=None, _7=None), size, None) == 1  # nothing asked for
    for i, by in ((0, 2), (1, 1), (2, 2), (3, 2), (4, 1), (5, 1), (6, 2), (7, 2), (8, 8)):
        assert b(c, *but(args, **{"_%d" % i: GOOD + by}), size, None) == 10, i
    assert A.accept_launch_count() == before


def test_micro_params_and_sizes(A):
    P, check = A.MicroParams, A.accept_micro_check_params
    assert check(P(0, 0)) == 0 and check(P(7, 9)) == 0
    assert check(P(1 << 31, 1)) == 9 and check(P(1, 1 << 31)) == 9 and check(P((1 << 31) - 1, (1 << 31) - 1)) == 9 and check(P(7, 9, ld=8)) == 9
    assert check(P(7, 9, dtype=3)) == 4 and check(P(7, 9, round=2)) == 4 and check(P(7, 9, block=2)) == 4
    p = P(130, 1000)
    assert A.accept_micro_data_size(p) == 130 * 512 and A.accept_micro_data_size(p, True) == 1000 * 80
    assert A.accept_micro_scale_size(p) == 512 * 2 * 8 and A.accept_micro_scale_size(p, True) == 512 * 8 * 2
    assert A.accept_micro_data_size(P(7, 9, dtype=3)) == 0 and A.accept_micro_workspace_size(p) == 16


def test_micro_refusals(A, lib):
    before = A.accept_launch_count()
    c, f, g = ctypes.byref(A.MicroParams(130, 1000).c()), lib.accept_micro_quantize, lib.accept_micro_dequantize
    assert f(c, None, GOOD, GOOD, GOOD, GOOD, GOOD, 16, None) == 1
    assert f(c, GOOD, None, None, None, None, GOOD, 16, None) == 1       # no output
    assert f(c, GOOD, GOOD, None, None, None, GOOD, 16, None) == 1       # codes without scales
    assert f(c, GOOD, GOOD, GOOD, None, GOOD, GOOD, 16, None) == 1
    assert f(c, GOOD, GOOD, GOOD, GOOD, GOOD, None, 16, None) == 1
    assert f(c, GOOD, GOOD, GOOD, GOOD, GOOD, GOOD, 15, None) == 5
    assert f(c, GOOD + 2, GOOD, GOOD, GOOD, GOOD, GOOD, 16, None) == 10
    for i in range(1, 5):
        assert f(c, *[GOOD + 8 if j == i else GOOD for j in range(6)], 16, None) == 10
    for i in range(3):
        assert g(c, *[None if j == i else GOOD for j in range(3)], None) == 1
    assert g(c, GOOD + 8, GOOD, GOOD, None) == 10 and g(c, GOOD, GOOD + 8, GOOD, None) == 10 and g(c, GOOD, GOOD, GOOD + 2, None) == 10
    assert g(None, GOOD, GOOD, GOOD, None) == 1
    assert f(ctypes.byref(A.MicroParams(130, 1000, round=7).c()), *[GOOD] * 6, 16, None) == 4
    assert A.accept_launch_count() == before


def test_micro_matmul_params_and_refusals(A, lib):
    P, check = A.MicroMatmulParams, A.accept_micro_matmul_check_params
    assert check(P(0, 0, 0)) == 0 and check(P(5, 6, 7)) == 0 and check(P(5, 6, 7, ldd=5)) == 9 and check(P(5, 6, 7, dtype_d=3)) == 4
    for i in range(3):
        assert check(P(*[1 << 31 if j == i else 1 for j in range(3)])) == 9
    assert check(P((1 << 31) - 1, (1 << 31) - 1, 1)) == 9  # more tiles than a grid has
    assert A.accept_micro_matmul_workspace_size(P(5, 6, 7, dtype_d=3)) == 0 and A.accept_micro_matmul_workspace_size(P(5, 6, 7)) >= 16
    before = A.accept_launch_count()
    p = P(50, 60, 70)
    c, size, f = ctypes.byref(p.c()), A.accept_micro_matmul_workspace_size(p), lib.accept_micro_matmul
    for i in (0, 1, 2, 3, 5, 6):  # a, its scales, b, its scales, d, workspace
        assert f(c, *[None if j == i else GOOD for j in range(7)], size, None) == 1
    assert f(c, *[GOOD] * 7, size - 1, None) == 5
    for i in range(4):
        assert f(c, *[GOOD + 8 if j == i else GOOD for j in range(7)], size, None) == 10
    assert f(c, GOOD, GOOD, GOOD, GOOD, GOOD + 2, GOOD, GOOD, size, None) == 10
    assert f(c, GOOD, GOOD, GOOD, GOOD, GOOD, GOOD + 1, GOOD, size, None) == 10
    assert f(None, *[GOOD] * 7, size, None) == 1
    assert A.accept_launch_count() == before
