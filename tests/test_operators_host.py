"""Refusals and size queries of the operators beside the codec: everything is decided on the host, without a GPU."""
import ctypes

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
    assert ctypes.sizeof(b.CLayerNormParams) == 48 and b.CLayerNormParams.eps.offset == 32 and b.CLayerNormParams.dtype_w.offset == 44
    assert ctypes.sizeof(b.CQuantizeParams) == 40 and b.CQuantizeParams.dtype.offset == 24 and b.CQuantizeParams.block.offset == 32
    assert ctypes.sizeof(b.CMatmulParams) == 48 and b.CMatmulParams.format_a.offset == 32 and b.CMatmulParams.accumulate.offset == 44


def test_layer_norm_params(A):
    P = A.LayerNormParams
    assert A.accept_layer_norm_check_params(P(3, 5)) == 0 and A.accept_layer_norm_check_params(P(0, 5)) == 0
    assert A.accept_layer_norm_check_params(P(3, 0)) == 9
    assert A.accept_layer_norm_check_params(P(3, 1 << 31)) == 9
    assert A.accept_layer_norm_check_params(P(3, 5, ld_x=4)) == 9
    assert A.accept_layer_norm_check_params(P(3, 5, ld_y=4)) == 9
    assert A.accept_layer_norm_check_params(P(1 << 40, 1 << 30)) == 9
    assert A.accept_layer_norm_check_params(P(3, 5, eps=-1.0)) == 9
    assert A.accept_layer_norm_check_params(P(3, 5, eps=float("nan"))) == 9
    assert A.accept_layer_norm_check_params(P(3, 5, eps=float("inf"))) == 9
    for name in ("dtype_x", "dtype_y", "dtype_w"):
        assert A.accept_layer_norm_check_params(P(3, 5, **{name: 3})) == 4
        assert A.accept_layer_norm_check_params(P(3, 5, **{name: -1})) == 4
    assert A.accept_layer_norm_workspace_size(P(3, 0)) == 0 and A.accept_layer_norm_workspace_size(P(3, 5)) >= 16


def test_layer_norm_refusals(A, lib):
    before = A.accept_launch_count()
    p = A.LayerNormParams(10, 100, dtype_x=A.DTYPE_BF16)
    c, size = ctypes.byref(p.c()), A.accept_layer_norm_workspace_size(p)
    f, b = lib.accept_layer_norm_forward, lib.accept_layer_norm_backward
    assert f(None, GOOD, GOOD, GOOD, GOOD, GOOD, GOOD, None) == 1
    assert f(c, None, GOOD, GOOD, GOOD, GOOD, GOOD, None) == 1 and f(c, GOOD, GOOD, GOOD, None, GOOD, GOOD, None) == 1
    assert f(c, GOOD + 1, GOOD, GOOD, GOOD, GOOD, GOOD, None) == 10   # x: 2-byte values
    assert f(c, GOOD, GOOD, GOOD, GOOD + 2, GOOD, GOOD, None) == 10   # y: 4-byte values
    assert f(c, GOOD, GOOD, GOOD + 2, GOOD, GOOD, GOOD, None) == 10 and f(c, GOOD, GOOD, GOOD, GOOD, GOOD + 2, GOOD, None) == 10
    assert f(ctypes.byref(A.LayerNormParams(3, 5, dtype_w=9).c()), GOOD, GOOD, GOOD, GOOD, GOOD, GOOD, None) == 4
    args = [GOOD] * 9
    assert b(c, *args, size - 1, None) == 5
    for i in (0, 1, 3, 4, 8):  # dy, x, mean, rstd, workspace
        assert b(c, *[None if j == i else v for j, v in enumerate(args)], size, None) == 1
    assert b(c, GOOD, GOOD, GOOD, GOOD, GOOD, None, None, None, GOOD, size, None) == 1  # nothing asked for
    assert b(c, *args[:8], GOOD + 4, size, None) == 10
    assert b(c, GOOD, GOOD, GOOD, GOOD, GOOD, GOOD + 1, GOOD, GOOD, GOOD, size, None) == 10
    assert A.accept_launch_count() == before


def test_block_params_and_sizes(A):
    P = A.QuantizeParams
    assert A.accept_block_check_params(P(0, 0)) == 0 and A.accept_block_check_params(P(7, 9)) == 0
    assert A.accept_block_check_params(P(1 << 31, 1)) == 9 and A.accept_block_check_params(P(1, 1 << 31)) == 9
    assert A.accept_block_check_params(P(7, 9, ld=8)) == 9
    assert A.accept_block_check_params(P(7, 9, dtype=3)) == 4 and A.accept_block_check_params(P(7, 9, format=2)) == 4
    assert A.accept_block_check_params(P(7, 9, block=2)) == 4
    p = P(130, 1000)
    assert A.accept_block_data_size(p) == 130 * 1008 and A.accept_block_data_size(p, True) == 1000 * 144
    assert A.accept_block_scale_size(p) == 512 * 2 * 2 and A.accept_block_scale_size(p, True) == 512 * 8 * 1
    assert A.accept_block_data_size(P(7, 9, dtype=3)) == 0 and A.accept_block_workspace_size(p) == 16


def test_block_refusals(A, lib):
    before = A.accept_launch_count()
    c = ctypes.byref(A.QuantizeParams(130, 1000).c())
    f = lib.accept_block_quantize
    assert f(c, None, GOOD, GOOD, GOOD, GOOD, GOOD, 16, None) == 1
    assert f(c, GOOD, None, None, None, None, GOOD, 16, None) == 1       # no output
    assert f(c, GOOD, GOOD, None, None, None, GOOD, 16, None) == 1       # codes without scales
    assert f(c, GOOD, GOOD, GOOD, None, GOOD, GOOD, 16, None) == 1
    assert f(c, GOOD, GOOD, GOOD, GOOD, GOOD, None, 16, None) == 1
    assert f(c, GOOD, GOOD, GOOD, GOOD, GOOD, GOOD, 15, None) == 5
    assert f(c, GOOD + 2, GOOD, GOOD, GOOD, GOOD, GOOD, 16, None) == 10
    for i in range(1, 5):
        assert f(c, *[GOOD + 8 if j == i else GOOD for j in range(6)], 16, None) == 10
    assert f(ctypes.byref(A.QuantizeParams(130, 1000, format=7).c()), *[GOOD] * 6, 16, None) == 4
    assert A.accept_launch_count() == before


def test_matmul_params(A):
    P = A.MatmulParams
    assert A.accept_matmul_check_params(P(0, 0, 0)) == 0 and A.accept_matmul_check_params(P(5, 6, 7)) == 0
    assert A.accept_matmul_check_params(P(5, 6, 7, ldd=5)) == 9
    for i in range(3):
        assert A.accept_matmul_check_params(P(*[1 << 31 if j == i else 1 for j in range(3)])) == 9
    assert A.accept_matmul_check_params(P((1 << 31) - 1, (1 << 31) - 1, 1)) == 9  # more tiles than a grid has
    assert A.accept_matmul_check_params(P(5, 6, 7, format_a=2)) == 4 and A.accept_matmul_check_params(P(5, 6, 7, format_b=-1)) == 4
    assert A.accept_matmul_check_params(P(5, 6, 7, dtype_d=3)) == 4
    assert A.accept_matmul_workspace_size(P(5, 6, 7, dtype_d=3)) == 0 and A.accept_matmul_workspace_size(P(5, 6, 7)) >= 16


def test_matmul_refusals(A, lib):
    before = A.accept_launch_count()
    p = A.MatmulParams(50, 60, 70)
    c, size = ctypes.byref(p.c()), A.accept_matmul_workspace_size(p)
    f = lib.accept_block_matmul
    for i in (0, 1, 2, 3, 5, 6):  # a, its scales, b, its scales, d, workspace
        assert f(c, *[None if j == i else GOOD for j in range(7)], size, None) == 1
    assert f(c, *[GOOD] * 7, size - 1, None) == 5
    for i in range(4):
        assert f(c, *[GOOD + 8 if j == i else GOOD for j in range(7)], size, None) == 10
    assert f(c, GOOD, GOOD, GOOD, GOOD, GOOD + 2, GOOD, GOOD, size, None) == 10
    assert f(c, GOOD, GOOD, GOOD, GOOD, GOOD, GOOD + 1, GOOD, size, None) == 10
    assert f(None, *[GOOD] * 7, size, None) == 1
    assert f(ctypes.byref(A.MatmulParams(5, 6, 7, dtype_d=5).c()), *[GOOD] * 7, size, None) == 4
    assert A.accept_launch_count() == before
