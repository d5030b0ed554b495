"""Layer norm where intermediate values pass the range of fp32 although the results do not."""
import pytest

from tests import operators_plain as plain
from tests import test_gpu_operators as ops

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def A():
    import paper_2311_05827_b200 as pkg
    return pkg


@pytest.mark.parametrize("dtype", [F32, BF16], ids=str)
@pytest.mark.parametrize("pad", [0, 1])
@pytest.mark.parametrize("cols", [1, 2, 32, 64, 100, 128, 256, 513, 1024, 4100, 8200, 20000])
def test_norm_grad_of_constant_rows_far_from_zero(A, cols, pad, dtype):
    """Rows of 2^120: x - mean is 0 and rstd is 1 / sqrt(eps), about 316, in the forward pass; mean times rstd is past the
    largest float.  The gradient is (h - mean(h)) rstd: xhat is 0 in every column that exists."""
    rows = 5
    _, x = ops.matrix(rows, cols, cols + pad, dtype, torch.full((rows, cols), 2.0 ** 120, device="cuda"))
    _, dy = ops.matrix(rows, cols, cols + pad, dtype, ops.random(1, rows, cols))
    _, dx = ops.matrix(rows, cols, cols + pad, dtype)
    mean, rstd = torch.full((rows,), 2.0 ** 120, device="cuda"), torch.full((rows,), 1e-5, device="cuda").rsqrt()
    dgamma, dbeta = torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
    p = A.LayerNormParams(rows, cols, 1e-5, ops.code_of(A, dtype), ops.code_of(A, dtype), A.DTYPE_F32, cols + pad, cols + pad)
    A.accept_layer_norm_backward(p, dy, x, None, mean, rstd, dx, dgamma, dbeta, A.new_workspace(p))
    h, s = dy.double(), rstd.double()[:, None]
    want = s * (h - h.mean(1, keepdim=True))
    # the roundings of a row's sum and of three operations on terms of its size
    tol = (64 + cols / 1024 + 4) * plain.E32 * s * (h.abs() + h.abs().mean(1, keepdim=True)) + plain.UNIT[dtype] * want.abs()
    assert bool(((dx.double() - want).abs() <= tol).all())
    assert bool((dgamma == 0).all())
    assert bool(((dbeta.double() - h.sum(0)).abs() <= 8 * plain.E32 * h.abs().sum(0)).all())
