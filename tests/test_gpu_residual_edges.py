"""Operators of a residual stage where sizes pass 32 bits, against 64-bit plain forms of parts of the matrix and against the same calls on
rows side by side."""
import pytest

from tests import residual_plain as plain
from tests.test_gpu_operators import code_of, random

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

F32, BF16 = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def A():
    import paper_2311_05827_b200 as pkg
    return pkg


@pytest.fixture(autouse=True)
def memory_goes_back():
    yield
    torch.cuda.empty_cache()


# (eight rows of a thread, four in fp32: the last starts more than 2^32 values after the first)
@pytest.mark.parametrize("dtype,rows,cols,first", [(BF16, 8, 1 << 30, 0), (BF16, 8, 1 << 30, 3), (F32, 4, 1_500_000_000, (1 << 34) - 400)], ids=str)
def test_stochastic_codes_of_very_wide_rows(A, dtype, rows, cols, first):
    """Every value is 0.3, 4.8 of its scale: the codes show the numbers that were drawn, whose counters are rng_offset + i cols + j."""
    seed, part = 0xFEDCBA9876543210, 4096
    x = torch.full((rows, cols), 0.3, dtype=dtype, device="cuda")
    p = A.MicroParams(rows, cols, code_of(A, dtype), A.ROUND_STOCHASTIC, seed=seed, rng_offset=first)
    q, s = (torch.empty(size(p), dtype=torch.uint8, device="cuda") for size in (A.accept_micro_data_size, A.accept_micro_scale_size))
    A.accept_micro_quantize(p, x, q, s, None, None, A.new_workspace(p))
    q = q.view(rows, -1)
    for r in range(rows):
        for c in (0, cols // 64 * 32, cols - part):
            codes, _ = plain.code4(x[r:r + 1, c:c + part], False, plain.draws(1, part, seed, first + r * cols + c))
            assert torch.equal(q[r:r + 1, c // 2:(c + part) // 2], plain.packed4(codes)), (r, c)
