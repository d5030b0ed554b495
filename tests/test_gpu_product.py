"""The paths of the block-scaled product that only some sizes take: many units of work for each pair of SMs, tiles cut along
k and joined, fp32 sums taken in chunks of k, long sums."""
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


# ---- many units of few products, whose results leave slowly --------------------------------------------------------------

@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("dtype,pad", [(BF16, 0), (F32, 1), (F16, 1)], ids=str)
@pytest.mark.parametrize("n,k", [(n, k) for n in (4100, 4160) for k in (64, 128, 1024)])
def test_sums_are_read_before_the_unit_after_next_takes_their_place(A, n, k, dtype, pad, accumulate):
    """8192 rows by 17 tiles of 256 columns: seven or eight units for each pair, one to eight blocks of k each.  In the last
    tile of columns half of the reading warps have nothing to store and run ahead of the others."""
    m = 8192
    ops.check_product(A, m, n, k, "e4m3", "e4m3", dtype, not accumulate, accumulate, pad)
    a, sa = ops.coded(3, m, k, "e4m3")
    b, sb = ops.coded(4, n, k, "e4m3", square=True)
    start = ops.random(5, m, n).to(dtype)
    p = A.MatmulParams(m, n, k, dtype_d=ops.code_of(A, dtype), accumulate=accumulate, ldd=n + pad)
    ws, first = A.new_workspace(p), None
    for _ in range(10):
        d = torch.zeros(m, n + pad, dtype=dtype, device="cuda")
        d[:, :n] = start
        A.accept_block_matmul(p, a, sa, b, sb, None, d, ws)
        first = d if first is None else first
        assert torch.equal(first.view(torch.uint8), d.view(torch.uint8))
    assert A.accept_last_device_status(ws) == 0
