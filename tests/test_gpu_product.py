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


# ---- tiles cut along k, and fp32 sums in chunks ---------------------------------------------------------------------------

# m, n, k, type of d, bias, accumulate, extra values between rows of d; then what the sizes are chosen for: tiles that are cut,
# their parts, their columns (0: none is cut)
CUTS = [
    (1280, 1100, 9000, BF16, True, False, 0, 25, 2, 256), (2560, 2560, 5000, F32, False, True, 0, 26, 2, 256),
    (1280, 1000, 6000, F16, True, False, 1, 20, 3, 256), (2048, 3000, 4000, F32, True, False, 1, 22, 3, 256),
    (1810, 300, 10000, BF16, False, True, 0, 24, 3, 128), (1810, 300, 10000, F32, True, True, 0, 24, 3, 128),
    (700, 1100, 12000, F32, True, False, 0, 15, 4, 256), (2560, 2100, 4000, BF16, False, True, 3, 16, 4, 256),
    (1570, 300, 10000, F32, False, False, 0, 14, 5, 256), (2590, 1800, 3500, BF16, True, False, 8, 14, 5, 256),
    (700, 1000, 8300, F16, False, True, 0, 12, 6, 256), (500, 700, 20000, F32, True, True, 1, 12, 6, 128),
    (500, 700, 20000, BF16, True, False, 0, 12, 6, 128),
    # whole tiles whose sums are taken over two and three chunks of k, with and without cut ones beside them
    (2304, 2100, 8300, F32, True, False, 0, 7, 6, 256), (2304, 2100, 8300, F32, True, True, 0, 7, 6, 256), (2304, 2100, 8300, F32, True, True, 1, 7, 6, 256),
    (2304, 2100, 8300, F32, False, False, 1, 7, 6, 256), (1280, 2000, 8300, F32, True, True, 0, 0, 1, 256),
    (1280, 2000, 8300, F32, True, False, 1, 0, 1, 256), (1280, 1100, 8300, F32, False, True, 0, 0, 1, 128), (2560, 2560, 16500, F32, True, True, 0, 0, 1, 256),
]


def bytes_of_parts(case):
    _, _, _, _, _, _, _, cut, parts, columns = case
    return cut * parts * 256 * columns * 4


@pytest.mark.parametrize("case", CUTS, ids=str)
def test_product_of_cut_tiles_and_chunks(A, case):
    m, n, k, dtype, bias, accumulate, pad = case[:7]
    # the workspace holds the parts' sums and what counts them: the sizes are dealt as this test means them to be
    beside = A.accept_matmul_workspace_size(A.MatmulParams(m, n, k, dtype_d=ops.code_of(A, dtype), accumulate=accumulate, ldd=n + pad)) - bytes_of_parts(case)
    assert 16 < beside < 32768 if case[7] else beside == 16
    ops.check_product(A, m, n, k, "e5m2" if accumulate else "e4m3", "e4m3", dtype, bias, accumulate, pad)


def test_cut_tiles_stay_inside_their_buffers(A):
    from tests import gpu_util
    with gpu_util.library_variant("bounds"):
        assert A.accept_bounds_check_report()[:2] == (0, 0)
        for case in CUTS:
            ops.check_product(A, *case[:3], "e4m3", "e4m3", *case[3:7])
        for m in (7, 32, 60, 128):  # long shares of few rows
            ops.check_product(A, m, 2100, 35000, "e4m3", "e4m3", F32, True, False, 1)
        assert A.accept_bounds_check_report()[:2] == (0, 0)


# ---- rows of d that end inside 16 bytes ------------------------------------------------------------------------------------------

# m, n, k, type of d, bias, accumulate, extra values between rows of d: rows start on 16-byte boundaries and end off them
ENDS = [
    (2560, 3980, 176, F16, False, False, 4), (2808, 9967, 1, BF16, True, False, 1), (9570, 4310, 1104, BF16, False, False, 2), (3056, 3444, 1, BF16, False, False, 4),
    (6168, 4407, 10, F32, True, False, 1), (11265, 138, 1672, F32, False, False, 2), (9600, 130, 128, F32, False, False, 2), (903, 1303, 3387, F32, False, False, 1),
    (428, 9906, 28, F32, True, False, 2), (2304, 2303, 300, F32, True, True, 1), (2304, 2305, 300, F32, False, True, 7), (2304, 2311, 300, F16, False, True, 1),
    (2304, 2257, 200, BF16, True, False, 7), (2304, 2271, 200, BF16, True, False, 1), (2304, 2289, 200, F16, True, False, 15), (2304, 2287, 200, F16, True, False, 1),
    # cut tiles, chunks of k
    (700, 1002, 8300, F16, True, False, 6), (1280, 1001, 6000, F32, True, False, 3), (1810, 301, 10000, BF16, False, False, 3), (1280, 1999, 8300, F32, True, True, 1),
    (2304, 2101, 8300, F32, True, False, 3), (2304, 2101, 8300, F32, False, True, 3), (1280, 1102, 8300, F32, False, False, 2),
]


@pytest.mark.parametrize("case", ENDS, ids=str)
def test_product_writes_nothing_behind_the_end_of_a_row(A, case):
    m, n, k, dtype, bias, accumulate, pad = case
    assert n * dtype.itemsize % 16 != 0 and (n + pad) * dtype.itemsize % 16 == 0
    ops.check_product(A, m, n, k, "e4m3", "e5m2", dtype, bias, accumulate, pad)
    # d as the first columns of a matrix whose other columns are someone else's
    a, sa = ops.coded(5, m, k, "e4m3")
    b, sb = ops.coded(6, n, k, "e4m3")
    whole = ops.random(7, m, n + pad).to(dtype)
    others = whole[:, n:].clone()
    p = A.MatmulParams(m, n, k, dtype_d=ops.code_of(A, dtype), accumulate=accumulate, ldd=n + pad)
    A.accept_block_matmul(p, a, sa, b, sb, None, whole, A.new_workspace(p))
    assert torch.equal(whole[:, n:], others)


def test_row_ends_stay_inside_their_buffers(A):
    """The checking build compares a tile store in units of 16 bytes, as it writes them."""
    from tests import gpu_util
    with gpu_util.library_variant("bounds"):
        assert A.accept_bounds_check_report()[:2] == (0, 0)
        for case in ENDS:
            ops.check_product(A, *case[:3], "e4m3", "e4m3", *case[3:])
        assert A.accept_bounds_check_report()[:2] == (0, 0)


# ---- waits that run out --------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("m,n,k,dtype", [(4, 300, 64, BF16), (64, 9600, 4096, F32), (300, 300, 100, F32), (2304, 2304, 64, BF16), (8192, 4160, 1024, BF16),
                                         (700, 1000, 8300, BF16), (2304, 2100, 8300, F32)], ids=str)
def test_products_whose_copies_do_not_arrive_end_and_leave_the_gpu_usable(A, m, n, k, dtype):
    """Fewer copies than stages and more of them, many units a pair, cut tiles, chunks of k: the call reports the wait that ran
    out, and the next call is right."""
    from tests import gpu_util
    a, sa = ops.coded(1, m, k, "e4m3")
    b, sb = ops.coded(2, n, k, "e4m3")
    p = A.MatmulParams(m, n, k, dtype_d=ops.code_of(A, dtype))
    d, want, ws = torch.zeros(m, n, dtype=dtype, device="cuda"), torch.zeros(m, n, dtype=dtype, device="cuda"), A.new_workspace(p)
    A.accept_block_matmul(p, a, sa, b, sb, None, want, ws)
    assert A.accept_last_device_status(ws) == 0
    with gpu_util.library_variant("stall"):
        A.accept_block_matmul(p, a, sa, b, sb, None, d, ws)
        assert A.accept_last_device_status(ws) == A.DEV_COPY_TIMEOUT
    ws[0] = 0
    A.accept_block_matmul(p, a, sa, b, sb, None, d, ws)
    assert A.accept_last_device_status(ws) == 0
    assert torch.equal(d, want)


# ---- long sums --------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("m", [5, 17, 64, 100, 128])
@pytest.mark.parametrize("n,k,bias,accumulate,pad", [(9600, 32768, False, False, 0), (9601, 20001, True, True, 0), (2000, 70000, True, False, 1), (300, 131072, False, True, 0)])
def test_few_rows_of_long_sums_are_single_precision(A, m, n, k, bias, accumulate, pad):
    """fp32 results of few rows, shares of up to 256 blocks of k.  The tensor cores' sums over 8192 values are off by less than
    10^-6 of their norm, so the sum of chunks of that length is too, whatever k is.  In one run, 20001 values are off by
    1.5e-6 and 32768 by 3.0e-6."""
    a, sa = ops.coded(1, m, k, "e4m3", spread=0)
    b, sb = ops.coded(2, n, k, "e4m3", spread=0)
    offset = ops.random(3, n) if bias else None
    start = ops.random(4, m, n)
    gd, d = ops.matrix(m, n, n + pad, F32, start)
    p = A.MatmulParams(m, n, k, dtype_d=A.DTYPE_F32, accumulate=accumulate, ldd=n + pad)
    A.accept_block_matmul(p, a, sa, b, sb, offset, d, A.new_workspace(p))
    gd.check("d")
    columns = 256  # of the result, the first ones: their scales are the first 128-row groups'
    whole = b.shape[0]
    r, at = torch.arange(columns, device="cuda")[:, None], torch.arange(-(-k // 128), device="cuda")[None]
    e = sb[plain.place(r, at, whole)].double() - 127
    vb = b[:columns, :k].contiguous().view(torch.float8_e4m3fn).double() * torch.ldexp(torch.ones_like(e), e.int()).repeat_interleave(128, 1)[:, :k]
    want = plain.decode(a, sa, "e4m3", k) @ vb.t()
    norm = want.norm()
    if bias:
        want += offset[:columns].double()
    if accumulate:
        want += start[:, :columns].double()
    assert float((d[:, :columns].double() - want).norm() / norm) < 1e-6
    assert bool(torch.isfinite(d).all())


def test_product_of_the_longest_rows(A):
    """k = 2^31 - 1, the largest that the header allows: sums that take longer (416 ms, measured) than
    a copy may (200 ms), and offsets past 31 bits."""
    k = 2 ** 31 - 1
    at = [0, 5, 2 ** 30 + 129, k - 1]
    a, b = torch.zeros(2 ** 31, dtype=torch.uint8, device="cuda"), torch.zeros(2 ** 31, dtype=torch.uint8, device="cuda")
    for i, c in enumerate(at):
        a[c], b[c] = 0x38, 0x38 + 8 * i  # 1 times 2^i
    p = A.MatmulParams(1, 1, k)
    scales = torch.full((A.accept_block_scale_size(A.QuantizeParams(1, k)),), 127, dtype=torch.uint8, device="cuda")
    d, ws = torch.zeros(1, 1, dtype=BF16, device="cuda"), A.new_workspace(p)
    A.accept_block_matmul(p, a, scales, b, scales, None, d, ws)
    assert A.accept_last_device_status(ws) == 0
    assert float(d) == 15.0
