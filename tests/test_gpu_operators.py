"""Layer norm, block quantisation and the block-scaled matrix product against 64-bit plain forms, through the C ABI.

Tolerances come from the number of roundings on the way (E32 = 2^-24 each, of the magnitudes that are added), plus one
rounding to the output's type; codes and scale bytes are compared bit for bit.
"""
import numpy as np
import pytest

from tests import gpu_util
from tests import operators_plain as plain

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def A():
    import paper_2311_05827_b200 as pkg
    return pkg


def code_of(A, dtype):
    return {F32: A.DTYPE_F32, BF16: A.DTYPE_BF16, F16: A.DTYPE_F16}[dtype]


def matrix(rows, cols, ld, dtype, values=None, offset=0):
    """A rows x cols view with row stride ld, `offset` values into a guarded buffer of exactly the bytes it spans."""
    size = torch.empty(0, dtype=dtype).element_size()
    n = ((rows - 1) * ld + cols) if rows else 0
    g = gpu_util.Guarded(torch, (n + offset) * size, 0x5B)
    flat = g.view(dtype)[offset:]
    v = torch.as_strided(flat, (rows, cols), (ld, 1)) if rows else flat.reshape(0, cols)
    if values is not None:
        v.copy_(values)
    return g, v


def gaps_untouched(g, rows, cols, ld, dtype, offset=0):
    """The bytes between the rows still hold what the buffer was filled with."""
    if not rows:
        return True
    size = torch.empty(0, dtype=dtype).element_size()
    keep = torch.ones(g.nbytes, dtype=torch.bool, device="cuda")
    at = (offset + torch.arange(rows, device="cuda")[:, None] * ld + torch.arange(cols, device="cuda")[None]).reshape(-1) * size
    for i in range(size):
        keep[at + i] = False
    return bool((g.bytes[keep] == 0x5B).all())


def random(seed, *shape, scale=1.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randn(*shape, device="cuda", generator=g) * scale


# ---- layer norm -----------------------------------------------------------------------------------------------------

# rows, cols, extra values between rows of x and of y, offset of x in its buffer, types of x, y, weights
NORMS = [
    (1, 1, 0, 0, 0, F32, F32, F32), (3, 2, 0, 0, 0, BF16, F32, BF16), (2, 7, 1, 0, 0, F16, F16, F16), (5, 33, 0, 3, 0, F32, BF16, F32),
    (9, 256, 0, 0, 0, BF16, BF16, BF16), (17, 257, 7, 7, 0, F16, F32, F32), (8, 512, 0, 0, 1, F32, F32, F32), (33, 513, 0, 0, 0, F32, F16, F16),
    (6, 1000, 24, 8, 0, BF16, BF16, F32), (300, 1024, 0, 0, 0, F32, F32, F32), (700, 1537, 7, 7, 0, F16, F16, F32), (40, 2047, 1, 1, 0, F16, F16, F16),
    (41, 2056, 0, 0, 0, BF16, F32, F32), (1200, 4096, 0, 0, 0, BF16, BF16, F32), (65, 4096, 0, 0, 3, F32, BF16, BF16), (12, 4104, 0, 0, 0, F32, BF16, F32),
    (10, 8192, 0, 0, 0, BF16, BF16, BF16), (7, 8200, 0, 1, 0, F32, F32, F32), (5, 16384, 0, 0, 0, F16, BF16, F32), (3, 16391, 0, 0, 0, F32, F32, F32),
    (70, 20000, 0, 0, 0, BF16, F16, BF16), (2, 40000, 0, 0, 0, F32, F32, F32),
    (5000, 64, 0, 0, 0, BF16, BF16, BF16), (3001, 128, 0, 0, 0, BF16, BF16, F32), (700, 100, 8, 8, 0, F32, BF16, F32), (601, 127, 0, 0, 1, F16, F16, F16),
    (1100, 9001, 0, 0, 0, BF16, BF16, F32), (600, 8200, 0, 0, 0, F32, F32, F32), (300, 4480, 0, 0, 0, F16, F16, F16),
    (50, 1030, 0, 0, 0, BF16, BF16, BF16), (33, 2051, 1, 3, 2, F16, F16, F16), (31, 1031, 0, 0, 0, BF16, BF16, F32), (400, 98, 0, 0, 0, BF16, BF16, BF16),
    (20, 515, 0, 1, 0, F32, BF16, F32), (20, 515, 2, 0, 1, F32, F32, F32), (9, 8190, 0, 0, 0, F16, BF16, F16), (3, 9003, 1, 1, 0, BF16, F32, BF16),
]


def check_norm(A, rows, cols, pad_x, pad_y, offset, tx, ty, tw, eps=1e-5, x=None, weights=True, seed=0):
    if x is None:
        x = random(seed, rows, cols) * (0.1 + 3 * torch.rand(cols, device="cuda")) + 0.5
    gx, vx = matrix(rows, cols, cols + pad_x, tx, x, offset)
    gy, vy = matrix(rows, cols, cols + pad_y, ty)
    gamma = (1 + 0.3 * random(seed + 1, cols)).to(tw) if weights else None
    beta = (0.3 * random(seed + 2, cols)).to(tw) if weights else None
    mean, rstd = gpu_util.guarded_floats(torch, rows), gpu_util.guarded_floats(torch, rows)
    p = A.LayerNormParams(rows, cols, eps, code_of(A, tx), code_of(A, ty), code_of(A, tw), cols + pad_x, cols + pad_y)
    A.accept_layer_norm_forward(p, vx, gamma, beta, vy, mean.view(F32), rstd.view(F32))
    torch.cuda.synchronize()
    y, m, s = plain.norm(vx, gamma, beta, eps)
    # a row's sums: at most 64 roundings a thread and a tree; more where a thread walks a longer row
    n = 64 + cols / 1024
    size_x = vx.double().abs().mean(1)
    assert bool(((mean.view(F32).double() - m).abs() <= n * plain.E32 * size_x + 1e-45).all())
    off_var = n * plain.E32 * (1 + 2 * size_x * s) + 4 * plain.E32       # relative, of var + eps
    assert bool(((rstd.view(F32).double() - s).abs() <= off_var * s).all())
    g = 1.0 if gamma is None else gamma.double().abs()
    b = 0.0 if beta is None else beta.double().abs()
    tol = (n * plain.E32 * size_x * s)[:, None] * g + (off_var[:, None] + 4 * plain.E32) * ((vx.double() - m[:, None]).abs() * s[:, None] * g) + 2 * plain.E32 * b
    assert bool(((vy.double() - y).abs() <= tol + plain.UNIT[ty] * y.abs() + plain.SMALLEST[ty]).all())
    for name, buf in (("x", gx), ("y", gy), ("mean", mean), ("rstd", rstd)):
        buf.check(name)
    assert gaps_untouched(gy, rows, cols, cols + pad_y, ty)
    return p, vx, gamma, mean.view(F32), rstd.view(F32)


def check_norm_grad(A, rows, cols, pad_x, pad_y, offset, tx, ty, tw, weights=True, seed=5):
    p, x, gamma, mean, rstd = check_norm(A, rows, cols, pad_x, pad_y, offset, tx, ty, tw, weights=weights, seed=seed)
    _, dy = matrix(rows, cols, cols + pad_y, ty, random(seed + 3, rows, cols, scale=0.1))
    gdx, dx = matrix(rows, cols, cols + pad_x, tx, None, offset)
    dgamma, dbeta = gpu_util.guarded_floats(torch, cols), gpu_util.guarded_floats(torch, cols)
    ws = gpu_util.Guarded(torch, A.accept_layer_norm_workspace_size(p), 0xEE)
    call = lambda a, b, c: A.accept_layer_norm_backward(p, dy, x, gamma, mean, rstd, a, b, c, ws.bytes)  # noqa: E731
    call(dx, dgamma.view(F32), dbeta.view(F32))
    torch.cuda.synchronize()
    want, wg, wb, size, size_g, size_b = plain.norm_grad(dy, x, gamma, mean, rstd)
    n = 64 + cols / 1024
    assert bool(((dx.double() - want).abs() <= n * plain.E32 * size + plain.UNIT[tx] * want.abs() + plain.SMALLEST[tx]).all())
    m = 64 + rows                                                        # at most one rounding a row, and a few of xhat
    assert bool(((dgamma.view(F32).double() - wg).abs() <= m * plain.E32 * size_g + 1e-45).all())
    assert bool(((dbeta.view(F32).double() - wb).abs() <= m * plain.E32 * size_b + 1e-45).all())
    for name, buf in (("dx", gdx), ("dgamma", dgamma), ("dbeta", dbeta), ("workspace", ws)):
        buf.check(name)
    assert gaps_untouched(gdx, rows, cols, cols + pad_x, tx, offset)
    # the same bits again, and in the calls that ask for one side alone
    first = [t.clone() for t in (dx, dgamma.view(F32), dbeta.view(F32))]
    dx.zero_(), dgamma.view(F32).zero_(), dbeta.view(F32).zero_()
    call(dx, None, None)
    call(None, dgamma.view(F32), None)
    call(None, None, dbeta.view(F32))
    torch.cuda.synchronize()
    for a, b in zip(first, (dx, dgamma.view(F32), dbeta.view(F32))):
        assert torch.equal(a, b)


@pytest.mark.parametrize("case", NORMS, ids=str)
def test_norm_forward_and_backward(A, case):
    check_norm_grad(A, *case)


def test_norm_without_weights_and_without_rows(A):
    check_norm_grad(A, 19, 777, 0, 0, 0, F32, F32, F32, weights=False)
    p = A.LayerNormParams(0, 100)
    dgamma, dbeta = torch.full((100,), 7.0, device="cuda"), torch.full((100,), 7.0, device="cuda")
    none = torch.empty(0, device="cuda")
    A.accept_layer_norm_forward(p, none, None, None, none, None, None)
    A.accept_layer_norm_backward(p, none, none, None, none, none, none, dgamma, dbeta, A.new_workspace(p))
    assert bool((dgamma == 0).all()) and bool((dbeta == 0).all())


def test_norm_of_rows_with_a_large_offset_and_of_constant_rows(A):
    """The squared distances are taken from the mean, so an offset of 10^4 spreads keeps the digits that x has."""
    x = random(3, 50, 1024) + 1e4
    check_norm(A, 50, 1024, 0, 0, 0, F32, F32, F32, x=x)
    x = torch.full((4, 640), 3.25, device="cuda")
    _, _, _, mean, rstd = check_norm(A, 4, 640, 0, 0, 0, F32, F32, F32, x=x)
    assert bool((mean == 3.25).all())


@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("cols", [100, 1024, 20000])
def test_norm_keeps_a_bad_row_to_itself(A, value, cols):
    x = random(4, 11, cols)
    x[5, cols // 2] = value
    p = A.LayerNormParams(11, cols)
    y, mean, rstd = torch.empty_like(x), torch.empty(11, device="cuda"), torch.empty(11, device="cuda")
    A.accept_layer_norm_forward(p, x, None, None, y, mean, rstd)
    assert bool(torch.isnan(y[5]).all())
    rest = [r for r in range(11) if r != 5]
    assert bool(torch.isfinite(y[rest]).all())
    dx = torch.empty_like(x)
    A.accept_layer_norm_backward(p, x, x, None, mean, rstd, dx, None, None, A.new_workspace(p))
    assert bool(torch.isnan(dx[5]).all()) and bool(torch.isfinite(dx[rest]).all())


def test_norm_gradient_against_differences(A):
    """dx, dgamma and dbeta against central differences of the forward kernel: step h = 2^-6, so the third-order term
    is about h^2 and the fp32 noise about 2^-24 / h of the loss' terms."""
    rows, cols, h = 3, 40, 2.0 ** -6
    x, gamma, beta, dy = random(1, rows, cols), 1 + 0.2 * random(2, cols), 0.2 * random(3, cols), random(4, rows, cols)
    p = A.LayerNormParams(rows, cols)
    y, mean, rstd = torch.empty_like(x), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    A.accept_layer_norm_forward(p, x, gamma, beta, y, mean, rstd)
    dx, dgamma, dbeta = torch.empty_like(x), torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
    A.accept_layer_norm_backward(p, dy, x, gamma, mean, rstd, dx, dgamma, dbeta, A.new_workspace(p))

    def loss(x_, gamma_, beta_):
        out = torch.empty_like(x_)
        A.accept_layer_norm_forward(p, x_, gamma_, beta_, out)
        return float((out.double() * dy.double()).sum())

    def difference(t, at, *rest):
        args = []
        for sign in (1, -1):
            moved = t.clone()
            moved[at] += sign * h
            args.append(rest[0](moved))
        return (args[0] - args[1]) / (2 * h)

    tol = 8 * h * h * float(dy.abs().max()) * 4
    for at in [(0, 0), (1, 17), (2, 39)]:
        assert abs(difference(x, at, lambda t: loss(t, gamma, beta)) - float(dx[at])) <= tol
    for at in [0, 21, 39]:
        assert abs(difference(gamma, at, lambda t: loss(x, t, beta)) - float(dgamma[at])) <= tol
        assert abs(difference(beta, at, lambda t: loss(x, gamma, t)) - float(dbeta[at])) <= tol


# ---- block quantisation ---------------------------------------------------------------------------------------------

# rows, cols, extra values between rows, type of x, format, square
BLOCKS = [
    (1, 1, 0, F32, "e4m3", False), (1, 127, 0, BF16, "e4m3", False), (2, 128, 0, F16, "e5m2", False), (3, 129, 0, F32, "e5m2", True),
    (31, 16, 0, BF16, "e4m3", True), (33, 520, 0, BF16, "e4m3", False), (128, 512, 8, F32, "e4m3", True), (130, 300, 1, F16, "e4m3", False),
    (129, 1, 0, F32, "e4m3", False), (200, 700, 0, BF16, "e5m2", False), (513, 144, 3, F32, "e5m2", False), (640, 257, 0, F16, "e4m3", True),
]


def check_quantize(A, x, pad, fmt, square, sides="both"):
    rows, cols = x.shape
    _, vx = matrix(rows, cols, cols + pad, x.dtype, x)
    p = A.QuantizeParams(rows, cols, code_of(A, x.dtype), {"e4m3": A.FORMAT_E4M3, "e5m2": A.FORMAT_E5M2}[fmt],
                         A.BLOCK_SQUARE if square else A.BLOCK_ROW, cols + pad)
    bufs = {}
    for t, side in enumerate(("rows", "columns")):
        if sides in (side, "both"):
            bufs[side] = (gpu_util.Guarded(torch, A.accept_block_data_size(p, bool(t)), 0x77), gpu_util.Guarded(torch, A.accept_block_scale_size(p, bool(t)), 0x77))
    ws = gpu_util.Guarded(torch, A.accept_block_workspace_size(p), 0)
    args = [b.bytes if b is not None else None for side in ("rows", "columns") for b in bufs.get(side, (None, None))]
    A.accept_block_quantize(p, vx, *args, ws.bytes)
    status = A.accept_last_device_status(ws.bytes)
    ws.check("workspace")
    cpu = vx.cpu()
    assert status == (0 if bool(torch.isfinite(cpu.double()).all()) else A.DEV_NONFINITE)
    for side, (q, s) in bufs.items():
        q.check("codes"), s.check("scales")
        want, e = plain.quantize(cpu if side == "rows" else cpu.t(), fmt, square)
        r, c = want.shape[0], (cols if side == "rows" else rows)
        assert np.array_equal(s.bytes.cpu().numpy(), plain.scale_bytes(e, r, c).numpy()), side
        got = q.bytes.cpu().view(r, -1)
        bad = torch.isnan(want.view(plain.FLOAT8[fmt]).float())
        assert torch.equal(torch.isnan(got.view(plain.FLOAT8[fmt]).float()), bad), side
        assert torch.equal(got[~bad], want[~bad]), side
    return p, bufs


@pytest.mark.parametrize("case", BLOCKS, ids=str)
def test_block_quantize(A, case):
    rows, cols, pad, dtype, fmt, square = case
    x = random(rows + cols, rows, cols) * torch.exp2(torch.randint(-9, 9, (rows, 1), device="cuda").float())
    x[torch.rand(rows, cols, device="cuda") < 0.1] = 0
    for sides in ("both", "rows", "columns"):
        check_quantize(A, x.to(dtype), pad, fmt, square, sides)


@pytest.mark.parametrize("fmt", ["e4m3", "e5m2"])
@pytest.mark.parametrize("square", [False, True])
def test_block_quantize_at_the_ends_of_the_range(A, fmt, square):
    """Blocks of zeros, of subnormals, of the largest floats, at and just past a power of two times the largest code,
    ties between two codes, and NaN and infinities among them and alone."""
    top = plain.LARGEST[fmt]
    x = torch.zeros(140, 400, device="cuda")
    x[1, 5] = 2.0 ** -149
    x[2, :128] = random(2, 128) * 2.0 ** -140
    x[3, 300] = 3.4028234e38
    x[4, 128:256] = -3.4028234e38
    for r in range(8):
        x[5 + r, :] = random(r, 400)
        x[5 + r, 17] = top * 2.0 ** (r - 4)
        x[5 + r, 140] = float(np.nextafter(np.float32(top * 2.0 ** (r - 4)), np.float32(np.inf)))
    x[20, :256] = torch.arange(256, device="cuda") * 0.0625 + 0.03125
    x[20, 0] = top
    x[21, :] = -x[20, :]
    x[22, 7] = 2.0 ** -126
    x[23, 7] = float(np.nextafter(np.float32(2.0 ** -126), np.float32(0)))
    check_quantize(A, x, 0, fmt, square)
    bad = random(9, 140, 400)
    bad[3, 3], bad[4, 200], bad[5, 399] = float("nan"), float("inf"), float("-inf")
    bad[6, 128:256] = float("inf")
    bad[7, :] = float("nan")
    check_quantize(A, bad, 0, fmt, square)
    check_quantize(A, bad.to(BF16), 0, fmt, square)
    check_quantize(A, torch.where(torch.isfinite(bad), bad, 0.0).to(F16) * 4000, 0, fmt, square)


def test_block_quantize_of_nothing(A):
    ws = torch.zeros(4, dtype=torch.int32, device="cuda")
    some = torch.zeros(16, dtype=torch.uint8, device="cuda")
    before = A.accept_launch_count()
    for rows, cols in ((0, 5), (5, 0)):
        A.accept_block_quantize(A.QuantizeParams(rows, cols), some, some, some, None, None, ws)
    assert A.accept_launch_count() == before


# ---- matrix product --------------------------------------------------------------------------------------------------

FORMATS = ("e4m3", "e5m2")
# m, n, k, formats of a and b, type of d, bias, accumulate, extra values between rows of d
PRODUCTS = [
    (1, 1, 1, "e4m3", "e4m3", F32, False, False, 0), (1, 130, 128, "e4m3", "e4m3", BF16, True, False, 0),
    (1, 4096, 4096, "e4m3", "e4m3", BF16, True, False, 0), (3, 200, 100, "e5m2", "e4m3", F16, False, True, 1),
    (16, 384, 640, "e4m3", "e5m2", F32, True, True, 0), (17, 129, 129, "e5m2", "e5m2", F32, False, False, 3),
    (32, 1000, 2000, "e4m3", "e4m3", BF16, False, False, 0), (33, 256, 513, "e4m3", "e4m3", BF16, True, False, 8),
    (64, 128, 4000, "e4m3", "e4m3", F32, False, False, 0), (65, 333, 777, "e4m3", "e4m3", F16, True, False, 0),
    (128, 512, 1024, "e4m3", "e4m3", BF16, False, True, 0), (129, 128, 384, "e4m3", "e4m3", F32, True, False, 0),
    (200, 1, 300, "e4m3", "e4m3", F32, False, False, 0), (300, 50, 260, "e5m2", "e4m3", BF16, True, False, 0),
    (257, 2050, 1544, "e4m3", "e4m3", F16, False, False, 0), (1000, 777, 91, "e4m3", "e4m3", F32, True, True, 7),
    (512, 512, 512, "e5m2", "e4m3", F32, False, True, 0), (1500, 1100, 700, "e4m3", "e4m3", BF16, True, False, 0),
    (2048, 2304, 640, "e4m3", "e4m3", BF16, True, False, 0), (640, 1280, 8300, "e5m2", "e4m3", F32, False, False, 0),
    (2600, 2600, 1160, "e4m3", "e4m3", F32, False, True, 0), (4100, 520, 2100, "e4m3", "e4m3", F16, True, False, 4),
    (2305, 2311, 300, "e5m2", "e5m2", BF16, True, False, 0), (2048, 2100, 257, "e4m3", "e5m2", F16, False, True, 0), (5000, 1900, 1000, "e4m3", "e4m3", F32, True, False, 0),
    (4000, 3333, 128, "e4m3", "e4m3", F32, False, True, 1), (7000, 2000, 1, "e5m2", "e4m3", BF16, True, False, 0),
]


def coded(seed, rows, k, fmt, square=False, spread=6):
    """Random codes and scale bytes as the quantiser writes them, on the GPU."""
    import paper_2311_05827_b200 as A
    x = random(seed, rows, k) * torch.exp2(torch.randint(-spread, spread + 1, (rows, 1), device="cuda").float())
    p = A.QuantizeParams(rows, k, A.DTYPE_F32, {"e4m3": A.FORMAT_E4M3, "e5m2": A.FORMAT_E5M2}[fmt], A.BLOCK_SQUARE if square else A.BLOCK_ROW)
    q = gpu_util.Guarded(torch, A.accept_block_data_size(p))
    s = gpu_util.Guarded(torch, A.accept_block_scale_size(p))
    A.accept_block_quantize(p, x, q.bytes, s.bytes, None, None, A.new_workspace(p))
    return q.bytes.view(rows, -1), s.bytes


def check_product(A, m, n, k, fa, fb, td, with_bias, accumulate, pad, seed=1):
    a, sa = coded(seed, m, k, fa)
    b, sb = coded(seed + 1, n, k, fb, square=True)
    bias = random(seed + 2, n) if with_bias else None
    start = random(seed + 3, m, n).to(td)
    gd, d = matrix(m, n, n + pad, td, start)
    p = A.MatmulParams(m, n, k, FORMATS.index(fa), FORMATS.index(fb), code_of(A, td), accumulate, n + pad)
    ws = gpu_util.Guarded(torch, A.accept_matmul_workspace_size(p), 0)
    A.accept_block_matmul(p, a, sa, b, sb, bias, d, ws.bytes)
    assert A.accept_last_device_status(ws.bytes) == 0
    gd.check("d"), ws.check("workspace")
    assert gaps_untouched(gd, m, n, n + pad, td)
    va, vb = plain.decode(a, sa, fa, k), plain.decode(b, sb, fb, k)
    want, size = va @ vb.t(), va.abs() @ vb.abs().t()
    if bias is not None:
        want, size = want + bias.double(), size + bias.double().abs()
    if accumulate:
        want, size = want + start.double(), size + start.double().abs()
    # one addition for each 32 products and some to join parts, each off by at most one unit in the last place
    tol = 2 * plain.E32 * (k / 32 + 16) * size
    tol = tol + plain.UNIT[td] * want.abs() + plain.SMALLEST[td]
    overflow = (want.abs() + tol >= torch.finfo(td).max) & (d.double() == want.sign() * float("inf"))  # past the type's largest value
    assert bool((((d.double() - want).abs() <= tol) | overflow).all())
    assert bool(torch.isfinite(d[want.abs() + tol < torch.finfo(td).max]).all())
    first = d.clone()
    d.copy_(start)
    A.accept_block_matmul(p, a, sa, b, sb, bias, d, ws.bytes)
    torch.cuda.synchronize()
    assert torch.equal(first, d)  # the same bits again


@pytest.mark.parametrize("case", PRODUCTS, ids=str)
def test_product(A, case):
    check_product(A, *case)


def test_product_sums_are_single_precision(A):
    """Sums over 16384 values of k keep the accuracy of fp32 sums: within 10^-6 of the result's norm, ten times the
    square root of the number of additions per partial sum times a rounding."""
    a, sa = coded(1, 256, 16384, "e4m3", spread=0)
    b, sb = coded(2, 384, 16384, "e4m3", spread=0)
    d = torch.empty(256, 384, device="cuda")
    p = A.MatmulParams(256, 384, 16384, dtype_d=A.DTYPE_F32)
    A.accept_block_matmul(p, a, sa, b, sb, None, d, A.new_workspace(p))
    want = plain.decode(a, sa, "e4m3", 16384) @ plain.decode(b, sb, "e4m3", 16384).t()
    assert float((d.double() - want).norm() / want.norm()) < 1e-6


def test_product_of_nothing(A):
    some = torch.zeros(512, dtype=torch.uint8, device="cuda")
    ws = torch.zeros(4, dtype=torch.int32, device="cuda")
    before = A.accept_launch_count()
    for m, n in ((0, 3), (3, 0)):
        A.accept_block_matmul(A.MatmulParams(m, n, 16), some, some, some, some, None, some, ws)
    assert A.accept_launch_count() == before
    bias = random(1, 5)
    d = torch.full((3, 5), 2.0, device="cuda")
    A.accept_block_matmul(A.MatmulParams(3, 5, 0, dtype_d=A.DTYPE_F32, accumulate=True), some, some, some, some, bias, d, ws)
    assert torch.equal(d, 2.0 + bias.expand(3, 5))
    A.accept_block_matmul(A.MatmulParams(3, 5, 0, dtype_d=A.DTYPE_F32), some, some, some, some, None, d, ws)
    assert bool((d == 0).all())


def test_product_with_scales_at_the_ends_and_bad_codes(A):
    """Scale bytes 0 and 200, and a NaN code that reaches its own row alone."""
    a, sa = coded(1, 140, 256, "e4m3", spread=0)
    b, sb = coded(2, 130, 256, "e4m3", spread=0)
    sa[plain.place(7, 0, 140)] = 0
    sa[plain.place(7, 1, 140)] = 0
    sa[plain.place(139, 1, 140)] = 200
    a[77, 200] = 0x7F
    p = A.MatmulParams(140, 130, 256, dtype_d=A.DTYPE_F32)
    d = torch.empty(140, 130, device="cuda")
    A.accept_block_matmul(p, a, sa, b, sb, None, d, A.new_workspace(p))
    want = plain.decode(a, sa, "e4m3", 256) @ plain.decode(b, sb, "e4m3", 256).t()
    size = plain.decode(a, sa, "e4m3", 256).abs() @ plain.decode(b, sb, "e4m3", 256).abs().t()
    assert bool(torch.isnan(d[77]).all()) and not bool(torch.isnan(torch.cat([d[:77], d[78:]])).any())
    good = [r for r in range(140) if r != 77]
    assert bool(((d.double() - want)[good].abs() <= (2 * plain.E32 * 24 * size + 1e-45)[good]).all())


def test_linear_layer_gradients_are_the_products_differences(A):
    """y = x W^T is linear in each coded value: moving one code moves y by the other operand's values, which is what
    the two gradient products (b by columns; both by columns) must contract."""
    m, n, k = 70, 140, 260
    x, w, dy = random(1, m, k), random(2, n, k, scale=0.1), random(3, m, n)
    qx, qw, qd = A.QuantizeParams(m, k), A.QuantizeParams(n, k, block=A.BLOCK_SQUARE), A.QuantizeParams(m, n)

    def code(p, t):
        bufs = [torch.zeros(size(p, side), dtype=torch.uint8, device="cuda") for side in (False, True) for size in (A.accept_block_data_size, A.accept_block_scale_size)]
        A.accept_block_quantize(p, t, *bufs, A.new_workspace(p))
        return bufs

    bx, bw, bd = code(qx, x), code(qw, w), code(qd, dy)

    def product(rows, cols, inner, a, sa, b, sb):
        p = A.MatmulParams(rows, cols, inner, dtype_d=A.DTYPE_F32)
        d = torch.empty(rows, cols, device="cuda")
        A.accept_block_matmul(p, a, sa, b, sb, None, d, A.new_workspace(p))
        return d

    y = product(m, n, k, bx[0], bx[1], bw[0], bw[1])
    dx = product(m, k, n, bd[0], bd[1], bw[2], bw[3])
    dw = product(n, k, m, bd[2], bd[3], bx[2], bx[3])
    vw = plain.decode(bw[0].view(n, -1), bw[1], "e4m3", k)
    assert torch.equal(plain.decode(bw[2].view(k, -1), bw[3], "e4m3", n).t(), vw)  # square blocks: one set of values both ways
    vd_rows, vd_cols = plain.decode(bd[0].view(m, -1), bd[1], "e4m3", n), plain.decode(bd[2].view(n, -1), bd[3], "e4m3", m).t()
    vx_cols = plain.decode(bx[2].view(k, -1), bx[3], "e4m3", m).t()
    for r, c in [(0, 0), (69, 259), (33, 128)]:
        moved = bx[0].clone().view(m, -1)
        moved[r, c] = 0x38  # one
        scale = 2.0 ** (float(bx[1][plain.place(r, c // 128, m)]) - 127)
        step = scale - float(plain.decode(bx[0].view(m, -1), bx[1], "e4m3", k)[r, c])
        moved_y = product(m, n, k, moved.view(-1), bx[1], bw[0], bw[1])
        difference = float(((moved_y.double() - y.double()) * vd_rows).sum()) / step
        noise = 4 * plain.E32 * float((y.double().abs() * vd_rows.abs())[r].sum()) * 24 / abs(step) + 1e-4
        assert abs(difference - float(dx[r, c])) <= noise
    assert bool(((dw.double() - vd_cols.t() @ vx_cols).abs() <= 2 * plain.E32 * 24 * (vd_cols.abs().t() @ vx_cols.abs())).all())


# ---- streams, the checking build, waits that run out ---------------------------------------------------------------

def test_operators_run_on_the_stream_they_are_given(A):
    side = torch.cuda.Stream()
    x = random(1, 300, 1024)
    p, q = A.LayerNormParams(300, 1024), A.QuantizeParams(300, 1024)
    y = torch.empty_like(x)
    bufs = [torch.zeros(size(q, False), dtype=torch.uint8, device="cuda") for size in (A.accept_block_data_size, A.accept_block_scale_size)]
    ws, wq = A.new_workspace(p), A.new_workspace(q)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        x2 = x * 2  # ordered before the operators on the side stream only
        A.accept_layer_norm_forward(p, x2, None, None, y)
        A.accept_block_quantize(q, y, bufs[0], bufs[1], None, None, wq)
    side.synchronize()
    want, _, _ = plain.norm(x.double() * 2, None, None, 1e-5)
    assert float((plain.decode(bufs[0].view(300, -1), bufs[1], "e4m3", 1024) - want).abs().max()) <= 0.3
    assert float((y.double() - want).abs().max()) < 1e-5
    assert ws is not None


def test_operators_stay_inside_their_buffers(A):
    with gpu_util.library_variant("bounds"):
        assert A.accept_bounds_check_report()[:2] == (0, 0)
        for case in NORMS:
            check_norm_grad(A, *case)
        assert A.accept_bounds_check_report()[:2] == (0, 0), "layer norm"
        for rows, cols, pad, dtype, fmt, square in BLOCKS:
            check_quantize(A, random(1, rows, cols).to(dtype), pad, fmt, square)
        assert A.accept_bounds_check_report()[:2] == (0, 0), "block quantisation"
        for case in PRODUCTS:
            check_product(A, *case)
        code, count, addr, size, write = A.accept_bounds_check_report()
        assert (code, count) == (0, 0), f"product: {count} accesses outside, first at {addr:#x} ({size} bytes, write={write})"


@pytest.mark.parametrize("m,n,k", [(4, 300, 4096), (300, 300, 2000), (2304, 2304, 1024)])
def test_product_whose_copies_do_not_arrive_reports_it_and_leaves_the_gpu_usable(A, m, n, k):
    a, sa = coded(1, m, k, "e4m3")
    b, sb = coded(2, n, k, "e4m3")
    p = A.MatmulParams(m, n, k)
    d, ws = torch.zeros(m, n, dtype=BF16, device="cuda"), A.new_workspace(p)
    with gpu_util.library_variant("stall"):
        A.accept_block_matmul(p, a, sa, b, sb, None, d, ws)
        assert A.accept_last_device_status(ws) == A.DEV_COPY_TIMEOUT
    check_product(A, m, n, k, "e4m3", "e4m3", BF16, True, False, 0)


# ---- the operators together ------------------------------------------------------------------------------------------

@pytest.mark.parametrize("tokens,width,features", [(256, 512, 384), (130, 328, 200)])
def test_linear_stage_step(tokens, width, features):
    """A training step of the example: 8-bit operands (E4M3: 2^-4 relative rounding at most, a third of that on average;
    E5M2: twice that) leave the products within 10 %, gradients of sums over tokens included."""
    from examples import linear_stage
    errors = linear_stage.run(tokens, width, features, seed=3)
    assert set(errors) == {"y", "dx", "dweight", "dgamma", "dbeta"}
    assert max(errors.values()) < 0.1, errors
