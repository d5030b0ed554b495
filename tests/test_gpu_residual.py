"""Dropout and the root-mean-square norm of a residual stream against 64-bit plain forms, through the C ABI.

What is dropped, and the sum that is kept, are compared bit for bit: the definition names each fp32 operation.  The tolerances of the
rest count roundings on the way (E32 = 2^-24 each, of the magnitudes that are added), plus one to the output's type.
"""
import pytest

from tests import gpu_util
from tests import operators_plain as plain8
from tests import residual_plain as plain
from tests.test_gpu_operators import code_of, gaps_untouched, matrix, random

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
BIG = (1 << 64) - 50  # counters that wrap


@pytest.fixture(scope="module")
def A():
    import paper_2311_05827_b200 as pkg
    return pkg


def same(a, b):
    """Equal bits, but that -0 is 0 and a NaN a NaN."""
    return bool(((a == b) | (torch.isnan(a) & torch.isnan(b))).all())


# ---- dropout ----------------------------------------------------------------------------------------------------------

# rows, cols, extra values between rows of x and of y, offset of x in its buffer, types, residual, p, first counter
DROPS = [
    (1, 1, 0, 0, 0, F32, F32, False, 0.5, 0), (3, 2, 0, 0, 0, BF16, F32, True, 0.5, 1), (2, 7, 1, 0, 0, F16, F16, False, 0.25, 3),
    (5, 33, 0, 3, 0, F32, BF16, True, 0.1, 2), (77, 1001, 0, 0, 0, BF16, BF16, False, 0.1, 77077), (64, 4096, 0, 0, 0, BF16, F32, True, 0.1, 0),
    (64, 4096, 8, 8, 0, BF16, BF16, True, 0.1, 6), (40, 1030, 2, 0, 0, F16, F32, False, 0.9, (1 << 34) - 1000), (300, 9, 0, 1, 1, F32, F16, True, 0.3, BIG),
    (1, 5000, 0, 0, 3, F16, BF16, False, 0.05, BIG), (1000, 100, 12, 4, 0, F32, F32, True, 0.2, (1 << 34) * 3 - 50001), (129, 515, 0, 0, 0, F32, F32, False, 1.0, 5),
    (20, 300, 0, 0, 0, BF16, F16, True, 0.0, 5), (20, 300, 0, 0, 0, F32, F32, True, 2.0 ** -25, 9), (33, 1000, 0, 0, 0, BF16, BF16, True, 1 - 2.0 ** -24, 1 << 63),
    (5003, 1537, 7, 7, 0, F16, F16, True, 0.1, 3),
]


@pytest.mark.parametrize("case", DROPS, ids=str)
def test_dropout(A, case):
    check_dropout(A, *case)


def check_dropout(A, rows, cols, pad_x, pad_y, offset, tx, ty, residual, rate, first, seed=0x1234567890ABCDEF):
    gx, x = matrix(rows, cols, cols + pad_x, tx, random(rows, rows, cols), offset)
    gy, y = matrix(rows, cols, cols + pad_y, ty)
    _, r = matrix(rows, cols, cols + pad_y, ty, random(cols, rows, cols)) if residual else (None, None)
    p = A.DropoutParams(rows, cols, rate, code_of(A, tx), code_of(A, ty), seed, first, cols + pad_x, cols + pad_y)
    A.accept_dropout(p, x, r, y)
    torch.cuda.synchronize()
    want = plain.dropped32(x, rate, seed, first)
    if residual:
        want = want + r.float()
    assert same(y, want.to(ty))
    gx.check("x"), gy.check("y")
    assert gaps_untouched(gy, rows, cols, cols + pad_y, ty)
    # the gradient is the same call on dy: what was dropped has none
    gdx, dx = matrix(rows, cols, cols + pad_x, tx)
    _, dy = matrix(rows, cols, cols + pad_y, ty, random(7, rows, cols))
    A.accept_dropout(A.DropoutParams(rows, cols, rate, code_of(A, ty), code_of(A, tx), seed, first, cols + pad_y, cols + pad_x), dy, None, dx)
    assert same(dx, plain.dropped32(dy, rate, seed, first).to(tx))
    gdx.check("dx")


def test_dropout_keeps_its_share_and_takes_fresh_numbers(A):
    """Of 2^20 values about (1 - p) are kept: within six standard deviations; calls with the next counters drop others."""
    n, rate = 1 << 20, 0.3
    x, y, z = torch.ones(n, device="cuda"), torch.empty(n, device="cuda"), torch.empty(n, device="cuda")
    A.accept_dropout(A.DropoutParams(1, n, rate, seed=11), x, None, y)
    A.accept_dropout(A.DropoutParams(1, n, rate, seed=11, rng_offset=n), x, None, z)
    sd = (n * rate * (1 - rate)) ** 0.5
    assert abs(int((y > 0).sum()) - n * (1 - rate)) < 6 * sd and abs(int((z > 0).sum()) - n * (1 - rate)) < 6 * sd
    both = int(((y > 0) & (z > 0)).sum())
    assert abs(both - n * (1 - rate) ** 2) < 6 * (n * 0.49 * 0.51) ** 0.5


def test_dropout_of_bad_values_and_in_place(A):
    rows, cols, rate = 30, 200, 0.5
    keep = plain.kept(rows, cols, rate, 3, 4)
    for tx in (F32, BF16, F16):
        x = random(1, rows, cols).to(tx)
        x[3], x[4], x[5] = float("nan"), float("inf"), torch.finfo(tx).max
        p = A.DropoutParams(rows, cols, rate, code_of(A, tx), code_of(A, tx), 3, 4)
        want = plain.dropped32(x, rate, 3, 4).to(tx)
        assert bool((want[~keep] == 0).all())
        y = x.clone()
        A.accept_dropout(p, y, None, y)
        assert same(y, want)
        y = x.clone()
        A.accept_dropout(p, x, y, y)  # the residual's place
        assert same(y, (plain.dropped32(x, rate, 3, 4) + x.float()).to(tx))
    before = A.accept_launch_count()
    A.accept_dropout(A.DropoutParams(0, 5, 0.1), x, None, x)
    A.accept_dropout(A.DropoutParams(5, 0, 0.1), x, None, x)
    assert A.accept_launch_count() == before


# ---- the root-mean-square norm ------------------------------------------------------------------------------------------

# rows, cols, extra values between rows of x and of y, offset of x in its buffer, types of x, y, weights, branch, p, first counter
NORMS = [
    (1, 1, 0, 0, 0, F32, F32, F32, False, 0.0, 0), (3, 2, 0, 0, 0, BF16, F32, BF16, True, 0.5, 1), (2, 7, 1, 0, 0, F16, F16, F16, True, 0.0, 0),
    (5, 33, 0, 3, 0, F32, BF16, F32, True, 0.1, 6), (9, 256, 0, 0, 0, BF16, BF16, BF16, False, 0.0, 0), (17, 257, 7, 7, 0, F16, F32, F32, True, 0.2, BIG),
    (8, 512, 0, 0, 1, F32, F32, F32, True, 0.1, 0), (33, 513, 0, 0, 0, F32, F16, F16, True, 0.1, (1 << 34) - 4000), (6, 1000, 24, 8, 0, BF16, BF16, F32, True, 0.1, 0),
    (300, 1024, 0, 0, 0, F32, F32, F32, False, 0.0, 0), (700, 1537, 7, 7, 0, F16, F16, F32, True, 0.1, 3), (40, 2047, 1, 1, 0, F16, F16, F16, False, 0.0, 0),
    (41, 2056, 0, 0, 0, BF16, F32, F32, True, 0.3, 2), (1200, 4096, 0, 0, 0, BF16, BF16, F32, True, 0.1, 0), (65, 4096, 0, 0, 3, F32, BF16, BF16, True, 0.1, 5),
    (12, 4104, 0, 0, 0, F32, BF16, F32, True, 0.0, 0), (10, 8192, 0, 0, 0, BF16, BF16, BF16, True, 0.1, (1 << 34) - 10000), (7, 8200, 0, 1, 0, F32, F32, F32, True, 0.1, 7),
    (5, 16384, 0, 0, 0, F16, BF16, F32, True, 0.1, 0), (3, 16391, 0, 0, 0, F32, F32, F32, True, 0.5, (1 << 34) - 20000), (70, 20000, 0, 0, 0, BF16, F16, BF16, False, 0.0, 0),
    (2, 40000, 0, 0, 0, F32, F32, F32, True, 0.1, 1), (5000, 64, 0, 0, 0, BF16, BF16, BF16, True, 0.1, 0), (3001, 128, 0, 0, 0, BF16, BF16, F32, True, 0.0, 0),
    (700, 100, 8, 8, 0, F32, BF16, F32, True, 0.1, 4), (601, 127, 0, 0, 1, F16, F16, F16, True, 0.1, 3), (1100, 9001, 0, 0, 0, BF16, BF16, F32, True, 0.1, 0),
    (600, 8200, 0, 0, 0, F32, F32, F32, False, 0.0, 0), (50, 1030, 0, 0, 0, BF16, BF16, BF16, True, 0.1, 0), (33, 2051, 1, 3, 2, F16, F16, F16, True, 0.1, 0),
    (31, 1031, 0, 0, 0, BF16, BF16, F32, False, 0.0, 0), (400, 98, 0, 0, 0, BF16, BF16, BF16, True, 0.1, 0), (20, 515, 0, 1, 0, F32, BF16, F32, True, 0.1, 0),
    (20, 515, 2, 0, 1, F32, F32, F32, True, 1.0, 0), (9, 8190, 0, 0, 0, F16, BF16, F16, True, 0.1, 0), (2000, 1000, 0, 0, 0, F32, BF16, F32, True, 0.1, 0),
    (260, 1500, 0, 0, 0, F16, F32, F16, True, 0.1, 0), (1000, 130, 0, 0, 0, BF16, F16, F32, True, 0.1, 0),
]


def stage(A, rows, cols, pad_x, pad_y, offset, tx, ty, tw, branch, rate, first, weights=True, eps=1e-5, x=None, b=None, seed=99):
    """Inputs of a case and its parameters."""
    if x is None:
        x = random(rows, rows, cols) * (0.1 + 3 * torch.rand(cols, device="cuda")) + 0.3
    if b is None:
        b = random(rows + 1, rows, cols)
    gx, vx = matrix(rows, cols, cols + pad_x, tx, x, offset)
    _, vb = matrix(rows, cols, cols + pad_y, ty, b) if branch else (None, None)
    gamma = (1 + 0.3 * random(cols, cols)).to(tw) if weights else None
    p = lambda fmt=0: A.RmsNormParams(rows, cols, eps, code_of(A, tx), code_of(A, ty), code_of(A, tw), rate, seed, first, fmt, cols + pad_x, cols + pad_y)  # noqa: E731
    return p, vx, vb, gamma


def rounds(cols):
    """Roundings of a row's sum: at most 64 a thread and a tree, more where a thread walks a longer row; rsqrt and the eps beside it."""
    return 72 + cols / 1024


def check_codes(A, q, scale, y, fmt, rows, cols, off):
    """Codes and scale bytes against y in 64 bits, each value of which is off by `off` relatively at most."""
    bits, low, top = (3, -6, 448.0) if fmt == 0 else (2, -14, 57344.0)
    blocks = -(-cols // 128)
    wide = torch.zeros(rows, blocks * 128, dtype=torch.float64, device="cuda")
    wide[:, :cols] = y
    most = wide.abs().view(rows, blocks, 128).amax(2)
    r, b = torch.arange(rows, device="cuda")[:, None], torch.arange(blocks, device="cuda")[None]
    e = scale[plain.place(r, b, rows)].double() - 127
    two = torch.ldexp(torch.ones_like(most), e.int())
    assert bool((((most / two <= top * (1 + off)) & (most / two * 2 >= top * (1 - off))) | (most == 0) | (e == -127)).all())
    held = plain8.up(cols, 16)
    v = q.view(torch.float8_e4m3fn if fmt == 0 else torch.float8_e5m2).float().double()
    two = two.repeat_interleave(128, 1)[:, :held]
    t = wide[:, :held] / two
    step = torch.ldexp(torch.ones_like(t), (torch.frexp(t)[1] - 1).clamp(min=low) - bits)
    assert bool(((v - t).abs() <= 0.5 * step + off * t.abs()).all())
    assert bool((q[:, cols:] == 0).all())
    rest = torch.ones(scale.numel(), dtype=torch.bool, device="cuda")
    rest[plain.place(r, b, rows)] = False
    assert bool((scale[rest] == 127).all())


def check_norm(A, case, **more):
    rows, cols, pad_x, pad_y, offset, tx, ty, tw, branch, rate, first = case
    p, x, b, gamma = stage(A, *case, **more)
    seed, eps = more.get("seed", 99), more.get("eps", 1e-5)
    gs, s = matrix(rows, cols, cols + pad_x, tx, None, offset)
    gy, y = matrix(rows, cols, cols + pad_y, ty)
    rstd = gpu_util.guarded_floats(torch, rows)
    A.accept_rms_norm_forward(p(), x, b, gamma, s, y, None, None, rstd.view(F32))
    torch.cuda.synchronize()
    want = x if b is None else (x.float() + plain.dropped32(b, rate, seed, first)).to(tx)
    assert same(s, want)
    wy, wr = plain.rms(s, gamma, eps)
    off = rounds(cols) * plain.E32
    assert bool(((rstd.view(F32).double() - wr).abs() <= off * wr + 2.0 ** -149).all())
    assert bool(((y.double() - wy).abs() <= (off + 4 * plain.E32) * wy.abs() + plain8.UNIT[ty] * wy.abs() + plain8.SMALLEST[ty]).all())
    for name, buf in (("sum", gs), ("y", gy), ("rstd", rstd)):
        buf.check(name)
    assert gaps_untouched(gs, rows, cols, cols + pad_x, tx, offset) and gaps_untouched(gy, rows, cols, cols + pad_y, ty)
    # 8-bit codes, alone and beside the other outputs
    size = A.QuantizeParams(rows, cols)
    for fmt in (0, 1):
        q, scale = gpu_util.Guarded(torch, A.accept_block_data_size(size), 0xA7), gpu_util.Guarded(torch, A.accept_block_scale_size(size), 0xA7)
        ws = gpu_util.Guarded(torch, 16, 0)
        A.accept_rms_norm_forward(p(fmt), x, b, gamma, None, None, q.bytes, scale.bytes, None, ws.bytes)
        torch.cuda.synchronize()
        check_codes(A, q.bytes.view(rows, -1), scale.bytes, wy, fmt, rows, cols, off + 4 * plain.E32)
        for buf in (q, scale, ws):
            buf.check()
        assert int(ws.bytes.sum()) == 0
        again = [t.clone() for t in (q.bytes, scale.bytes)]
        s2, y2, r2 = torch.empty_strided(s.shape, s.stride(), dtype=tx, device="cuda"), torch.empty_strided(y.shape, y.stride(), dtype=ty, device="cuda"), torch.empty(rows, device="cuda")
        A.accept_rms_norm_forward(p(fmt), x, b, gamma, s2, y2, q.bytes, scale.bytes, r2, ws.bytes)
        assert torch.equal(s2, s) and torch.equal(y2, y) and torch.equal(r2, rstd.view(F32))
        assert all(torch.equal(u, v) for u, v in zip(again, (q.bytes, scale.bytes)))
        if ty == F32:  # y is not rounded before: the codes are the quantiser's
            qq = [torch.empty_like(t) for t in again]
            y3 = y.contiguous()
            A.accept_block_quantize(A.QuantizeParams(rows, cols, format=fmt), y3, qq[0], qq[1], None, None, ws.bytes)
            assert all(torch.equal(u, v) for u, v in zip(again, qq))
    return p, s, gamma, rstd.view(F32)


def check_norm_grad(A, case, **more):
    rows, cols, pad_x, pad_y, offset, tx, ty, tw, branch, rate, first = case
    p, s, gamma, rstd = check_norm(A, case, **more)
    seed = more.get("seed", 99)
    _, dy = matrix(rows, cols, cols + pad_y, ty, random(5, rows, cols, scale=0.1))
    _, dsum = matrix(rows, cols, cols + pad_x, tx, random(6, rows, cols, scale=0.1)) if branch else (None, None)
    gdx, dx = matrix(rows, cols, cols + pad_x, tx, None, offset)
    gdb, db = matrix(rows, cols, cols + pad_y, ty)
    dgamma = gpu_util.guarded_floats(torch, cols)
    ws = gpu_util.Guarded(torch, A.accept_rms_norm_workspace_size(p()), 0xEE)
    call = lambda a, b, c: A.accept_rms_norm_backward(p(), dy, s, gamma, rstd, dsum, a, b, c, ws.bytes)  # noqa: E731
    call(dx, db, dgamma.view(F32))
    torch.cuda.synchronize()
    want, wg, size, size_g = plain.rms_grad(dy, s, gamma, rstd, dsum)
    off = rounds(cols) * plain.E32
    assert bool(((dx.double() - want).abs() <= off * size + plain8.UNIT[tx] * want.abs() + plain8.SMALLEST[tx]).all())
    keep = plain.kept(rows, cols, rate, seed, first) if rate > 0 else torch.ones_like(dx, dtype=torch.bool)
    scale = 1 / (1 - plain.single(rate)) if plain.single(rate) < 1 else 0.0
    wb = torch.where(keep, want * scale, 0.0)
    assert bool(((db.double() - wb).abs() <= (off * size + 4 * plain.E32 * want.abs()) * scale + plain8.UNIT[ty] * wb.abs() + plain8.SMALLEST[ty]).all())
    assert bool((db[~keep] == 0).all())
    m = 64 + rows                                                        # at most one rounding a row, and a few of xhat
    assert bool(((dgamma.view(F32).double() - wg).abs() <= m * plain.E32 * size_g + 1e-45).all())
    for name, buf in (("dx", gdx), ("dbranch", gdb), ("dgamma", dgamma), ("workspace", ws)):
        buf.check(name)
    assert gaps_untouched(gdx, rows, cols, cols + pad_x, tx, offset) and gaps_untouched(gdb, rows, cols, cols + pad_y, ty)
    # the same bits again, and in the calls that ask for one output alone
    first_bits = [t.clone() for t in (dx, db, dgamma.view(F32))]
    dx.zero_(), db.zero_(), dgamma.view(F32).zero_()
    call(dx, None, None)
    call(None, db, None)
    call(None, None, dgamma.view(F32))
    torch.cuda.synchronize()
    for a, b in zip(first_bits, (dx, db, dgamma.view(F32))):
        assert torch.equal(a, b)


@pytest.mark.parametrize("case", NORMS, ids=str)
def test_norm_forward_and_backward(A, case):
    check_norm_grad(A, case)


def test_norm_without_weights_and_without_rows(A):
    check_norm_grad(A, (19, 777, 0, 0, 0, F32, F32, F32, True, 0.1, 0), weights=False)
    p = A.RmsNormParams(0, 100)
    ws, dgamma = A.new_workspace(p), torch.ones(100, device="cuda")
    nothing = torch.empty(0, 100, device="cuda")
    before = A.accept_launch_count()
    A.accept_rms_norm_forward(p, nothing, None, None, None, nothing)
    assert A.accept_launch_count() == before
    A.accept_rms_norm_backward(p, nothing, nothing, None, nothing, None, None, None, dgamma, ws)
    assert bool((dgamma == 0).all())
    wide = A.RmsNormParams(0, 10000)
    dgamma = torch.ones(10000, device="cuda")
    A.accept_rms_norm_backward(wide, nothing, nothing, None, nothing, None, None, None, dgamma, A.new_workspace(wide))
    assert bool((dgamma == 0).all())


@pytest.mark.parametrize("cols", [100, 1500, 9000])
def test_norm_of_rows_past_the_range_of_squares(A, cols):
    """Values from 2^-100 to 2^126: their squares are not fp32 values, y is."""
    x = random(1, 8, cols)
    for i, e in enumerate((126, 100, 65, 40, -40, -70, -100, 0)):
        x[i] *= 2.0 ** (e - 3 if e > 120 else e)
    for tx in (F32, BF16):
        for eps in (0.0, 1e-5):
            case = (8, cols, 0, 0, 0, tx, F32, F32, False, 0.0, 0)
            p, vx, _, gamma = stage(A, *case, eps=eps, x=x)
            y, rstd = torch.empty(8, cols, device="cuda"), torch.empty(8, device="cuda")
            A.accept_rms_norm_forward(p(), vx, None, gamma, None, y, None, None, rstd)
            wy, wr = plain.rms(vx, gamma, eps)
            off = rounds(cols) * plain.E32
            # rstd may be a subnormal: half of the smallest step beside the relative error
            assert bool(((rstd.double() - wr).abs() <= off * wr + 2.0 ** -150).all())
            tol = (off + 6 * plain.E32) * wy.abs() + 2.0 ** -149 * vx.double().abs() * (gamma.double().abs() + 1) + 2.0 ** -149
            assert bool(((y.double() - wy).abs() <= tol).all())


@pytest.mark.parametrize("cols", [100, 1500, 9000])
def test_norm_of_bad_rows(A, cols):
    x = random(1, 200, cols)
    x[3, 7], x[50, 0], x[60] = float("nan"), float("inf"), 0.0
    p, vx, _, gamma = stage(A, 200, cols, 0, 0, 0, BF16, F32, F32, False, 0.0, 0, x=x)
    y, rstd = torch.empty(200, cols, device="cuda"), torch.empty(200, device="cuda")
    size = A.QuantizeParams(200, cols)
    q, scale, ws = (torch.empty(n, dtype=torch.uint8, device="cuda") for n in (A.accept_block_data_size(size), A.accept_block_scale_size(size), 16))
    ws.zero_()
    A.accept_rms_norm_forward(p(), vx, None, gamma, None, y, q, scale, rstd, ws)
    assert A.accept_last_device_status(ws) == A.DEV_NONFINITE
    assert bool(torch.isnan(y[3]).all()) and bool(torch.isnan(y[50, 0])) and bool((y[50, 1:] == 0).all()) and bool((y[60] == 0).all())
    rest = [i for i in range(200) if i not in (3, 50, 60)]
    assert bool(torch.isfinite(y[rest]).all())
    want = [torch.empty_like(t) for t in (q, scale)]
    A.accept_block_quantize(size, y, want[0], want[1], None, None, ws)
    assert torch.equal(q, want[0]) and torch.equal(scale, want[1])


@pytest.mark.parametrize("tx,ty", [(F32, F32), (BF16, BF16)])
@pytest.mark.parametrize("rows,cols", [(30, 1000), (700, 77), (400, 9000)])
def test_norm_in_place(A, rows, cols, tx, ty):
    """sum in x's place, y in the branch's; dx in that of s or dsum, dbranch in dy's."""
    case = (rows, cols, 0, 0, 0, tx, ty, F32, True, 0.1, 0)
    p, x, b, gamma = stage(A, *case)
    s, y, rstd = torch.empty_like(x), torch.empty_like(b), torch.empty(rows, device="cuda")
    A.accept_rms_norm_forward(p(), x, b, gamma, s, y, None, None, rstd)
    x2, b2 = x.clone(), b.clone()
    A.accept_rms_norm_forward(p(), x2, b2, gamma, x2, b2)
    assert torch.equal(x2, s) and torch.equal(b2, y)
    dy, dsum = random(3, rows, cols).to(ty), random(4, rows, cols).to(tx)
    dx, db, dg, ws = torch.empty_like(x), torch.empty_like(b), torch.empty(cols, device="cuda"), A.new_workspace(p())
    A.accept_rms_norm_backward(p(), dy, s, gamma, rstd, dsum, dx, db, dg, ws)
    for place in ("s", "dsum"):
        s2, dsum2, dy2, dg2 = s.clone(), dsum.clone(), dy.clone(), torch.empty_like(dg)
        into = s2 if place == "s" else dsum2
        A.accept_rms_norm_backward(p(), dy2, s2, gamma, rstd, dsum2, into, dy2, dg2, ws)
        assert torch.equal(into, dx) and torch.equal(dy2, db) and torch.equal(dg2, dg)


def test_norm_gradient_is_that_of_differences(A):
    """dx and dbranch against differences of the 64-bit forward form with the library's own mask: sum(dy y + dsum s) moves by the gradient
    where one value of x or of the branch moves (central differences, h = 1e-4: off by h^2 and rounding of dx)."""
    rows, cols, rate = 6, 50, 0.3
    p, x, b, gamma = stage(A, rows, cols, 0, 0, 0, F32, F32, F32, True, rate, 8)
    s, y, rstd = torch.empty_like(x), torch.empty_like(b), torch.empty(rows, device="cuda")
    A.accept_rms_norm_forward(p(), x, b, gamma, s, y, None, None, rstd)
    dy, dsum = random(3, rows, cols), random(4, rows, cols)
    dx, db, dg = torch.empty_like(x), torch.empty_like(b), torch.empty(cols, device="cuda")
    A.accept_rms_norm_backward(p(), dy, s, gamma, rstd, dsum, dx, db, dg, A.new_workspace(p()))
    keep = plain.kept(rows, cols, rate, 99, 8).double() / (1 - plain.single(rate))

    def loss(x, b, g):
        s = x + b * keep
        y = s / torch.sqrt(s.square().mean(1, keepdim=True) + 1e-5) * g
        return float((dy.double() * y + dsum.double() * s).sum())

    x, b, g, h = x.double(), b.double(), gamma.double(), 1e-4
    for r, c in ((0, 0), (2, 31), (5, 49), (3, 7)):
        for i, grad in enumerate((dx, db, dg)):
            ends = []
            for sign in (1, -1):
                args = [x.clone(), b.clone(), g.clone()]
                args[i][(r, c) if i < 2 else c] += sign * h
                ends.append(loss(*args))
            got = float(grad[r, c] if i < 2 else grad[c])
            assert abs((ends[0] - ends[1]) / (2 * h) - got) <= 1e-5 * (1 + abs(got))


# ---- streams, graphs, the checking build --------------------------------------------------------------------------------------

def test_residual_operators_run_on_their_stream_and_in_graphs(A):
    rows, cols = 300, 1024
    case = (rows, cols, 0, 0, 0, F32, BF16, F32, True, 0.1, 0)
    p, x, b, gamma = stage(A, *case)
    outs = [torch.empty_like(x), torch.empty_like(b), torch.empty(rows, device="cuda")]
    grads = [torch.empty_like(x), torch.empty_like(b), torch.empty(cols, device="cuda")]
    drop = A.DropoutParams(rows, cols, 0.2, A.DTYPE_F32, A.DTYPE_F32, 5)
    dropped, ws = torch.empty_like(x), A.new_workspace(p())

    def step(x):
        A.accept_rms_norm_forward(p(), x, b, gamma, outs[0], outs[1], None, None, outs[2])
        A.accept_rms_norm_backward(p(), outs[1], outs[0], gamma, outs[2], x, *grads, ws)
        A.accept_dropout(drop, grads[0], x, dropped)

    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        x2 = x * 2  # ordered before the operators on the side stream only
        step(x2)
    side.synchronize()
    want = [t.clone() for t in outs + grads + [dropped]]
    assert same(want[0], x * 2 + plain.dropped32(b, 0.1, 99, 0))
    for t in outs + grads + [dropped]:
        t.zero_()
    graph = torch.cuda.CUDAGraph()
    held = x * 2
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        step(held)
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    for u, v in zip(want, outs + grads + [dropped]):
        assert torch.equal(u, v)


def test_residual_operators_stay_inside_their_buffers(A):
    with gpu_util.library_variant("bounds"):
        assert A.accept_bounds_check_report()[:2] == (0, 0)
        for case in DROPS:
            check_dropout(A, *case)
        assert A.accept_bounds_check_report()[:2] == (0, 0), "dropout"
        for case in NORMS:
            check_norm_grad(A, case)
        code, count, addr, size, write = A.accept_bounds_check_report()
        assert (code, count) == (0, 0), f"norm: {count} accesses outside, first at {addr:#x} ({size} bytes, write={write})"
