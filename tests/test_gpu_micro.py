"""4-bit floating point with a scale for each 32 values: codes, values and products against 64-bit plain forms, through the C ABI.

Codes and scale bytes are compared bit for bit, stochastic rounding included; a product's tolerance counts the additions of its sums.
"""
import pytest

from tests import gpu_util
from tests import operators_plain as plain8
from tests import residual_plain as plain
from tests.test_gpu_operators import code_of, gaps_untouched, matrix, random

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def A():
    import paper_2311_05827_b200 as pkg
    return pkg


# ---- codes ------------------------------------------------------------------------------------------------------------------

# rows, cols, extra values between rows, offset of x in its buffer, type, square blocks
BLOCKS = [
    (1, 1, 0, 0, F32, False), (1, 31, 0, 0, BF16, True), (33, 33, 0, 0, F16, False), (32, 64, 0, 0, F32, True), (128, 128, 0, 0, BF16, False),
    (129, 257, 7, 0, F32, False), (130, 1000, 24, 0, BF16, True), (77, 4096, 0, 0, BF16, False), (300, 100, 0, 1, F16, False), (1001, 515, 1, 1, F32, True),
    (97, 161, 0, 0, BF16, True), (5, 2049, 0, 3, BF16, False), (640, 384, 8, 0, F32, False), (260, 31, 0, 0, F16, True), (2, 16384, 0, 0, F32, False),
]


def sides(A, p):
    return [gpu_util.Guarded(torch, size(p, side), 0xA7) for side in (False, True) for size in (A.accept_micro_data_size, A.accept_micro_scale_size)]


def check_quantize(A, x, pad, offset, square, stochastic, first=0, seed=0xFEDCBA9876543210, bad=False):
    rows, cols = x.shape
    gx, vx = matrix(rows, cols, cols + pad, x.dtype, x, offset)
    p = A.MicroParams(rows, cols, code_of(A, x.dtype), A.ROUND_STOCHASTIC if stochastic else A.ROUND_NEAREST, A.BLOCK_SQUARE if square else A.BLOCK_ROW, seed, first, cols + pad)
    q, s, qt, st = bufs = sides(A, p)
    ws = gpu_util.Guarded(torch, A.accept_micro_workspace_size(p), 0)
    A.accept_micro_quantize(p, vx, q.bytes, s.bytes, qt.bytes, st.bytes, ws.bytes)
    assert A.accept_last_device_status(ws.bytes) == (A.DEV_NONFINITE if bad else 0)
    r = plain.draws(rows, cols, seed, first) if stochastic else None
    for data, scale, v, n in ((q, s, vx, r), (qt, st, vx.t(), None if r is None else r.t())):
        codes, byte = plain.code4(v, square, n)
        assert torch.equal(data.bytes.view(v.shape[0], -1), plain.packed4(codes))
        assert torch.equal(scale.bytes, plain.scales4(byte, *v.shape))
    for buf in bufs + [ws, gx]:
        buf.check()
    # one side alone
    first_bits = [b.bytes.clone() for b in bufs]
    for b in bufs:
        b.bytes.fill_(0xA7)
    A.accept_micro_quantize(p, vx, q.bytes, s.bytes, None, None, ws.bytes)
    assert bool((qt.bytes == 0xA7).all())
    A.accept_micro_quantize(p, vx, None, None, qt.bytes, st.bytes, ws.bytes)
    assert all(torch.equal(a, b.bytes) for a, b in zip(first_bits, bufs))
    # and the values again
    for dtype in (F32, BF16, F16):
        for data, scale, v in ((q, s, vx), (qt, st, vx.t())):
            gv, back = matrix(*v.shape, v.shape[1] + pad, dtype, None, offset)
            A.accept_micro_dequantize(A.MicroParams(*v.shape, code_of(A, dtype), ld=v.shape[1] + pad), data.bytes, scale.bytes, back)
            want = plain.decode4(data.bytes.view(v.shape[0], -1), scale.bytes, v.shape[1]).to(dtype)
            assert bool(((back == want) | (torch.isnan(back) & torch.isnan(want))).all())
            gv.check(), data.check(), scale.check()
            assert gaps_untouched(gv, *v.shape, v.shape[1] + pad, dtype, offset)


@pytest.mark.parametrize("stochastic", [False, True])
@pytest.mark.parametrize("case", BLOCKS, ids=str)
def test_codes(A, case, stochastic):
    rows, cols, pad, offset, dtype, square = case
    x = random(rows, rows, cols) * torch.exp2(torch.randint(-9, 9, (rows, 1), device="cuda").float())
    check_quantize(A, x.to(dtype), pad, offset, square, stochastic, first=(0, 5, (1 << 34) - 700, (1 << 64) - 50)[rows % 4])


@pytest.mark.parametrize("square", [False, True])
@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=str)
def test_codes_at_the_ends_of_the_range(A, dtype, square):
    """Ties and borders of every step at several scales, zeros of both signs, subnormals, the largest values."""
    steps = torch.tensor([0, 0.25, 0.5, 0.75, 1, 1.25, 1.5, 1.75, 2, 2.5, 3, 3.5, 4, 5, 6, 0.2499, 0.2501, 4.99, 5.01, 1e-3], device="cuda")
    x = torch.zeros(160, 64, device="cuda")
    x[:, 0:20], x[:, 20:40], x[:, 40:60] = steps, -steps, steps * 0.999
    x[:, 63] = -0.0
    x[5:10] = 0.0
    e = torch.randint(-14, 12, (160, 1), device="cuda", generator=torch.Generator(device="cuda").manual_seed(3)).float()
    x = (x * torch.exp2(e)).to(dtype)
    info = torch.finfo(dtype)
    x[100, 3], x[101, 33], x[102, 3:9] = info.max, -info.max, torch.arange(6, device="cuda").to(dtype) * info.smallest_normal
    x[103] = 0
    x[103, 1] = {F32: 2.0 ** -149, BF16: 2.0 ** -133, F16: 2.0 ** -24}[dtype]
    for stochastic in (False, True):
        check_quantize(A, x, 0, 0, square, stochastic)


def test_codes_of_bad_values_and_of_nothing(A):
    for square in (False, True):
        x = random(1, 200, 300)
        x[3, 40], x[77, 0], x[199, 299], x[130, 131] = float("nan"), float("inf"), float("-inf"), float("nan")
        for dtype in (F32, BF16, F16):
            for stochastic in (False, True):
                check_quantize(A, x.to(dtype), 0, 0, square, stochastic, bad=True)
    before = A.accept_launch_count()
    ws, some = torch.zeros(4, dtype=torch.int32, device="cuda"), torch.zeros(512, dtype=torch.uint8, device="cuda")
    for rows, cols in ((0, 5), (5, 0)):
        A.accept_micro_quantize(A.MicroParams(rows, cols), x, some, some, None, None, ws)
        A.accept_micro_dequantize(A.MicroParams(rows, cols), some, some, x)
    assert A.accept_launch_count() == before


def test_stochastic_codes_are_unbiased(A):
    """Over 4096 draws the mean of a value's codes is the value: within six standard deviations of a two-point distribution (at most
    half a step each)."""
    t = torch.tensor([0.1, 0.25, 0.9, 1.2, 2.3, 3.9, 4.5, 5.9, -0.3, -2.6, 6.0, 0.01], device="cuda")
    x = torch.zeros(4096, 32, device="cuda")
    x[:, :12] = t
    p = A.MicroParams(4096, 32, round=A.ROUND_STOCHASTIC, seed=17)
    q, s = (torch.zeros(size(p), dtype=torch.uint8, device="cuda") for size in (A.accept_micro_data_size, A.accept_micro_scale_size))
    A.accept_micro_quantize(p, x, q, s, None, None, A.new_workspace(p))
    mean = plain.decode4(q.view(4096, -1), s, 12).mean(0)
    step = torch.where(t.abs() < 2, 0.5, torch.where(t.abs() < 4, 1.0, 2.0)).double()
    assert bool(((mean - t.double()).abs() <= 6 * 0.5 * step / 64).all())


# ---- products ------------------------------------------------------------------------------------------------------------------

# m, n, k, type of d, bias, accumulate, extra values between rows of d
PRODUCTS = [
    (1, 1, 1, F32, False, False, 0), (1, 128, 32, BF16, True, False, 0), (3, 130, 100, F16, True, True, 1), (16, 4096, 4096, BF16, True, False, 0),
    (17, 100, 257, F32, False, True, 0), (33, 4100, 900, BF16, True, False, 0), (64, 128, 4000, F32, False, False, 0), (65, 333, 777, F16, True, False, 0),
    (128, 512, 1024, BF16, False, True, 0), (129, 128, 384, F32, True, False, 0), (200, 1, 300, F32, False, False, 0), (300, 50, 260, BF16, True, False, 0),
    (257, 2050, 1544, F16, False, False, 0), (1000, 777, 91, F32, True, True, 7), (512, 512, 512, F32, False, True, 0), (1500, 1100, 700, BF16, True, False, 0),
    (2048, 2304, 640, BF16, True, False, 0), (640, 1280, 8300, F32, False, False, 0), (2600, 2600, 1160, F32, False, True, 0), (4100, 520, 2100, F16, True, False, 4),
    (2305, 2311, 300, BF16, True, False, 0), (2048, 2100, 257, F16, False, True, 0), (5000, 1900, 1000, F32, True, False, 0), (4000, 3333, 128, F32, False, True, 1),
    (7000, 2000, 1, BF16, True, False, 0), (8192, 4100, 64, BF16, True, False, 0), (8192, 4160, 300, F32, False, True, 1), (8192, 4100, 2048, F16, True, False, 1),
    # long sums: shares of few rows, chunks of k, tiles cut along k into two to six parts
    (7, 2100, 35000, F32, True, False, 1), (60, 2100, 35000, F32, False, True, 0), (128, 2100, 35000, BF16, True, False, 0),
    (1280, 1100, 18000, BF16, True, False, 0), (2560, 2560, 10000, F32, False, True, 0), (1280, 1000, 12000, F16, True, False, 1),
    (700, 1100, 24000, F32, True, False, 1), (2590, 1800, 7000, BF16, True, False, 8), (500, 700, 40000, F32, True, True, 1), (2304, 2100, 16600, F32, True, False, 3),
    # rows of d that end inside 16 bytes, behind which someone else's values lie
    (2560, 3980, 176, F16, False, False, 4), (2304, 2303, 300, F32, True, True, 1), (2304, 2271, 200, BF16, True, False, 1),
]


def coded(seed, rows, k, square=False, spread=6):
    """Random codes and scale bytes as the quantiser writes them."""
    import paper_2311_05827_b200 as A
    x = random(seed, rows, k) * torch.exp2(torch.randint(-spread, spread + 1, (rows, 1), device="cuda").float())
    p = A.MicroParams(rows, k, A.DTYPE_F32, A.ROUND_NEAREST, A.BLOCK_SQUARE if square else A.BLOCK_ROW)
    q, s = gpu_util.Guarded(torch, A.accept_micro_data_size(p)), gpu_util.Guarded(torch, A.accept_micro_scale_size(p))
    A.accept_micro_quantize(p, x, q.bytes, s.bytes, None, None, A.new_workspace(p))
    return q.bytes.view(rows, -1), s.bytes


def check_product(A, m, n, k, td, with_bias, accumulate, pad, seed=1):
    a, sa = coded(seed, m, k)
    b, sb = coded(seed + 1, n, k, square=True)
    bias = random(seed + 2, n) if with_bias else None
    start = random(seed + 3, m, n).to(td)
    gd, d = matrix(m, n, n + pad, td, start)
    p = A.MicroMatmulParams(m, n, k, code_of(A, td), accumulate, n + pad)
    ws = gpu_util.Guarded(torch, A.accept_micro_matmul_workspace_size(p), 0)
    A.accept_micro_matmul(p, a, sa, b, sb, bias, d, ws.bytes)
    assert A.accept_last_device_status(ws.bytes) == 0
    gd.check("d"), ws.check("workspace")
    assert gaps_untouched(gd, m, n, n + pad, td)
    va, vb = plain.decode4(a, sa, k), plain.decode4(b, sb, k)
    want, size = va @ vb.t(), va.abs() @ vb.abs().t()
    if bias is not None:
        want, size = want + bias.double(), size + bias.double().abs()
    if accumulate:
        want, size = want + start.double(), size + start.double().abs()
    # one addition for each 32 products and some to join parts, each off by at most one unit in the last place
    tol = 2 * plain.E32 * (k / 32 + 16) * size
    tol = tol + plain8.UNIT[td] * want.abs() + plain8.SMALLEST[td]
    overflow = (want.abs() + tol >= torch.finfo(td).max) & (d.double() == want.sign() * float("inf"))  # past the type's largest value
    assert bool((((d.double() - want).abs() <= tol) | overflow).all())
    assert bool(torch.isfinite(d[want.abs() + tol < torch.finfo(td).max]).all())
    first = d.clone()
    for _ in range(3):
        d.copy_(start)
        A.accept_micro_matmul(p, a, sa, b, sb, bias, d, ws.bytes)
        torch.cuda.synchronize()
        assert torch.equal(first, d)  # the same bits again


@pytest.mark.parametrize("case", PRODUCTS, ids=str)
def test_product(A, case):
    check_product(A, *case)


def test_product_of_one_pair_of_values(A):
    """Each code of a against each code of b, at one place of k after the other: every nibble, scale byte and group of scales is taken
    from its own place (sums of one product are exact)."""
    k = 600
    for m, n in ((16, 128), (300, 16)):
        for at in (0, 1, 31, 32, 63, 64, 95, 127, 128, 191, 255, 256, 300, 511, 512, 599):
            a, b = torch.zeros(m, k, dtype=torch.long, device="cuda"), torch.zeros(n, k, dtype=torch.long, device="cuda")
            a[:, at], b[:, at] = torch.arange(m, device="cuda") % 16, torch.arange(n, device="cuda") // 3 % 16
            blocks = -(-k // 32)
            ea = 120 + (torch.arange(m, device="cuda")[:, None] * 7 + torch.arange(blocks, device="cuda") * 3) % 13
            eb = 121 + (torch.arange(n, device="cuda")[:, None] * 5 + torch.arange(blocks, device="cuda")) % 11
            d = torch.empty(m, n, device="cuda")
            p = A.MicroMatmulParams(m, n, k, A.DTYPE_F32)
            A.accept_micro_matmul(p, plain.packed4(a), plain.scales4(ea, m, k), plain.packed4(b), plain.scales4(eb, n, k), None, d, A.new_workspace(p))
            want = plain.values4(a, ea, k) @ plain.values4(b, eb, k).t()
            assert torch.equal(d.double(), want), (m, n, at)


def test_product_sums_are_single_precision(A):
    """Sums over 32768 values of k keep the accuracy of fp32 sums: within 10^-6 of the result's norm."""
    a, sa = coded(1, 256, 32768, spread=0)
    b, sb = coded(2, 384, 32768, spread=0)
    d = torch.empty(256, 384, device="cuda")
    p = A.MicroMatmulParams(256, 384, 32768, A.DTYPE_F32)
    A.accept_micro_matmul(p, a, sa, b, sb, None, d, A.new_workspace(p))
    want = plain.decode4(a, sa, 32768) @ plain.decode4(b, sb, 32768).t()
    assert float((d.double() - want).norm() / want.norm()) < 1e-6


@pytest.mark.parametrize("m,n", [(9, 130), (140, 130), (2400, 2304)])
def test_product_with_scales_at_the_ends(A, m, n):
    """Scale bytes 0, 200 and 255: the last makes the sums of its own row NaN, and no others."""
    k = 320
    a, sa = coded(1, m, k, spread=0)
    b, sb = coded(2, n, k, spread=0)
    sa[plain.place(7, 0, m)] = 0
    sa[plain.place(8, 9, m)] = 200
    sa[plain.place(5, 3, m)] = 255
    sb[plain.place(100, 8, n)] = 255
    p = A.MicroMatmulParams(m, n, k, A.DTYPE_F32)
    d = torch.empty(m, n, device="cuda")
    A.accept_micro_matmul(p, a, sa, b, sb, None, d, A.new_workspace(p))
    bad = torch.zeros(m, n, dtype=torch.bool, device="cuda")
    bad[5], bad[:, 100] = True, True
    assert torch.equal(torch.isnan(d), bad)
    va, vb = plain.decode4(a, sa, k), plain.decode4(b, sb, k)
    want, size = va @ vb.t(), va.abs() @ vb.abs().t()
    assert bool(((d.double() - want).abs() <= 2 * plain.E32 * 26 * size + 1e-45)[~bad].all())


def test_product_of_nothing(A):
    some = torch.zeros(512, dtype=torch.uint8, device="cuda")
    ws = torch.zeros(4, dtype=torch.int32, device="cuda")
    before = A.accept_launch_count()
    for m, n in ((0, 3), (3, 0)):
        A.accept_micro_matmul(A.MicroMatmulParams(m, n, 16), some, some, some, some, None, some, ws)
    assert A.accept_launch_count() == before
    bias = random(1, 5)
    d = torch.full((3, 5), 2.0, device="cuda")
    A.accept_micro_matmul(A.MicroMatmulParams(3, 5, 0, A.DTYPE_F32, accumulate=True), some, some, some, some, bias, d, ws)
    assert torch.equal(d, 2.0 + bias.expand(3, 5))


def test_linear_layer_gradients(A):
    """y = x W^T in 4 bits: the gradient products contract what the codes stand for, square blocks of W being one set of values both
    ways, and dW is the difference quotient of sum(dy y) in the values of W (which is linear in them)."""
    m, n, k = 70, 140, 260

    def code(t, **more):
        p = A.MicroParams(*t.shape, **more)
        bufs = [torch.zeros(size(p, side), dtype=torch.uint8, device="cuda") for side in (False, True) for size in (A.accept_micro_data_size, A.accept_micro_scale_size)]
        A.accept_micro_quantize(p, t, *bufs, A.new_workspace(p))
        return bufs

    def product(rows, cols, inner, a, sa, b, sb):
        p = A.MicroMatmulParams(rows, cols, inner, A.DTYPE_F32)
        d = torch.empty(rows, cols, device="cuda")
        A.accept_micro_matmul(p, a, sa, b, sb, None, d, A.new_workspace(p))
        return d

    x, w, dy = code(random(1, m, k)), code(random(2, n, k, scale=0.1), block=A.BLOCK_SQUARE), code(random(3, m, n), round=A.ROUND_STOCHASTIC, seed=4)
    vw = plain.decode4(w[0].view(n, -1), w[1], k)
    assert torch.equal(plain.decode4(w[2].view(k, -1), w[3], n).t(), vw)
    dx, dw = product(m, k, n, dy[0], dy[1], w[2], w[3]), product(n, k, m, dy[2], dy[3], x[2], x[3])
    vd, vdt, vxt = plain.decode4(dy[0].view(m, -1), dy[1], n), plain.decode4(dy[2].view(n, -1), dy[3], m), plain.decode4(x[2].view(k, -1), x[3], m)
    assert bool(((dx.double() - vd @ vw).abs() <= 2 * plain.E32 * 24 * (vd.abs() @ vw.abs())).all())
    assert bool(((dw.double() - vdt @ vxt.t()).abs() <= 2 * plain.E32 * 24 * (vdt.abs() @ vxt.abs().t())).all())
    for r, c in ((0, 0), (139, 259), (33, 128)):
        h = torch.zeros(n, k, dtype=torch.float64, device="cuda")
        h[r, c] = 0.5
        difference = float((vdt.t() * (vxt.t() @ h.t())).sum()) / 0.5
        assert abs(difference - float(dw[r, c])) <= 2 * plain.E32 * 24 * float((vdt.abs() @ vxt.abs().t())[r, c])


# ---- streams, graphs, the checking build, waits that run out ----------------------------------------------------------------------

@pytest.mark.parametrize("k", [12000, 24000])
def test_micro_operators_run_on_their_stream_and_in_graphs(A, k):
    """Quantise and multiply on a side stream; then two captured graphs that share one workspace, replayed in turn, with other operators'
    calls between: of whole tiles, and of tiles cut along k."""
    m, n = 700, 1100
    x = random(1, m, k)
    b, sb = coded(2, n, k, square=True)
    p, g = A.MicroParams(m, k), A.MicroMatmulParams(m, n, k, A.DTYPE_F32)
    assert (A.accept_micro_matmul_workspace_size(g) > 16) == (k == 24000)  # cut tiles
    q, s = (torch.zeros(size(p), dtype=torch.uint8, device="cuda") for size in (A.accept_micro_data_size, A.accept_micro_scale_size))
    d, ws = torch.empty(m, n, device="cuda"), A.new_workspace(g)

    def step(x, d):
        A.accept_micro_quantize(p, x, q, s, None, None, ws)
        A.accept_micro_matmul(g, q, s, b, sb, None, d, ws)

    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        x2 = x * 2
        step(x2, d)
    side.synchronize()
    want = d.clone()
    graphs, outs, xs = [], [], [x * 2, x.clone()]
    torch.cuda.synchronize()
    for i in range(2):
        outs.append(torch.zeros(m, n, device="cuda"))
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[i]):
            step(xs[i], outs[i])
    norm, y = A.LayerNormParams(m, k), torch.empty(m, k, device="cuda")
    for _ in range(3):
        graphs[0].replay()
        A.accept_layer_norm_forward(norm, x, None, None, y)
        graphs[1].replay()
    torch.cuda.synchronize()
    assert torch.equal(outs[0], want) and torch.equal(outs[1] * 2, want)  # a power of two moves the scales alone
    assert A.accept_last_device_status(ws) == 0


def test_micro_operators_stay_inside_their_buffers(A):
    with gpu_util.library_variant("bounds"):
        assert A.accept_bounds_check_report()[:2] == (0, 0)
        for rows, cols, pad, offset, dtype, square in BLOCKS:
            for stochastic in (False, True):
                check_quantize(A, random(1, rows, cols).to(dtype), pad, offset, square, stochastic)
        assert A.accept_bounds_check_report()[:2] == (0, 0), "codes"
        for case in PRODUCTS:
            check_product(A, *case)
        code, count, addr, size, write = A.accept_bounds_check_report()
        assert (code, count) == (0, 0), f"product: {count} accesses outside, first at {addr:#x} ({size} bytes, write={write})"


@pytest.mark.parametrize("m,n,k", [(4, 300, 4096), (300, 300, 2000), (2304, 2304, 1024)])
def test_product_whose_copies_do_not_arrive_reports_it_and_leaves_the_gpu_usable(A, m, n, k):
    a, sa = coded(1, m, k)
    b, sb = coded(2, n, k)
    p = A.MicroMatmulParams(m, n, k)
    d, ws = torch.zeros(m, n, dtype=BF16, device="cuda"), A.new_workspace(p)
    with gpu_util.library_variant("stall"):
        A.accept_micro_matmul(p, a, sa, b, sb, None, d, ws)
        assert A.accept_last_device_status(ws) == A.DEV_COPY_TIMEOUT
    check_product(A, m, n, k, BF16, True, False, 0)
