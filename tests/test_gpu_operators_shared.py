"""What calls share: one workspace for several entry points and sizes, results in the place of inputs, and kernels that several
host threads launch."""
import ctypes
import threading

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


def test_one_workspace_serves_all_operators_by_turns(A):
    """A buffer that held anything before, used by products of different cuts (2, 3 and 6 parts), layer norms' backward
    passes and the quantiser in turn: every result is the one that a fresh workspace gives, bit for bit."""
    sizes = [(700, 1000, 8300, BF16), (1810, 300, 10000, F32), (1280, 1100, 9000, BF16), (700, 1000, 8300, BF16)]
    products = []
    for i, (m, n, k, dtype) in enumerate(sizes):
        p = A.MatmulParams(m, n, k, dtype_d=ops.code_of(A, dtype))
        assert A.accept_matmul_workspace_size(p) > 4096
        operands = ops.coded(2 * i, m, k, "e4m3") + ops.coded(2 * i + 1, n, k, "e4m3")
        want = torch.empty(m, n, dtype=dtype, device="cuda")
        A.accept_block_matmul(p, *operands, None, want, A.new_workspace(p))
        products.append((p, operands, want))
    norm, q = A.LayerNormParams(900, 1500), A.QuantizeParams(900, 1500)
    x, dy = ops.random(20, 900, 1500), ops.random(21, 900, 1500)
    y, mean, rstd = torch.empty_like(x), torch.empty(900, device="cuda"), torch.empty(900, device="cuda")
    A.accept_layer_norm_forward(norm, x, None, None, y, mean, rstd)

    def backward(ws):
        out = torch.empty_like(x), torch.empty(1500, device="cuda"), torch.empty(1500, device="cuda")
        A.accept_layer_norm_backward(norm, dy, x, None, mean, rstd, *out, ws)
        return out

    def quantize(ws):
        out = [torch.empty(size(q, side), dtype=torch.uint8, device="cuda") for side in (False, True) for size in (A.accept_block_data_size, A.accept_block_scale_size)]
        A.accept_block_quantize(q, x, *out, ws)
        return out

    grads, codes = backward(A.new_workspace(norm)), quantize(A.new_workspace(q))
    size = max([A.accept_matmul_workspace_size(p) for p, _, _ in products] + [A.accept_layer_norm_workspace_size(norm)])
    for fill in (0, 1, 0x33, 0xFF):
        ws = torch.full((size,), fill, dtype=torch.uint8, device="cuda")
        ws[:4] = 0  # the status word is the caller's
        for p, operands, want in products:
            d = torch.full_like(want, float("nan"))
            A.accept_block_matmul(p, *operands, None, d, ws)
            assert torch.equal(d, want)
            for a, b in zip(grads, backward(ws)):
                assert torch.equal(a, b)
            for a, b in zip(codes, quantize(ws)):
                assert torch.equal(a, b)
        assert A.accept_last_device_status(ws) == 0


def test_a_captured_product_of_cut_tiles_repeats(A):
    """A CUDA graph repeats one call: the same result each time, whatever else the workspace served in between."""
    m, n, k = 700, 1000, 8300
    p = A.MatmulParams(m, n, k)
    operands = ops.coded(1, m, k, "e4m3") + ops.coded(2, n, k, "e4m3")
    want, d, ws = torch.empty(m, n, dtype=BF16, device="cuda"), torch.empty(m, n, dtype=BF16, device="cuda"), A.new_workspace(p)
    A.accept_block_matmul(p, *operands, None, want, ws)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        A.accept_block_matmul(p, *operands, None, d, ws)
    for fill in (None, None, 1, -1, 0x33333333):
        if fill is not None:
            ws[1:] = fill
        d.fill_(float("nan"))
        graph.replay()
        assert torch.equal(d, want)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=str)
@pytest.mark.parametrize("rows,cols,pad", [(70, 64, 0), (300, 1024, 0), (1200, 1037, 0), (40, 8192, 8), (600, 8200, 0), (1100, 9001, 0), (33, 16384, 0), (70, 20000, 1), (5, 20001, 0)])
def test_norm_results_may_take_the_place_of_inputs(A, rows, cols, pad, dtype):
    """y in the place of x, and dx in the place of x or of dy, give the bits that they give apart."""
    p = A.LayerNormParams(rows, cols, 1e-5, ops.code_of(A, dtype), ops.code_of(A, dtype), A.DTYPE_F32, cols + pad, cols + pad)
    place = lambda v: ops.matrix(rows, cols, cols + pad, dtype, v)[1]  # noqa: E731
    x, dy = place(ops.random(1, rows, cols) + 0.5), place(ops.random(2, rows, cols, scale=0.1))
    gamma, beta = 1 + 0.2 * ops.random(3, cols), 0.2 * ops.random(4, cols)
    y, mean, rstd = place(None), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    A.accept_layer_norm_forward(p, x, gamma, beta, y, mean, rstd)
    over = place(x)
    A.accept_layer_norm_forward(p, over, gamma, beta, over)
    assert torch.equal(over, y)

    def backward(dy_, x_, dx):
        dgamma, dbeta = torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
        A.accept_layer_norm_backward(p, dy_, x_, gamma, mean, rstd, dx, dgamma, dbeta, A.new_workspace(p))
        return dx, dgamma, dbeta

    want = backward(dy, x, place(None))
    over_x, over_dy = place(x), place(dy)
    for got in (backward(dy, over_x, over_x), backward(over_dy, x, over_dy)):
        for a, b in zip(got, want):
            assert torch.equal(a, b)


@pytest.mark.parametrize("backward", [False, True])
def test_norms_of_different_shapes_from_four_threads(A, backward):
    """Four host threads with streams and buffers of their own, whose calls run the same kernel with different amounts of
    shared memory: every call is accepted, and right."""
    from paper_2311_05827_b200 import binding
    lib = binding.lib()
    shapes = [(2048, 1024), (40, 4096), (300, 513), (2048, 4096)]
    refused, calls = [0] * len(shapes), []
    for i, (rows, cols) in enumerate(shapes):
        p, stream = A.LayerNormParams(rows, cols), torch.cuda.Stream()
        x, out, mean, rstd = ops.random(i, rows, cols), torch.empty(rows, cols, device="cuda"), torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
        ws = A.new_workspace(p)
        A.accept_layer_norm_forward(p, x, None, None, out, mean, rstd)
        handle, c, size = stream.cuda_stream, ctypes.byref(p.c()), 4 * ws.numel()
        if backward:
            call = (lib.accept_layer_norm_backward, (c, x.data_ptr(), x.data_ptr(), None, mean.data_ptr(), rstd.data_ptr(), out.data_ptr(), None, None, ws.data_ptr(), size, handle))
        else:
            call = (lib.accept_layer_norm_forward, (c, x.data_ptr(), None, None, out.data_ptr(), None, None, handle))
        calls.append((call, stream, x, mean, rstd, out, p, ws))
    torch.cuda.synchronize()

    def work(i):
        (f, args), stream = calls[i][:2]
        for turn in range(10000):
            refused[i] += f(*args) != 0
            if turn % 500 == 0:
                stream.synchronize()

    threads = [threading.Thread(target=work, args=(i,)) for i in range(len(shapes))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert refused == [0] * len(shapes)
    for _, _, x, mean, rstd, out, _, _ in calls:
        want = plain.norm_grad(x, x, None, mean, rstd)[0] if backward else plain.norm(x, None, None, 1e-5)[0]
        assert float((out.double() - want).abs().max()) < 1e-4
