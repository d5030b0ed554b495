"""One training step of the stage that receives a boundary tensor: layer norm and a linear layer in 8 bits.

    python examples/linear_stage.py [tokens] [width] [features]

Forward: the codec's stream is decompressed, normalised, quantised in blocks of 128 (along the width for the product,
along the tokens for the gradient of the weight: one read) and multiplied by the quantised weight.  Backward: the gradient
of the output is quantised both ways, two products give the gradients of the normalised input and of the weight, the layer
norm's backward pass gives the gradient of the boundary tensor, and the codec compresses that for the stage before.
Everything runs on the library's kernels; torch holds the memory.  The same step in fp32 torch operations on the
decompressed tensor says how far 8 bits are off.
"""
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch

import paper_2311_05827_b200 as A

EPS = 1e-5


class Coded:
    """A matrix in 8-bit blocks: codes and scales by rows and by columns."""

    def __init__(self, p):
        self.p = p
        self.ws = A.new_workspace(p)
        sizes = [size(p, side) for side in (False, True) for size in (A.accept_block_data_size, A.accept_block_scale_size)]
        self.q, self.scale, self.qt, self.scale_t = (torch.empty(n, dtype=torch.uint8, device="cuda") for n in sizes)

    def take(self, x):
        A.accept_block_quantize(self.p, x, self.q, self.scale, self.qt, self.scale_t, self.ws)
        return self


class Stage:
    """Layer norm and a linear layer y = norm(x) W^T + b over `tokens` rows; fp32 master weights."""

    def __init__(self, tokens, width, features, weight, bias, gamma, beta):
        self.tokens, self.width, self.features = tokens, width, features
        self.weight, self.bias, self.gamma, self.beta = weight, bias, gamma, beta
        self.norm = A.LayerNormParams(tokens, width, EPS, A.DTYPE_F32, A.DTYPE_BF16, A.DTYPE_F32)
        self.norm_ws = A.new_workspace(self.norm)
        self.x_coded = Coded(A.QuantizeParams(tokens, width, A.DTYPE_BF16))
        self.w_coded = Coded(A.QuantizeParams(features, width, A.DTYPE_F32, block=A.BLOCK_SQUARE))
        self.dy_coded = Coded(A.QuantizeParams(tokens, features, A.DTYPE_BF16, A.FORMAT_E5M2))
        self.products = [A.MatmulParams(tokens, features, width),
                         A.MatmulParams(tokens, width, features, A.FORMAT_E5M2),
                         A.MatmulParams(features, width, tokens, A.FORMAT_E5M2, A.FORMAT_E4M3, A.DTYPE_F32, accumulate=True)]
        self.product_ws = [A.new_workspace(p) for p in self.products]
        f32, bf16 = dict(device="cuda"), dict(dtype=torch.bfloat16, device="cuda")
        self.normed, self.y, self.dnormed = torch.empty(tokens, width, **bf16), torch.empty(tokens, features, **bf16), torch.empty(tokens, width, **bf16)
        self.mean, self.rstd = torch.empty(tokens, **f32), torch.empty(tokens, **f32)
        self.dx = torch.empty(tokens, width, **f32)
        self.dgamma, self.dbeta, self.dweight = torch.empty(width, **f32), torch.empty(width, **f32), torch.zeros(features, width, **f32)
        self.w_coded.take(weight)

    def forward(self, x):
        self.x = x
        A.accept_layer_norm_forward(self.norm, x, self.gamma, self.beta, self.normed, self.mean, self.rstd)
        a, b = self.x_coded.take(self.normed), self.w_coded
        A.accept_block_matmul(self.products[0], a.q, a.scale, b.q, b.scale, self.bias, self.y, self.product_ws[0])
        return self.y

    def backward(self, dy):
        """Adds to dweight; writes dgamma, dbeta and the gradient of x, which it returns."""
        d, w, x = self.dy_coded.take(dy), self.w_coded, self.x_coded
        A.accept_block_matmul(self.products[1], d.q, d.scale, w.qt, w.scale_t, None, self.dnormed, self.product_ws[1])
        A.accept_block_matmul(self.products[2], d.qt, d.scale_t, x.qt, x.scale_t, None, self.dweight, self.product_ws[2])
        A.accept_layer_norm_backward(self.norm, self.dnormed, self.x, self.gamma, self.mean, self.rstd, self.dx, self.dgamma, self.dbeta, self.norm_ws)
        return self.dx

    def status(self):
        """The device status words of all calls, joined."""
        bits = 0
        for ws in [c.ws for c in (self.x_coded, self.w_coded, self.dy_coded)] + self.product_ws:
            bits |= A.accept_last_device_status(ws)
        return bits


def run(tokens=1024, width=4096, features=4096, seed=0):
    """One step; returns the relative errors of y and of each gradient against fp32 torch operations."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    randn = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    boundary = randn(tokens, width) * (0.1 + 9.9 * torch.rand(width, device="cuda", generator=g))
    weight, bias = randn(features, width) * width ** -0.5, 0.1 * randn(features)
    gamma, beta = 1 + 0.1 * randn(width), 0.1 * randn(width)
    dy = (1e-3 * randn(tokens, features)).to(torch.bfloat16)

    # the boundary tensor arrives as the codec's stream: 8 bits, one range for 4096 values
    p = A.Params(tokens * width, 4096, 8)
    stream, ws = A.new_stream_buffer(p), A.new_workspace(p)
    x = torch.empty(tokens, width, device="cuda")
    A.accept_compress(p, boundary, stream, ws)
    A.accept_decompress(p, stream, x, ws)

    stage = Stage(tokens, width, features, weight, bias, gamma, beta)
    y = stage.forward(x)
    dx = stage.backward(dy)

    # the gradient goes back as a stream too: 4 bits, stochastic rounding
    pg = A.Params(tokens * width, 4096, 4, round=A.ROUND_STOCHASTIC, seed=seed)
    back = A.new_stream_buffer(pg)
    A.accept_compress(pg, dx, back, ws)
    status = stage.status() | A.accept_last_device_status(ws)
    if status:
        raise RuntimeError(f"device status {status:#x}")

    xr, wr, gr, br = (t.detach().clone().requires_grad_() for t in (x, weight, gamma, beta))
    yr = torch.nn.functional.layer_norm(xr, (width,), gr, br, EPS) @ wr.t() + bias
    yr.backward(dy.float())
    error = lambda a, b: float((a.detach().double() - b.detach().double()).norm() / b.detach().double().norm())  # noqa: E731
    return {"y": error(y, yr), "dx": error(dx, xr.grad), "dweight": error(stage.dweight, wr.grad),
            "dgamma": error(stage.dgamma, gr.grad), "dbeta": error(stage.dbeta, br.grad)}


if __name__ == "__main__":
    for name, e in run(*map(int, sys.argv[1:4])).items():
        print(f"{name:8s} relative error {e:.4f}")
