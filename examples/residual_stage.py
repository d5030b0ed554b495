"""One training step of a residual stage: dropout of a branch, its addition to the residual stream, root-mean-square norm and a linear
layer in 4 bits; and the same stage as it answers, with 8-bit codes straight from the norm.

    python examples/residual_stage.py [tokens] [width] [features]

Forward: the branch is dropped and added to the fp32 stream (the sum is kept), normalised, coded in blocks of 32 along the width for the
product and along the tokens for the gradient of the weight (one read), and multiplied by the coded weight.  Backward: the gradient of the
output is coded both ways with stochastic rounding, two products give the gradients of the normalised sum and of the weight, and the
norm's backward pass gives those of the stream, of the branch (its mask is drawn again) and of gamma.  Everything runs on the library's kernels;
torch holds the memory.  The same step in fp32 torch operations, with the same mask, says how far 4 bits are off.
"""
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch

import paper_2311_05827_b200 as A

EPS = 1e-5

# Relative errors that coding explains for inputs() of 256 tokens, 512 values, 384 features, and a sixth (answer: a third) above them.  Coding in
# 4 bits costs normal values 0.115 in blocks of 32, weights 0.126 in squares, the gradient with stochastic rounding 0.166; the errors of a
# product's two sides are independent: y 0.17, dweight 0.20, dnormed and so dgamma 0.21, of which dx and dbranch carry half beside dsum,
# 0.107.  In 8 bits each side costs 0.026, so the answer 0.037.
LIMITS = {"y": 0.2, "dx": 0.125, "dbranch": 0.125, "dweight": 0.235, "dgamma": 0.25, "answer": 0.05}


class Coded:
    """A matrix in 4-bit blocks: codes and scales by rows and by columns."""

    def __init__(self, p):
        self.p = p
        self.ws = A.new_workspace(p)
        sizes = [size(p, side) for side in (False, True) for size in (A.accept_micro_data_size, A.accept_micro_scale_size)]
        self.q, self.scale, self.qt, self.scale_t = (torch.empty(n, dtype=torch.uint8, device="cuda") for n in sizes)

    def take(self, x, p=None):
        A.accept_micro_quantize(p or self.p, x, self.q, self.scale, self.qt, self.scale_t, self.ws)
        return self


class Stage:
    """y = norm(x + drop(branch)) W^T + b over `tokens` rows of the fp32 stream x; bf16 branch, fp32 master weights."""

    def __init__(self, tokens, width, features, weight, bias, gamma, rate, seed):
        self.shape = tokens, width, features
        self.weight, self.bias, self.gamma, self.rate, self.seed = weight, bias, gamma, rate, seed
        self.y_coded = Coded(A.MicroParams(tokens, width, A.DTYPE_BF16))
        self.w_coded = Coded(A.MicroParams(features, width, A.DTYPE_F32, block=A.BLOCK_SQUARE)).take(weight)
        self.d_coded = Coded(A.MicroParams(tokens, features, A.DTYPE_BF16, A.ROUND_STOCHASTIC))
        self.products = [A.MicroMatmulParams(tokens, features, width), A.MicroMatmulParams(tokens, width, features),
                         A.MicroMatmulParams(features, width, tokens, A.DTYPE_F32, accumulate=True)]
        self.product_ws = [A.new_workspace(p) for p in self.products]
        bf16 = dict(dtype=torch.bfloat16, device="cuda")
        self.sum, self.rstd = torch.empty(tokens, width, device="cuda"), torch.empty(tokens, device="cuda")
        self.normed, self.out, self.dnormed = torch.empty(tokens, width, **bf16), torch.empty(tokens, features, **bf16), torch.empty(tokens, width, **bf16)
        self.dx, self.dbranch = torch.empty(tokens, width, device="cuda"), torch.empty(tokens, width, **bf16)
        self.dgamma, self.dweight = torch.empty(width, device="cuda"), torch.zeros(features, width, device="cuda")
        self.norm_ws = A.new_workspace(self._norm(0))
        # as it answers: an 8-bit weight, codes from the norm
        q = A.QuantizeParams(features, width, A.DTYPE_F32, block=A.BLOCK_SQUARE)
        self.w8, self.w8_scale = (torch.empty(size(q), dtype=torch.uint8, device="cuda") for size in (A.accept_block_data_size, A.accept_block_scale_size))
        A.accept_block_quantize(q, weight, self.w8, self.w8_scale, None, None, A.new_workspace(q))
        q = A.QuantizeParams(tokens, width)
        self.y8, self.y8_scale = (torch.empty(size(q), dtype=torch.uint8, device="cuda") for size in (A.accept_block_data_size, A.accept_block_scale_size))
        self.product8 = A.MatmulParams(tokens, features, width)
        self.product8_ws = A.new_workspace(self.product8)

    def _norm(self, step, rate=None):
        tokens, width, _ = self.shape
        return A.RmsNormParams(tokens, width, EPS, A.DTYPE_F32, A.DTYPE_BF16, A.DTYPE_F32, self.rate if rate is None else rate, self.seed, step * tokens * width)

    def forward(self, x, branch, step):
        A.accept_rms_norm_forward(self._norm(step), x, branch, self.gamma, self.sum, self.normed, None, None, self.rstd, self.norm_ws)
        a, b = self.y_coded.take(self.normed), self.w_coded
        A.accept_micro_matmul(self.products[0], a.q, a.scale, b.q, b.scale, self.bias, self.out, self.product_ws[0])
        return self.out

    def backward(self, dout, dsum, step):
        """Adds to dweight; writes dgamma and the gradients of x and of the branch, which it returns.  dsum: what reaches the sum by the
        stream itself."""
        tokens, width, features = self.shape
        p = A.MicroParams(tokens, features, A.DTYPE_BF16, A.ROUND_STOCHASTIC, seed=self.seed + 1, rng_offset=step * tokens * features)
        d, w, y = self.d_coded.take(dout, p), self.w_coded, self.y_coded
        A.accept_micro_matmul(self.products[1], d.q, d.scale, w.qt, w.scale_t, None, self.dnormed, self.product_ws[1])
        A.accept_micro_matmul(self.products[2], d.qt, d.scale_t, y.qt, y.scale_t, None, self.dweight, self.product_ws[2])
        A.accept_rms_norm_backward(self._norm(step), self.dnormed, self.sum, self.gamma, self.rstd, dsum, self.dx, self.dbranch, self.dgamma, self.norm_ws)
        return self.dx, self.dbranch

    def answer(self, x, branch):
        """The stage without dropout: the sum, and the output from 8-bit codes that the norm itself writes."""
        A.accept_rms_norm_forward(self._norm(0, 0.0), x, branch, self.gamma, self.sum, None, self.y8, self.y8_scale, None, self.norm_ws)
        A.accept_block_matmul(self.product8, self.y8, self.y8_scale, self.w8, self.w8_scale, self.bias, self.out, self.product8_ws)
        return self.sum, self.out

    def status(self):
        """The device status words of all calls, joined."""
        bits = A.accept_last_device_status(self.norm_ws) | A.accept_last_device_status(self.product8_ws)
        for ws in [c.ws for c in (self.y_coded, self.w_coded, self.d_coded)] + self.product_ws:
            bits |= A.accept_last_device_status(ws)
        return bits


def inputs(tokens, width, features, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    randn = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    return {"x": randn(tokens, width), "branch": randn(tokens, width).to(torch.bfloat16), "weight": randn(features, width) * width ** -0.5, "bias": 0.1 * randn(features),
            "gamma": 1 + 0.1 * randn(width), "dout": (1e-3 * randn(tokens, features)).to(torch.bfloat16), "dsum": 1e-3 * randn(tokens, width)}


def run(tokens=1024, width=4096, features=4096, seed=0, rate=0.1):
    """Two steps; returns the relative errors of the second one's output and gradients against fp32 torch operations."""
    i = inputs(tokens, width, features, seed)
    stage = Stage(tokens, width, features, i["weight"], i["bias"], i["gamma"], rate, seed)
    for step in range(2):
        stage.dweight.zero_()
        y = stage.forward(i["x"], i["branch"], step)
        dx, dbranch = stage.backward(i["dout"], i["dsum"], step)
    xr, br, wr, gr, cr = (i[k].detach().float().requires_grad_() for k in ("x", "branch", "weight", "gamma", "bias"))
    kept = torch.empty_like(i["x"])  # the mask, as the library draws it, times 1 / (1 - rate)
    A.accept_dropout(A.DropoutParams(tokens, width, rate, seed=seed, rng_offset=tokens * width), torch.ones_like(kept), None, kept)
    s = xr + br * kept
    yr = s * torch.rsqrt(s.square().mean(1, keepdim=True) + EPS) * gr @ wr.t() + cr
    torch.autograd.backward([yr, s], [i["dout"].float(), i["dsum"]])
    error = lambda a, b: float((a.detach().double() - b.detach().double()).norm() / b.detach().double().norm())  # noqa: E731
    found = {"y": error(y, yr), "dx": error(dx, xr.grad), "dbranch": error(dbranch, br.grad), "dweight": error(stage.dweight, wr.grad),
             "dgamma": error(stage.dgamma, gr.grad)}
    s = i["x"] + i["branch"].float()
    answer = s * torch.rsqrt(s.square().mean(1, keepdim=True) + EPS) * i["gamma"] @ i["weight"].t() + i["bias"]
    found["answer"] = error(stage.answer(i["x"], i["branch"])[1], answer)
    status = stage.status()
    if status:
        raise RuntimeError(f"device status {status:#x}")
    return found


if __name__ == "__main__":
    for name, e in run(*map(int, sys.argv[1:4])).items():
        print(f"{name:8s} relative error {e:.4f}")
