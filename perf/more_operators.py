"""The operators of a residual stage beside layer norm and the 8-bit product, as workloads: dropout whose mask is never
stored, the root-mean-square norm that adds a branch to the residual stream first (with 8-bit codes as its output where a
product follows) and its gradient, and 4-bit floating point with one power-of-two scale for each 32 values: coding,
decoding, and the products of a linear layer in that form, forward and backward.  Sizes are those of the hidden states that
the codec's own transformer workload moves (16 x 1024 tokens of 4096 values), of single tokens, and of ragged shapes between.

`own` false computes the operators from elementary torch operations in fp32; `own` true calls the library.
"""
import math
import struct

import torch

own = False

EPS = 1e-5
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
FORMATS = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
TOP_EXPONENT = {"e4m3": 9, "e5m2": 16}             # the largest finite value is 0.875 * 2^TOP_EXPONENT
BLOCK = {"e4m3": 128, "e5m2": 128, "e2m1": 32}     # values that share a scale
LARGEST = 16384 * 4096                             # values of the transformer boundary tensor
LARGEST_PRODUCT = 16384 * 4096 * 4096


def listed():
    return [
        # hidden states of a small odd batch: a call's own time
        {"name": "dropout_small", "op": "dropout", "rows": 77, "cols": 1001, "pad": 0, "x": "bf16", "y": "bf16", "residual": False, "p": 0.1, "offset": 77077},
        # a sublayer's bf16 output into the fp32 residual stream of the full micro-batch
        {"name": "dropout_boundary", "op": "dropout", "rows": 16384, "cols": 4096, "pad": 0, "x": "bf16", "y": "f32", "residual": True, "p": 0.1, "offset": 0},
        # a few tokens of a decoding step: residual addition and norm, no dropout
        {"name": "rms_tokens", "op": "rms", "rows": 8, "cols": 4096, "pad": 0, "x": "bf16", "y": "bf16", "w": "bf16", "branch": True, "p": 0.0, "codes": "", "offset": 0},
        # ragged token count, odd width, rows with a stride of their own (a slice of a wider tensor)
        {"name": "rms_ragged", "op": "rms", "rows": 5003, "cols": 1537, "pad": 7, "x": "f16", "y": "f16", "w": "f32", "branch": True, "p": 0.1, "codes": "", "offset": 3},
        # training on the full micro-batch: fp32 stream, bf16 branch with dropout, 8-bit codes for the next product
        {"name": "rms_codes_boundary", "op": "rms", "rows": 16384, "cols": 4096, "pad": 0, "x": "f32", "y": "bf16", "w": "f32", "branch": True, "p": 0.1, "codes": "e4m3", "offset": 0},
        # a small micro-batch: the reduction over rows has few rows to share
        {"name": "rms_grad_small", "op": "rms_grad", "rows": 64, "cols": 1024, "pad": 0, "x": "f32", "y": "f32", "w": "f32", "branch": False, "p": 0.0, "offset": 0},
        # the gradient of the full micro-batch's step
        {"name": "rms_grad_boundary", "op": "rms_grad", "rows": 16384, "cols": 4096, "pad": 0, "x": "f32", "y": "bf16", "w": "f32", "branch": True, "p": 0.1, "offset": 0},
        # fp32 master weights of odd height in 32 x 32 blocks, both ways and back
        {"name": "store4_weight", "op": "store4", "rows": 1001, "cols": 4096, "x": "f32", "square": True, "stochastic": False, "side": "columns", "offset": 0},
        # activations of the full micro-batch kept in 4 bits until the backward pass reads them
        {"name": "store4_activations", "op": "store4", "rows": 16384, "cols": 4096, "x": "bf16", "square": False, "stochastic": False, "side": "rows", "offset": 0},
        # single tokens against a weight: the weight's bytes bound it
        {"name": "linear4_tokens", "op": "linear4", "m": 4, "n": 4096, "k": 4096, "x": "bf16", "d": "bf16", "bias": True},
        # forward product of the full micro-batch, activations coded on the way
        {"name": "linear4_forward", "op": "linear4", "m": 16384, "n": 4096, "k": 4096, "x": "bf16", "d": "bf16", "bias": True},
        # its backward pass: the gradient coded both ways from one read with stochastic rounding, two products
        {"name": "linear4_grad", "op": "linear4_grad", "m": 16384, "n": 4096, "k": 4096, "x": "bf16", "offset": 0},
    ]


def _spread(rng, lo, hi):
    """A size between lo and hi, even over the logarithm; a third of them multiples of 320 where they can be."""
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    if rng.random() < 0.34 and v >= 320:
        v -= v % 320
    return max(lo, min(hi, v))


def draw(rng):
    op = rng.choice(["dropout", "rms", "rms_grad", "store4", "linear4", "linear4_grad"])
    offset = rng.choice([0, 4 * rng.randrange(1 << 38), rng.randrange(1 << 40)])  # what calls before this one have drawn
    if op in ("dropout", "rms", "rms_grad"):
        cols = _spread(rng, 33, 16384)
        x = rng.choice(["f32", "bf16", "f16"])
        case = {"op": op, "rows": _spread(rng, 1, min(16384, LARGEST // cols)), "cols": cols, "pad": rng.choice([0, 0, 1, 8, 24]), "x": x,
                "y": rng.choice([x, x, "bf16"]), "offset": offset}
        if op == "dropout":
            return {**case, "residual": rng.random() < 0.5, "p": rng.choice([0.05, 0.1, 0.25, 0.5])}
        branch = rng.random() < 0.7
        case |= {"w": rng.choice([x, "f32"]), "branch": branch, "p": rng.choice([0.0, 0.1, 0.3]) if branch else 0.0}
        return case if op == "rms_grad" else {**case, "codes": rng.choice(["", "e4m3", "e5m2"])}
    if op == "store4":
        cols = _spread(rng, 16, 16384)
        return {"op": op, "rows": _spread(rng, 1, min(16384, LARGEST // cols)), "cols": cols, "x": rng.choice(["f32", "bf16", "f16"]),
                "square": rng.random() < 0.4, "stochastic": rng.random() < 0.5, "side": rng.choice(["rows", "columns"]), "offset": offset}
    n, k = _spread(rng, 32, 16384), _spread(rng, 64, 16384)
    m = _spread(rng, 1, max(1, min(16384, LARGEST_PRODUCT // (n * k))))
    if op == "linear4":
        return {"op": op, "m": m, "n": n, "k": k, "x": rng.choice(["bf16", "f16", "f32"]), "d": rng.choice(["bf16", "f16", "f32"]), "bias": rng.random() < 0.5}
    return {"op": op, "m": m, "n": n, "k": k, "x": rng.choice(["bf16", "f16", "f32"]), "offset": offset}


# ---- inputs ---------------------------------------------------------------------------------------------------

def _generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _hidden(g, rows, cols):
    """Hidden states: N(0,1) with a scale for each channel and an offset, as a boundary tensor of a transformer."""
    scale = torch.rand(cols, device="cuda", generator=g) * 3.9 + 0.1
    return torch.randn(rows, cols, device="cuda", generator=g).mul_(scale).add_(0.25)


def _gradient(g, rows, cols):
    """Gradients of hidden states: small, some tokens many binades below others."""
    return torch.randn(rows, cols, device="cuda", generator=g).mul_(torch.exp2(-6 - 6 * torch.rand(rows, 1, device="cuda", generator=g)))


def _padded(v, dtype, pad):
    """v in `dtype` as the first columns of rows that are `pad` values longer."""
    whole = torch.zeros(v.shape[0], v.shape[1] + pad, dtype=dtype, device="cuda")
    whole[:, :v.shape[1]] = v
    return whole[:, :v.shape[1]]


def _room(rows, cols, dtype, pad=0):
    return torch.zeros(rows, cols + pad, dtype=DTYPES[dtype], device="cuda")[:, :cols]


def _bytes(n):
    return torch.zeros(n, dtype=torch.uint8, device="cuda")


def _coded_room(rows, cols):
    """Room for the 4-bit codes of a matrix and their scales."""
    return _bytes(rows * (_up(cols, 32) // 2)).view(rows, -1), _bytes(_scale_bytes(rows, cols, "e2m1"))


def prepare(case, seed):
    g = _generator(seed)
    op = case["op"]
    state = {"case": case, "seed": seed}           # the seed of the counter-based numbers, too
    if op in ("dropout", "rms", "rms_grad"):
        rows, cols, pad, x, y = (case[k] for k in ("rows", "cols", "pad", "x", "y"))
        if op == "dropout":
            state["x"] = _padded(_hidden(g, rows, cols), DTYPES[x], pad)
            state["residual"] = _padded(_hidden(g, rows, cols), DTYPES[y], pad) if case["residual"] else None
            state["out"] = _room(rows, cols, y, pad)
            return state
        state["gamma"] = (1 + 0.2 * torch.randn(cols, device="cuda", generator=g)).to(DTYPES[case["w"]])
        state["x"] = _padded(_hidden(g, rows, cols), DTYPES[x], pad)
        if op == "rms":
            state["branch"] = _padded(_hidden(g, rows, cols), DTYPES[y], pad) if case["branch"] else None
            state["sum"] = _room(rows, cols, x, pad) if case["branch"] else None
            state["rstd"] = torch.zeros(rows, device="cuda")
            if case["codes"]:
                state["y"], state["q"], state["scale"] = None, _bytes(rows * _up(cols, 16)).view(rows, -1), _bytes(_scale_bytes(rows, cols, case["codes"]))
            else:
                state["y"], state["q"], state["scale"] = _room(rows, cols, y, pad), None, None
        else:
            state["rstd"] = torch.rsqrt(state["x"].float().square().mean(1) + EPS)
            state["dy"] = _padded(_gradient(g, rows, cols), DTYPES[y], pad)
            state["dsum"] = _padded(_gradient(g, rows, cols), DTYPES[x], pad) if case["branch"] else None
            state["dx"] = _room(rows, cols, x, pad)
            state["dbranch"] = _room(rows, cols, y, pad) if case["branch"] else None
            state["dgamma"] = torch.zeros(cols, device="cuda")
    elif op == "store4":
        rows, cols = case["rows"], case["cols"]
        state["x"] = (_gradient if case["stochastic"] else _hidden)(g, rows, cols).to(DTYPES[case["x"]])
        r, c = (rows, cols) if case["side"] == "rows" else (cols, rows)
        state["q"], state["scale"] = _coded_room(r, c)
        state["back"] = _room(r, c, case["x"])
    else:
        m, n, k = case["m"], case["n"], case["k"]
        w = torch.randn(n, k, device="cuda", generator=g).mul_(0.02)
        if op == "linear4":
            state["x"] = _hidden(g, m, k).to(DTYPES[case["x"]])
            state["w"], state["w_scale"] = _packed4(*_coded4(w, True))
            state["bias"] = 0.1 * torch.randn(n, device="cuda", generator=g) if case["bias"] else None
            state["q"], state["scale"] = _coded_room(m, k)
            state["d"] = _room(m, n, case["d"])
        else:
            state["dy"] = _gradient(g, m, n).to(DTYPES[case["x"]])
            state["wt"], state["wt_scale"] = _packed4(*_coded4(w.t(), True))              # as the forward pass coded them
            state["xt"], state["xt_scale"] = _packed4(*_coded4(_hidden(g, m, k).t(), False))
            state["q"], state["scale"] = _coded_room(m, n)
            state["qt"], state["scale_t"] = _coded_room(n, m)
            state["dx"], state["dw"] = _room(m, k, case["x"]), _room(n, k, "f32")
    return state


# ---- the operators in their plain form --------------------------------------------------------------------------

def _up(v, to):
    return -(-v // to) * to


def _scale_bytes(rows, cols, fmt):
    return 512 * (_up(rows, 128) // 128) * (_up(cols, 4 * BLOCK[fmt]) // (4 * BLOCK[fmt]))


def _single(v):
    """v rounded to fp32."""
    return struct.unpack("f", struct.pack("f", v))[0]


MIX = 0xFFFFFFFF


def _finalise(h):
    """The 32-bit finaliser of MurmurHash3 on 32-bit words held in 64 bits."""
    h = ((h ^ (h >> 16)) * 0x85EBCA6B) & MIX
    h = ((h ^ (h >> 13)) * 0xC2B2AE35) & MIX
    return h ^ (h >> 16)


def _random24(rows, cols, seed, offset):
    """The upper 24 bits of the generator's words for a rows x cols matrix: counter offset + row * cols + column, four
    neighbouring counters share a hash."""
    ctr = torch.arange(rows * cols, device="cuda") + offset
    quad = ctr >> 2
    key = _finalise((quad >> 32) ^ (seed & MIX) ^ 0x9E3779B9) ^ (seed >> 32 & MIX)
    h = _finalise((quad & MIX) ^ key)
    lane = torch.tensor([1, 0x9E3779B1, 0x85EBCA77, 0xC2B2AE3D], device="cuda")[ctr & 3]
    return ((h * lane & MIX) >> 8).view(rows, cols)


def _dropped(x, case, seed):
    """x / (1 - p) where the element's number is at least p, else 0."""
    p = _single(case["p"])
    keep = _random24(*x.shape, seed, case["offset"]) >= math.ceil(p * 2 ** 24)
    return torch.where(keep, x.float() * _single(1 / (1 - p)), 0.0)


def _dropout(state):
    c = state["case"]
    y = _dropped(state["x"], c, state["seed"])
    if state["residual"] is not None:
        y = y + state["residual"].float()
    return {"y": y.to(DTYPES[c["y"]])}


def _rms(state):
    c = state["case"]
    x, out = state["x"], {}
    if c["branch"]:
        added = _dropped(state["branch"], c, state["seed"]) if c["p"] > 0 else state["branch"].float()
        out["sum"] = x = (x.float() + added).to(DTYPES[c["x"]])
    x = x.float()
    out["rstd"] = torch.rsqrt(x.square().mean(1) + EPS)
    y = x * out["rstd"][:, None] * state["gamma"].float()
    if c["codes"]:
        out["q"], scale = _coded8(y, c["codes"])
        out["scale"] = scale.view(torch.float8_e8m0fnu)
    else:
        out["y"] = y.to(DTYPES[c["y"]])
    return out


def _rms_grad(state):
    c = state["case"]
    dy, rstd = state["dy"].float(), state["rstd"][:, None]
    xhat = state["x"].float() * rstd
    h = dy * state["gamma"].float()
    dx = (h - xhat * (h * xhat).mean(1, keepdim=True)) * rstd
    if c["branch"]:
        dx = dx + state["dsum"].float()
    out = {"dx": dx.to(DTYPES[c["x"]]), "dgamma": (dy * xhat).sum(0)}
    if c["branch"]:
        out["dbranch"] = (_dropped(dx, c, state["seed"]) if c["p"] > 0 else dx).to(DTYPES[c["y"]])
    return out


def _pack_scales(e):
    """Scale bytes (rows x blocks) in the order the library keeps them: 512 bytes for each 128 rows and four blocks,
    row r of the 128 at 16 * (r % 32) + 4 * (r // 32), one byte for each block."""
    rows, blocks = e.shape
    full = torch.full((_up(rows, 128), _up(blocks, 4)), 127, dtype=torch.uint8, device=e.device)
    full[:rows, :blocks] = e
    return full.view(-1, 4, 32, full.shape[1] // 4, 4).permute(3, 0, 2, 1, 4).reshape(-1)


def _unpack_scales(s, rows, blocks):
    """The scale bytes of rows x blocks."""
    atoms = _up(rows, 128) // 128
    return s.view(-1, atoms, 32, 4, 4).permute(1, 3, 2, 0, 4).reshape(atoms * 128, -1)[:rows, :blocks]


def _exponents(largest, top, above):
    """The least e with largest * 2^-e within the format: 2^top * above is one past, above the fraction of its largest value."""
    mantissa, exponent = torch.frexp(largest)
    e = exponent - top + (mantissa > above).int()
    return torch.where(largest > 0, e.clamp(-127, 127), 0)


def _coded8(x, fmt):
    """8-bit codes along the rows of x (rows padded to a multiple of 16 with zeros) and their scale bytes."""
    rows, cols = x.shape
    x = torch.nn.functional.pad(x, (0, _up(cols, 128) - cols)).view(rows, -1, 128)
    e = _exponents(x.abs().amax(2), TOP_EXPONENT[fmt], 0.875)
    inverse = ((127 - e) << 23).view(torch.float32)  # 2^-e, exact
    codes = (x * inverse[:, :, None]).view(rows, -1)[:, :_up(cols, 16)].to(FORMATS[fmt])
    return codes, _pack_scales((e + 127).to(torch.uint8))


def _coded4(x, square, random=None):
    """What the 4-bit codes along the rows of x stand for before the scale (rows padded to a multiple of 32), and the
    exponents; `random`: 24-bit numbers for stochastic rounding."""
    rows, cols = x.shape
    wide = _up(cols, 32)
    x = torch.nn.functional.pad(x.float(), (0, wide - cols)).view(rows, -1, 32)
    largest = x.abs().amax(2)
    if square:
        padded = torch.nn.functional.pad(largest, (0, 0, 0, _up(rows, 32) - rows))
        largest = padded.view(-1, 32, padded.shape[1]).amax(1).repeat_interleave(32, 0)[:rows]
    e = _exponents(largest, 3, 0.75)
    t = (x * ((127 - e) << 23).view(torch.float32)[:, :, None]).view(rows, wide)
    size = t.abs()
    step = torch.where(size < 2, 0.5, torch.where(size < 4, 1.0, 2.0))
    units = size / step
    if random is None:
        units = torch.round(units)                 # ties to even
    else:
        whole = torch.floor(units)
        units = whole + (torch.nn.functional.pad(random, (0, wide - cols)) < (units - whole) * 2.0 ** 24)
    return torch.copysign(units * step, t), e


def _packed4(values, e):
    """Codes, two to a byte (the even column in the lower half), and scale bytes as the library keeps them."""
    size = values.abs()
    code = torch.where(size < 2, size * 2, torch.where(size < 4, size + 2, size / 2 + 4)).to(torch.uint8) | (torch.signbit(values).to(torch.uint8) << 3)
    return (code[:, 0::2] | code[:, 1::2] << 4).contiguous(), _pack_scales((e + 127).to(torch.uint8))


def _two(e):
    """2^e in fp32, e from -127 to 127."""
    return torch.where(e > -127, (e + 127) << 23, 1 << 22).view(torch.float32)


def _scaled4(values, e, cols):
    return (values * _two(e).repeat_interleave(32, 1))[:, :cols]


def _unpacked4(q, scales, cols):
    """The values that packed codes stand for."""
    table = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0], device="cuda")
    values = table[torch.stack([q & 15, q >> 4], 2).view(q.shape[0], -1).int()]
    return _scaled4(values, _unpack_scales(scales, q.shape[0], _up(cols, 32) // 32).int() - 127, cols)


def _store4(state):
    c = state["case"]
    x, random = state["x"], None
    if c["stochastic"]:
        random = _random24(*x.shape, state["seed"], c["offset"])
    if c["side"] == "columns":
        x, random = x.t(), None if random is None else random.t()
    return {"back": _scaled4(*_coded4(x, c["square"], random), x.shape[1]).to(DTYPES[c["x"]])}


def _linear4(state):
    c = state["case"]
    x = _scaled4(*_coded4(state["x"], False), c["k"])
    d = torch.matmul(x, _unpacked4(state["w"], state["w_scale"], c["k"]).t())
    if state["bias"] is not None:
        d = d + state["bias"]
    return {"d": d.to(DTYPES[c["d"]])}


def _linear4_grad(state):
    c = state["case"]
    m, n = c["m"], c["n"]
    random = _random24(m, n, state["seed"], c["offset"])
    dy = _scaled4(*_coded4(state["dy"], False, random), n)
    dyt = _scaled4(*_coded4(state["dy"].t(), False, random.t()), m)
    dx = torch.matmul(dy, _unpacked4(state["wt"], state["wt_scale"], n).t())
    dw = torch.matmul(dyt, _unpacked4(state["xt"], state["xt_scale"], m).t())
    return {"dx": dx.to(DTYPES[c["x"]]), "dw": dw}


# ---- the library's operators ------------------------------------------------------------------------------------

def _plan(state):
    """What a program keeps from call to call: the library, the parameters and the workspace."""
    import paper_2311_05827_b200 as A
    c, seed = state["case"], state["seed"]
    types = {"f32": A.DTYPE_F32, "bf16": A.DTYPE_BF16, "f16": A.DTYPE_F16}
    op = c["op"]
    if op == "dropout":
        return A, [A.DropoutParams(c["rows"], c["cols"], c["p"], types[c["x"]], types[c["y"]], seed, c["offset"], c["cols"] + c["pad"], c["cols"] + c["pad"])], None
    if op in ("rms", "rms_grad"):
        fmt = A.FORMAT_E5M2 if c.get("codes") == "e5m2" else A.FORMAT_E4M3
        p = [A.RmsNormParams(c["rows"], c["cols"], EPS, types[c["x"]], types[c["y"]], types[c["w"]], c["p"], seed, c["offset"], fmt,
                             c["cols"] + c["pad"], c["cols"] + c["pad"])]
    elif op == "store4":
        rounding = A.ROUND_STOCHASTIC if c["stochastic"] else A.ROUND_NEAREST
        r, k = (c["rows"], c["cols"]) if c["side"] == "rows" else (c["cols"], c["rows"])
        p = [A.MicroParams(c["rows"], c["cols"], types[c["x"]], rounding, A.BLOCK_SQUARE if c["square"] else A.BLOCK_ROW, seed, c["offset"]),
             A.MicroParams(r, k, types[c["x"]])]
    elif op == "linear4":
        p = [A.MicroParams(c["m"], c["k"], types[c["x"]]), A.MicroMatmulParams(c["m"], c["n"], c["k"], types[c["d"]])]
    else:
        p = [A.MicroParams(c["m"], c["n"], types[c["x"]], A.ROUND_STOCHASTIC, A.BLOCK_ROW, seed, c["offset"]),
             A.MicroMatmulParams(c["m"], c["k"], c["n"], types[c["x"]]), A.MicroMatmulParams(c["n"], c["k"], c["m"], A.DTYPE_F32)]
    return A, p, [A.new_workspace(each) for each in p]


def _own(state):
    if "plan" not in state:
        state["plan"] = _plan(state)
    A, p, ws = state["plan"]
    s, c = state, state["case"]
    op = c["op"]
    if op == "dropout":
        A.accept_dropout(p[0], s["x"], s["residual"], s["out"])
        return {"y": s["out"]}
    if op == "rms":
        A.accept_rms_norm_forward(p[0], s["x"], s["branch"], s["gamma"], s["sum"], s["y"], s["q"], s["scale"], s["rstd"], ws[0])
        out = {"sum": s["sum"], "rstd": s["rstd"]} if c["branch"] else {"rstd": s["rstd"]}
        return {**out, "q": s["q"].view(FORMATS[c["codes"]]), "scale": s["scale"].view(torch.float8_e8m0fnu)} if c["codes"] else {**out, "y": s["y"]}
    if op == "rms_grad":
        A.accept_rms_norm_backward(p[0], s["dy"], s["x"], s["gamma"], s["rstd"], s["dsum"], s["dx"], s["dbranch"], s["dgamma"], ws[0])
        return {k: s[k] for k in (("dx", "dgamma", "dbranch") if c["branch"] else ("dx", "dgamma"))}
    if op == "store4":
        sides = (s["q"], s["scale"], None, None) if c["side"] == "rows" else (None, None, s["q"], s["scale"])
        A.accept_micro_quantize(p[0], s["x"], *sides, ws[0])
        A.accept_micro_dequantize(p[1], s["q"], s["scale"], s["back"])
        return {"back": s["back"]}
    if op == "linear4":
        A.accept_micro_quantize(p[0], s["x"], s["q"], s["scale"], None, None, ws[0])
        A.accept_micro_matmul(p[1], s["q"], s["scale"], s["w"], s["w_scale"], s["bias"], s["d"], ws[1])
        return {"d": s["d"]}
    A.accept_micro_quantize(p[0], s["dy"], s["q"], s["scale"], s["qt"], s["scale_t"], ws[0])
    A.accept_micro_matmul(p[1], s["q"], s["scale"], s["wt"], s["wt_scale"], None, s["dx"], ws[1])
    A.accept_micro_matmul(p[2], s["qt"], s["scale_t"], s["xt"], s["xt_scale"], None, s["dw"], ws[2])
    return {"dx": s["dx"], "dw": s["dw"]}


def run(state):
    if own:
        return _own(state)
    return {"dropout": _dropout, "rms": _rms, "rms_grad": _rms_grad, "store4": _store4, "linear4": _linear4, "linear4_grad": _linear4_grad}[state["case"]["op"]](state)


# ---- work, and the definitions in 64 bits -------------------------------------------------------------------------

def _coded_bytes(rows, cols):
    return rows * (_up(cols, 32) // 2) + _scale_bytes(rows, cols, "e2m1")


def work(case):
    size = {"f32": 4, "bf16": 2, "f16": 2}
    op = case["op"]
    if op in ("dropout", "rms", "rms_grad"):
        rows, cols, x, y = case["rows"], case["cols"], size[case["x"]], size[case["y"]]
        v = rows * cols
        if op == "dropout":
            return {"bytes": v * (x + y + (y if case["residual"] else 0)), "flops": 3 * v}
        w = cols * size[case["w"]] + 4 * rows
        if op == "rms":
            out = rows * _up(cols, 16) + _scale_bytes(rows, cols, case["codes"]) if case["codes"] else v * y
            return {"bytes": v * x + (v * (x + y) if case["branch"] else 0) + out + w, "flops": 6 * v}
        return {"bytes": v * (2 * x + y) + (v * (x + y) if case["branch"] else 0) + w + 4 * cols, "flops": 12 * v}
    if op == "store4":  # values in and out, codes and scales written and read
        rows, cols = case["rows"], case["cols"]
        coded = _coded_bytes(rows, cols) if case["side"] == "rows" else _coded_bytes(cols, rows)
        return {"bytes": 2 * rows * cols * size[case["x"]] + 2 * coded, "flops": 6 * rows * cols}
    m, n, k = case["m"], case["n"], case["k"]
    if op == "linear4":
        return {"bytes": m * k * size[case["x"]] + 2 * _coded_bytes(m, k) + _coded_bytes(n, k) + m * n * size[case["d"]] + (4 * n if case["bias"] else 0),
                "flops": 2 * m * n * k}
    return {"bytes": m * n * size[case["x"]] + 2 * _coded_bytes(m, n) + 2 * _coded_bytes(n, m) + _coded_bytes(k, n) + _coded_bytes(k, m)
            + m * k * size[case["x"]] + 4 * n * k, "flops": 4 * m * n * k}


def _two64(e):
    """2^e in 64 bits, from its exponent field."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _wrapped(v):
    """A 32-bit constant as the int32 of the same bits."""
    return v - (1 << 32) if v >> 31 else v


def _numbers(rows, cols, seed, offset):
    """U of the generator for each element, as multiples of 2^-24 in 64 bits, in wrapping 32-bit arithmetic."""
    def shifted(h, by):  # without the sign
        return (h >> by) & ((1 << (32 - by)) - 1)

    def mixed(h):
        h = (h ^ shifted(h, 16)) * _wrapped(0x85EBCA6B)
        h = (h ^ shifted(h, 13)) * _wrapped(0xC2B2AE35)
        return h ^ shifted(h, 16)

    first = torch.arange(rows, device="cuda")[:, None] * cols + offset
    at = first + torch.arange(cols, device="cuda")
    high, low, lane = (at >> 34).int(), (at >> 2).int(), at % 4
    key = mixed(high ^ _wrapped(seed % (1 << 32)) ^ _wrapped(0x9E3779B9)) ^ _wrapped(seed >> 32)
    h = mixed(low ^ key)
    for m, times in ((1, 0x9E3779B1), (2, 0x85EBCA77), (3, 0xC2B2AE3D)):
        h = torch.where(lane == m, mixed(low ^ key) * _wrapped(times), h)
    return shifted(h, 8).double() * 2.0 ** -24


def _exact_dropped(x, case, seed):
    p = struct.unpack("f", struct.pack("f", case["p"]))[0]
    if p == 0:
        return x
    return x * (_numbers(*x.shape, seed, case["offset"]) >= p) / (1 - p)


def _exact8(x, fmt):
    """What the 8-bit codes of x stand for before the scale, and the scales (64 bits), as rows x blocks."""
    rows, cols = x.shape
    bits, low, top = (3, -6, 448.0) if fmt == "e4m3" else (2, -14, 57344.0)
    blocks = -(-cols // 128)
    x = torch.cat([x, torch.zeros(rows, blocks * 128 - cols, dtype=torch.float64, device="cuda")], 1).view(rows, blocks, 128)
    e = _exact_exponents(x.abs().amax(2), top)
    x = x * _two64(-e)[:, :, None]
    step = _two64((torch.frexp(x)[1] - 1).clamp(min=low) - bits)
    return (torch.round(x / step) * step).view(rows, -1)[:, :-(-cols // 16) * 16], _two64(e)


def _exact_exponents(largest, top):
    e = torch.ceil(torch.log2(torch.where(largest > 0, largest, top) / top)).long()
    e = e + (largest * _two64(-e) > top).long()          # where the logarithm was rounded to a whole number
    e = e - (largest * _two64(1 - e) <= top).long()
    return torch.where(largest > 0, e.clamp(-127, 127), 0)


GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _exact4(x, square, u=None):
    """The values that x has in 4 bits, scale included; u: the numbers of stochastic rounding."""
    x = x.double()
    rows, cols = x.shape
    blocks = -(-cols // 32)
    parts = torch.stack([piece.abs().amax(1) for piece in x.split(32, 1)], 1)
    if square:
        parts = torch.cat([piece.amax(0, keepdim=True).expand(piece.shape[0], blocks) for piece in parts.split(32)])
    two = _two64(_exact_exponents(parts, 6.0)).repeat_interleave(32, 1)[:, :cols]
    grid = torch.tensor(GRID, dtype=torch.float64, device="cuda")
    t = x.abs() / two
    below = (torch.searchsorted(grid, t.contiguous(), right=True) - 1).clamp(max=6)
    lower, upper = grid[below], grid[below + 1]
    share = (t - lower) / (upper - lower)
    if u is None:
        up = (share > 0.5) | ((share == 0.5) & (below % 2 == 1))
    else:
        up = (u < share) | (share == 1)
    return torch.sign(x) * torch.where(up, upper, lower) * two


def _exact_values4(q, scales, cols):
    """The 64-bit values of packed codes."""
    rows = q.shape[0]
    grid = torch.tensor(GRID + tuple(-v for v in GRID), dtype=torch.float64, device="cuda")
    c = torch.arange(cols, device="cuda")
    code = (q[:, c // 2].int() >> (c % 2 * 4)) & 15
    r, b = torch.arange(rows, device="cuda")[:, None], c[None] // 32
    at = ((b // 4) * (-(-rows // 128)) + r // 128) * 512 + (r % 32) * 16 + (r // 32) % 4 * 4 + b % 4
    return grid[code] * _two64(scales[at].int() - 127)


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "dropout":
        y = _exact_dropped(s["x"].double(), case, seed)
        return {"y": y if s["residual"] is None else y + s["residual"].double()}
    if op == "rms":
        x, out = s["x"].double(), {}
        if case["branch"]:
            out["sum"] = x + _exact_dropped(s["branch"].double(), case, seed)
            x = out["sum"].to(s["x"].dtype).double()     # the norm is that of the sum as it is kept
        out["rstd"] = 1 / torch.sqrt((x * x).sum(1) / case["cols"] + EPS)
        y = x * (out["rstd"][:, None] * s["gamma"].double())
        if case["codes"]:
            out["q"], out["scale"] = _exact8(y, case["codes"])[0], None
        else:
            out["y"] = y
        return out
    if op == "rms_grad":
        rstd = s["rstd"].double()[:, None]
        xhat, dy = s["x"].double() * rstd, s["dy"].double()
        h = dy * s["gamma"].double()
        dx = rstd * (h - xhat * ((h * xhat).sum(1, keepdim=True) / case["cols"]))
        out = {"dgamma": (dy * xhat).sum(0)}
        if case["branch"]:
            dx = dx + s["dsum"].double()
            out["dbranch"] = _exact_dropped(dx, case, seed)
        return {**out, "dx": dx}
    if op == "store4":
        u = _numbers(case["rows"], case["cols"], seed, case["offset"]) if case["stochastic"] else None
        x = s["x"]
        if case["side"] == "columns":
            x, u = x.t(), None if u is None else u.t()
        return {"back": _exact4(x, case["square"], u)}
    m, n, k = case["m"], case["n"], case["k"]
    if op == "linear4":
        d = _exact4(s["x"], False) @ _exact_values4(s["w"], s["w_scale"], k).t()
        return {"d": d if s["bias"] is None else d + s["bias"].double()}
    u = _numbers(m, n, seed, case["offset"])
    return {"dx": _exact4(s["dy"], False, u) @ _exact_values4(s["wt"], s["wt_scale"], n).t(),
            "dw": _exact4(s["dy"].t(), False, u.t()) @ _exact_values4(s["xt"], s["xt_scale"], m).t()}
