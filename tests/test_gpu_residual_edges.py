"""Operators of a residual stage at the ends of their matrices and where sizes pass 32 bits, against 64-bit plain forms."""
import pytest

from tests import gpu_util
from tests import residual_plain as plain
from tests.test_gpu_micro import check_quantize
from tests.test_gpu_operators import code_of, matrix, random
from tests.test_gpu_residual import check_dropout, same

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16


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


def test_nothing_is_read_behind_a_matrix_that_ends_one_value_past_a_unit(A):
    """16-bit values read as words off 16-byte boundaries, the last unit of eight on a 4-byte one: the word behind it holds the last value
    and one that does not exist.  On the checking build, which compares each access with the bytes of the call's matrices."""
    with gpu_util.library_variant("bounds"):
        assert A.accept_bounds_check_report()[:2] == (0, 0)
        for dtype in (BF16, F16):
            for rows, cols, pad, offset in ((8, 1001, 1, 0), (16, 1001, 1, 2), (8, 9, 1, 0), (136, 137, 1, 4), (8, 1001, 0, 1)):
                for stochastic in (False, True):
                    check_quantize(A, random(rows, rows, cols).to(dtype), pad, offset, False, stochastic)
            for rows, cols, pad, offset in ((1, 5001, 0, 2), (1, 9, 0, 2), (3, 1001, 7, 2), (31, 25, 7, 4), (1, 5001, 0, 3), (2, 5000, 1, 1)):
                for to in (dtype, F32):
                    check_dropout(A, rows, cols, pad, pad, offset, dtype, to, True, 0.1, 5)
            # the residual off a boundary, beside x and y on one
            x, r = random(1, 1, 5001).to(dtype), random(2, 1, 5001).to(dtype)
            for offset in (2, 3, 4):
                (_, vx), (_, vr), (gy, y) = matrix(1, 5001, 5001, dtype, x), matrix(1, 5001, 5001, dtype, r, offset), matrix(1, 5001, 5001, dtype)
                A.accept_dropout(A.DropoutParams(1, 5001, 0.1, code_of(A, dtype), code_of(A, dtype), 3, 6), vx, vr, y)
                assert same(y, (plain.dropped32(x, 0.1, 3, 6) + r.float()).to(dtype))
                gy.check()
        code, count, addr, size, write = A.accept_bounds_check_report()
        assert (code, count) == (0, 0), f"{count} accesses outside, first at {addr:#x} ({size} bytes, write={write})"


def test_example_is_as_near_as_its_codes(A, monkeypatch):
    """The example's outputs and gradients against fp32 operations: no further off than coding explains.  Where those draw the mask of
    other counters, as a wrong mask in the library would look, all that depends on it is."""
    from examples import residual_stage as example
    for seed in range(3):
        errors = example.run(256, 512, 384, seed=seed)
        assert set(errors) == set(example.LIMITS) and all(errors[k] < limit for k, limit in example.LIMITS.items()), errors
    params = A.DropoutParams
    monkeypatch.setattr(example.A, "DropoutParams", lambda *a, rng_offset, **more: params(*a, rng_offset=rng_offset + 4, **more))
    errors = example.run(256, 512, 384)
    assert all(errors[k] > example.LIMITS[k] for k in ("y", "dbranch", "dweight")), errors


def test_values_at_the_top_of_the_range_round_up_past_it(A):
    """From 1.75 2^127 on the nearest code stands for 4 2^126, which neither fp32 nor bf16 has; from 1.75 2^15 on for 2^16, which fp16 has not:
    infinities, of which the status word says nothing.  As a factor such a code is 2^128."""
    for dtype, top in ((F32, 127), (BF16, 127), (F16, 15)):
        x = torch.zeros(4, 32, dtype=dtype, device="cuda")
        x[0, 3], x[1, 4], x[2, 5], x[3, 6] = 1.75 * 2.0 ** top, -torch.finfo(dtype).max, 1.5 * 2.0 ** top, 1.625 * 2.0 ** top
        p = A.MicroParams(4, 32, code_of(A, dtype))
        q, s = (torch.empty(size(p), dtype=torch.uint8, device="cuda") for size in (A.accept_micro_data_size, A.accept_micro_scale_size))
        ws, back = A.new_workspace(p), torch.empty_like(x)
        A.accept_micro_quantize(p, x, q, s, None, None, ws)
        A.accept_micro_dequantize(p, q, s, back)
        assert A.accept_last_device_status(ws) == 0
        want = torch.zeros_like(x)
        want[0, 3], want[1, 4], want[2, 5], want[3, 6] = float("inf"), -float("inf"), 1.5 * 2.0 ** top, 1.5 * 2.0 ** top
        assert torch.equal(back, want)
        b = torch.full((16, 32), 2.0 ** -20, device="cuda")
        pb, d = A.MicroParams(16, 32), torch.empty(4, 16, device="cuda")
        qb, sb = (torch.empty(size(pb), dtype=torch.uint8, device="cuda") for size in (A.accept_micro_data_size, A.accept_micro_scale_size))
        A.accept_micro_quantize(pb, b, qb, sb, None, None, A.new_workspace(pb))
        g = A.MicroMatmulParams(4, 16, 32, A.DTYPE_F32)
        A.accept_micro_matmul(g, q, s, qb, sb, None, d, A.new_workspace(g))
        assert torch.equal(d, torch.tensor([2.0, -2.0, 1.5, 1.5], device="cuda")[:, None].expand(4, 16) * 2.0 ** (top - 20))


def test_stochastic_codes_of_values_far_below_their_block(A):
    """Where U = 0 any t above 0 is coded 0.5, but for t that fp32 has no value for, 2^-150 and less: those count as 0."""
    seed, n = 5, 1 << 24
    first = next(at + int(hit[0]) for at in range(0, 64 * n, n) for hit in [torch.nonzero(plain.draws(1, n, seed, at)[0] == 0)[:, 0]] if len(hit) and at + int(hit[0]) >= 5)
    for dtype in (F32, BF16):
        for t, code in ((2.0 ** -100, 1), (2.0 ** -149, 1), (1.5 * 2.0 ** -150, 1), (2.0 ** -150, 0), (2.0 ** -155, 0), (0.0, 0)):
            for sign in (1, -1):
                x = torch.zeros(1, 32, dtype=dtype, device="cuda")
                x[0, 0], x[0, 5] = 2.0 ** 127, sign * t * 2.0 ** 125  # the block's scale is 2^125
                p = A.MicroParams(1, 32, code_of(A, dtype), A.ROUND_STOCHASTIC, seed=seed, rng_offset=first - 5)
                q, s = (torch.empty(size(p), dtype=torch.uint8, device="cuda") for size in (A.accept_micro_data_size, A.accept_micro_scale_size))
                A.accept_micro_quantize(p, x, q, s, None, None, A.new_workspace(p))
                assert int(s[0]) == 125 + 127 and int(q[2] >> 4) == code + (8 if sign < 0 else 0), (dtype, t, sign)


def test_masks_are_the_codecs_own_numbers(A):
    """What dropout keeps, against the words of the codec's CPU implementation: U = (word >> 8) 2^-24."""
    import oracle
    n = 100_003
    for seed, first, rate in ((1, 0, 0.1), (0xFEDCBA9876543210, (1 << 34) - 50_001, 0.5), (77, (1 << 64) - 1000, 0.9)):
        y = torch.empty(n, device="cuda")
        A.accept_dropout(A.DropoutParams(1, n, rate, seed=seed, rng_offset=first), torch.ones(n, device="cuda"), None, y)
        numbers = torch.from_numpy(oracle.rng_words(seed, first, n).astype("int64") >> 8).cuda()
        assert torch.equal(y > 0, numbers * 2.0 ** -24 >= plain.single(rate))


def test_operators_on_rows_that_lie_far_apart(A):
    """Row strides of 2^31 values and more, all matrices in one buffer: the bits of the same calls on rows side by side."""
    rows, cols, ld = 3, 300, (1 << 31) + 8
    room = torch.empty(2 * ld + 9 * 512, dtype=BF16, device="cuda")
    far = lambda k: torch.as_strided(room, (rows, cols), (ld, 1), 512 * k)  # noqa: E731
    x, branch, dsum, dy = (random(k, rows, cols).to(BF16) for k in range(4))
    gamma, results = 1 + 0.1 * random(5, cols), []
    for apart in (False, True):
        place = far if apart else lambda k: torch.empty(rows, cols, dtype=BF16, device="cuda")
        step, names = ld if apart else cols, ("x", "branch", "dsum", "dy", "sum", "y", "dx", "dbranch", "out")
        m = {name: place(k) for k, name in enumerate(names)}
        for name, v in (("x", x), ("branch", branch), ("dsum", dsum), ("dy", dy)):
            m[name].copy_(v)
        p = A.RmsNormParams(rows, cols, 1e-5, A.DTYPE_BF16, A.DTYPE_BF16, A.DTYPE_F32, 0.2, 7, 11, ld_x=step, ld_y=step)
        rstd, dgamma = torch.empty(rows, device="cuda"), torch.empty(cols, device="cuda")
        A.accept_rms_norm_forward(p, m["x"], m["branch"], gamma, m["sum"], m["y"], None, None, rstd)
        A.accept_rms_norm_backward(p, m["dy"], m["sum"], gamma, rstd, m["dsum"], m["dx"], m["dbranch"], dgamma, A.new_workspace(p))
        A.accept_dropout(A.DropoutParams(rows, cols, 0.3, A.DTYPE_BF16, A.DTYPE_BF16, 5, 6, step, step), m["x"], m["branch"], m["out"])
        found = [m[name].clone() for name in ("sum", "y", "dx", "dbranch", "out")] + [rstd, dgamma]
        p = A.MicroParams(rows, cols, A.DTYPE_BF16, A.ROUND_STOCHASTIC, seed=3, rng_offset=4, ld=step)
        codes = [torch.empty(size(p, side), dtype=torch.uint8, device="cuda") for side in (False, True) for size in (A.accept_micro_data_size, A.accept_micro_scale_size)]
        A.accept_micro_quantize(p, m["x"], *codes, A.new_workspace(p))
        A.accept_micro_dequantize(p, codes[0], codes[1], m["out"])
        results.append(found + codes + [m["out"].clone()])
    assert all(torch.equal(a, b) for a, b in zip(*results))


def test_values_of_the_longest_row(A):
    """2^31 - 1 values, off a 16-byte boundary: first, middle and last ones."""
    cols, part = (1 << 31) - 1, 4096
    p = A.MicroParams(1, cols, A.DTYPE_BF16)
    q = torch.randint(0, 256, (A.accept_micro_data_size(p),), dtype=torch.uint8, device="cuda")
    s = torch.randint(120, 130, (A.accept_micro_scale_size(p),), dtype=torch.uint8, device="cuda")
    x = torch.full((cols + 18,), 7.0, dtype=BF16, device="cuda")
    A.accept_micro_dequantize(p, q, s, x[9:9 + cols])
    for c in (0, cols // 64 * 32, (cols - 1) // 32 * 32 - part):
        n = min(2 * part, cols - c)
        blocks = torch.arange(c // 32, -(-(c + n) // 32), device="cuda")
        code = torch.stack([q[c // 2:c // 2 + part] & 15, q[c // 2:c // 2 + part] >> 4], 1).view(1, -1)[:, :n].long()
        byte = s[plain.place(torch.zeros_like(blocks), blocks, 1)].long().view(1, -1)
        assert torch.equal(x[9 + c:9 + c + n].double(), plain.values4(code, byte, n)[0]), c
    assert bool((x[:9] == 7).all()) and bool((x[9 + cols:] == 7).all())
