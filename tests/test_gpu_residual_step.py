"""The operators of a residual stage together, as the example uses them: its output and gradients against 64-bit formulas on what the
codes stand for."""
import threading

import pytest

from tests import operators_plain as plain8
from tests import residual_plain as plain

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

BF16 = torch.bfloat16


def step(tokens, width, features, rate=0.2, seed=5, number=3):
    from examples import residual_stage as example
    i = example.inputs(tokens, width, features, seed)
    stage = example.Stage(tokens, width, features, i["weight"], i["bias"], i["gamma"], rate, seed)
    out = stage.forward(i["x"], i["branch"], number)
    dx, dbranch = stage.backward(i["dout"], i["dsum"], number)
    return i, stage, out, dx, dbranch


def within(got, want, tol):
    return bool(((got.double() - want).abs() <= tol).all())


@pytest.mark.parametrize("tokens,width,features", [(128, 256, 384), (130, 328, 200), (1, 64, 33), (700, 1001, 515)])
def test_step(tokens, width, features):
    rate, seed, number = 0.2, 5, 3
    i, stage, out, dx, dbranch = step(tokens, width, features, rate, seed, number)
    assert stage.status() == 0
    e32, unit = plain.E32, plain8.UNIT[BF16]
    # the sum, its norm, the codes of the norm both ways
    first = number * tokens * width
    assert torch.equal(stage.sum, i["x"] + plain.dropped32(i["branch"], rate, seed, first))
    y, rstd = plain.rms(stage.sum, i["gamma"], 1e-5)
    off = (72 + width / 1024) * e32
    assert within(stage.normed, y, (off + 4 * e32 + unit) * y.abs() + plain8.SMALLEST[BF16])
    r = plain.draws(tokens, features, seed + 1, number * tokens * features)
    for coded, v, square, n in ((stage.y_coded, stage.normed, False, None), (stage.w_coded, i["weight"], True, None), (stage.d_coded, i["dout"], False, r)):
        for q, s, m, k in ((coded.q, coded.scale, v, n), (coded.qt, coded.scale_t, v.t(), None if n is None else n.t())):
            codes, byte = plain.code4(m, square, k)
            assert torch.equal(q.view(m.shape[0], -1), plain.packed4(codes)) and torch.equal(s, plain.scales4(byte, *m.shape))
    # the products, from what the codes stand for: an addition for each 32 values of k and some to join parts
    a, w = plain.decode4(stage.y_coded.q.view(tokens, -1), stage.y_coded.scale, width), plain.decode4(stage.w_coded.q.view(features, -1), stage.w_coded.scale, width)
    d, dt = plain.decode4(stage.d_coded.q.view(tokens, -1), stage.d_coded.scale, features), plain.decode4(stage.d_coded.qt.view(features, -1), stage.d_coded.scale_t, tokens)
    at = plain.decode4(stage.y_coded.qt.view(width, -1), stage.y_coded.scale_t, tokens)
    for got, u, v, bias in ((out, a, w.t(), i["bias"].double()), (stage.dnormed, d, w, 0.0), (stage.dweight, dt, at.t(), 0.0)):
        want, size = u @ v + bias, u.abs() @ v.abs() + (bias.abs() if torch.is_tensor(bias) else 0.0)
        rounding = unit if got.dtype == BF16 else e32
        assert within(got, want, 2 * e32 * (u.shape[1] / 32 + 16) * size + rounding * want.abs() + plain8.SMALLEST[BF16])
    # the norm's gradients
    want, wg, size, size_g = plain.rms_grad(stage.dnormed, stage.sum, i["gamma"], stage.rstd, i["dsum"])
    assert within(dx, want, off * size + e32 * want.abs() + 1e-45)
    keep = plain.kept(tokens, width, rate, seed, first)
    scale = 1 / (1 - plain.single(rate))
    assert within(dbranch, torch.where(keep, want * scale, 0.0), (off * size + (4 * e32 + unit) * want.abs()) * scale + plain8.SMALLEST[BF16])
    assert within(stage.dgamma, wg, (64 + tokens) * e32 * size_g + 1e-45)


def test_step_accumulates_and_draws_again():
    """A second backward pass adds to the gradient of the weight; another step draws another mask and other roundings."""
    i, stage, _, dx, _ = step(256, 320, 128)
    once, sum0, codes0 = stage.dweight.clone(), stage.sum.clone(), stage.d_coded.q.clone()
    stage.backward(i["dout"], i["dsum"], 3)
    assert bool(((stage.dweight.double() - 2 * once.double()).abs() <= 2 * plain.E32 * once.abs()).all()) and torch.equal(codes0, stage.d_coded.q)
    stage.forward(i["x"], i["branch"], 4)
    stage.backward(i["dout"], i["dsum"], 4)
    assert not torch.equal(sum0, stage.sum) and not torch.equal(codes0, stage.d_coded.q)


def test_answer_is_the_eight_bit_product_of_the_norms_codes():
    i, stage, _, _, _ = step(130, 328, 200)
    s, out = stage.answer(i["x"], i["branch"])
    assert torch.equal(s, i["x"] + i["branch"].float())
    a, w = plain8.decode(stage.y8.view(130, -1), stage.y8_scale, "e4m3", 328), plain8.decode(stage.w8.view(200, -1), stage.w8_scale, "e4m3", 328)
    want, size = a @ w.t() + i["bias"].double(), a.abs() @ w.abs().t() + i["bias"].double().abs()
    assert within(out, want, 2 * plain.E32 * 28 * size + plain8.UNIT[BF16] * want.abs())
    y, _ = plain.rms(s, i["gamma"], 1e-5)
    # E4M3 is off by at most 2^-4 of a value, or half of its smallest step, 2^-10, below 2^-6 of the scale (which is at most 2^-7 of the largest)
    assert within(a, y, (2.0 ** -4 + 1e-5) * y.abs() + 2.0 ** -17 * y.abs().amax(1, keepdim=True))


def test_example_runs():
    from examples import residual_stage as example
    errors = example.run(256, 512, 384, seed=3)
    assert set(errors) == {"y", "dx", "dbranch", "dweight", "dgamma", "answer"} and all(e == e for e in errors.values())


def test_two_streams_and_several_host_threads_at_once():
    """Stages of different sizes, each with buffers and workspaces of its own, stepped by four host threads on their own streams at the same
    time: the bits of each are those of the same steps made one after the other."""
    from examples import residual_stage as example
    sizes = [(300, 520, 200), (64, 4096, 128), (1000, 77, 260), (129, 2048, 1030)]

    def stages():
        made = []
        for k, (tokens, width, features) in enumerate(sizes):
            i = example.inputs(tokens, width, features, k)
            made.append((i, example.Stage(tokens, width, features, i["weight"], i["bias"], i["gamma"], 0.1, k)))
        torch.cuda.synchronize()
        return made

    def steps(i, stage):
        for number in range(8):
            stage.forward(i["x"], i["branch"], number)
            stage.backward(i["dout"], i["dsum"], number)

    results = lambda stage: [stage.sum, stage.normed, stage.out, stage.dnormed, stage.dweight, stage.dx, stage.dbranch, stage.dgamma]  # noqa: E731
    one, errors = stages(), []
    for i, stage in one:
        steps(i, stage)
    torch.cuda.synchronize()
    many = stages()

    def work(i, stage):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                steps(i, stage)
        except Exception as e:  # noqa: BLE001
            errors.append(e)

    threads = [threading.Thread(target=work, args=m) for m in many]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not errors
    for (_, a), (_, b) in zip(one, many):
        assert b.status() == 0 and all(torch.equal(u, v) for u, v in zip(results(a), results(b)))


def test_captured_step_is_replayed():
    """A whole step in a graph, replayed on new inputs: the bits of the calls themselves, the numbers of the captured counters."""
    i, stage, _, _, _ = step(200, 328, 264)
    other = {k: v.clone() for k, v in i.items()}
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        stage.forward(other["x"], other["branch"], 6)
        stage.backward(other["dout"], other["dsum"], 6)
    for scale in (1.0, 0.5):
        for k in ("x", "branch", "dout", "dsum"):
            other[k].copy_(i[k] * scale)
        stage.dweight.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (stage.out, stage.dx, stage.dbranch, stage.dgamma, stage.dweight)]
        stage.dweight.zero_()
        stage.forward(other["x"], other["branch"], 6)
        stage.backward(other["dout"], other["dsum"], 6)
        torch.cuda.synchronize()
        assert all(torch.equal(u, v) for u, v in zip(got, (stage.out, stage.dx, stage.dbranch, stage.dgamma, stage.dweight)))
