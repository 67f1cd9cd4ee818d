"""Calls of layer norm, gated layer and dropout beyond those of test_gpu_sublayer.py.

Rounding to storage is off by at most HALF relative to the value; U is that of a float."""
import numpy as np
import pytest
import torch

from gpu_harness import DEV, GpuStage, compare_minibatch, gpu_minibatch, stage_io, tdtype
from oracle import ops
from oracle.stage import OracleStage
from paper_2012_12544_amd import binding as B
from stage_inputs import configs as C
from stage_inputs import gen
from test_gpu_sublayer import HALF, U, _f64, _one, _rows, _run, _stage
from test_oracle_sublayer import sublayer

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------ positions folded into the batch
MANY = [dict(c=64, units=1600, micro_batch=2060), dict(c=96, units=1608, micro_batch=2050, act=C.GATE_GELU),
        dict(c=32, units=1600, micro_batch=2060, bias=0),       # one panel: the same order as rows
        dict(c=40, units=1608, micro_batch=2050),               # no panels
        dict(c=128, units=3200, micro_batch=1000, act=C.GATE_SIGMOID), dict(c=64, units=1604, micro_batch=2060)]


@pytest.mark.parametrize("kw", MANY)
def test_sublayer_of_many_maps_of_one_pixel(kw):
    """A 1x1 convolution of single pixels keeps its filters in panels, which the products that fill the chip meet as well."""
    compare_minibatch(sublayer(seq=1, n_micro=1, stage_index=1, n_stages=1, **kw))


@pytest.mark.parametrize("kw", MANY)
def test_positions_in_the_batch_or_in_a_sequence_are_the_same(kw):
    """(C, 1, 1) x rows and (C, rows, 1) x 1 are the same elements in the same order: two mini-batches, with the update between them."""
    rows = kw["micro_batch"]
    folded = sublayer(seq=1, n_micro=2, stage_index=1, n_stages=1, **kw)
    along = sublayer(seq=rows, n_micro=2, stage_index=1, n_stages=1, **dict(kw, micro_batch=1))
    params = gen.all_params(folded, perturb=True)
    xs, gs = stage_io(folded)
    out = []
    for st in (folded, along):
        to = lambda a: np.ascontiguousarray(a if st is folded else a[:, :, 0, 0].T[None, :, :, None])  # noqa: E731
        g, got = GpuStage(st, params), []
        for _ in range(2):
            for m in range(2):
                got += [_rows(g.forward(m, to(xs[m]))), _rows(g.backward(m, to(gs[m])))]
            got += [a for i, (w, _) in enumerate(params) if w is not None for a in g.grads(i) if a is not None]
            B.bapipe_stage_step(g.h, 0.05)
        g.close()
        out.append(got)
    for a, b in zip(*out):
        assert np.array_equal(a, b) and np.any(a)


@pytest.mark.parametrize("kw", [dict(c=64, units=320, micro_batch=70), dict(c=96, units=352, micro_batch=500), dict(c=160, units=640, micro_batch=1500),
                                dict(c=1024, units=2048, micro_batch=130), dict(c=72, units=328, micro_batch=333, act=C.GATE_RELU)])
def test_sublayer_of_some_maps_of_one_pixel(kw):
    """Too few tiles for that kernel: gradients between the layers are float sums of products whose filters are in panels."""
    compare_minibatch(sublayer(seq=1, n_micro=2, stage_index=1, n_stages=1, **kw))


def test_a_large_sublayer_on_the_static_workspace():
    """The same bits as on the stage's own."""
    st = sublayer(c=1024, units=4096, seq=512, micro_batch=4, n_micro=2, stage_index=1, n_stages=2)
    ref, got = gpu_minibatch(st), gpu_minibatch(st, static=True)
    for k in ref:
        assert np.array_equal(got[k], ref[k]) and np.any(ref[k]), k


# ------------------------------------------------------------------------------ what is not finite
@pytest.mark.parametrize("c,units,seq", [(16, 40, 6), (16, 4096, 2048), (15, 40, 6)])
def test_an_infinite_gradient_of_a_narrow_layer_norm(c, units, seq):
    """dy that overflowed in one element: the gradients that it reaches are infinite, as the sums say, not NaN, and rows that it does
    not reach are what they were.  Narrow layer norms take what rounding took from the projections' gradients as well."""
    b = C._Builder()
    b.layernorm(c, src=-1)
    b.gated(c, units, act=C.GATE_SIGMOID, bias=1)
    b.conv(units, 8, 1)
    st = _stage(b.layers, C.BF16, (c, seq, 1), 1, 1)
    params = gen.all_params(st, perturb=True)
    # positive weights and linear parts, moderate gates: every product that dy enters is positive
    w = np.abs(params[1][0]) * np.float32(0.5) + np.float32(0.01)
    bias = np.concatenate([np.zeros(units), np.full(units, 16 * w.sum(1).max())]).astype(np.float32)
    params[1] = (w, bias)
    params[2] = (np.abs(params[2][0]) + np.float32(0.01), params[2][1])
    xs, gs = stage_io(st)
    dy = gs[0].copy()
    dy[0, 0, 3] = np.inf
    g = GpuStage(st, params)
    g.forward(0, xs[0])
    dx = _rows(g.backward(0, dy))
    dgamma, dbeta = g.grads(0)
    g.close()
    xhat = ops.layernorm_fwd(_f64(torch.from_numpy(xs[0]).bfloat16().float().numpy()), np.ones(c), np.zeros(c), 1e-5)[1]
    assert np.all(np.isfinite(dx[[0, 1, 2, 4, 5]]))
    assert np.all(dbeta == np.inf), dbeta
    assert np.array_equal(dgamma, np.sign(_rows(xhat)[3]) * np.inf), dgamma


def test_an_infinite_output_of_a_layer_norm_in_front_of_a_relu():
    """What rounding took from it is nothing."""
    c, units = 24, 40
    b = C._Builder()
    b.layernorm(c, src=-1)
    b.gated(c, units, act=C.GATE_RELU, bias=1)
    st = _stage(b.layers, C.BF16, (c, 5, 1), 2, 1)
    params = gen.all_params(st, perturb=True)
    gamma, beta = params[0]
    beta = beta.copy()
    beta[7] = np.inf
    params[0], params[1] = (gamma, beta), (np.abs(params[1][0]) + np.float32(0.01), params[1][1])
    g = GpuStage(st, params)
    y = g.forward(0, stage_io(st)[0][0])
    g.close()
    assert np.all(y == np.inf)


@pytest.mark.parametrize("dtype,c,units,rows", [(C.FP32, 24, 40, 9), (C.FP32, 16, 2056, 2050), (C.BF16, 24, 40, 9), (C.BF16, 25, 41, 9), (C.BF16, 64, 1600, 2060)])
def test_a_relu_gate_that_is_no_number(dtype, c, units, rows):
    """max(g, 0) of NaN is NaN: a parameter that went wrong shows in the output and in the gradients that the unit's value enters."""
    st = _stage(_one("gated", c, units, act=C.GATE_RELU, bias=1), dtype, (c, rows, 1), 1, 1)
    (w, bias), = params = gen.all_params(st, perturb=True)
    xs, gs = stage_io(st)
    ref = _run(st, xs, gs, params)
    bias = bias.copy()
    bias[3] = np.nan
    g = GpuStage(st, [(w, bias)])
    y = _rows(g.forward(0, xs[0]))
    g.backward(0, gs[0])
    dw, db = g.grads(0)
    g.close()
    others = np.arange(units) != 3
    assert np.all(np.isnan(y[:, 3])) and np.array_equal(y[:, others], _rows(ref["y0"])[:, others])
    assert np.isnan(db[units + 3]) and np.all(np.isnan(dw[units + 3]))
    keep = np.concatenate([others, others])
    assert np.array_equal(dw[keep], ref["dw0"][keep]) and np.array_equal(db[keep], ref["db0"][keep])


# ------------------------------------------------------------------------------ saturated gates
@pytest.mark.parametrize("dtype", [C.FP32, C.BF16])
@pytest.mark.parametrize("at", [-15.0, -9.0, 9.0, 12.0, 15.0])
def test_the_derivative_of_a_saturated_sigmoid(dtype, at):
    """s (1 - s) of s within rounding of 1: the gates' weight gradients have all their digits."""
    c, units, seq = 8, 16, 40
    st = _stage(_one("gated", c, units, act=C.GATE_SIGMOID, bias=1), dtype, (c, seq, 1), 1, 1)
    (w, bias), = params = gen.all_params(st, perturb=True)
    bias = np.concatenate([np.full(units, at, np.float32), bias[units:]])
    xs, gs = stage_io(st)
    got = _f64(_run(st, xs, gs, [(w, bias)])["dw0"])[:units]
    orc = OracleStage(dict(st), [(w, bias)])
    W, x, dy = orc.q(_f64(w)), _rows(torch.from_numpy(xs[0]).to(tdtype(st)).double().numpy()), _rows(torch.from_numpy(gs[0]).to(tdtype(st)).double().numpy())
    both = x @ W.T + bias
    e = np.exp(-np.abs(both[:, :units]))
    dg = dy * both[:, units:] * e / (1 + e) ** 2
    # an error of the gate's argument is one of dg, relative; of exp's argument, scaled by log2 e, the hardware's exp2 has |g| 2U more.  32 U
    # for the products; the other projection's own error enters in absolute terms; a chain of seq additions; bf16: D is rounded once
    size = np.abs(x) @ np.abs(W).T + np.abs(bias)
    eg, eu = (c + 2) * U * size[:, :units], (c + 2) * U * size[:, units:]
    off = np.abs(dg) * (eg + (4 * abs(at) + 32) * U + (HALF[dtype] if dtype == C.BF16 else 0)) + np.abs(dy) * eu * e / (1 + e) ** 2
    bound = off.T @ np.abs(x) + seq * U * (np.abs(dg).T @ np.abs(x))
    worst = float(np.max(np.abs(got - dg.T @ x) / bound))
    assert worst <= 1


# ------------------------------------------------------------------------------ dx over dy
def _over(b, kind, c):
    if kind == "sublayer":
        b.layernorm(c, src=-1)
        b.gated(c, 2 * c, act=C.GATE_SILU, bias=1)
        b.conv(2 * c, c, 1)
        b.dropout(0.2)
        b.addl(3, -1, relu=0)
    elif kind == "side by side":       # two readers of the input, whose gradients share dy's place
        b.layernorm(c, src=-1)
        b.gated(c, c, act=C.GATE_GELU, bias=1, src=-1)
        b.addl(0, 1, relu=0)
    elif kind == "dropped twice":
        b.dropout(0.2, src=-1)
        b.dropout(0.3, src=-1)
        b.addl(0, 1, relu=0)
    elif kind == "dropout and sum":
        b.dropout(0.2, src=-1)
        b.addl(0, -1, relu=0)
    elif kind == "norm and sum":
        b.layernorm(c, src=-1)
        b.addl(-1, 0, relu=0)
    elif kind == "gated and sum":
        b.gated(c, c, act=C.GATE_SIGMOID, src=-1)
        b.addl(0, -1, relu=0)
    elif kind == "convolutions":
        b.conv(c, c, 1, src=-1)
        b.conv(c, c, 3, src=-1)
        b.addl(0, 1, relu=0)
    else:
        getattr(b, kind)(*dict(layernorm=(c,), gated=(c, c), dropout=(0.2,), conv=(c, c, 3), bn=(c,), relu=())[kind], src=-1)


@pytest.mark.parametrize("dtype", [C.FP32, C.BF16])
@pytest.mark.parametrize("streams", [1, 3])
@pytest.mark.parametrize("kind", ["sublayer", "side by side", "dropped twice", "dropout and sum", "norm and sum", "gated and sum", "convolutions", "layernorm",
                                  "gated", "dropout", "conv", "bn", "relu"])
def test_dx_over_dy(kind, streams, dtype):
    """At dy's address, rows behind it and rows in front of it: the gradients that dx apart from dy gives, bit for bit."""
    c, rows = 64, 700
    b = C._Builder()
    _over(b, kind, c)
    st = C._stage("over", b.layers, dtype, (c, 1, rows), 2, 1, 1, 1, 1, C.BASE_SEED + 82, "xavier")
    xs, gs = stage_io(st)
    dy = torch.from_numpy(gs[0]).permute(0, 2, 3, 1).reshape(-1).to(DEV, tdtype(st))
    n, room = dy.numel(), 3 * c
    ref = None
    for shift in (None, 0, 3 * c, -3 * c, c // 2):
        g = GpuStage(st, gen.all_params(st, perturb=True), backward_stream=streams == 3)
        g.forward(0, xs[0])
        buf = torch.zeros(n + 2 * room, device=DEV, dtype=dy.dtype)
        buf[room:room + n] = dy
        dx = torch.zeros_like(dy) if shift is None else buf[room + shift:room + shift + n]
        torch.cuda.synchronize()
        B.bapipe_stage_backward(g.h, 0, buf[room:].data_ptr(), dx.data_ptr())
        torch.cuda.synchronize()
        got = [dx.clone().cpu().float().numpy()] + [a for i, (w, _) in enumerate(g.params) if w is not None for a in g.grads(i) if a is not None]
        g.close()
        ref = ref or got
        for a, r in zip(got, ref):
            assert np.array_equal(a, r) and np.any(a), (kind, shift)


# ------------------------------------------------------------------------------ filters that are streamed
@pytest.mark.parametrize("c,units,rows", [
    (2048, 4128, 1), (2048, 4128, 64), (2048, 4128, 65),         # both copies in panels, the last ones of rows that take them
    (2080, 4104, 5), (2056, 4112, 5),                            # only the one that forward reads, only the other
])
def test_gated_of_filters_that_are_streamed(c, units, rows):
    st = _stage(_one("gated", c, units, act=C.GATE_SILU, bias=1), C.BF16, (c, rows, 1), 1, 1)
    compare_minibatch(st)


def test_sublayer_of_filters_that_are_streamed():
    compare_minibatch(sublayer(c=2080, units=4112, seq=1, micro_batch=3, n_micro=1, stage_index=1, n_stages=1))


# ------------------------------------------------------------------------------ a slope and the library's own difference quotient
@pytest.mark.parametrize("act", [C.GATE_SIGMOID, C.GATE_SILU, C.GATE_GELU])
def test_the_slope_along_many_directions(act):
    """Float, along directions of one coordinate each and random ones: (f(x + h v) - f(x - h v)) / 2h of the library's own forward pass
    against its dx.  What the third derivative leaves of it is the oracle's alone: its quotient at h against its own dx."""
    st = sublayer(c=16, units=24, seq=2, micro_batch=64, n_micro=1, act=act, dtype=C.FP32, stage_index=1, n_stages=1, p=0.2)
    params = gen.all_params(st, perturb=True)
    xs, gs = stage_io(st)
    h, x0 = 2.0 ** -4, _f64(xs[0])
    # 64 samples of 2 x 16 elements: 32 directions along one coordinate of one position, 32 random ones
    v = np.random.default_rng(5).standard_normal((64, 16, 2, 1))
    for i in range(32):
        v[i] = 0
        v[i, i % 16, i // 16] = 1
    plus, minus = (np.float32(x0 + s * h * v) for s in (1, -1))
    v = (_f64(plus) - _f64(minus)) / (2 * h)                      # what the floats are apart
    per_sample = lambda a, b: np.sum(_f64(a) * _f64(b), axis=(1, 2, 3))  # noqa: E731

    def values(x):
        g, o = GpuStage(st, params), OracleStage(st, params)
        y = per_sample(g.forward(0, x), gs[0])
        g.close()
        return y, per_sample(o.forward(0, _f64(x)), gs[0])

    g, orc = GpuStage(st, params), OracleStage(st, params)
    y = g.forward(0, xs[0])
    orc.forward(0, x0)
    slope, exact = per_sample(g.backward(0, gs[0]), v), per_sample(orc.backward(0, gs[0]), v)
    g.close()
    (yp, op), (ym, om) = values(plus), values(minus)
    got, curve = (yp - ym) / (2 * h), np.abs((op - om) / (2 * h) - exact)
    # 64 U of every output, either side of the quotient: sums of 24 and 16 terms, the layer norm's, the activation's
    noise = 64 * U * np.sum(np.abs(gs[0]) * (1 + np.abs(y)), axis=(1, 2, 3)) / h
    size = np.abs(exact) + 1e-3 * np.linalg.norm(gs[0].reshape(64, -1), axis=1)
    assert np.all(np.abs(got - slope) <= curve + noise + 1e-4 * size), float(np.max((np.abs(got - slope) - curve - noise) / size))
    assert np.median((curve + noise) / size) <= 0.01             # a wrong dx would not hide in what is allowed
