"""Pins of the oracle's layer norm, gated linear layer and dropout: torch in 64 bits, central differences, published words of the
generator; and what bapipe_stage_create and bapipe_stage_set_dropout refuse, which takes no GPU."""
import ctypes as ct

import numpy as np
import pytest
import torch

from oracle import ops
from oracle.stage import OracleStage, one_f_one_b_order
from paper_2012_12544_amd import binding as B
from stage_inputs import configs as C
from stage_inputs import gen

rng = np.random.default_rng(7)
F = torch.nn.functional


def sublayer(c=24, units=40, seq=5, micro_batch=2, n_micro=3, act=C.GATE_SILU, bias=1, p=0.3, dtype=C.BF16, stage_index=2, n_stages=3):
    """x + dropout(W2 gated(layer norm(x))): the feed-forward sublayer of a transformer"""
    b = C._Builder()
    b.layernorm(c, src=-1)
    b.gated(c, units, act=act, bias=bias)
    b.conv(units, c, 1, bias=bias)
    b.dropout(p)
    b.addl(3, -1, relu=0)
    return C._stage("sublayer", b.layers, dtype, (c, seq, 1), micro_batch, n_micro, stage_index, n_stages, 1, C.BASE_SEED + 70, "xavier")


@pytest.mark.parametrize("words,counter,key", [
    ("6627e8d5 e169c58d bc57ac4c 9b00dbd8", "00000000 00000000 00000000 00000000", "00000000 00000000"),
    ("408f276d 41c83b0e a20bc7c6 6d5451fd", "ffffffff ffffffff ffffffff ffffffff", "ffffffff ffffffff"),
    ("d16cfe09 94fdcceb 5001e420 24126ea1", "243f6a88 85a308d3 13198a2e 03707344", "a4093822 299f31d0"),
])
def test_the_generator_gives_the_published_words(words, counter, key):
    c = np.array([[int(v, 16) for v in counter.split()]], np.uint32)
    got = ops.philox4x32(c, [int(v, 16) for v in key.split()])[0]
    assert " ".join("%08x" % v for v in got) == words


def test_dropout_factor():
    a = ops.dropout_factor((3, 5, 7, 2), 0.25, 9, 4, 1, 2)
    assert set(np.unique(a)) == {0.0, 1 / 0.75}
    assert np.array_equal(a, ops.dropout_factor((3, 5, 7, 2), 0.25, 9, 4, 1, 2))
    for other in ((8, 4, 1, 2), (9 + (1 << 32), 4, 1, 2), (9, 5, 1, 2), (9, 4, 0, 2), (9, 4, 1, 3)):
        assert not np.array_equal(a, ops.dropout_factor((3, 5, 7, 2), 0.25, *other))
    assert np.all(ops.dropout_factor((1, 3, 1, 1), 0.0, 1, 0, 0, 0) == 1)
    # 10^5 draws: within six standard deviations
    kept = np.mean(ops.dropout_factor((10, 100, 100, 1), 0.2, 5, 0, 0, 0) > 0)
    assert abs(kept - 0.8) < 6 * np.sqrt(0.16 / 1e5)
    # channels run fastest
    w = ops.philox4x32(np.array([[0, 4, 1, 2]], np.uint32), (9, 0))[0]
    assert np.array_equal(ops.dropout_factor((1, 2, 2, 1), 0.25, 9, 4, 1, 2)[0, :, :, 0].T.reshape(-1) > 0, w >= 2 ** 30)


def test_layernorm_against_torch():
    x, dy, w, b = rng.standard_normal((2, 7, 3, 4)) * 3 + 1, rng.standard_normal((2, 7, 3, 4)), rng.standard_normal(7), rng.standard_normal(7)
    t = [torch.from_numpy(v).requires_grad_() for v in (x, w, b)]
    yt = F.layer_norm(t[0].permute(0, 2, 3, 1), (7,), t[1], t[2], 1e-3).permute(0, 3, 1, 2)
    yt.backward(torch.from_numpy(dy))
    y, xhat, inv = ops.layernorm_fwd(x, w, b, 1e-3)
    dg, db = np.ones(7), np.ones(7)
    dx = ops.layernorm_bwd(xhat, inv, dy, w, dg, db)
    for got, want in ((y, yt), (dx, t[0].grad), (dg - 1, t[1].grad), (db - 1, t[2].grad)):
        np.testing.assert_allclose(got, want.detach().numpy(), rtol=1e-10, atol=1e-11)


@pytest.mark.parametrize("act", range(4))
def test_gated_against_torch(act):
    x, dy = rng.standard_normal((2, 6, 3, 2)), rng.standard_normal((2, 5, 3, 2))
    w, b = rng.standard_normal((10, 6)), rng.standard_normal(10)
    t = [torch.from_numpy(v).requires_grad_() for v in (x, w, b)]
    both = F.linear(t[0].permute(0, 2, 3, 1), t[1], t[2])
    yt = ([torch.sigmoid, F.silu, F.gelu, F.relu][act](both[..., :5]) * both[..., 5:]).permute(0, 3, 1, 2)
    yt.backward(torch.from_numpy(dy))
    y, saved = ops.gated_fwd(x, w, b, act)
    dw, db = np.ones((10, 6)), np.ones(10)
    dx = ops.gated_bwd(x, w, saved, act, dy, dw, db)
    for got, want in ((y, yt), (dx, t[0].grad), (dw - 1, t[1].grad), (db - 1, t[2].grad)):
        np.testing.assert_allclose(got, want.detach().numpy(), rtol=1e-10, atol=1e-11)


@pytest.mark.parametrize("act", [C.GATE_SIGMOID, C.GATE_SILU, C.GATE_GELU])
def test_sublayer_gradients_by_central_differences(act):
    st = sublayer(c=6, units=5, seq=3, n_micro=2, act=act)
    params = gen.all_params(st, perturb=True)
    xs = [np.float64(gen.stage_input(st, m)) for m in range(2)]
    gs = [np.float64(gen.upstream_grad(st, m)) for m in range(2)]

    def run(xs, params, back=False):
        o = OracleStage(st, params, storage="exact")
        o.dropout_seed, total, dx = 11, 0.0, []
        for t, m in one_f_one_b_order(2, o.depth):
            if t == "F":
                total += float(np.sum(o.forward(m, xs[m]) * gs[m]))
            else:
                dx.append(o.backward(m, gs[m]))
        return (total, dx, o) if back else total

    _, dx, o = run(xs, params, True)
    h = 1e-5
    for m in range(2):
        v = rng.standard_normal(xs[m].shape)
        moved = [[x + s * h * v if i == m else x for i, x in enumerate(xs)] for s in (1, -1)]
        assert (run(moved[0], params) - run(moved[1], params)) / (2 * h) == pytest.approx(float(np.sum(dx[m] * v)), rel=1e-7)
    for i, (w, b) in enumerate(params):
        for k, p in enumerate((w, b)):
            if p is None:
                continue
            v = rng.standard_normal(p.shape)
            f = [run(xs, [tuple(np.float64(q) + s * h * v if (j, n) == (i, k) else q for n, q in enumerate(pair)) for j, pair in enumerate(params)])
                 for s in (1, -1)]
            assert (f[0] - f[1]) / (2 * h) == pytest.approx(float(np.sum((o.dw, o.db)[k][i] * v)), rel=1e-7)


# ------------------------------------------------------------------------------ refusals
def _status(layers, shape=(8, 4, 1), micro_batch=2, dtype=C.BF16, n_stages=1, stage_index=1):
    """Of creating the stage with an allocator that has nothing: E_OOM where the description is in order."""
    st = C._stage("refused", layers, dtype, shape, micro_batch, 1, stage_index, n_stages, 1, 0, "xavier")
    o = B.make_opts(st)
    o.mem.alloc, o.mem.free = B.ALLOC_FN(lambda n, ctx: None), B.FREE_FN(lambda ptr, ctx: None)
    with pytest.raises(B.BapipeError) as e:
        B.bapipe_stage_create(layers, micro_batch, 1, o)
    return e.value.status


def _one(method, *args, **changed):
    b = C._Builder()
    getattr(b, method)(*args, src=-1)
    b.layers[0].update(changed)
    return b.layers


def test_what_create_takes_and_refuses():
    assert _status(_one("layernorm", 8)) == B.E_OOM
    assert _status(_one("layernorm", 9)) == B.E_SHAPE
    assert _status(_one("layernorm", 8, cout=4)) == B.E_SHAPE
    for eps in (0.0, -1.0, float("nan"), float("inf")):
        assert _status(_one("layernorm", 8, eps=eps)) == B.E_INVALID
    assert _status(_one("layernorm", 8, fuse_relu=1)) == B.E_UNSUPPORTED

    assert _status(_one("gated", 8, 3)) == B.E_OOM
    assert _status(_one("gated", 7, 3)) == B.E_SHAPE
    for bad in (dict(cout=0), dict(cout=-8), dict(cin=0), dict(kh=-1), dict(kh=4), dict(cout=2 ** 31 - 1)):
        assert _status(_one("gated", 8, 3, **bad)) == B.E_INVALID
    assert _status(_one("gated", 8, 3, fuse_relu=1)) == B.E_UNSUPPORTED
    # both projections of a micro-batch: 2 * 2^14 positions * 2 * 2^14 units of 2 bytes are 2 GiB, of 4 bytes twice that
    assert _status(_one("gated", 8, 2 ** 14), shape=(8, 2 ** 14, 1)) == B.E_UNSUPPORTED
    assert _status(_one("gated", 8, 2 ** 14 - 8), shape=(8, 2 ** 14, 1)) == B.E_OOM
    assert _status(_one("gated", 8, 2 ** 14 - 8), shape=(8, 2 ** 14, 1), dtype=C.FP32) == B.E_UNSUPPORTED
    assert _status(_one("gated", 2 ** 15, 2 ** 13 + 1), shape=(2 ** 15, 1, 1)) == B.E_UNSUPPORTED        # 2 GiB of weights

    for p in (0.0, 0.5, np.nextafter(np.float32(1), np.float32(0))):
        assert _status(_one("dropout", p)) == B.E_OOM
    for p in (-0.1, 1.0, 2.0, float("nan"), float("inf")):
        assert _status(_one("dropout", p)) == B.E_INVALID
    assert _status(_one("dropout", 0.5, fuse_relu=1)) == B.E_UNSUPPORTED
    assert _status(_one("dropout", 0.5), n_stages=65537) == B.E_UNSUPPORTED
    assert _status(_one("dropout", 0.5), n_stages=65536, stage_index=65536) == B.E_OOM


@pytest.mark.parametrize("method,args", [("layernorm", (32,)), ("gated", (32, 8)), ("dropout", (0.5,))])
def test_a_flattened_map_is_refused(method, args):
    """Its elements lie in the map's order, not in that of the features; one of single pixels is a tensor like any other."""
    def layers(flattened):
        b = C._Builder()
        b.layernorm(8 if flattened else 32, src=-1)
        b.flatten()
        getattr(b, method)(*args)
        return b.layers

    assert _status(layers(True), shape=(8, 4, 1)) == B.E_UNSUPPORTED
    assert _status(layers(False), shape=(32, 1, 1)) == B.E_OOM


def test_set_dropout_without_a_stage():
    assert B.load().bapipe_stage_set_dropout(None, ct.c_uint64(1), ct.c_uint32(0)) == B.E_INVALID


def test_the_binding_names_the_layer_kinds_of_the_descriptions():
    for name in C.KIND_NAMES:
        assert getattr(B, name.upper()) == getattr(C, name.upper())
    for name in ("SIGMOID", "SILU", "GELU", "RELU"):
        assert getattr(B, "GATE_" + name) == getattr(C, "GATE_" + name)
