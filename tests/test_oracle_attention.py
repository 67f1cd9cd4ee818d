"""The oracle's rotary positions and attention pinned: forward formulas and gradients against torch's in 64 bits, gradients against
differences, masks that leave a row empty; and what bapipe_stage_create, bapipe_stage_set_spans and bapipe_stage_set_rotary refuse,
which takes no GPU."""
import ctypes as ct
import math

import numpy as np
import pytest
import torch

from oracle import ops
from oracle.stage import OracleStage
from paper_2012_12544_amd import binding as B
from stage_inputs import configs as C
from stage_inputs import gen
from test_oracle_sublayer import _status

rng = np.random.default_rng(11)


def attention_sublayer(heads=4, groups=2, d=8, c=24, seq=6, micro_batch=2, n_micro=2, norm=1, mask=C.MASK_CAUSAL, cap=0.0, bias=0,
                       turning=None, layout=C.ROTARY_HALVES, dtype=C.BF16, stage_index=1, n_stages=2):
    """x + W2 attention(rotary(W1 layer norm(x))): the attention sublayer of a transformer"""
    b = C._Builder()
    b.layernorm(c, src=-1)
    b.conv(c, (heads + 2 * groups) * d, 1)
    b.rotary(heads, groups, d, turning, layout, norm)
    b.attention(heads, groups, d, mask, cap, bias)
    b.conv(heads * d, c, 1)
    b.addl(4, -1, relu=0)
    return C._stage("attention_sublayer", b.layers, dtype, (c, seq, 1), micro_batch, n_micro, stage_index, n_stages, 1, C.BASE_SEED + 90, "xavier")


def some_spans(kind, N, T, r):
    """Documents with padding behind, a window, a prefix, or spans at random, some of them empty or outside: int32 (N, T, 2)."""
    at = np.arange(T)
    spans = np.zeros((N, T, 2), np.int32)
    for n in range(N):
        if kind == "documents":
            used = T - int(r.integers(0, T // 4 + 1))
            cuts = np.unique(np.concatenate([[0, used], r.integers(0, used + 1, size=T // 20 + 1)]))
            for lo, hi in zip(cuts[:-1], cuts[1:]):
                spans[n, lo:hi, 0], spans[n, lo:hi, 1] = lo, at[lo:hi] + 1
        elif kind == "window":
            w = int(r.integers(1, T + 1))
            spans[n, :, 0], spans[n, :, 1] = np.maximum(at + 1 - w, 0), at + 1
        elif kind == "prefix":
            spans[n, :, 1] = np.maximum(at + 1, int(r.integers(0, T + 1)))
        else:
            spans[n] = r.integers(-T // 2, T + T // 2 + 1, size=(T, 2))
    return spans


@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("heads,groups,d,T,r", [(3, 1, 6, 4, 6), (2, 2, 9, 1, 4), (4, 2, 5, 7, 0)])
def test_rotary(heads, groups, d, T, r, norm, pairs):
    x, dy = (rng.standard_normal((2, (heads + 2 * groups) * d, T, 1)) for _ in range(2))
    gains = 1 + 0.3 * rng.standard_normal((2, d)) if norm else None
    by = ops.rotary_angles(T, r, base=50.0, first_position=3)
    dg = np.zeros((2, d))
    y = ops.rotary_fwd(x, heads, groups, by, pairs, gains, 1e-3)
    dx = ops.rotary_bwd(x, dy, heads, groups, by, pairs, gains, 1e-3, dg)
    # by one matrix for each position, by the definition
    tx = torch.tensor(x, requires_grad=True)
    tg = torch.tensor(gains if norm else np.ones((2, d)), requires_grad=True)
    rows = []
    for t in range(T):
        turn = torch.eye(d, dtype=torch.float64)
        for j in range(r // 2):
            a, b = (2 * j, 2 * j + 1) if pairs else (j, j + r // 2)
            angle = (3 + t) * 50.0 ** (-2 * j / r)
            turn[a, a] = turn[b, b] = math.cos(angle)
            turn[a, b], turn[b, a] = -math.sin(angle), math.sin(angle)
        for h in range(heads + 2 * groups):
            z = tx[:, h * d:(h + 1) * d, t, 0]
            if h < heads + groups:
                if norm:
                    z = z / torch.sqrt((z * z).mean(1, keepdim=True) + 1e-3) * tg[0 if h < heads else 1]
                z = z @ turn.T
            rows.append(z)
    ty = torch.stack(rows).reshape(T, heads + 2 * groups, 2, d).permute(2, 1, 3, 0).reshape(x.shape)
    (ty * torch.tensor(dy)).sum().backward()
    np.testing.assert_allclose(y, ty.detach().numpy(), rtol=1e-12, atol=1e-12)
    np.testing.assert_allclose(dx, tx.grad.numpy(), rtol=1e-11, atol=1e-12)
    if norm:
        np.testing.assert_allclose(dg, tg.grad.numpy(), rtol=1e-11, atol=1e-12)


def test_angles_of_stretched_contexts():
    plain = np.angle(ops.rotary_angles(2, 64)[1])
    np.testing.assert_allclose(plain, 10000.0 ** (-np.arange(32) / 32), rtol=1e-13)
    np.testing.assert_allclose(np.angle(ops.rotary_angles(2, 64, factor=8.0)[1]), plain / 8, rtol=1e-12)
    changed = dict(factor=8.0, original_length=1000.0, low_turns=1.0, high_turns=4.0)
    turns, got = 1000 * plain / (2 * math.pi), np.angle(ops.rotary_angles(2, 64, **changed)[1])
    assert (turns > 4).any() and (turns < 1).any() and ((turns > 1) & (turns < 4)).any()
    np.testing.assert_allclose(got[turns >= 4], plain[turns >= 4], rtol=1e-12)
    np.testing.assert_allclose(got[turns <= 1], plain[turns <= 1] / 8, rtol=1e-12)
    between = (turns > 1) & (turns < 4)
    assert np.all(got[between] < plain[between]) and np.all(got[between] > plain[between] / 8)
    far = ops.rotary_angles(2, 64, first_position=10 ** 6, magnitude=1.25)
    np.testing.assert_allclose(np.abs(far), 1.25, rtol=1e-13)
    np.testing.assert_allclose(far[1] / far[0], np.exp(1j * plain), rtol=1e-9)


@pytest.mark.parametrize("mask", ["none", "causal", "documents", "window", "prefix", "random"])
@pytest.mark.parametrize("cap,bias", [(0.0, 0), (2.0, 0), (0.0, 8), (3.0, 4)])
def test_attention(mask, cap, bias):
    heads, groups, d, T, N = 4, 2, 5, 9, 2
    x, dy = (rng.standard_normal((N, c * d, T, 1)) for c in (heads + 2 * groups, heads))
    x[:, :heads * d] *= 2
    spans = some_spans(mask, N, T, rng)
    sees = ops.attention_sees({"none": 0, "causal": 1}.get(mask, 2), N, T, spans)
    p, slope = ops.attention_probabilities(x, heads, groups, sees, cap, bias)
    y, dx = ops.attention_fwd(x, heads, groups, p), ops.attention_bwd(x, dy, heads, groups, p, slope)
    tx, ty = torch.tensor(x, requires_grad=True), []
    for n in range(N):
        for h in range(heads):
            g = h // (heads // groups)
            q, k, v = (tx[n, i * d:(i + 1) * d, :, 0].T for i in (h, heads + g, heads + groups + g))
            for t in range(T):
                lo, hi = {"none": (0, T), "causal": (0, t + 1)}.get(mask, (max(int(spans[n, t, 0]), 0), min(int(spans[n, t, 1]), T)))
                if lo >= hi:
                    ty.append(torch.zeros(d, dtype=torch.float64))
                    continue
                s = k[lo:hi] @ q[t] / math.sqrt(d)
                s = cap * torch.tanh(s / cap) if cap else s
                s = s - (2.0 ** (-bias * (h + 1) / heads) if bias else 0.0) * (torch.arange(lo, hi) - t).abs()
                ty.append(torch.softmax(s, 0) @ v[lo:hi])
    ty = torch.stack(ty).reshape(N, heads, T, d).transpose(2, 3).reshape(y.shape)
    (ty * torch.tensor(dy)).sum().backward()
    np.testing.assert_allclose(y, ty.detach().numpy(), rtol=1e-12, atol=1e-12)
    np.testing.assert_allclose(dx, tx.grad.numpy(), rtol=1e-11, atol=1e-12)


@pytest.mark.parametrize("norm,layout,mask,cap,bias", [(1, 0, C.MASK_CAUSAL, 0.0, 0), (0, 1, C.MASK_SPANS, 2.0, 8)])
def test_the_sublayers_gradients_against_differences(norm, layout, mask, cap, bias):
    st = attention_sublayer(norm=norm, layout=layout, mask=mask, cap=cap, bias=bias, dtype=C.FP32, n_micro=1, n_stages=1)
    params = gen.all_params(st, perturb=True)
    x, dy = gen.stage_input(st, 0), gen.upstream_grad(st, 0)
    spans = some_spans("random", 2, 6, np.random.default_rng(5))

    def loss(xs, ps):
        o = OracleStage(st, ps, storage="exact")
        o.spans[0] = spans
        return float((o.forward(0, xs) * dy).sum())

    o = OracleStage(st, params, storage="exact")
    o.spans[0] = spans
    o.forward(0, x)
    dx = o.backward(0, dy)
    h = 1e-5
    for _ in range(12):
        u = rng.standard_normal(x.shape)
        u /= np.linalg.norm(u)
        slope = (loss(x + h * u, params) - loss(x - h * u, params)) / (2 * h)
        assert abs(slope - float((dx * u).sum())) <= 1e-7 * (1 + np.linalg.norm(dx))
    for i, (w, _) in enumerate(params):
        if w is None:
            continue
        u = rng.standard_normal(w.shape)
        u /= np.linalg.norm(u)
        moved = [[p if j != i else (p[0].astype(np.float64) + e * u, p[1]) for j, p in enumerate(params)] for e in (h, -h)]
        slope = (loss(x, moved[0]) - loss(x, moved[1])) / (2 * h)
        assert abs(slope - float((o.dw[i] * u).sum())) <= 1e-7 * (1 + np.linalg.norm(o.dw[i]))


def test_what_the_oracle_rounds():
    """Between a ROTARY and the ATTENTION that alone reads it nothing; with another reader all of it."""
    def run(second):
        b = C._Builder()
        b.rotary(2, 1, 4, norm=1, src=-1)
        b.attention(2, 1, 4)
        if second:
            b.conv(16, 8, 1, src=0)
            b.addl(1, 2, relu=0)
        st = C._stage("s", b.layers, C.BF16, (16, 5, 1), 1, 1, 1, 1, 1, 3, "xavier")
        o = OracleStage(st, gen.all_params(st))
        o.trace = {}
        o.forward(0, gen.stage_input(st, 0))
        o.backward(0, gen.upstream_grad(st, 0))
        return o

    for second in (0, 1):
        o = run(second)
        for t in (o.trace[(0, 1)]["x"], o.trace[(0, 1)]["dx"]):
            t = t[:, :12]                                    # queries and keys
            assert np.array_equal(t, ops.round_bf16(t)) == bool(second)
        assert (0 in o.float_grads) == (not second)


# ------------------------------------------------------------------------------ refusals
def _layer(method, *args, **changed):
    b = C._Builder()
    getattr(b, method)(*args, src=-1)
    b.layers[0].update(changed)
    return b.layers


@pytest.mark.parametrize("method", ["rotary", "attention"])
def test_what_create_takes_and_refuses_of_heads(method):
    shape = dict(shape=(32, 4, 1))
    assert _status(_layer(method, 4, 2, 4), **shape) == B.E_OOM
    assert _status(_layer(method, 4, 2, 4), dtype=C.FP32, **shape) == B.E_OOM
    assert _status(_layer(method, 1, 1, 256), shape=(768, 1, 1)) == B.E_OOM
    assert _status(_layer(method, 1, 1, 1), shape=(3, 1, 1), dtype=C.FP32) == B.E_OOM
    assert _status(_layer(method, 1, 1, 257), shape=(771, 1, 1)) == B.E_UNSUPPORTED
    for bad in (dict(kh=0), dict(kw=0), dict(kh=-4), dict(kw=-2), dict(kh=2 ** 21)):
        assert _status(_layer(method, 4, 2, 4, **bad), **shape) == B.E_INVALID
    assert _status(_layer(method, 4, 2, 4, kh=5), **shape) == B.E_SHAPE            # heads that are shared unevenly
    assert _status(_layer(method, 4, 2, 4, cin=24), **shape) == B.E_SHAPE
    assert _status(_layer(method, 4, 2, 4, cout=8), **shape) == B.E_SHAPE
    assert _status(_layer(method, 4, 2, 4), shape=(33, 4, 1)) == B.E_SHAPE
    assert _status(_layer(method, 4, 2, 4, cin=33), shape=(33, 4, 1)) == B.E_SHAPE
    assert _status(_layer(method, 4, 2, 4), shape=(32, 4, 2)) == B.E_SHAPE         # a map, not a sequence
    assert _status(_layer(method, 4, 2, 4, fuse_relu=1), **shape) == B.E_UNSUPPORTED
    # a tensor of 2 GiB
    assert _status(_layer(method, 4, 2, 4), shape=(32, 2 ** 24, 1)) == B.E_UNSUPPORTED


def test_what_create_refuses_of_a_rotary():
    shape = dict(shape=(32, 4, 1))
    for good in (dict(pad=0), dict(pad=2), dict(stride=1), dict(has_bias=1, eps=1e-6)):
        assert _status(_layer("rotary", 4, 2, 4, **good), **shape) == B.E_OOM
    for bad in (dict(pad=-2), dict(pad=3), dict(pad=6), dict(stride=2), dict(stride=-1), dict(eps=1e-6), dict(has_bias=1, eps=0.0),
                dict(has_bias=1, eps=-1.0), dict(has_bias=1, eps=float("nan")), dict(has_bias=1, eps=float("inf")), dict(eps=float("nan"))):
        assert _status(_layer("rotary", 4, 2, 4, **bad), **shape) == B.E_INVALID


def test_what_create_refuses_of_an_attention():
    shape = dict(shape=(32, 4, 1))
    for good in (dict(stride=0), dict(stride=2), dict(eps=50.0), dict(pad=64), dict(pad=8, eps=1e30)):
        assert _status(_layer("attention", 4, 2, 4, **good), **shape) == B.E_OOM
    for bad in (dict(stride=3), dict(stride=-1), dict(pad=-1), dict(pad=65), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf"))):
        assert _status(_layer("attention", 4, 2, 4, **bad), **shape) == B.E_INVALID
    assert _status(_layer("attention", 4, 2, 4, has_bias=1), **shape) == B.E_UNSUPPORTED

    def two(seq2):                                           # spans of sequences of two lengths
        b = C._Builder()
        b.attention(4, 2, 4, mask=C.MASK_SPANS, src=-1)
        b.conv(16, 32, 1)
        if seq2 != 8:
            b.add(kind=C.MAXPOOL2D, k=2, stride=2)
            b.layers[-1].update(kw=1)
        b.attention(4, 2, 4, mask=C.MASK_SPANS)
        return b.layers

    assert _status(two(8), shape=(32, 8, 1)) == B.E_OOM
    assert _status(two(4), shape=(32, 8, 1)) == B.E_SHAPE


def test_what_create_takes_and_refuses_of_caps():
    """Of one below 2^-100 the reciprocal, times the score's factors, may be infinite, and a score of 0 times that is none."""
    for cap in (2.0 ** -100, 1.0, 2.0 ** 100, float(np.finfo(np.float32).max)):
        assert _status(_layer("attention", 4, 2, 4, eps=cap), shape=(32, 4, 1)) == B.E_OOM, cap
    for cap in (2.0 ** -101, 2.0 ** -126, 1e-40, 2.0 ** -149):
        assert _status(_layer("attention", 4, 2, 4, eps=cap), shape=(32, 4, 1)) == B.E_INVALID, cap


def test_what_create_refuses_of_many_blocks():
    """A launch holds less than 2^24 blocks of 256 threads; a block is 128 positions of a head, or what there are of them."""
    for heads, micro_batch, seq, want in ((256, 65535, 1, B.E_OOM), (256, 65536, 1, B.E_UNSUPPORTED), (256, 65536, 60, B.E_UNSUPPORTED), (4096, 4095, 1, B.E_OOM),
                                          (4096, 4096, 1, B.E_UNSUPPORTED), (2 ** 20, 16, 1, B.E_UNSUPPORTED), (2 ** 20, 15, 8, B.E_OOM)):
        d = 1 if heads * micro_batch * seq > 2 ** 26 else 4
        for mask in (C.MASK_NONE, C.MASK_SPANS):
            assert _status(_layer("attention", heads, 1, d, mask), shape=((heads + 2) * d, seq, 1), micro_batch=micro_batch) == want, (heads, micro_batch, seq)


@pytest.mark.parametrize("method", ["rotary", "attention"])
def test_a_flattened_sequence_is_refused(method):
    b = C._Builder()
    b.layernorm(8, src=-1)
    b.flatten()
    getattr(b, method)(4, 2, 4)
    assert _status(b.layers, shape=(8, 4, 1)) == B.E_UNSUPPORTED


def test_calls_without_a_stage():
    lib = B.load()
    assert lib.bapipe_stage_set_spans(None, ct.c_int(0), None) == B.E_INVALID
    assert lib.bapipe_stage_set_rotary(None, ct.c_int(0), None) == B.E_INVALID


def test_the_binding_names_what_the_descriptions_do():
    for name in ("ROTARY_HALVES", "ROTARY_PAIRS", "MASK_NONE", "MASK_CAUSAL", "MASK_SPANS"):
        assert getattr(B, name) == getattr(C, name)
