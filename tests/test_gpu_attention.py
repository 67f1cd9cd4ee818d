"""Rotary positions and attention on the GPU against the oracle in 64 bits, through the C ABI: head widths, head counts, lengths,
masks, caps, slopes; angles and norms; the sublayer of a transformer that they make up.

Rounding to storage is off by at most HALF relative to the value; U is that of a float.  Two kinds of bounds:

element by element, the sum of what every rounding on the way can do at most (first order, 5 % on top for the second): _bounds;

in the 2-norm, where roundings are independent: one of relative size up to h has a root mean square of at most h / sqrt(3), so k of
them give sqrt(k / 3) h, and twice that is allowed.  An output of a bf16 stage has been through two (a probability, itself), a
gradient through five (a probability, the output in dout . o, its own, the gradient of a score, itself).  Floats: the sums over d
channels and T keys are random walks of steps U, on scores of size s: 4 (sqrt(d) + sqrt(T) + 8) (1 + s) U."""
import math

import numpy as np
import pytest
import torch

from gpu_harness import DEV, GpuStage, from_dev, stage_io, tdtype, to_dev
from oracle import ops
from oracle.stage import OracleStage, one_f_one_b_order
from paper_2012_12544_amd import binding as B
from stage_inputs import configs as C
from stage_inputs import gen
from test_oracle_attention import attention_sublayer, some_spans

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {C.FP32: 2.0 ** -24, C.BF16: 2.0 ** -8}
BOTH = pytest.mark.parametrize("dtype", [C.FP32, C.BF16])


def _stage(layers, dtype, shape, micro_batch=2, n_micro=1, stage_index=1, n_stages=1, seed=95):
    return C._stage("one", layers, dtype, shape, micro_batch, n_micro, stage_index, n_stages, 1, C.BASE_SEED + seed, "xavier")


def _norm(a):
    return float(np.linalg.norm(a))


def _spans(st, kind, seed=3):
    r = np.random.default_rng(seed)
    return [some_spans(kind, st["micro_batch"], st["in_h"], r) for _ in range(st["n_micro"])]


def _has_spans(st):
    return any(L["kind"] == C.ATTENTION and L["stride"] == C.MASK_SPANS for L in st["layers"])


def run(st, params, xs, gs, spans=None, angles=None, static=False, layout=B.NHWC, backward_stream=False):
    """One mini-batch in 1F1B order: y, dx per micro-batch, accumulated gradients."""
    g = GpuStage(st, params, layout=layout, backward_stream=backward_stream)
    for i, a in (angles or {}).items():
        B.bapipe_stage_set_rotary(g.h, i, **a)
    out, keep = {}, []
    for t, m in one_f_one_b_order(st["n_micro"], B.bapipe_stage_stash_bytes(g.h)[1]):
        if t == "F":
            if spans is not None:
                keep.append(torch.from_numpy(spans[m]).to(DEV))
                torch.cuda.synchronize()
                B.bapipe_stage_set_spans(g.h, m, keep[-1].data_ptr())
            out["y%d" % m] = g.forward(m, xs[m])
            if spans is not None:
                keep[-1].fill_(1)                            # the pass keeps a copy
        else:
            out["dx%d" % m] = g.backward(m, gs[m], static=static)
    for i, (w, b) in enumerate(params):
        if w is not None:
            out["dw%d" % i], db = g.grads(i)
            if db is not None:
                out["db%d" % i] = db
    g.close()
    return out


def oracle(st, params, xs, gs, spans=None, angles=None, trace=None):
    o = OracleStage(st, params)
    o.trace = trace
    o.angles = angles or {}
    out = {}
    for t, m in one_f_one_b_order(st["n_micro"], o.depth):
        if t == "F":
            if spans is not None:
                o.spans[m] = spans[m]
            out["y%d" % m] = o.forward(m, xs[m])
        else:
            out["dx%d" % m] = o.backward(m, gs[m])
    for i, (w, b) in enumerate(params):
        if w is not None:
            out["dw%d" % i] = o.dw[i]
            if b is not None:
                out["db%d" % i] = o.db[i]
    return out


def _within(got, ref, bound, what):
    assert got.shape == ref.shape and np.all(np.isfinite(got)), what
    worst = np.max(np.abs(got - ref) - bound)
    assert worst <= 0, (what, float(worst), float(np.max(np.abs(got - ref))))


# ------------------------------------------------------------------------------ attention
def _bounds(st, x, dy, spans):
    """Exact y and dx of a stage of one ATTENTION, and what they may be off by, element by element."""
    L = st["layers"][0]
    H, G, cap, bias = L["kh"], L["kw"], L["eps"], L["pad"]
    h = 0.0 if st["dtype"] == C.FP32 else HALF[C.BF16]       # of an operand
    x, dy = np.asarray(x, np.float64), np.asarray(dy, np.float64)
    z, do = ops.split_heads(x, H + 2 * G), ops.split_heads(dy, H)
    N, _, T, d = z.shape
    per = H // G
    q = z[:, :H]
    k, v = (np.repeat(t, per, axis=1) for t in (z[:, H:H + G], z[:, H + G:]))
    turn = lambda t: t.transpose(0, 1, 3, 2)                 # noqa: E731
    sees = ops.attention_sees(L["stride"], N, T, spans)
    p, slope = ops.attention_probabilities(x, H, G, sees, cap, bias)
    raw = q @ turn(k) / math.sqrt(d)
    i = np.arange(T)
    fall = (2.0 ** (-bias * np.arange(1, H + 1) / H))[:, None, None] * np.abs(i[:, None] - i) if bias else np.zeros((1, T, T))
    size = np.abs(raw) if not cap else np.minimum(np.abs(raw), cap)
    # of a score: its product, the cap, the bias; 16 roundings of arguments and of the exponential; the sum it is taken relative to
    delta = (d + 16) * U * (np.abs(q) @ turn(np.abs(k))) / math.sqrt(d) + 16 * U * (1 + size + fall) + (8 * U * min(cap, 4096.0) if cap else 0)
    delta = np.where(sees, delta, 0.0)
    rho = delta + (p * delta).sum(-1, keepdims=True) + (T + 16) * U + 16 * U * (size + fall)
    y = p @ v
    dy_err = (p * (rho + h)) @ np.abs(v) + (T + 16) * U * (p @ np.abs(v))
    dp = do @ turn(v)
    D = (do * y).sum(-1, keepdims=True)
    o_err = dy_err + HALF[st["dtype"]] * np.abs(y)
    gap_err = (d + 8) * U * (np.abs(do) @ turn(np.abs(v))) + (np.abs(do) * (o_err + d * U * np.abs(y))).sum(-1, keepdims=True)
    gap = dp - D
    # the cap's slope 4 r (1 - r), off by as much as r is
    slope_err = 16 * U + (2 * delta / cap if cap else 0) + 8 * U
    ds = p * gap * slope / math.sqrt(d)
    ds_err = (p * (rho * np.abs(gap) + gap_err) * slope + p * np.abs(gap) * slope_err) / math.sqrt(d)
    op_err = ds_err + (h + 8 * U) * np.abs(ds)

    def shared(t):
        return t.reshape(N, G, per, T, d).sum(2)

    dv, dv_err = shared(turn(p) @ do), shared(turn(p * (rho + h + (per * T + 16) * U)) @ np.abs(do))
    dq, dq_err = ds @ k, (op_err + (T + 16) * U * np.abs(ds)) @ np.abs(k)
    dk, dk_err = shared(turn(ds) @ q), shared(turn(op_err + (per * T + 16) * U * np.abs(ds)) @ np.abs(q))
    half = HALF[st["dtype"]]
    dx, dx_err = np.concatenate([dq, dk, dv], 1), np.concatenate([dq_err, dk_err, dv_err], 1)
    join = ops.join_heads
    return (join(y), join(1.05 * dy_err + half * np.abs(y) + 1e-30), join(dx), join(1.05 * dx_err + half * np.abs(dx) + 1e-30),
            float(np.std(raw) + np.max(fall) * 0.01))


def _check_attention(st, kind="random", static=False, layout=B.NHWC, scale=1.0):
    xs, gs = stage_io(st)
    if scale != 1.0:                                         # queries and keys: a power of two, so that bf16 holds it
        n = st["in_c"] - st["layers"][0]["kw"] * (st["in_c"] // (st["layers"][0]["kh"] + 2 * st["layers"][0]["kw"]))
        for x in xs:
            x[:, :n] *= scale
    spans = _spans(st, kind) if _has_spans(st) else None
    got = run(st, [(None, None)], xs, gs, spans, static=static, layout=layout)
    H, G = st["layers"][0]["kh"], st["layers"][0]["kw"]
    d, T = st["in_c"] // (H + 2 * G), st["in_h"]
    for m in range(st["n_micro"]):
        y, y_err, dx, dx_err, s = _bounds(st, xs[m], gs[m], None if spans is None else spans[m])
        _within(got["y%d" % m], y, y_err, "y")
        _within(got["dx%d" % m], dx, dx_err, "dx")
        loose = 4 * (math.sqrt(d) + math.sqrt(T) + 8) * (1 + s) * U
        walk = (lambda k: loose) if st["dtype"] == C.FP32 else (lambda k: 2 * math.sqrt(k / 3) * HALF[C.BF16] + loose)
        assert _norm(got["y%d" % m] - y) <= walk(2) * _norm(y), (_norm(got["y%d" % m] - y) / _norm(y), walk(2))
        cut = [0, H * d, (H + G) * d, (H + 2 * G) * d]
        for name, lo, hi in zip("qkv", cut, cut[1:]):
            a, r = got["dx%d" % m][:, lo:hi], dx[:, lo:hi]
            # gradients of queries and keys are differences: measured against what they are made of where little of it is left
            against = max(_norm(r), 0.2 * _norm(dx) * math.sqrt((hi - lo) / (cut[3])))
            assert _norm(a - r) <= walk(5) * against, (name, _norm(a - r) / against, walk(5))


def _attention(dtype, heads, groups, d, T, mask=C.MASK_CAUSAL, cap=0.0, bias=0, micro_batch=2, n_micro=1, stage_index=1, n_stages=1):
    b = C._Builder()
    b.attention(heads, groups, d, mask, cap, bias, src=-1)
    return _stage(b.layers, dtype, ((heads + 2 * groups) * d, T, 1), micro_batch, n_micro, stage_index, n_stages)


@BOTH
@pytest.mark.parametrize("d", [1, 2, 7, 8, 24, 32, 33, 40, 64, 72, 75, 80, 96, 100, 128, 136, 160, 192, 200, 250, 256])
def test_attention_of_heads_of_every_width(dtype, d):
    _check_attention(_attention(dtype, 2, 1, d, 70))


@BOTH
@pytest.mark.parametrize("T", [1, 2, 31, 32, 33, 63, 64, 65, 127, 128, 129, 200, 300])
@pytest.mark.parametrize("mask", [C.MASK_NONE, C.MASK_CAUSAL])
def test_attention_of_sequences_of_every_length(dtype, T, mask):
    _check_attention(_attention(dtype, 2, 2, 40, T, mask))


@BOTH
@pytest.mark.parametrize("kind", ["documents", "window", "prefix", "random"])
@pytest.mark.parametrize("d,T", [(16, 5), (45, 90), (64, 257), (128, 140), (256, 70)])
def test_attention_with_spans(dtype, kind, d, T):
    _check_attention(_attention(dtype, 4, 2, d, T, C.MASK_SPANS, n_micro=2), kind)


@BOTH
@pytest.mark.parametrize("heads,groups", [(1, 1), (3, 3), (8, 1), (12, 4), (10, 2)])
def test_attention_with_shared_key_heads(dtype, heads, groups):
    _check_attention(_attention(dtype, heads, groups, 24, 150, C.MASK_NONE, micro_batch=3))


@BOTH
@pytest.mark.parametrize("cap,bias,scale", [(2.0, 0, 1.0), (30.0, 0, 4.0), (5000.0, 0, 1.0), (0.0, 8, 1.0), (0.0, 64, 1.0), (4.0, 3, 2.0), (0.0, 0, 8.0)])
@pytest.mark.parametrize("mask,d", [(C.MASK_NONE, 32), (C.MASK_CAUSAL, 80), (C.MASK_SPANS, 56)])
def test_attention_with_caps_and_slopes(dtype, cap, bias, scale, mask, d):
    _check_attention(_attention(dtype, 6, 2, d, 100, mask, cap, bias), scale=scale)


@BOTH
@pytest.mark.parametrize("bias", [0, 6])
@pytest.mark.parametrize("rotary", [0, 1])
def test_caps_that_no_score_comes_near(dtype, rotary, bias):
    """c tanh(s / c) is s - s^3 / 3 c^2 ..: for c of 2^100 and more a float's s up to 2^87.  The same bits as without a cap, up to the largest float."""
    def stage(cap):
        b = C._Builder()
        if rotary:
            b.rotary(4, 2, 40, norm=1, src=-1)
        b.attention(4, 2, 40, C.MASK_CAUSAL, cap, bias, src=0 if rotary else -1)
        return _stage(b.layers, dtype, (320, 90, 1))

    params = gen.all_params(stage(0.0), perturb=True)
    xs, gs = stage_io(stage(0.0))
    ref = run(stage(0.0), params, xs, gs)
    for cap in (2.0 ** 100, 2.0 ** 127, float(np.finfo(np.float32).max)):
        got = run(stage(cap), params, xs, gs)
        assert all(np.array_equal(got[k], ref[k]) for k in ref), cap


@BOTH
@pytest.mark.parametrize("cap", [2.0 ** -100, 2.0 ** 99])
def test_the_smallest_cap_and_a_large_one(dtype, cap):
    _check_attention(_attention(dtype, 4, 2, 40, 90, C.MASK_CAUSAL, cap))


@BOTH
@pytest.mark.parametrize("heads,groups,d,T,mask,micro_batch", [
    (4, 1, 64, 1100, C.MASK_CAUSAL, 1),                      # one key head for all: the queries of a key's sums in parts
    (4, 2, 75, 700, C.MASK_NONE, 1),
    (2, 1, 160, 900, C.MASK_SPANS, 1),
    (2, 2, 256, 600, C.MASK_CAUSAL, 1),
])
def test_attention_over_many_tiles(dtype, heads, groups, d, T, mask, micro_batch):
    _check_attention(_attention(dtype, heads, groups, d, T, mask, micro_batch=micro_batch), "documents")


# Up to here blocks of rows are fewer than the chip has units, and two waves share 32 rows.  Below, 264 and more of them, a wave to 32 rows.
@BOTH
@pytest.mark.parametrize("d", [1, 8, 24, 33, 64, 75, 96, 128, 136, 192, 250, 256])
def test_attention_of_many_sequences(dtype, d):
    _check_attention(_attention(dtype, 4, 4, d, 66, micro_batch=66))


@BOTH
@pytest.mark.parametrize("mask,cap,bias", [(C.MASK_NONE, 0.0, 8), (C.MASK_CAUSAL, 3.0, 0), (C.MASK_SPANS, 0.0, 0), (C.MASK_SPANS, 5000.0, 2)])
@pytest.mark.parametrize("d", [30, 32, 80, 128, 200])
def test_attention_of_many_sequences_with_masks_caps_and_slopes(dtype, mask, cap, bias, d):
    _check_attention(_attention(dtype, 8, 4, d, 130, mask, cap, bias, micro_batch=33), "random" if cap else "documents")


@pytest.mark.parametrize("dtype,kind", [(C.FP32, "documents"), (C.BF16, "documents"), (C.BF16, "random")])
def test_blocks_in_the_order_of_their_work(dtype, kind):
    _check_attention(_attention(dtype, 36, 36, 8, 900, C.MASK_SPANS, micro_batch=1), kind)


@BOTH
def test_attention_over_micro_batches_in_flight(dtype):
    _check_attention(_attention(dtype, 4, 2, 32, 70, C.MASK_SPANS, n_micro=4, stage_index=1, n_stages=3), "documents")


@BOTH
@pytest.mark.parametrize("heads,groups,d", [(2, 1, 20), (4, 2, 64)])
def test_attention_from_nchw(dtype, heads, groups, d):
    _check_attention(_attention(dtype, heads, groups, d, 45, C.MASK_CAUSAL), layout=B.NCHW)


@BOTH
def test_positions_that_see_nothing_and_keys_that_nobody_sees(dtype):
    """Rows of zeros and gradients of exactly zero; spans that are reversed, empty or beyond the ends."""
    st = _attention(dtype, 4, 2, 32, 130, C.MASK_SPANS)
    xs, gs = stage_io(st)
    spans = np.zeros((2, 130, 2), np.int32)
    spans[0, :, :] = (-5, 200)                               # all of them
    spans[0, 40:50] = (20, 20)
    spans[0, 64:100] = (90, 10)
    spans[1, 30:60] = (17, 33)                               # one sample of which few see few
    got = run(st, [(None, None)], xs, gs, [spans])
    y, y_err, dx, dx_err, _ = _bounds(st, xs[0], gs[0], np.clip(spans, 0, 130))
    _within(got["y0"], y, y_err, "y")
    _within(got["dx0"], dx, dx_err, "dx")
    none = np.ones((2, 130), bool)
    none[0, :], none[0, 40:50], none[0, 64:100], none[1, 30:60] = False, True, True, False
    unseen = np.zeros((2, 130), bool)
    unseen[1] = True
    unseen[1, 17:33] = False
    assert not np.any(got["y0"].transpose(0, 2, 1, 3)[none])
    assert not np.any(got["dx0"][:, :128].transpose(0, 2, 1, 3)[none])
    assert not np.any(got["dx0"][:, 128:].transpose(0, 2, 1, 3)[unseen])
    # a mini-batch of nothing but padding
    got = run(st, [(None, None)], xs, gs, [np.zeros((2, 130, 2), np.int32)])
    assert not np.any(got["y0"]) and not np.any(got["dx0"])


@BOTH
@pytest.mark.parametrize("d,used", [(64, 100), (128, 64), (45, 33), (200, 127)])
@pytest.mark.parametrize("poison", [math.nan, math.inf])
@pytest.mark.parametrize("rotary", [0, 1])
@pytest.mark.parametrize("cap", [0.0, 3.0])
def test_what_padding_holds_has_no_effect(dtype, d, used, poison, rotary, cap):
    _padding(dtype, d, used, poison, rotary, cap, 2, 2)


@BOTH
@pytest.mark.parametrize("d", [45, 64, 128])
@pytest.mark.parametrize("rotary", [0, 1])
def test_what_padding_of_many_sequences_holds_has_no_effect(dtype, d, rotary):
    _padding(dtype, d, 70, math.nan, rotary, 0.0, 40, 4)


def _padding(dtype, d, used, poison, rotary, cap, micro_batch, groups):
    b = C._Builder()
    if rotary:
        b.rotary(4, groups, d, src=-1)
    b.attention(4, groups, d, C.MASK_SPANS, cap, src=-1 if not rotary else 0)
    st = _stage(b.layers, dtype, ((4 + 2 * groups) * d, 130, 1), micro_batch)
    params = gen.all_params(st)
    xs, gs = stage_io(st)
    spans = np.zeros((micro_batch, 130, 2), np.int32)
    spans[:, :used, 0], spans[:, :used, 1] = 0, np.arange(1, used + 1)
    spans[1, 20:40] = 0                                      # the other sample also has positions in between that see nothing
    clean = run(st, params, xs, gs, [spans])
    for a in (xs[0], gs[0]):
        a[:, :, used:] = poison
    got = run(st, params, xs, gs, [spans])
    for k in clean:
        assert np.array_equal(got[k][:, :, :used], clean[k][:, :, :used]), k
        if not rotary or k != "dx0":
            assert not np.any(got[k][:, :, used:]) and not np.any(clean[k][:, :, used:]), k


@BOTH
def test_large_scores_and_equal_ones(dtype):
    """Scores of thousands, where a probability is one or nothing, and queries of zeros, where all are alike."""
    st = _attention(dtype, 2, 1, 64, 96, C.MASK_CAUSAL)
    xs, gs = stage_io(st)
    zero = [xs[0].copy()]
    zero[0][:, :128] = 0
    got = run(st, [(None, None)], zero, gs)
    y, y_err, dx, dx_err, _ = _bounds(st, zero[0], gs[0], None)
    _within(got["y0"], y, y_err, "y")
    _within(got["dx0"], dx, dx_err, "dx")
    big = [xs[0].copy()]
    big[0][:, :192] *= 64                                    # scores of up to 64 * 64 * 8
    got = run(st, [(None, None)], big, gs)
    p, _ = ops.attention_probabilities(big[0], 2, 1, ops.attention_sees(1, 2, 96))
    sure = p.max(-1) > 1 - 1e-6                              # [n][head][position]; one key takes it all
    assert sure.mean() > 0.9
    y = got["y0"].reshape(2, 2, 64, 96).transpose(0, 1, 3, 2)
    taken = np.take_along_axis(ops.split_heads(big[0], 4)[:, [3, 3]], p.argmax(-1)[..., None], 2)
    assert np.max(np.abs(y - taken)[sure]) <= 2e-6 * 6 + HALF[dtype] * np.max(np.abs(taken))
    assert all(np.all(np.isfinite(v)) for v in got.values())


# ------------------------------------------------------------------------------ rotary
def _rotary(dtype, heads, groups, d, T, turning=None, layout=0, norm=0, eps=1e-6, micro_batch=2, n_micro=1, stage_index=1, n_stages=1):
    b = C._Builder()
    b.rotary(heads, groups, d, turning, layout, norm, eps, src=-1)
    return _stage(b.layers, dtype, ((heads + 2 * groups) * d, T, 1), micro_batch, n_micro, stage_index, n_stages)


def _check_rotary(st, angles=None, layout=B.NHWC, static=False):
    L, half = st["layers"][0], HALF[st["dtype"]]
    H, G, pairs, eps = L["kh"], L["kw"], bool(L["stride"]), L["eps"]
    d, T = st["in_c"] // (H + 2 * G), st["in_h"]
    params = gen.all_params(st, perturb=True)
    gains = None if params[0][0] is None else params[0][0].astype(np.float64)
    xs, gs = stage_io(st)
    got = run(st, params, xs, gs, angles={0: angles} if angles else None, layout=layout, static=static)
    by = ops.rotary_angles(T, L["pad"], **(angles or {}))
    # An angle t f is a double on either side: f = base^(..) is off by two roundings of 2^-53, the product by one.  At t = 2^40 and f = 1 that
    # is 2 * 3 * 2^-53 * 2^40 = 7.3e-4 between the two.
    angle_err = 6 * 2.0 ** -53 * ((angles or {}).get("first_position", 0) + T)
    size = np.ones((T, d))                                   # a turning channel is a sum of two products: |a| |cos| + |b| |sin|, twice that of one
    size[:, :L["pad"]] = np.abs(by).max(initial=0.0)
    dg, dg_err, terms = np.zeros((2, d)), np.zeros((2, d)), st["n_micro"] * st["micro_batch"] * T * H

    def spread(z):                                           # |a| + |b| at both channels of a pair
        r, a = L["pad"], np.abs(z)
        out = a.copy()
        if pairs:
            out[..., 0:r:2] = out[..., 1:r:2] = a[..., 0:r:2] + a[..., 1:r:2]
        else:
            out[..., :r // 2] = out[..., r // 2:r] = a[..., :r // 2] + a[..., r // 2:r]
        return out * size

    k = (d + 24) * U                                         # of a norm: the sum over the channels, the root, the products
    for m in range(st["n_micro"]):
        x, dy = (ops.split_heads(a, H + 2 * G) for a in (xs[m], gs[m]))
        y = ops.rotary_fwd(xs[m], H, G, by, pairs, gains, eps)
        mine = np.zeros((2, d))
        dx = ops.rotary_bwd(xs[m], gs[m], H, G, by, pairs, gains, eps, mine)
        dg += mine
        qk, dqk = x[:, :H + G], ops._turn(ops.split_heads(gs[m], H + 2 * G)[:, :H + G], by.conj(), pairs)
        turned = spread(dy[:, :H + G]) * (6 * U + angle_err)
        if gains is None:
            y_err, dx_err = spread(qk) * (6 * U + angle_err), turned
        else:
            gain, r = np.repeat(gains, [H, G], axis=0)[:, None], ops._rms(qk, eps)
            xhat = qk * r
            y_err = spread(xhat * gain) * (6 * U + k + angle_err)
            g, g_err = dqk * gain, turned * np.abs(gain)
            mean = (np.abs(g * xhat)).mean(-1, keepdims=True)
            dx_err = r * (g_err + np.abs(xhat) * (g_err * np.abs(xhat)).mean(-1, keepdims=True) + 3 * k * (np.abs(g) + np.abs(xhat) * mean))
            by_head = (np.abs(xhat) * (turned + k * np.abs(dqk)) + terms * U * np.abs(dqk * xhat)).sum((0, 2))
            dg_err += np.stack([by_head[:H].sum(0), by_head[H:].sum(0)])
        zero = np.zeros_like(x[:, H + G:])
        y_err, dx_err = (ops.join_heads(np.concatenate([e, zero], 1)) for e in (y_err, dx_err))
        _within(got["y%d" % m], y, 1.05 * y_err + half * np.abs(y), "y")
        _within(got["dx%d" % m], dx, 1.05 * dx_err + half * np.abs(dx), "dx")
        values = np.s_[:, (H + G) * d:]
        assert np.array_equal(got["y%d" % m][values], xs[m][values]) and np.array_equal(got["dx%d" % m][values], gs[m][values])
    if gains is not None:
        _within(got["dw0"], dg, 1.05 * dg_err + U * np.abs(dg), "dgains")


@BOTH
@pytest.mark.parametrize("norm,layout", [(0, 0), (0, 1), (1, 0), (1, 1)])
@pytest.mark.parametrize("heads,groups,d,T,turning", [
    (1, 1, 1, 3, 0), (1, 1, 2, 1, 2), (2, 1, 7, 5, 6), (4, 2, 8, 9, 8), (3, 3, 33, 20, 16), (8, 8, 64, 1, 64), (6, 2, 75, 19, 30),
    (5, 1, 80, 33, 80), (4, 4, 128, 40, 128), (4, 1, 128, 21, 32), (2, 2, 250, 11, 250), (2, 1, 256, 37, 256), (2, 2, 96, 13, 2), (3, 1, 48, 13, 36)])
def test_rotary(dtype, norm, layout, heads, groups, d, T, turning):
    _check_rotary(_rotary(dtype, heads, groups, d, T, turning, layout, norm))


@BOTH
@pytest.mark.parametrize("angles", [
    dict(base=500000.0), dict(factor=4.0), dict(factor=8.0, original_length=16.0, low_turns=0.25, high_turns=2.0, base=100.0),
    dict(magnitude=1.375), dict(first_position=1 << 20), dict(first_position=1 << 40, base=50.0, magnitude=0.5), dict(base=1.0)])
def test_rotary_with_other_angles(dtype, angles):
    _check_rotary(_rotary(dtype, 4, 2, 64, 40, norm=1), angles)


@BOTH
def test_rotary_of_many_positions_and_micro_batches(dtype):
    _check_rotary(_rotary(dtype, 5, 1, 64, 700, norm=1, micro_batch=3, n_micro=3, stage_index=1, n_stages=2), dict(base=5e5))
    _check_rotary(_rotary(dtype, 12, 4, 40, 501, 20, 1, micro_batch=2, n_micro=2))


@BOTH
def test_rotary_of_many_heads(dtype):
    _check_rotary(_rotary(dtype, 700, 20, 4, 3, norm=1))
    _check_rotary(_rotary(dtype, 70000, 1, 1, 1, micro_batch=1))
    _check_rotary(_rotary(dtype, 40000, 10000, 2, 2, norm=1, micro_batch=1))


@BOTH
@pytest.mark.parametrize("norm", [0, 1])
def test_rotary_from_nchw(dtype, norm):
    _check_rotary(_rotary(dtype, 2, 1, 24, 17, norm=norm), layout=B.NCHW)


@BOTH
def test_rotary_of_zeros_and_of_large_rows(dtype):
    st = _rotary(dtype, 2, 1, 32, 8, norm=1)
    params = gen.all_params(st, perturb=True)
    xs, gs = stage_io(st)
    xs[0][0, :, 0] = 0                                       # x / sqrt(eps), so gradients of 1 / sqrt(eps) = 1000
    xs[0][0, :, 1] *= 2.0 ** 40
    got, ref = run(st, params, xs, gs), oracle(st, params, xs, gs)
    assert not np.any(got["y0"][0, :96, 0])
    for k in ("y0", "dx0"):
        for t in range(8):
            a, r = got[k][0, :96, t], ref[k][0, :96, t]
            assert _norm(a - r) <= (2 * HALF[dtype] + 100 * U) * _norm(r), (k, t)


# ------------------------------------------------------------------------------ as they are used
def _close(st, got, ref, roundings):
    """2-norms; a float stage's products over up to 300 terms, four of them chained: 4 * 4 (sqrt(300) + sqrt(300) + 8) U"""
    limit = 2 * math.sqrt(roundings / 3) * HALF[C.BF16] if st["dtype"] == C.BF16 else 4e-5
    if st["layers"][-1]["fuse_relu"]:
        # Outputs that round to either side of zero: there the gate lets dy pass on one side only.  Of all elements a share f, of those that
        # pass (half of them) 2 f, so the gradient behind the gate is off by sqrt(2 f) in the 2-norm, and twice that is allowed.  y is off by
        # less than 2^-8 of its spread, so f is below that.
        ys = [k for k in ref if k[0] == "y"]
        f = float(np.mean([np.mean((got[k] > 0) != (ref[k] > 0)) for k in ys]))
        assert f <= 2.0 ** -8
        for k in ys:
            assert _norm(got[k] - ref[k]) <= limit * _norm(ref[k])
        limit += 2 * math.sqrt(2 * f * st["n_micro"])        # all of them may be in one micro-batch
    bad = {}
    for k, r in ref.items():
        assert np.all(np.isfinite(got[k])), k
        e = _norm(got[k] - r)
        if not e <= limit * _norm(r) + 1e-30:
            bad[k] = e / max(_norm(r), 1e-300)
    assert not bad, (bad, limit)


def _compare(st, spans=None, angles=None, roundings=16, **how):
    params = gen.all_params(st, perturb=True)
    xs, gs = stage_io(st)
    trace = {}
    got, ref = run(st, params, xs, gs, spans, angles, **how), oracle(st, params, xs, gs, spans, angles, trace)
    if st["in_h"] == 1:
        # One position: gradients of scores are dout . v - dout . o with o = v, exactly zero, and so are those of gains.  The two sums over d
        # channels are off by (d + 8) U sum |dout| |v| each; a gain's gradient is a sum over heads of that times |k| (or |q|) / sqrt(d) times
        # a normalised row, of 2-norm sqrt(d).
        for i, L in enumerate(st["layers"]):
            if L["kind"] == C.ROTARY and L["has_bias"]:
                H, G, bound = L["kh"], L["kw"], 0.0
                for m in range(st["n_micro"]):
                    at = trace[(m, i + 1)]
                    z, do = ops.split_heads(at["x"], H + 2 * G)[:, :, 0], ops.split_heads(at["g"], H)[:, :, 0]
                    d, q, (k, v) = z.shape[-1], z[:, :H], (np.repeat(z[:, a:a + G], H // G, axis=1) for a in (H, H + G))
                    off = 2 * (d + 8) * U * (np.abs(do) * np.abs(v)).sum(-1)
                    bound += float((off * (np.linalg.norm(q, axis=-1) + np.linalg.norm(k, axis=-1))).sum())
                assert _norm(ref.pop("dw%d" % i)) <= 1e-12 and _norm(got.pop("dw%d" % i)) <= bound
    _close(st, got, ref, roundings)


@BOTH
@pytest.mark.parametrize("kw", [
    dict(), dict(norm=0), dict(norm=0, layout=1, mask=C.MASK_NONE), dict(mask=C.MASK_SPANS, heads=6, groups=3, d=24, c=48, seq=70),
    dict(d=64, heads=4, groups=1, c=96, seq=130, turning=32), dict(d=64, norm=0, cap=5.0, bias=4, seq=65, c=64),
    dict(d=128, heads=2, groups=1, c=128, seq=140, layout=1), dict(d=256, heads=2, groups=2, c=32, seq=40, mask=C.MASK_SPANS),
    dict(d=200, heads=1, groups=1, c=40, seq=75), dict(d=7, heads=3, groups=3, c=13, seq=9), dict(seq=1), dict(d=160, heads=3, groups=3, seq=33, c=40)])
def test_the_sublayer(dtype, kw):
    st = attention_sublayer(dtype=dtype, **kw)
    _compare(st, _spans(st, "documents") if _has_spans(st) else None)


@BOTH
@pytest.mark.parametrize("norm", [0, 1])
@pytest.mark.parametrize("d,heads,groups,T,mask", [(64, 4, 2, 100, C.MASK_CAUSAL), (128, 4, 1, 70, C.MASK_SPANS), (33, 2, 2, 40, C.MASK_NONE),
                                                   (96, 2, 1, 130, C.MASK_CAUSAL), (256, 2, 1, 90, C.MASK_NONE), (192, 2, 2, 300, C.MASK_CAUSAL)])
def test_rotary_and_attention(dtype, norm, d, heads, groups, T, mask):
    b = C._Builder()
    b.rotary(heads, groups, d, norm=norm, src=-1)
    b.attention(heads, groups, d, mask)
    st = _stage(b.layers, dtype, ((heads + 2 * groups) * d, T, 1), n_micro=2)
    _compare(st, _spans(st, "window") if _has_spans(st) else None, {0: dict(base=1000.0, first_position=7)}, roundings=8)


@BOTH
@pytest.mark.parametrize("norm,conv", [(0, 0), (1, 0), (0, 1), (1, 1)])
@pytest.mark.parametrize("turned,read", [((8, 4, 64), (12, 2, 64)), ((8, 4, 64), (4, 2, 128)), ((2, 1, 12), (6, 3, 4)), ((5, 1, 9), (1, 1, 21)), ((4, 4, 30), (8, 1, 36))])
def test_an_attention_of_other_heads_than_the_rotary_in_front(dtype, turned, read, norm, conv):
    """Channels that one layer turns as keys are queries of the other, and so on.  Both sides round what the ROTARY stores, so what differs is a
    gradient's roundings: a probability, the output in dout . o, its own, the gradient of a score, itself, and once more behind the ROTARY; with a
    convolution in front the product's.  Eight."""
    c = (turned[0] + 2 * turned[1]) * turned[2]
    assert c == (read[0] + 2 * read[1]) * read[2]
    b = C._Builder()
    if conv:
        b.conv(c, c, 1, src=-1)
    b.rotary(*turned, norm=norm, src=None if conv else -1)
    b.attention(*read)
    _compare(_stage(b.layers, dtype, (c, 70, 1), n_micro=3, stage_index=1, n_stages=2), roundings=8)


@BOTH
@pytest.mark.parametrize("d,norm,mask,cap", [(24, 1, C.MASK_CAUSAL, 0.0), (33, 0, C.MASK_NONE, 0.0), (64, 1, C.MASK_SPANS, 0.0), (64, 0, C.MASK_CAUSAL, 4.0), (96, 1, C.MASK_CAUSAL, 0.0),
                                             (128, 1, C.MASK_CAUSAL, 0.0), (128, 0, C.MASK_SPANS, 4.0), (192, 0, C.MASK_CAUSAL, 0.0), (256, 1, C.MASK_SPANS, 0.0)])
def test_rotary_and_attention_of_many_sequences(dtype, d, norm, mask, cap):
    b = C._Builder()
    b.rotary(4, 4, d, norm=norm, src=-1)
    b.attention(4, 4, d, mask, cap)
    st = _stage(b.layers, dtype, (12 * d, 66, 1), micro_batch=66)
    _compare(st, _spans(st, "documents") if _has_spans(st) else None, roundings=8)


def _graphs():
    """Around the two layers: others that read the same tensor, ReLUs in front, sums behind, a second attention, ends of a stage."""
    H, G, d = 4, 2, 8
    wide = (H + 2 * G) * d

    def two_readers_of_the_input(b):
        b.attention(H, G, d, src=-1)
        b.conv(wide, H * d, 1, src=-1)
        b.addl(0, 1, relu=0)

    def rotary_with_two_readers(b):
        b.conv(wide, wide, 1, src=-1)
        b.rotary(H, G, d, norm=1)
        b.attention(H, G, d)
        b.conv(wide, H * d, 1, src=1)
        b.addl(2, 3, relu=0)

    def projection_with_two_readers(b):
        b.conv(wide, wide, 1, src=-1)
        b.rotary(H, G, d)
        b.attention(H, G, d, src=1)
        b.conv(wide, H * d, 1, src=0)
        b.addl(2, 3, relu=1)

    def behind_a_relu(b):
        b.conv(wide, wide, 1, relu=1, src=-1)
        b.rotary(H, G, d)
        b.attention(H, G, d)

    def attention_behind_a_relu(b):
        b.conv(wide, wide, 1, relu=1, src=-1)
        b.attention(H, G, d)

    def rotary_of_a_relu_layer(b):
        b.relu(src=-1)
        b.rotary(H, G, d, norm=1)
        b.relu()

    def two_in_a_row(b):
        b.rotary(H, G, d, norm=1, src=-1)
        b.rotary(H, G, d)
        b.attention(H, G, d)
        b.conv(H * d, wide, 1)
        b.rotary(H, G, d, layout=1)
        b.attention(H, G, d, C.MASK_NONE)

    def attention_twice(b):
        b.attention(H, G, d, src=-1)
        b.attention(H, G, d, C.MASK_NONE, 2.0, src=-1)
        b.addl(0, 1, relu=0)

    def two_attentions_of_a_rotary(b):
        b.rotary(H, G, d, src=-1)
        b.attention(H, G, d, src=0)
        b.attention(H, G, d, C.MASK_NONE, src=0)
        b.addl(1, 2, relu=0)

    def rotary_last(b):
        b.conv(wide, wide, 1, src=-1)
        b.rotary(H, G, d)

    def gated_behind(b):
        b.layernorm(wide, src=-1)
        b.rotary(H, G, d)
        b.attention(H, G, d)
        b.gated(H * d, 24)
        b.dropout(0.0)

    def sum_in_front(b):
        b.conv(wide, wide, 1, src=-1)
        b.addl(0, -1, relu=1)
        b.rotary(H, G, d, norm=1)
        b.attention(H, G, d)

    def turned_in_place_for_two(b):
        b.conv(wide, wide, 1, src=-1)
        b.rotary(H, G, d)
        b.attention(H, G, d, src=1)
        b.conv(wide, H * d, 1, src=1)
        b.addl(2, 3, relu=0)

    def turned_in_place_for_a_sum(b):
        b.conv(wide, wide, 1, src=-1)
        b.rotary(H, G, d, layout=1)
        b.addl(1, -1, relu=0)
        b.attention(H, G, d)

    def two_rotaries_of_one(b):
        b.conv(wide, wide, 1, src=-1)
        b.rotary(H, G, d, norm=1, src=0)
        b.rotary(H, G, d, src=0)
        b.attention(H, G, d, src=1)
        b.attention(H, G, d, C.MASK_NONE, src=2)
        b.addl(3, 4, relu=0)

    def a_recurrence_and_a_loss_behind(b):
        b.bn(wide, src=-1)
        b.attention(H, G, d)
        b.lstm(H * d, 16)
        b.flatten()
        b.linear(16 * 37, 10)
        b.xent()

    def rotary_before_a_linear_layer(b):
        b.conv(wide, wide, 1, src=-1)
        b.rotary(H, G, d)
        b.flatten()
        b.linear(wide * 37, 10)

    return {f.__name__: f for f in (two_readers_of_the_input, rotary_with_two_readers, projection_with_two_readers, behind_a_relu,
                                    attention_behind_a_relu, rotary_of_a_relu_layer, two_in_a_row, attention_twice,
                                    two_attentions_of_a_rotary, rotary_last, gated_behind, sum_in_front, turned_in_place_for_two,
                                    turned_in_place_for_a_sum, two_rotaries_of_one, a_recurrence_and_a_loss_behind, rotary_before_a_linear_layer)}


@BOTH
@pytest.mark.parametrize("name", list(_graphs()))
def test_among_other_layers(name, dtype):
    b = C._Builder()
    _graphs()[name](b)
    st = _stage(b.layers, dtype, (64, 37, 1), n_micro=3, stage_index=1, n_stages=2)
    _compare(st)


@pytest.mark.parametrize("spans", [0, 1])
def test_gradients_of_a_float_stage_against_differences(spans):
    """Of the GPU's own outputs: (L(x + h u) - L(x - h u)) / 2 h, L = <dy, y>.  L is off by U-sized roundings of ~|dy| |y|, so the
    slope by that over h; what is left of the third derivative is h^2."""
    st = attention_sublayer(d=16, c=32, seq=20, dtype=C.FP32, n_micro=1, n_stages=1, mask=C.MASK_SPANS if spans else C.MASK_CAUSAL, cap=4.0, bias=2)
    params = gen.all_params(st, perturb=True)
    xs, gs = stage_io(st)
    sp = _spans(st, "random") if spans else None
    base = run(st, params, xs, gs, sp)
    r = np.random.default_rng(2)
    h = 2.0 ** -6
    for _ in range(4):
        u = (base["dx0"] * r.random(xs[0].shape)).astype(np.float32)       # along which the slope is large
        u /= _norm(u)
        step = lambda e: float((run(st, params, [(xs[0] + e * h * u).astype(np.float32)], gs, sp)["y0"] * gs[0]).sum())  # noqa: E731
        slope = (step(1) - step(-1)) / (2 * h)
        noise = 64 * U * _norm(gs[0]) * _norm(base["y0"]) / h
        assert abs(slope - float((base["dx0"] * u).sum())) <= noise + 4 * h * h * _norm(base["dx0"]), (slope, noise)
