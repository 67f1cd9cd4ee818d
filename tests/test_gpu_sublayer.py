"""Layer norm, gated linear layer and dropout on the GPU against the oracle in 64 bits, through the C ABI: single layers at the sizes
where they can go wrong, gradients that meet other layers' epilogues, and the sublayer of a transformer that they make up.

Rounding to storage is off by at most HALF relative to the value; U is that of a float.  A sum of n terms in floats, in whatever
order, is off by at most (its longest chain of additions) * U * the sum of the terms' magnitudes."""
import numpy as np
import pytest
import torch

from gpu_harness import DEV, GpuStage, compare_minibatch, gpu_minibatch, stage_io, tdtype
from oracle import ops
from oracle.stage import OracleStage, one_f_one_b_order
from paper_2012_12544_amd import binding as B
from stage_inputs import configs as C
from stage_inputs import gen
from test_oracle_sublayer import sublayer

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
HALF = {C.FP32: 2.0 ** -24, C.BF16: 2.0 ** -8}


def _stage(layers, dtype, shape, micro_batch=2, n_micro=1, stage_index=1, n_stages=1, seed=80):
    return C._stage("one", layers, dtype, shape, micro_batch, n_micro, stage_index, n_stages, 1, C.BASE_SEED + seed, "xavier")


def _one(method, *args, **kw):
    b = C._Builder()
    getattr(b, method)(*args, src=-1, **kw)
    return b.layers


def _f64(a):
    return np.asarray(a, np.float64)


def _rows(a):
    """[N][C][H][W] -> [rows][C]"""
    a = np.asarray(a, np.float64)
    return a.transpose(0, 2, 3, 1).reshape(-1, a.shape[1])


def _within(got, ref, bound):
    assert got.shape == ref.shape and np.all(np.isfinite(got))
    worst = np.max((np.abs(got - ref) - bound) / np.maximum(bound, 1e-300))
    assert worst <= 0, float(worst)


# ------------------------------------------------------------------------------ layer norm
def _check_layernorm(st, xs, gs, got, gamma, beta, eps):
    half, Cn = HALF[st["dtype"]], st["in_c"]
    # the longest chain of a row's sums: a thread's share of a row (64 threads at the least, or 32 values) and the tree above it
    k = (max(Cn / 64, 32) + 24) * U
    dg, db, dg_err, db_err = (np.zeros(Cn) for _ in range(4))
    for m in range(st["n_micro"]):
        x, dy = _rows(xs[m]), _rows(gs[m])
        n = len(x)
        mean = x.mean(1, keepdims=True)
        d = x - mean
        var = (d * d).mean(1, keepdims=True)
        inv = 1 / np.sqrt(var + eps)
        xhat = d * inv
        d_mean = k * np.abs(x).mean(1, keepdims=True)
        rel_inv = 0.5 * (k + d_mean ** 2 * inv ** 2) + 4 * U
        e_x = inv * d_mean + np.abs(xhat) * (rel_inv + 4 * U)
        y = xhat * gamma + beta
        _within(_rows(got["y%d" % m]), y, np.abs(gamma) * e_x + 4 * U * (np.abs(gamma * xhat) + np.abs(beta)) + half * np.abs(y) + 1e-40)
        a = dy * gamma
        m1, m2 = a.mean(1, keepdims=True), (a * xhat).mean(1, keepdims=True)
        e1 = k * np.abs(a).mean(1, keepdims=True)
        e2 = k * np.abs(a * xhat).mean(1, keepdims=True) + (np.abs(a) * e_x).mean(1, keepdims=True)
        dx = inv * (a - m1 - xhat * m2)
        parts = np.abs(a) + np.abs(m1) + np.abs(xhat * m2)
        bound = inv * (e1 + np.abs(xhat) * e2 + e_x * (np.abs(m2) + e2) + 6 * U * parts + rel_inv * parts) + half * np.abs(dx)
        _within(_rows(got["dx%d" % m]), dx, bound + 1e-40)
        kr = (n / 64 + 128) * U
        dg += (dy * xhat).sum(0)
        db += dy.sum(0)
        dg_err += (np.abs(dy) * e_x).sum(0) + kr * np.abs(dy * xhat).sum(0)
        db_err += kr * np.abs(dy).sum(0)
    _within(_f64(got["dw0"]), dg, dg_err + 4 * U * np.abs(dg) + 1e-40)
    _within(_f64(got["db0"]), db, db_err + 4 * U * np.abs(db) + 1e-40)


@pytest.mark.parametrize("dtype", [C.FP32, C.BF16])
@pytest.mark.parametrize("c,seq,micro_batch,n_micro", [
    (1, 3, 2, 1), (2, 1, 1, 1), (3, 700, 2, 1), (5, 1, 1, 3), (7, 9, 3, 1), (8, 5, 1, 2), (31, 40, 2, 1), (64, 33, 3, 2), (65, 20, 2, 1),
    (72, 129, 2, 1), (100, 50, 3, 1), (256, 1, 1, 1), (257, 33, 2, 1), (500, 70, 2, 1), (512, 65, 2, 2), (520, 64, 2, 1), (1000, 17, 2, 1),
    (1024, 50, 4, 2), (1003, 11, 2, 1), (2048, 9, 2, 1), (2056, 9, 2, 1), (4096, 5, 2, 1), (4100, 5, 1, 1), (8192, 3, 2, 1),
    (8200, 2, 1, 1), (16384, 2, 1, 1), (16385, 3, 1, 1), (33000, 2, 1, 1), (40001, 1, 2, 1), (16, 4000, 2, 1), (128, 2100, 2, 1),
])
def test_layernorm(dtype, c, seq, micro_batch, n_micro):
    st = _stage(_one("layernorm", c), dtype, (c, seq, 1), micro_batch, n_micro)
    (gamma, beta), = gen.all_params(st, perturb=True)
    xs, gs = stage_io(st)
    _check_layernorm(st, xs, gs, gpu_minibatch(st), _f64(gamma), _f64(beta), np.float64(np.float32(1e-5)))


@pytest.mark.parametrize("dtype", [C.FP32, C.BF16])
@pytest.mark.parametrize("shape", [(24, 5, 7), (1000, 3, 2), (3, 8, 8)])
def test_layernorm_of_images_from_nchw(dtype, shape):
    st = _stage(_one("layernorm", shape[0]), dtype, shape, 3, 2)
    (gamma, beta), = gen.all_params(st, perturb=True)
    xs, gs = stage_io(st)
    _check_layernorm(st, xs, gs, gpu_minibatch(st, layout=B.NCHW), _f64(gamma), _f64(beta), np.float64(np.float32(1e-5)))


def _run(st, xs, gs, params=None, layout=B.NHWC):
    """One mini-batch of given inputs: y, dx, gradients by name."""
    g = GpuStage(st, gen.all_params(st, perturb=True) if params is None else params, layout=layout)
    out = {}
    for t, m in one_f_one_b_order(st["n_micro"], B.bapipe_stage_stash_bytes(g.h)[1]):
        if t == "F":
            out["y%d" % m] = g.forward(m, xs[m])
        else:
            out["dx%d" % m] = g.backward(m, gs[m])
    for i, (w, b) in enumerate(g.params):
        if w is not None:
            out["dw%d" % i], out["db%d" % i] = g.grads(i)
    g.close()
    return out


@pytest.mark.parametrize("dtype", [C.FP32, C.BF16])
@pytest.mark.parametrize("c", [40, 1003, 2048])
def test_layernorm_of_rows_far_from_zero_and_of_constant_rows(dtype, c):
    """Offsets that E[x^2] - mean^2 would not survive; rows without variance, whose 1/std is 1/sqrt(eps)."""
    st = _stage(_one("layernorm", c), dtype, (c, 6, 1), 2, 1)
    (gamma, beta), = gen.all_params(st, perturb=True)
    xs, gs = stage_io(st)
    x = xs[0].copy()
    x[0, :, 0] = 1000 + 8 * x[0, :, 0]
    x[0, :, 1] = -3e4
    x[0, :, 2] = 0
    x[1, :, 3] *= 1e-6
    x[1, :, 4] *= 1e6
    x = torch.from_numpy(x).to(tdtype(st)).float().numpy()
    _check_layernorm(st, [x], gs, _run(st, [x], gs), _f64(gamma), _f64(beta), np.float64(np.float32(1e-5)))


@pytest.mark.parametrize("dtype", [C.FP32, C.BF16])
def test_layernorm_keeps_what_is_not_finite_in_its_row(dtype):
    st = _stage(_one("layernorm", 96), dtype, (96, 8, 1), 1, 1)
    xs, gs = stage_io(st)
    x = xs[0].copy()
    ref = _run(st, [x], gs)
    x[0, 5, 2], x[0, 90, 6] = np.inf, np.nan
    g = GpuStage(st, gen.all_params(st, perturb=True))
    y, dx = g.forward(0, x), g.backward(0, gs[0])
    g.close()
    fine = [0, 1, 3, 4, 5, 7]
    assert np.array_equal(y[:, :, fine], ref["y0"][:, :, fine]) and np.array_equal(dx[:, :, fine], ref["dx0"][:, :, fine])
    assert np.all(np.isnan(y[:, :, 6])) and not np.all(np.isfinite(y[:, :, 2]))


# ------------------------------------------------------------------------------ gated
def _check_gated(st, layout=B.NHWC):
    L, dtype = st["layers"][0], st["dtype"]
    c, f, act = L["cin"], L["cout"], L["kh"]
    xs, gs = stage_io(st)
    params = gen.all_params(st, perturb=True)
    got = _run(st, xs, gs, layout=layout)
    orc = OracleStage(st, params)
    w, b = orc.q(_f64(params[0][0])), params[0][1]
    rows = st["micro_batch"] * st["in_h"] * st["in_w"]
    errs = {}
    for t, m in one_f_one_b_order(st["n_micro"], orc.depth):
        if t == "F":
            orc.forward(m, xs[m])
            x = _rows(xs[m])
            both = x @ w.T + (0 if b is None else b)
            # a projection is a chain of at most cin + 1 additions; the activations' slopes are below 1.13, their own errors 32 U
            e = (c + 2) * U * (np.abs(x) @ np.abs(w).T + (0 if b is None else np.abs(b)))
            g, u, eg, eu = both[:, :f], both[:, f:], e[:, :f], e[:, f:]
            a = ops.gate(act, g)[0]
            bound = 1.13 * (np.abs(u) + eu) * eg + np.abs(a) * eu + 32 * U * (1 + np.abs(g)) * np.abs(u) + HALF[dtype] * np.abs(a * u)
            _within(_rows(got["y%d" % m]), a * u, bound + 1e-38)
        else:
            errs["dx%d" % m] = (got["dx%d" % m], orc.backward(m, gs[m]))
    errs["dw"] = (_f64(got["dw0"]), orc.dw[0])
    if b is not None:
        errs["db"] = (_f64(got["db0"]), orc.db[0])
    # Gradients in the 2-norm.  Float: chains of cin, 2 cout and rows additions.  bf16: the gradients of the projections are
    # rounded, and where the sums of the two sides lie on both sides of a rounding border (noise of sqrt(cin) U against steps of 2^-7:
    # a share below 3e-3 at these sizes) they are a step apart: sqrt(3e-3) 2^-7 = 4e-4 of a tensor; each is rounded to dx once more,
    # where noise of that size flips a tenth of the elements by a step: sqrt(0.1) 2^-7 = 2.5e-3.
    loose = (c + 2 * f + rows * st["n_micro"]) * U
    for name, (a, r) in errs.items():
        off = np.linalg.norm(a - r) / max(np.linalg.norm(r), 1e-300)
        assert off <= (loose if dtype == C.FP32 else 3e-3 if name[:2] == "dx" else 1e-3), (name, off)


@pytest.mark.parametrize("dtype", [C.FP32, C.BF16])
@pytest.mark.parametrize("c,units,seq,micro_batch,bias", [
    (1, 1, 1, 1, 1), (3, 5, 2, 1, 0), (8, 8, 1, 1, 0), (8, 8, 3, 2, 1), (17, 33, 130, 1, 1), (64, 64, 1, 1, 1), (64, 128, 40, 2, 0), (64, 128, 64, 2, 1),
    (72, 200, 77, 3, 0), (100, 36, 129, 2, 1), (128, 64, 256, 1, 0), (256, 96, 300, 1, 1), (500, 133, 77, 1, 1), (512, 8, 200, 1, 0),
    (8, 512, 600, 2, 0), (1024, 256, 1, 2, 1), (96, 1032, 65, 1, 1), (320, 320, 512, 2, 1), (768, 512, 7, 1, 0),
])
def test_gated(dtype, c, units, seq, micro_batch, bias):
    _check_gated(_stage(_one("gated", c, units, act=(c + units) % 4, bias=bias), dtype, (c, seq, 1), micro_batch, 1))


@pytest.mark.parametrize("dtype,c,units,seq,bias", [
    (C.BF16, 72, 1600, 515, 1), (C.BF16, 72, 1601, 515, 0), (C.BF16, 200, 1603, 513, 1), (C.BF16, 40, 10240, 150, 0), (C.BF16, 16, 19201, 64, 1),
    (C.BF16, 32, 4096, 1024, 1), (C.BF16, 8, 4097, 1000, 0), (C.FP32, 20, 2050, 1023, 1), (C.FP32, 4, 19203, 150, 0), (C.FP32, 36, 4096, 1023, 0),
    (C.FP32, 512, 8, 8192, 1), (C.FP32, 516, 38, 8200, 0),
])
def test_gated_of_many_tiles(dtype, c, units, seq, bias):
    """Products that fill the chip unsplit: tiles of every size, a K that ends inside one, rows and units that do."""
    _check_gated(_stage(_one("gated", c, units, act=(c + units) % 4, bias=bias), dtype, (c, seq, 1), 2, 1))


@pytest.mark.parametrize("dtype", [C.FP32, C.BF16])
@pytest.mark.parametrize("act", range(4))
@pytest.mark.parametrize("c,units,seq", [(48, 80, 70), (30, 41, 33), (64, 64, 300)])
def test_gated_activations_over_micro_batches(dtype, act, c, units, seq):
    _check_gated(_stage(_one("gated", c, units, act=act, bias=1), dtype, (c, seq, 1), 2, 3, 2, 3))


@pytest.mark.parametrize("dtype", [C.FP32, C.BF16])
def test_gated_images_from_nchw(dtype):
    _check_gated(_stage(_one("gated", 40, 56, act=C.GATE_GELU, bias=1), dtype, (40, 6, 5), 3, 2), layout=B.NCHW)


@pytest.mark.parametrize("dtype", [C.FP32, C.BF16])
@pytest.mark.parametrize("act", range(4))
def test_gated_far_from_zero(dtype, act):
    """Gates of +-10^2 and +-10^4, where exp under- and overflows: values and gradients stay finite and right."""
    st = _stage(_one("gated", 8, 16, act=act), dtype, (8, 4, 1), 2, 1)
    x = np.zeros((2, 8, 4, 1), np.float32)
    x[:, 0, :, 0] = [[100, -100, 1e4, -1e4], [90, -90, 87, -88]]
    x[:, 1] = 1
    w = np.zeros((32, 8), np.float32)
    w[:16, 0] = 1
    w[16:, 1] = 2
    x = torch.from_numpy(x).to(tdtype(st)).float().numpy()
    dy = np.ones((2, 16, 4, 1), np.float32)
    got = _run(st, [x], [dy], [(w, None)])
    g = _rows(x)[:, :1]
    a, da = ops.gate(act, np.broadcast_to(g, (8, 16)))
    half = HALF[dtype]
    # single products: no sums to be off; a saturated sigmoid's derivative is 0 or below 1e-37.  The hardware's exp2 and reciprocal,
    # which a bf16 layer takes, give 0 for results below the smallest normal float: 1 / (1 + exp(88)) = 6.1e-39 < 2^-126 = 1.2e-38, so
    # that u silu(g) may be |u| |g| 2^-126 off, 2.1e-36 at g = -88, u = 2.
    _within(_rows(got["y0"]), 2 * a, 2 * (half + 64 * U) * np.abs(2 * a) + 1e-36 + (2 * np.abs(g) * 2.0 ** -126 if dtype == C.BF16 else 0))
    assert np.all(np.isfinite(got["dx0"])) and np.all(np.isfinite(got["dw0"]))
    # 16 units of dg = 2 da, each rounded, and of du = a in x's second channel
    _within(_rows(got["dx0"])[:, 0], 32 * da[:, 0], 2 * (half + 64 * U) * np.abs(32 * da[:, 0]) + 64 * U * (1 + np.abs(g[:, 0])) * (da[:, 0] > 0) + 1e-34)
    _within(_rows(got["dx0"])[:, 1], 32 * a[:, 0], 2 * (half + 64 * U) * np.abs(32 * a[:, 0]) + 1e-34)


# ------------------------------------------------------------------------------ dropout
def _dropped(st, a, p, m, seed=0, mini_batch=0, layer=0):
    """What is stored of a: elements times the float 1/(1-p), rounded once more, or 0."""
    f = ops.dropout_factor(a.shape, p, seed, layer + 65536 * (st["stage_index"] - 1), m, mini_batch)
    scale = np.float32(1 / (1 - float(np.float32(p))))
    v = (torch.from_numpy(np.float32(a)) * float(scale)).to(tdtype(st)).double().numpy()
    return np.where(f > 0, v, 0.0)


@pytest.mark.parametrize("dtype", [C.FP32, C.BF16])
@pytest.mark.parametrize("shape,micro_batch,p", [
    ((1, 1, 1), 1, 0.5), ((3, 1, 1), 1, 0.5), ((5, 3, 1), 1, 0.25), ((7, 3, 2), 3, 0.1), ((8, 1, 1), 1, 0.5), ((64, 50, 1), 4, 0.2),
    ((1003, 31, 1), 2, 0.6), ((1024, 50, 1), 8, 0.0), ((12, 9, 1), 2, 1e-9), ((40, 33, 1), 3, 0.999999), ((2048, 600, 1), 2, 0.1),
])
def test_dropout(dtype, shape, micro_batch, p):
    st = _stage(_one("dropout", p), dtype, shape, micro_batch, 3, 2, 3)
    xs, gs = stage_io(st)
    got = _run(st, xs, gs, [(None, None)])
    for m in range(3):
        assert np.array_equal(got["y%d" % m], _dropped(st, xs[m], p, m))
        assert np.array_equal(got["dx%d" % m], _dropped(st, gs[m], p, m))


@pytest.mark.parametrize("dtype", [C.FP32, C.BF16])
@pytest.mark.parametrize("seq", [40, 1101])
def test_dropout_in_a_residual_sum_of_any_size(dtype, seq):
    """x + dropout(x) and its gradient, below and above the size from which loads pass by the caches."""
    b = C._Builder()
    b.dropout(0.3, src=-1)
    b.addl(0, -1, relu=0)
    st = _stage(b.layers, dtype, (2047, seq, 1), 2, 2)
    xs, gs = stage_io(st)
    got = _run(st, xs, gs, [(None, None)] * 2)
    for m in range(2):
        for name, v in (("y", xs[m]), ("dx", gs[m])):
            dropped = torch.from_numpy(np.float32(_dropped(st, v, 0.3, m)))
            want = (dropped + torch.from_numpy(np.float32(v))).to(tdtype(st)).double().numpy()
            assert np.array_equal(got["%s%d" % (name, m)], want), (name, m)


@pytest.mark.parametrize("dtype", [C.FP32, C.BF16])
def test_dropout_from_nchw_numbers_the_same_elements(dtype):
    st = _stage(_one("dropout", 0.3), dtype, (24, 5, 7), 3, 2)
    xs, gs = stage_io(st)
    got = _run(st, xs, gs, [(None, None)], layout=B.NCHW)
    assert np.array_equal(got["y1"], _dropped(st, xs[1], 0.3, 1)) and np.array_equal(got["dx1"], _dropped(st, gs[1], 0.3, 1))


def test_dropout_seeds_and_mini_batches():
    st = _stage(_one("dropout", 0.4), C.BF16, (40, 9, 1), 2, 2)
    xs, gs = stage_io(st)
    g = GpuStage(st, [(None, None)])

    def mini_batch(seed, number):
        for m in range(2):
            assert np.array_equal(g.forward(m, xs[m]), _dropped(st, xs[m], 0.4, m, seed, number)), (seed, number, m)
            if m == 0:
                with pytest.raises(B.BapipeError) as e:
                    B.bapipe_stage_set_dropout(g.h, 1, 1)
                assert e.value.status == B.E_ORDER
            assert np.array_equal(g.backward(m, gs[m]), _dropped(st, gs[m], 0.4, m, seed, number)), (seed, number, m)
        B.bapipe_stage_step(g.h, 0.1)

    mini_batch(0, 0)
    mini_batch(0, 1)
    B.bapipe_profile_layers(g.h, 0, 1, 1)                        # draws, and leaves the number as it is
    mini_batch(0, 2)
    seed = 0xFEDCBA9876543210
    B.bapipe_stage_set_dropout(g.h, seed, 2 ** 32 - 1)
    mini_batch(seed, 2 ** 32 - 1)
    mini_batch(seed, 0)
    B.bapipe_stage_set_dropout(g.h, seed, 2 ** 32 - 1)
    mini_batch(seed, 2 ** 32 - 1)
    g.close()
    g = GpuStage(_stage(_one("layernorm", 40), C.BF16, (40, 9, 1)), [(None, None)])
    with pytest.raises(B.BapipeError) as e:
        B.bapipe_stage_set_dropout(g.h, 1, 1)
    assert e.value.status == B.E_INVALID
    g.close()


@pytest.mark.parametrize("dtype", [C.FP32, C.BF16])
def test_dropout_drops_what_is_not_finite(dtype):
    st = _stage(_one("dropout", 0.5), dtype, (64, 20, 1), 1, 1)
    x = np.full((1, 64, 20, 1), np.nan, np.float32)
    x[:, ::2] = np.inf
    g = GpuStage(st, [(None, None)])
    y = torch.empty(1 * 20 * 64, dtype=tdtype(st), device=DEV)
    xd = torch.from_numpy(x).permute(0, 2, 3, 1).contiguous().to(DEV, tdtype(st))
    torch.cuda.synchronize()
    B.bapipe_stage_forward(g.h, 0, xd.data_ptr(), y.data_ptr())
    torch.cuda.synchronize()
    g.close()
    keep = _rows(ops.dropout_factor(x.shape, 0.5, 0, 0, 0, 0)) > 0
    y = y.float().cpu().numpy().reshape(20, 64)
    assert np.all(y[~keep] == 0) and not np.any(np.isfinite(y[keep]))


@pytest.mark.parametrize("dtype", [C.FP32, C.BF16])
@pytest.mark.parametrize("method,args", [("dropout", (0.3,)), ("layernorm", (24,)), ("gated", (24, 24))])
def test_buffers_at_odd_addresses_and_in_place_of_one_another(dtype, method, args):
    """x, y, dy and dx one element behind an aligned address, y over x, dx over dy: the same bits."""
    st = _stage(_one(method, *args), dtype, (24, 33, 1), 2, 1)
    xs, gs = stage_io(st)
    ref = _run(st, xs, gs)
    n, t = 2 * 33 * 24, tdtype(st)

    def host(a):
        return torch.from_numpy(a).permute(0, 2, 3, 1).reshape(-1).to(DEV, t)

    for offset in (0, 1):
        for in_place in (False, True):
            g = GpuStage(st, gen.all_params(st, perturb=True))
            bufs = [torch.full((n + 16,), 7.0, dtype=t, device=DEV) for _ in range(4)]
            x, y, dy, dx = (b[offset:offset + n] for b in bufs)
            x.copy_(host(xs[0]))
            dy.copy_(host(gs[0]))
            if in_place:
                y, dx = x, dy
            torch.cuda.synchronize()
            B.bapipe_stage_forward(g.h, 0, x.data_ptr(), y.data_ptr())
            torch.cuda.synchronize()
            got_y = y.clone()
            B.bapipe_stage_backward(g.h, 0, dy.data_ptr(), dx.data_ptr())
            torch.cuda.synchronize()
            assert torch.equal(got_y.cpu(), host(np.float32(ref["y0"])).cpu()) and torch.equal(dx.cpu(), host(np.float32(ref["dx0"])).cpu())
            for b in bufs:                                       # nothing in front of the tensors or behind them
                assert torch.all(b[:offset] == 7) and torch.all(b[offset + n:] == 7)
            g.close()


# ------------------------------------------------------------------------------ among other layers
def _graphs():
    def gates(b, c):          # every one of them behind a fused ReLU, whose gate the gradient has to meet
        b.conv(c, c, 1, relu=1, src=-1)
        b.layernorm(c)
        b.conv(c, c, 1, relu=1)
        b.gated(c, c, act=C.GATE_SILU, bias=1)
        b.conv(c, c, 1, relu=1)
        b.dropout(0.25)

    def fan_out(b, c):        # tensors with two readers: gradients are added to what is there
        b.layernorm(c, src=-1)
        b.gated(c, c, act=C.GATE_GELU, src=0)
        b.dropout(0.5, src=0)
        b.addl(1, 2, relu=0)
        b.layernorm(c, src=-1)
        b.addl(3, 4, relu=1)
        b.dropout(0.1, src=5)
        b.addl(6, 5, relu=0)

    def post_norm(b, c):      # the older order, and dropout in front
        b.dropout(0.1, src=-1)
        b.gated(c, 2 * c, act=C.GATE_SIGMOID, bias=1)
        b.conv(2 * c, c, 1)
        b.dropout(0.2)
        b.addl(3, 0, relu=0)
        b.layernorm(c)

    def lstm(b, c):           # GNMT's layers as they are trained
        b.dropout(0.2, src=-1)
        b.lstm(c, c)
        b.addl(1, -1, relu=0)
        b.layernorm(c)
        b.dropout(0.2)
        b.lstm(c, c)
        b.addl(5, 2, relu=0)

    def norms(b, c):          # beside batch-norm and pooling
        b.conv(c, c, 1, bias=0, src=-1)
        b.bn(c, relu=1)
        b.dropout(0.3)
        b.layernorm(c)
        b.addl(3, 1, relu=1)

    def loss(b, c):           # the end of a network
        b.layernorm(c, src=-1)
        b.dropout(0.1)
        b.flatten()
        b.linear(6 * c, 10)
        b.xent()
    return dict(gates=gates, fan_out=fan_out, post_norm=post_norm, lstm=lstm, norms=norms, loss=loss)


@pytest.mark.parametrize("dtype,c", [(C.FP32, 12), (C.FP32, 32), (C.BF16, 24), (C.BF16, 64)])
@pytest.mark.parametrize("name", list(_graphs()))
def test_among_other_layers(name, dtype, c):
    b = C._Builder()
    _graphs()[name](b, c)
    st = C._stage(name, b.layers, dtype, (c, 6, 1), 3, 2, 1, 1, 1, C.BASE_SEED + 81, "xavier")
    compare_minibatch(st)
    compare_minibatch(st, layout=B.NCHW)


@pytest.mark.parametrize("dtype", [C.FP32, C.BF16])
@pytest.mark.parametrize("kw", [
    dict(c=24, units=40, seq=5), dict(c=33, units=50, seq=7), dict(c=64, units=176, seq=40, micro_batch=3, act=C.GATE_GELU, bias=0),
    dict(c=128, units=352, seq=1, micro_batch=1), dict(c=256, units=704, seq=65, n_micro=2), dict(c=520, units=1000, seq=9, act=C.GATE_RELU),
    dict(c=33, units=50, seq=70, act=C.GATE_RELU), dict(c=64, units=96, seq=130, n_micro=2, act=C.GATE_RELU), dict(c=8, units=24, seq=1, micro_batch=1),
])
def test_sublayer(dtype, kw):
    compare_minibatch(sublayer(dtype=dtype, **kw))


@pytest.mark.parametrize("dtype,kw", [
    (C.BF16, dict(c=64, units=1600, seq=1030)), (C.BF16, dict(c=40, units=1608, seq=1025, bias=0)), (C.BF16, dict(c=24, units=19200, seq=150)),
    (C.BF16, dict(c=16, units=4096, seq=2048, act=C.GATE_GELU)), (C.BF16, dict(c=72, units=1608, seq=520, act=C.GATE_RELU)),
    (C.FP32, dict(c=16, units=2056, seq=2050)),
])
def test_sublayer_of_many_tiles(dtype, kw):
    """The products that fill the chip unsplit, the convolution's input gradient that makes the projections' gradients among them."""
    compare_minibatch(sublayer(dtype=dtype, n_micro=1, stage_index=1, n_stages=1, **kw))


def test_a_large_weight_gradient_over_micro_batches():
    """dw of 8192 x 1024 from two micro-batches of 1024 rows, against a product in 64 bits of what the device itself holds: x and D,
    each D worked out from the device's own forward product in 64 bits and rounded as the layer rounds it."""
    c, f, rows = 1024, 4096, 1024
    st = _stage(_one("gated", c, f, act=C.GATE_SIGMOID), C.BF16, (c, rows, 1), 1, 2)
    (w, _), = params = gen.all_params(st, perturb=True)
    xs, gs = stage_io(st)
    got = _run(st, xs, gs, params)["dw0"]
    on = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(DEV).to(tdtype(st)).double()  # noqa: E731
    W, ref, size = on(w), 0, 0
    for x, dy in zip(xs, gs):
        x, dy = on(_rows(x)), on(_rows(dy))
        P = x @ W.t()
        a = torch.sigmoid(P[:, :f])
        D = torch.cat([dy * P[:, f:] * a * (1 - a), dy * a], 1)
        ref = ref + D.t() @ x
        size = size + D.abs().t() @ x.abs()
    off = (torch.from_numpy(_f64(got)).to(DEV) - ref).abs()
    # D rounded once, and values 1e-4 of themselves off in it; 2048 additions in floats
    assert torch.all(off <= (HALF[C.BF16] + 1e-4 + 2048 * U) * size)
    # roundings are independent: the norm of their sum over n terms is HALF / sqrt(3) of the terms' norm, not of the terms' sum
    assert float(off.norm() / ref.norm()) <= HALF[C.BF16]


def test_sublayer_without_an_input_gradient():
    """The first stage of a network: no dx, and nothing behind the layer norm's parameters."""
    st = dict(sublayer(), need_input_grad=0)
    compare_minibatch(st)


@pytest.mark.parametrize("dtype", [C.FP32, C.BF16])
def test_further_streams_and_the_static_workspace_change_nothing(dtype):
    st = sublayer(c=128, units=320, seq=33, n_micro=5, dtype=dtype, stage_index=1, n_stages=3)
    ref = gpu_minibatch(st)
    for kw in (dict(backward_stream=True, eager_sync=False), dict(backward_stream="no wgrad stream", eager_sync=False),
               dict(wgrad_stream=True, eager_sync=False), dict(static=True), dict(static=True, backward_stream=True, eager_sync=False)):
        got = gpu_minibatch(st, **kw)
        for k in ref:
            assert np.array_equal(got[k], ref[k]), (kw, k)


def test_large_products_are_the_same_on_every_stream():
    """Enough rows and weights for the kernels that fill the chip by themselves, and a weight gradient that is not split like a convolution's."""
    st = sublayer(c=1024, units=4096, seq=512, micro_batch=2, n_micro=2, stage_index=1, n_stages=2)
    ref = gpu_minibatch(st)
    assert all(np.all(np.isfinite(v)) for v in ref.values())
    for kw in (dict(backward_stream=True, eager_sync=False), dict(wgrad_stream=True, eager_sync=False)):
        got = gpu_minibatch(st, **kw)
        for k in ref:
            assert np.array_equal(got[k], ref[k]), (kw, k)


def _device_io(st):
    xs, gs = stage_io(st)
    to = lambda a: torch.from_numpy(a).permute(0, 2, 3, 1).contiguous().to(DEV, tdtype(st))  # noqa: E731
    xs, gs = [to(a) for a in xs], [to(a) for a in gs]
    return xs, gs, [torch.zeros_like(a) for a in gs], [torch.zeros_like(a) for a in xs]


def _enqueue(g, st, io, step=True, static=False):
    xs, gs, ys, dxs = io
    for t, m in one_f_one_b_order(st["n_micro"], B.bapipe_stage_stash_bytes(g.h)[1]):
        if t == "F":
            B.bapipe_stage_forward(g.h, m, xs[m].data_ptr(), ys[m].data_ptr())
        else:
            (B.bapipe_stage_backward_static if static else B.bapipe_stage_backward)(g.h, m, gs[m].data_ptr(), dxs[m].data_ptr())
    if step:
        B.bapipe_stage_step(g.h, 0.01)


@pytest.mark.parametrize("dtype,c,units", [(C.BF16, 128, 320), (C.FP32, 40, 56), (C.BF16, 33, 50)])
def test_a_captured_mini_batch_draws_anew_at_every_replay(dtype, c, units):
    """Forward, backward and update captured into one graph: each replay is the next mini-batch, masks and weights included."""
    st = sublayer(c=c, units=units, seq=17, n_micro=3, dtype=dtype)
    params = gen.all_params(st, perturb=True)
    eager, captured = GpuStage(st, params), GpuStage(st, params)
    io_e, io_c = _device_io(st), _device_io(st)
    torch.cuda.synchronize()
    for g in (eager, captured):
        B.bapipe_stage_set_dropout(g.h, 77, 5)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=captured.stream):
        _enqueue(captured, st, io_c)
    outs = []
    for replay in range(4):
        _enqueue(eager, st, io_e)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(io_e[2] + io_e[3], io_c[2] + io_c[3]):
            assert torch.equal(a, b), replay
        for i, (w, b) in enumerate(params):
            if w is not None:
                for a, r in zip(captured.get_params(i), eager.get_params(i)):
                    assert a is None or np.array_equal(a, r), (replay, i)
        outs.append(io_c[2][0].clone())
        io_c[2][0].zero_()
    assert not torch.equal(outs[0], outs[1])
    del graph
    eager.close()
    captured.close()


def test_captured_where_the_convolution_makes_the_projections_gradients():
    """The large products captured before anything ran them, profiled and replayed."""
    st = sublayer(c=64, units=1600, seq=1030, n_micro=2, stage_index=1, n_stages=1)
    params = gen.all_params(st, perturb=True)
    captured, eager = GpuStage(st, params), GpuStage(st, params)
    io_c, io_e = _device_io(st), _device_io(st)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=captured.stream):
        _enqueue(captured, st, io_c)
    for replay in range(3):
        graph.replay()
        rec = B.bapipe_profile_layers(eager.h, 0, 1, len(st["layers"]))
        assert all(r["fwd_ms"] > 0 for r in rec[:3]) and all(r["bwd_ms"] > 0 for r in rec[:4])
        _enqueue(eager, st, io_e)
        torch.cuda.synchronize()
        for a, b in zip(io_c[2] + io_c[3], io_e[2] + io_e[3]):
            assert torch.equal(a, b), replay
        for i, (w, b) in enumerate(params):
            if w is not None:
                for a, r in zip(captured.get_params(i), eager.get_params(i)):
                    assert a is None or np.array_equal(a, r), (replay, i)
    del graph
    captured.close()
    eager.close()


def test_two_stages_at_once():
    """Handles are independent: two stages on two streams, and one of them alone."""
    sts = [sublayer(c=128, units=320, seq=65, n_micro=4), sublayer(c=256, units=192, seq=33, n_micro=4, act=C.GATE_GELU)]
    params = [gen.all_params(st, perturb=True) for st in sts]
    alone = []
    for st, ps in zip(sts, params):
        g, io = GpuStage(st, ps), _device_io(st)
        torch.cuda.synchronize()
        _enqueue(g, st, io)
        torch.cuda.synchronize()
        alone.append([t.clone() for t in io[2] + io[3]])
        g.close()
    gs, ios = [GpuStage(st, ps) for st, ps in zip(sts, params)], [_device_io(st) for st in sts]
    torch.cuda.synchronize()
    for g, st, io in zip(gs, sts, ios):
        _enqueue(g, st, io)
    torch.cuda.synchronize()
    for io, ref in zip(ios, alone):
        for a, b in zip(io[2] + io[3], ref):
            assert torch.equal(a, b)
    for g in gs:
        g.close()


def test_profile_and_timing_tap():
    st = sublayer(c=64, units=128, seq=33)
    g = GpuStage(st, gen.all_params(st, perturb=True))
    rec = B.bapipe_profile_layers(g.h, 1, 2, len(st["layers"]))
    rows = 2 * 33
    assert [r["weight_bytes"] for r in rec] == [4 * 128, 4 * (256 * 64 + 256), 4 * (128 * 64 + 64), 0, 0]
    assert rec[0]["stash_bytes"] >= 8 * rows and rec[1]["stash_bytes"] >= rows * 256 * 2
    assert all(r["fwd_ms"] > 0 for r in rec[:3]) and all(r["bwd_ms"] > 0 for r in rec[:4])
    B.bapipe_stage_kernel_timing(g.h, B.KC_BATCHNORM)
    xs, gs = stage_io(st)
    g.forward(0, xs[0])
    g.backward(0, gs[0])
    t = B.bapipe_stage_kernel_timing_read(g.h)
    assert t["launches"] == 2 and t["bytes"] >= 5 * rows * 64 * 2
    g.close()


def test_gradients_by_central_differences():
    """Of the library's own forward pass, in float, along a random direction of the input."""
    st = sublayer(c=16, units=24, seq=3, micro_batch=1, n_micro=1, act=C.GATE_SILU, dtype=C.FP32, stage_index=1, n_stages=1)
    xs, gs = stage_io(st)
    v = np.random.default_rng(3).standard_normal(xs[0].shape).astype(np.float32)
    h = 2.0 ** -7

    def value(x):
        g = GpuStage(st, gen.all_params(st, perturb=True))
        y = g.forward(0, x)
        g.close()
        return float(np.sum(y * gs[0]))

    g = GpuStage(st, gen.all_params(st, perturb=True))
    g.forward(0, xs[0])
    dx = g.backward(0, gs[0])
    g.close()
    # the oracle's difference quotient at the same h says what the curve's third derivative leaves; floats add 48 outputs' 64 U / h
    o = []
    for s in (1, -1):
        orc = OracleStage(st, gen.all_params(st, perturb=True))
        o.append(float(np.sum(orc.forward(0, _f64(xs[0]) + s * h * v) * gs[0])))
    slope = float(np.sum(dx * v))
    curve = abs((o[0] - o[1]) / (2 * h) - slope)
    got = (value(xs[0] + np.float32(h) * v) - value(xs[0] - np.float32(h) * v)) / (2 * h)
    assert curve <= 0.02 * np.linalg.norm(dx) * np.linalg.norm(v)
    assert abs(got - slope) <= curve + 64 * U / h * float(np.sum(np.abs(gs[0]) * 4))
