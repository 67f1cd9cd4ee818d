"""ctypes access to the CPU oracle's layer functions (oracle/bapipe_oracle.c).

TEST INFRASTRUCTURE ONLY.  Arrays are float64 numpy, activations NCHW."""
import ctypes as ct
import math
import os

import numpy as np

from . import build as _build

_lib = None
_D = ct.POINTER(ct.c_double)


def lib():
    global _lib
    if _lib is None:
        path = _build.build(force=False)
        _lib = ct.CDLL(path)
        _lib.orc_xent_bwd.restype = ct.c_double
        _lib.orc_num_threads.restype = ct.c_int
    return _lib


def _p(a):
    if a is None:
        return None
    assert a.dtype == np.float64 and a.flags["C_CONTIGUOUS"], (a.dtype, a.flags)
    return a.ctypes.data_as(_D)


def _f64(a):
    return np.ascontiguousarray(a, dtype=np.float64)


def num_threads():
    return lib().orc_num_threads()


def round_bf16(a):
    """Round every element to the nearest-even bf16 value (returns a new float64 array)."""
    out = _f64(a).copy()
    lib().orc_round_bf16(_p(out), ct.c_size_t(out.size))
    return out


def _out_hw(H, W, k, st, pad):
    return (H + 2 * pad - k[0]) // st + 1, (W + 2 * pad - k[1]) // st + 1


def conv2d_fwd(x, w, b, stride, pad):
    x, w = _f64(x), _f64(w)
    b = None if b is None else _f64(b)
    N, Cin, H, W = x.shape
    Cout, Cin2, kh, kw = w.shape
    assert Cin == Cin2
    Ho, Wo = _out_hw(H, W, (kh, kw), stride, pad)
    y = np.empty((N, Cout, Ho, Wo))
    lib().orc_conv2d_fwd(_p(x), _p(w), _p(b), _p(y), N, Cin, H, W, Cout, kh, kw, stride, pad)
    return y


def conv2d_dgrad(dy, w, x_shape, stride, pad):
    dy, w = _f64(dy), _f64(w)
    N, Cin, H, W = x_shape
    Cout, _, kh, kw = w.shape
    assert dy.shape == (N, Cout) + _out_hw(H, W, (kh, kw), stride, pad)
    dx = np.empty(x_shape)
    lib().orc_conv2d_dgrad(_p(dy), _p(w), _p(dx), N, Cin, H, W, Cout, kh, kw, stride, pad)
    return dx


def conv2d_wgrad(x, dy, dw, db, stride, pad):
    """Accumulates into dw (OIHW float64) and db (may be None)."""
    x, dy = _f64(x), _f64(dy)
    N, Cin, H, W = x.shape
    Cout, _, kh, kw = dw.shape
    assert dy.shape == (N, Cout) + _out_hw(H, W, (kh, kw), stride, pad)
    lib().orc_conv2d_wgrad(_p(x), _p(dy), _p(dw), _p(db), N, Cin, H, W, Cout, kh, kw, stride, pad)


def relu_fwd(x):
    x = _f64(x)
    y = np.empty_like(x)
    lib().orc_relu_fwd(_p(x), _p(y), ct.c_size_t(x.size))
    return y


def relu_bwd(y, dy):
    y, dy = _f64(y), _f64(dy)
    dx = np.empty_like(y)
    lib().orc_relu_bwd(_p(y), _p(dy), _p(dx), ct.c_size_t(y.size))
    return dx


def maxpool_fwd(x, k=2, stride=2, pad=0):
    x = _f64(x)
    N, C, H, W = x.shape
    Ho, Wo = _out_hw(H, W, (k, k), stride, pad)
    y = np.empty((N, C, Ho, Wo))
    idx = np.empty((N, C, Ho, Wo), np.uint8)
    lib().orc_maxpool_fwd(_p(x), _p(y), idx.ctypes.data_as(ct.POINTER(ct.c_uint8)),
                          N, C, H, W, k, k, stride, pad)
    return y, idx


def maxpool_bwd(dy, idx, x_shape, k=2, stride=2, pad=0):
    dy = _f64(dy)
    idx = np.ascontiguousarray(idx, np.uint8)
    N, C, H, W = x_shape
    dx = np.empty(x_shape)
    lib().orc_maxpool_bwd(_p(dy), idx.ctypes.data_as(ct.POINTER(ct.c_uint8)), _p(dx),
                          N, C, H, W, k, k, stride, pad)
    return dx


def avgpool_fwd(x, k):
    x = _f64(x)
    N, C, H, W = x.shape
    y = np.empty((N, C, H // k, W // k))
    lib().orc_avgpool_fwd(_p(x), _p(y), N, C, H, W, k, k)
    return y


def avgpool_bwd(dy, x_shape, k):
    dy = _f64(dy)
    N, C, H, W = x_shape
    assert dy.shape == (N, C, H // k, W // k)
    dx = np.empty(x_shape)
    lib().orc_avgpool_bwd(_p(dy), _p(dx), N, C, H, W, k, k)
    return dx


def bn_fwd(x, gamma, beta, eps):
    x, gamma, beta = _f64(x), _f64(gamma), _f64(beta)
    N, C, H, W = x.shape
    y = np.empty_like(x)
    mean = np.empty(C)
    invstd = np.empty(C)
    lib().orc_bn_fwd(_p(x), _p(gamma), _p(beta), ct.c_double(eps), _p(y), _p(mean), _p(invstd),
                     N, C, H * W)
    return y, mean, invstd


def bn_bwd(x, dy, gamma, mean, invstd, dgamma, dbeta):
    """Returns dx; accumulates into dgamma, dbeta."""
    x, dy, gamma = _f64(x), _f64(dy), _f64(gamma)
    N, C, H, W = x.shape
    dx = np.empty_like(x)
    lib().orc_bn_bwd(_p(x), _p(dy), _p(gamma), _p(mean), _p(invstd), _p(dx), _p(dgamma),
                     _p(dbeta), N, C, H * W)
    return dx


def lstm_fwd(x, w, b, round16=False):
    """x [N][In][T][1], w [4*Hd][In+Hd], b [4*Hd] or None -> (y [N][Hd][T][1], (gates, cells))."""
    x, w = _f64(x), _f64(w)
    b = None if b is None else _f64(b)
    N, In, T, one = x.shape
    assert one == 1 and w.shape[0] % 4 == 0
    Hd = w.shape[0] // 4
    assert w.shape[1] == In + Hd
    y = np.empty((N, Hd, T, 1))
    gates = np.empty((N, T, 4 * Hd))
    cells = np.empty((N, T, Hd))
    lib().orc_lstm_fwd(_p(x), _p(w), _p(b), _p(y), _p(gates), _p(cells), N, In, Hd, T, int(bool(round16)))
    return y, (gates, cells)


def lstm_bwd(x, y, w, saved, dy, dw, db, want_dx=True, round16=False):
    """Returns dx (or None); accumulates into dw, db."""
    x, y, w, dy = _f64(x), _f64(y), _f64(w), _f64(dy)
    gates, cells = saved
    N, In, T, _ = x.shape
    Hd = w.shape[0] // 4
    dx = np.empty_like(x) if want_dx else None
    D = np.empty((N, T, 4 * Hd))
    lib().orc_lstm_bwd(_p(x), _p(y), _p(w), _p(gates), _p(cells), _p(dy), _p(dx), _p(dw), _p(db), _p(D),
                       N, In, Hd, T, int(bool(round16)))
    return dx


def linear_fwd(x, w, b):
    x, w = _f64(x), _f64(w)
    b = None if b is None else _f64(b)
    N, In = x.shape
    Out = w.shape[0]
    assert w.shape[1] == In
    y = np.empty((N, Out))
    lib().orc_linear_fwd(_p(x), _p(w), _p(b), _p(y), N, In, Out)
    return y


def linear_dgrad(dy, w):
    dy, w = _f64(dy), _f64(w)
    N, Out = dy.shape
    In = w.shape[1]
    dx = np.empty((N, In))
    lib().orc_linear_dgrad(_p(dy), _p(w), _p(dx), N, In, Out)
    return dx


def linear_wgrad(x, dy, dw, db):
    x, dy = _f64(x), _f64(dy)
    N, In = x.shape
    Out = dy.shape[1]
    assert dw.shape == (Out, In)
    lib().orc_linear_wgrad(_p(x), _p(dy), _p(dw), _p(db), N, In, Out)


# Layers that act on every position by itself; x [N][C][H][W]
def layernorm_fwd(x, gamma, beta, eps):
    """Returns y, xhat, 1/std (biased variance over the channels of a position)."""
    x = _f64(x)
    d = x - x.mean(axis=1, keepdims=True)
    inv = 1.0 / np.sqrt((d * d).mean(axis=1, keepdims=True) + eps)
    xhat = d * inv
    return xhat * gamma[:, None, None] + beta[:, None, None], xhat, inv


def layernorm_bwd(xhat, inv, dy, gamma, dgamma, dbeta):
    """Returns dx; accumulates into dgamma, dbeta."""
    dgamma += (dy * xhat).sum(axis=(0, 2, 3))
    dbeta += dy.sum(axis=(0, 2, 3))
    a = dy * gamma[:, None, None]
    return inv * (a - a.mean(axis=1, keepdims=True) - xhat * (a * xhat).mean(axis=1, keepdims=True))


_erf = np.vectorize(math.erf, otypes=[np.float64])


def gate(act, g):
    """act(g) and its derivative; act: 0 sigmoid, 1 SiLU, 2 GELU, 3 ReLU."""
    if act == 3:
        return np.maximum(g, 0.0), (g > 0).astype(np.float64)
    if act == 2:
        cdf = 0.5 * (1.0 + _erf(g / np.sqrt(2.0)))
        return g * cdf, cdf + g * np.exp(-0.5 * g * g) / np.sqrt(2.0 * np.pi)
    e = np.exp(-np.abs(g))
    s = np.where(g < 0, e, 1.0) / (1.0 + e)
    if act == 0:
        return s, s * (1.0 - s)
    return g * s, s + g * s * (1.0 - s)


def gated_fwd(x, w, b, act):
    """w [2*F][C], gate rows first.  Returns y [N][F][H][W] and the projections [N][2*F][H][W]."""
    x = _f64(x)
    both = np.tensordot(w, x, axes=([1], [1])).transpose(1, 0, 2, 3)
    if b is not None:
        both = both + b[:, None, None]
    F = w.shape[0] // 2
    return gate(act, both[:, :F])[0] * both[:, F:], both


def gated_bwd(x, w, both, act, dy, dw, db, q=lambda a: a, fine=False):
    """Returns dx; accumulates into dw, db.  q rounds the gradients of the projections, which are stored; fine: not those that dx is made of."""
    F = w.shape[0] // 2
    a, da = gate(act, both[:, :F])
    exact = np.concatenate([dy * both[:, F:] * da, dy * a], axis=1)
    D = q(exact)
    dw += np.tensordot(D, x, axes=([0, 2, 3], [0, 2, 3]))
    if db is not None:
        db += D.sum(axis=(0, 2, 3))
    return np.tensordot(exact if fine else D, w, axes=([1], [0])).transpose(0, 3, 1, 2)


def philox4x32(counter, key):
    """Ten rounds.  counter: uint32 array [..., 4], key: two numbers.  Returns uint32 [..., 4]."""
    c = [counter[..., i].astype(np.uint64) for i in range(4)]
    low, w32 = np.uint64(0xFFFFFFFF), np.uint64(32)
    k = [int(key[0]), int(key[1])]
    for _ in range(10):
        a, b = np.uint64(0xD2511F53) * c[0], np.uint64(0xCD9E8D57) * c[2]
        c = [(b >> w32) ^ c[1] ^ np.uint64(k[0]), b & low, (a >> w32) ^ c[3] ^ np.uint64(k[1]), a & low]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return np.stack(c, axis=-1).astype(np.uint32)


def dropout_factor(shape, p, seed, layer, micro_batch, mini_batch):
    """0 or 1/(1-p) per element of [N][C][H][W]; elements are numbered in NHWC order."""
    N, C, H, W = shape
    n, p = N * C * H * W, float(np.float32(p))
    c = np.zeros(((n + 3) // 4, 4), np.uint32)
    c[:, 0] = np.arange(len(c))
    c[:, 1:] = layer, micro_batch, mini_batch
    words = philox4x32(c, (seed & 0xFFFFFFFF, seed >> 32)).reshape(-1)[:n]
    keep = words.astype(np.int64) >= min(int(np.floor(p * 2.0 ** 32 + 0.5)), 2 ** 32 - 1)
    return (keep / (1.0 - p)).reshape(N, H, W, C).transpose(0, 3, 1, 2)


def softmax_fwd(z):
    z = _f64(z)
    p = np.empty_like(z)
    lib().orc_softmax_fwd(_p(z), _p(p), z.shape[0], z.shape[1])
    return p


def xent_bwd(z, labels, scale):
    """Returns (loss, dz) with loss = -scale*sum_n log softmax(z)[n,label_n]."""
    z = _f64(z)
    labels = np.ascontiguousarray(labels, np.int32)
    dz = np.empty_like(z)
    loss = lib().orc_xent_bwd(_p(z), labels.ctypes.data_as(ct.POINTER(ct.c_int32)),
                              ct.c_double(scale), _p(dz), z.shape[0], z.shape[1])
    return loss, dz


def sgd_step(w, g, lr):
    """In place: w <- w - lr*g."""
    lib().orc_sgd_step(_p(w), _p(_f64(g)), ct.c_double(lr), ct.c_size_t(w.size))


# ------------------------------------------------------------------------------ rotary positions and attention
def split_heads(x, heads):
    """(N, C, T, 1) -> (N, heads, T, d) of as many heads in all."""
    x = _f64(x)
    N, Cn, T, _ = x.shape
    return x[..., 0].reshape(N, heads, Cn // heads, T).transpose(0, 1, 3, 2)


def join_heads(z):
    N, heads, T, d = z.shape
    return np.ascontiguousarray(z.transpose(0, 1, 3, 2)).reshape(N, heads * d, T, 1)


ANGLES = dict(base=10000.0, factor=1.0, original_length=0.0, low_turns=1.0, high_turns=4.0, magnitude=1.0, first_position=0)


def rotary_angles(T, turning, **changed):
    """(T, turning / 2) complex numbers magnitude exp(i t f_j)"""
    a = dict(ANGLES, **changed)
    f = a["base"] ** (-2.0 * np.arange(turning // 2) / max(turning, 1))
    if a["original_length"] == 0:
        f = f / a["factor"]
    else:
        turns = a["original_length"] * f / (2 * math.pi)
        s = np.clip((turns - a["low_turns"]) / (a["high_turns"] - a["low_turns"]), 0.0, 1.0)
        f = f * (s + (1 - s) / a["factor"])
    t = a["first_position"] + np.arange(T, dtype=np.float64)
    return a["magnitude"] * np.exp(1j * t[:, None] * f)


def _turn(z, by, pairs):
    r = 2 * by.shape[1]
    a, b = (z[..., 0:r:2], z[..., 1:r:2]) if pairs else (z[..., :r // 2], z[..., r // 2:r])
    c = (a + 1j * b) * by
    out = z.copy()
    if pairs:
        out[..., 0:r:2], out[..., 1:r:2] = c.real, c.imag
    else:
        out[..., :r // 2], out[..., r // 2:r] = c.real, c.imag
    return out


def _rms(z, eps):
    return 1.0 / np.sqrt((z * z).mean(-1, keepdims=True) + eps)


def rotary_fwd(x, heads, groups, by, pairs, gains=None, eps=0.0):
    z = split_heads(x, heads + 2 * groups)
    qk = z[:, :heads + groups]
    if gains is not None:
        gain = np.repeat(gains, [heads, groups], axis=0)[:, None]
        qk = qk * _rms(qk, eps) * gain
    return join_heads(np.concatenate([_turn(qk, by, pairs), z[:, heads + groups:]], 1))


def rotary_bwd(x, dy, heads, groups, by, pairs, gains=None, eps=0.0, dgains=None):
    """dx; accumulates into dgains [2][d]"""
    z, g = split_heads(x, heads + 2 * groups), split_heads(dy, heads + 2 * groups)
    qk, dqk = z[:, :heads + groups], _turn(g[:, :heads + groups], by.conj(), pairs)
    if gains is not None:
        gain, r = np.repeat(gains, [heads, groups], axis=0)[:, None], _rms(qk, eps)
        xhat = qk * r
        by_head = (dqk * xhat).sum((0, 2))
        dgains += np.stack([by_head[:heads].sum(0), by_head[heads:].sum(0)])
        dqk = dqk * gain
        dqk = r * (dqk - xhat * (dqk * xhat).mean(-1, keepdims=True))
    return join_heads(np.concatenate([dqk, g[:, heads + groups:]], 1))


def attention_sees(mask, N, T, spans=None):
    """(N or 1, 1, T, T) of booleans: whether a position (third axis) sees a key.  mask: 0 all, 1 up to itself, 2 spans (N, T, 2)."""
    i = np.arange(T)
    if mask == 0:
        return np.ones((1, 1, T, T), bool)
    if mask == 1:
        return (i <= i[:, None])[None, None]
    spans = np.asarray(spans).reshape(N, 1, T, 1, 2)
    return (i >= spans[..., 0]) & (i < spans[..., 1])


def attention_probabilities(x, heads, groups, sees, cap=0.0, bias=0):
    """(N, heads, T, T) probabilities and the cap's slope there, of the queries and keys in x"""
    z = split_heads(x, heads + 2 * groups)
    d, T = z.shape[-1], z.shape[2]
    q, k = z[:, :heads], np.repeat(z[:, heads:heads + groups], heads // groups, axis=1)
    s = q @ k.transpose(0, 1, 3, 2) / math.sqrt(d)
    slope = np.ones_like(s)
    if cap:
        t = np.tanh(s / cap)
        s, slope = cap * t, 1 - t * t
    if bias:
        i = np.arange(T)
        s = s - 2.0 ** (-bias * np.arange(1, heads + 1) / heads)[:, None, None] * np.abs(i[:, None] - i)
    s = np.where(sees, s, -np.inf)
    top = s.max(-1, keepdims=True)
    p = np.exp(s - np.where(np.isneginf(top), 0.0, top))
    total = p.sum(-1, keepdims=True)
    return p / np.where(total == 0, 1.0, total), slope


def attention_fwd(x, heads, groups, p):
    v = np.repeat(split_heads(x, heads + 2 * groups)[:, heads + groups:], heads // groups, axis=1)
    return join_heads(p @ v)


def attention_bwd(x, dy, heads, groups, p, slope):
    z, do = split_heads(x, heads + 2 * groups), split_heads(dy, heads)
    N, _, T, d = z.shape
    per = heads // groups
    q = z[:, :heads]
    k, v = (np.repeat(t, per, axis=1) for t in (z[:, heads:heads + groups], z[:, heads + groups:]))
    dp = do @ v.transpose(0, 1, 3, 2)
    ds = p * (dp - (p * dp).sum(-1, keepdims=True)) * slope / math.sqrt(d)

    def shared(t):
        return t.reshape(N, groups, per, T, d).sum(2)

    return join_heads(np.concatenate([ds @ k, shared(ds.transpose(0, 1, 3, 2) @ q), shared(p.transpose(0, 1, 3, 2) @ do)], 1))
