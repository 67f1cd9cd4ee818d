"""How rotary positions and attention are called: captured into graphs, on further streams, on the static workspace, at odd addresses and
in place, with spans that change, out of order; long sequences; profiles and timings."""
import ctypes as ct
import math

import numpy as np
import pytest
import torch

from gpu_harness import DEV, GpuStage, gpu_minibatch, stage_io, tdtype
from oracle import ops
from oracle.stage import one_f_one_b_order
from paper_2012_12544_amd import binding as B
from stage_inputs import configs as C
from stage_inputs import gen
from test_gpu_attention import BOTH, HALF, U, _attention, _rotary, _spans, _stage, run
from test_oracle_attention import attention_sublayer, some_spans

pytestmark = pytest.mark.gpu


def _device_io(st):
    xs, gs = stage_io(st)
    to = lambda a: torch.from_numpy(a).permute(0, 2, 3, 1).contiguous().to(DEV, tdtype(st))  # noqa: E731
    xs, gs = [to(a) for a in xs], [to(a) for a in gs]
    return xs, gs, [torch.zeros_like(a) for a in gs], [torch.zeros_like(a) for a in xs]


def _enqueue(g, st, io, spans=None, static=False, step=True):
    xs, gs, ys, dxs = io
    for t, m in one_f_one_b_order(st["n_micro"], B.bapipe_stage_stash_bytes(g.h)[1]):
        if t == "F":
            if spans is not None:
                B.bapipe_stage_set_spans(g.h, m, spans[m].data_ptr())
            B.bapipe_stage_forward(g.h, m, xs[m].data_ptr(), ys[m].data_ptr())
        else:
            (B.bapipe_stage_backward_static if static else B.bapipe_stage_backward)(g.h, m, gs[m].data_ptr(), dxs[m].data_ptr())
    if step:
        # <dy, y> has no lower end: at a rate of 0.01 the exact weights pass a float's range in six steps (the oracle's are at 1e16 there and
        # their gradients at 1e36), at this one they stay below 2
        B.bapipe_stage_step(g.h, 2e-4)


def _graph_stages():
    return {
        "spans": dict(mask=C.MASK_SPANS, heads=6, groups=2, d=64, c=48, seq=130, n_micro=3),
        "causal": dict(heads=4, groups=1, d=128, c=64, seq=200, n_micro=3),
        "no norm": dict(norm=0, d=40, c=40, seq=75, n_micro=3, cap=3.0, bias=4),
        "parts": dict(heads=4, groups=1, d=32, c=32, seq=1100, n_micro=2, micro_batch=1),
    }


@BOTH
@pytest.mark.parametrize("static", [False, True])
@pytest.mark.parametrize("name", list(_graph_stages()))
def test_a_captured_mini_batch(name, static, dtype):
    """Forward, backward and update in one graph, replayed on other inputs and other spans each time, with the eager stage, a profile and
    synchronizations between: weights, outputs and gradients as the eager stage's, bit for bit."""
    st = attention_sublayer(dtype=dtype, **_graph_stages()[name])
    params = gen.all_params(st, perturb=True)
    eager, captured = GpuStage(st, params), GpuStage(st, params)
    io_e, io_c = _device_io(st), _device_io(st)
    with_spans = st["layers"][3]["stride"] == C.MASK_SPANS
    spans_e, spans_c = ([torch.from_numpy(s).to(DEV) for s in _spans(st, "documents")] if with_spans else None for _ in range(2))
    torch.cuda.synchronize()
    _enqueue(eager, st, io_e, spans_e, static)               # the eager stage lives, with work behind it
    torch.cuda.synchronize()                                 # (the static workspace is one per GPU)
    _enqueue(captured, st, io_c, spans_c, static)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=captured.stream):
        _enqueue(captured, st, io_c, spans_c, static)
    r = np.random.default_rng(8)
    for replay in range(4):
        for m in range(st["n_micro"]):
            io_c[0][m].mul_(0.75), io_e[0][m].mul_(0.75)
            if with_spans:
                new = torch.from_numpy(some_spans(["random", "prefix", "window", "documents"][replay], st["micro_batch"], st["in_h"], r)).to(DEV)
                spans_c[m].copy_(new), spans_e[m].copy_(new)
        torch.cuda.synchronize()
        _enqueue(eager, st, io_e, spans_e, static)
        if static:
            torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(io_e[2] + io_e[3], io_c[2] + io_c[3]):
            assert torch.equal(a, b) and torch.all(torch.isfinite(a)), replay
        for i, (w, b) in enumerate(params):
            if w is not None:
                for a, e in zip(captured.get_params(i), eager.get_params(i)):
                    assert a is None or np.array_equal(a, e), (replay, i)
        if replay == 1:
            rec = B.bapipe_profile_layers(eager.h, 0, 1, len(st["layers"]))
            assert all(x["fwd_ms"] > 0 for x in rec) and all(x["bwd_ms"] > 0 for x in rec[:5])
        for t in io_c[2] + io_c[3]:
            t.zero_()
    del graph
    eager.close()
    captured.close()


def test_two_captured_stages_replayed_at_once():
    """Each handle has its own workspace: two graphs on two streams, overlapping."""
    sts = [attention_sublayer(heads=4, groups=1, d=64, c=64, seq=600, n_micro=2), attention_sublayer(heads=8, groups=2, d=32, c=32, seq=500, n_micro=2, norm=0)]
    alone, graphs, stages, ios = [], [], [], []
    for st in sts:
        params = gen.all_params(st, perturb=True)
        g, io = GpuStage(st, params), _device_io(st)
        torch.cuda.synchronize()
        _enqueue(g, st, io)
        torch.cuda.synchronize()
        alone.append([t.clone() for t in io[2] + io[3]])
        g.close()
        g = GpuStage(st, params)
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=g.stream):
            _enqueue(g, st, io, step=False)
        # without the step the next replay would add to the gradients only; the handle is left mid-mini-batch and only replayed
        graphs.append(graph), stages.append(g), ios.append(io)
    for _ in range(3):
        for io in ios:
            for t in io[2] + io[3]:
                t.zero_()
        torch.cuda.synchronize()
        for g, graph in zip(stages, graphs):
            with torch.cuda.stream(g.stream):
                graph.replay()
        torch.cuda.synchronize()
        for io, ref in zip(ios, alone):
            assert all(torch.equal(a, b) for a, b in zip(io[2] + io[3], ref))
    del graphs, graph
    for g in stages:
        g.close()


@BOTH
@pytest.mark.parametrize("kw", [dict(heads=4, groups=1, d=128, c=64, seq=260), dict(norm=0, d=40, c=40, seq=75), dict(d=24, heads=6, groups=3, seq=400, c=24)])
def test_further_streams_and_the_static_workspace_change_nothing(dtype, kw):
    st = attention_sublayer(dtype=dtype, n_micro=4, **kw)
    ref = gpu_minibatch(st)
    for how in (dict(), dict(static=True), dict(backward_stream=True), dict(backward_stream="no wgrad stream", eager_sync=False),
                dict(backward_stream=True, eager_sync=False), dict(wgrad_stream=True, eager_sync=False)):
        got = gpu_minibatch(st, **how)
        for k in ref:
            assert np.array_equal(got[k], ref[k]), (how, k)


def test_two_stages_at_once():
    sts = [attention_sublayer(heads=4, groups=2, d=64, c=64, seq=300, n_micro=3), attention_sublayer(heads=2, groups=1, d=96, c=32, seq=500, n_micro=3, mask=0)]
    params = [gen.all_params(st, perturb=True) for st in sts]
    alone = []
    for st, p in zip(sts, params):
        g, io = GpuStage(st, p), _device_io(st)
        torch.cuda.synchronize()
        _enqueue(g, st, io)
        torch.cuda.synchronize()
        alone.append([t.clone() for t in io[2] + io[3]])
        g.close()
    gs, ios = [GpuStage(st, p) for st, p in zip(sts, params)], [_device_io(st) for st in sts]
    torch.cuda.synchronize()
    for g, st, io in zip(gs, sts, ios):
        _enqueue(g, st, io)
    torch.cuda.synchronize()
    for io, ref in zip(ios, alone):
        assert all(torch.equal(a, b) for a, b in zip(io[2] + io[3], ref))
    for g in gs:
        g.close()


# ------------------------------------------------------------------------------ addresses
def _address_stages(dtype):
    return {
        "rotary": _rotary(dtype, 4, 2, 32, 33, norm=1),
        "rotary plain": _rotary(dtype, 3, 3, 20, 17, 10),
        "rotary odd": _rotary(dtype, 2, 1, 7, 17, 6, 1, 1),
        "attention": _attention(dtype, 4, 2, 32, 70),
        "attention wide": _attention(dtype, 2, 1, 128, 150, C.MASK_NONE),
        "attention odd": _attention(dtype, 2, 1, 9, 70, C.MASK_SPANS),
        "sublayer": attention_sublayer(dtype=dtype, n_micro=1, n_stages=1, d=32, c=64, seq=70),
    }


@BOTH
@pytest.mark.parametrize("name", list(_address_stages(C.FP32)))
def test_buffers_at_odd_addresses_and_over_one_another(dtype, name):
    """x, y, dy and dx some elements behind an aligned address, dx over dy, rows behind it and rows in front of it; y over x where their
    sizes are the same: the same bits, and nothing outside of the tensors touched."""
    st = _address_stages(dtype)[name]
    params = gen.all_params(st, perturb=True)
    (x0,), (g0,) = stage_io(st)
    t = tdtype(st)
    host = lambda a: torch.from_numpy(a).permute(0, 2, 3, 1).reshape(-1).to(DEV, t)  # noqa: E731
    x0, g0 = host(x0), host(g0)
    has_spans = any(L["kind"] == C.ATTENTION and L["stride"] == C.MASK_SPANS for L in st["layers"])
    spans = torch.zeros(1 + 2 * 2 * st["in_h"], dtype=torch.int32, device=DEV)
    spans[1:] = torch.from_numpy(_spans(st, "random")[0]).to(DEV).reshape(-1)
    ref = None
    for offset in (0, 1, 4):
        for over in (None, 0, 24, -24):
            g = GpuStage(st, params)
            bufs = [torch.full((n + 128,), 7.0, dtype=t, device=DEV) for n in (len(x0), len(g0), len(g0), len(x0))]
            at = 64 + offset
            x, y, dy, dx = (b[at:at + n] for b, n in zip(bufs, (len(x0), len(g0), len(g0), len(x0))))
            x.copy_(x0)
            if over is not None and len(x0) == len(g0):
                y = x
            if over is not None:
                bufs[3] = torch.full((max(len(x0), len(g0)) + 128,), 7.0, dtype=t, device=DEV)
                dy, dx = bufs[3][at:at + len(g0)], bufs[3][at + over:at + over + len(x0)]
            dy.copy_(g0)
            torch.cuda.synchronize()
            if has_spans:
                B.bapipe_stage_set_spans(g.h, 0, spans[1:].data_ptr())         # aligned to 4 bytes only
            B.bapipe_stage_forward(g.h, 0, x.data_ptr(), y.data_ptr())
            torch.cuda.synchronize()
            got = [y.clone()]
            B.bapipe_stage_backward(g.h, 0, dy.data_ptr(), dx.data_ptr())
            torch.cuda.synchronize()
            got += [dx.clone()] + [torch.from_numpy(a) for i, (w, _) in enumerate(params) if w is not None for a in g.grads(i) if a is not None]
            ref = ref or got
            for a, b in zip(got, ref):
                assert torch.equal(a, b) and torch.any(a != 0), (offset, over)
            if over is None:
                for b, n in zip(bufs, (len(x0), len(g0), len(g0), len(x0))):
                    assert torch.all(b[:at] == 7) and torch.all(b[at + n:] == 7)
            else:
                lo, hi = at + min(over, 0), at + max(len(g0), over + len(x0))
                assert torch.all(bufs[3][:lo] == 7) and torch.all(bufs[3][hi:] == 7)
            g.close()


@BOTH
@pytest.mark.parametrize("d", [12, 20])
def test_sums_in_parts_for_a_dx_at_an_odd_address(dtype, d):
    """Keys' sums in parts, joined four channels at a time where dx allows it: the same bits at every address, nothing beside dx touched."""
    st = _attention(dtype, 4, 1, d, 700, micro_batch=1)
    (x0,), (g0,) = stage_io(st)
    host = lambda a: torch.from_numpy(a).permute(0, 2, 3, 1).reshape(-1).to(DEV, tdtype(st))  # noqa: E731
    x, dy = host(x0), host(g0)
    ref = None
    for offset in (0, 1, 2, 3, 4):
        g = GpuStage(st, [(None, None)])
        y, buf = torch.zeros_like(dy), torch.full((len(x) + 128,), 7.0, dtype=x.dtype, device=DEV)
        dx = buf[64 + offset:64 + offset + len(x)]
        torch.cuda.synchronize()
        B.bapipe_stage_forward(g.h, 0, x.data_ptr(), y.data_ptr())
        B.bapipe_stage_backward(g.h, 0, dy.data_ptr(), dx.data_ptr())
        torch.cuda.synchronize()
        ref = dx.clone() if ref is None else ref
        assert torch.equal(dx, ref) and torch.any(dx != 0) and torch.all(torch.isfinite(dx)), offset
        assert torch.all(buf[:64 + offset] == 7) and torch.all(buf[64 + offset + len(x):] == 7), offset
        g.close()


@BOTH
@pytest.mark.parametrize("name", list(_address_stages(C.FP32)))
def test_a_stage_that_hands_no_gradient_on(dtype, name):
    st = _address_stages(dtype)[name]
    params = gen.all_params(st, perturb=True)
    xs, gs = stage_io(st)
    spans = _spans(st, "random") if any(L["kind"] == C.ATTENTION and L["stride"] == C.MASK_SPANS for L in st["layers"]) else None
    ref = run(st, params, xs, gs, spans)
    got = run(dict(st, need_input_grad=0), params, xs, gs, spans)
    assert got["dx0"] is None
    for k in ref:
        if k != "dx0":
            assert np.array_equal(got[k], ref[k]), k


# ------------------------------------------------------------------------------ order and refusals
def _status(call, *args, **kw):
    with pytest.raises(B.BapipeError) as e:
        call(*args, **kw)
    return e.value.status


def test_spans_belong_to_the_next_forward():
    st = _attention(C.FP32, 2, 1, 16, 20, C.MASK_SPANS, n_micro=3, stage_index=1, n_stages=2)
    xs, gs = stage_io(st)
    spans = _spans(st, "random")
    ref = run(st, [(None, None)], xs, gs, spans)
    g = GpuStage(st, [(None, None)])
    dev = [torch.from_numpy(s).to(DEV) for s in spans]
    x = torch.from_numpy(xs[0]).permute(0, 2, 3, 1).contiguous().to(DEV)
    y = torch.zeros(2 * 20 * 32, device=DEV)
    torch.cuda.synchronize()
    assert _status(B.bapipe_stage_forward, g.h, 0, x.data_ptr(), y.data_ptr()) == B.E_ORDER          # none given
    assert _status(B.bapipe_stage_set_spans, g.h, 1, dev[1].data_ptr()) == B.E_ORDER                  # not the next one
    assert _status(B.bapipe_stage_set_spans, g.h, -1, dev[1].data_ptr()) == B.E_ORDER
    assert _status(B.bapipe_stage_set_spans, g.h, 0, None) == B.E_INVALID
    assert _status(B.bapipe_stage_set_spans, g.h, 0, dev[0].data_ptr() + 2) == B.E_INVALID
    for mini_batch in range(2):
        for t, m in one_f_one_b_order(3, 2):
            if t == "F":
                B.bapipe_stage_set_spans(g.h, m, dev[(m + 1) % 3].data_ptr())
                B.bapipe_stage_set_spans(g.h, m, dev[m].data_ptr())            # the last one counts
                assert np.array_equal(g.forward(m, xs[m]), ref["y%d" % m])
                if m < 2:                                                      # given once, for one micro-batch
                    assert _status(B.bapipe_stage_forward, g.h, m + 1, x.data_ptr(), y.data_ptr()) == B.E_ORDER
            else:
                assert np.array_equal(g.backward(m, gs[m]), ref["dx%d" % m])
        assert _status(B.bapipe_stage_set_spans, g.h, 3, dev[0].data_ptr()) == B.E_ORDER
        B.bapipe_stage_step(g.h, 0.1)
    g.close()
    g = GpuStage(_attention(C.FP32, 2, 1, 16, 20), [(None, None)])
    assert _status(B.bapipe_stage_set_spans, g.h, 0, dev[0].data_ptr()) == B.E_INVALID                # no layer with spans
    g.close()


def test_angles_are_set_between_mini_batches():
    st = _rotary(C.FP32, 2, 1, 8, 6, norm=1)
    params = gen.all_params(st)
    xs, gs = stage_io(st)
    g = GpuStage(st, params)
    nan, inf = math.nan, math.inf
    for bad in (dict(base=0.0), dict(base=-1.0), dict(base=nan), dict(base=inf), dict(factor=0.0), dict(factor=inf), dict(factor=nan), dict(magnitude=0.0),
                dict(magnitude=nan), dict(magnitude=1e39), dict(original_length=-1.0), dict(original_length=nan), dict(original_length=inf),
                dict(original_length=8.0, low_turns=2.0, high_turns=2.0), dict(original_length=8.0, low_turns=nan, high_turns=2.0),
                dict(original_length=8.0, low_turns=0.0, high_turns=inf), dict(first_position=-1), dict(first_position=2 ** 40 + 1)):
        assert _status(B.bapipe_stage_set_rotary, g.h, 0, **bad) == B.E_INVALID, bad
    for layer in (-1, 1):
        assert _status(B.bapipe_stage_set_rotary, g.h, layer) == B.E_INVALID
    assert B.load().bapipe_stage_set_rotary(g.h, 0, None) == B.E_INVALID
    y = g.forward(0, xs[0])                                  # a refused call has changed nothing
    assert np.array_equal(y, run(st, params, xs, gs)["y0"])
    assert _status(B.bapipe_stage_set_rotary, g.h, 0, base=50.0) == B.E_ORDER
    g.backward(0, gs[0])
    assert _status(B.bapipe_stage_set_rotary, g.h, 0, base=50.0) == B.E_ORDER
    B.bapipe_stage_step(g.h, 0.0)
    B.bapipe_stage_set_rotary(g.h, 0, base=50.0)
    assert np.array_equal(g.forward(0, xs[0]), run(st, params, xs, gs, angles={0: dict(base=50.0)})["y0"])
    g.backward(0, gs[0])
    B.bapipe_stage_step(g.h, 0.0)
    B.bapipe_stage_set_rotary(g.h, 0)
    assert np.array_equal(g.forward(0, xs[0]), y)
    g.close()
    g = GpuStage(_attention(C.FP32, 2, 1, 16, 20), [(None, None)])
    assert _status(B.bapipe_stage_set_rotary, g.h, 0) == B.E_INVALID
    g.close()


def test_gains():
    st = _rotary(C.BF16, 2, 1, 12, 6, norm=1)
    xs, gs = stage_io(st)
    g = GpuStage(st, [(None, None)])
    w, _ = B.bapipe_stage_get_params(g.h, 0, (2, 12), None)
    assert np.array_equal(w, np.ones((2, 12)))
    assert _status(B.bapipe_stage_set_params, g.h, 0, None, np.zeros(12, np.float32)) == B.E_INVALID
    new = np.random.default_rng(1).standard_normal((2, 12)).astype(np.float32)
    B.bapipe_stage_set_params(g.h, 0, new, None)
    assert np.array_equal(B.bapipe_stage_get_params(g.h, 0, (2, 12), None)[0], new)
    g.forward(0, xs[0])
    g.backward(0, gs[0])
    dw, _ = B.bapipe_stage_get_grads(g.h, 0, (2, 12), None)
    B.bapipe_stage_step(g.h, 0.5)
    assert np.array_equal(B.bapipe_stage_get_params(g.h, 0, (2, 12), None)[0], np.float32(new - np.float32(0.5) * dw))
    assert not B.bapipe_stage_get_grads(g.h, 0, (2, 12), None)[0].any()
    g.close()
    for st in (_rotary(C.BF16, 2, 1, 12, 6), _attention(C.BF16, 2, 1, 12, 6)):
        g = GpuStage(st, [(None, None)])
        assert _status(B.bapipe_stage_set_params, g.h, 0, np.ones((2, 12), np.float32), None) == B.E_INVALID
        g.close()


# ------------------------------------------------------------------------------ long sequences
@BOTH
@pytest.mark.parametrize("T,window", [(20000, 40), (70000, 3)])
def test_a_window_over_a_long_sequence(dtype, T, window):
    """Positions whose queries are those of others further on, too: a window's rows are gathered and computed in 64 bits."""
    H, d = 2, 16
    st = _attention(dtype, H, 1, d, T, C.MASK_SPANS, micro_batch=1)
    xs, gs = stage_io(st)
    at = np.arange(T)
    first = np.maximum(at + 1 - window, 0)
    spans = np.stack([first, at + 1], -1).astype(np.int32)[None]
    got = run(st, [(None, None)], xs, gs, [spans])
    z = torch.from_numpy(ops.split_heads(xs[0], H + 2)[0])
    do = torch.from_numpy(ops.split_heads(gs[0], H)[0])
    q, k, v = (t.clone().requires_grad_() for t in (z[:H], z[H], z[H + 1]))
    near = torch.from_numpy(at[:, None] + 1 - window + np.arange(window))
    s = (q[:, :, None] * k[near.clamp(min=0)]).sum(-1) / math.sqrt(d)
    p = torch.softmax(s.masked_fill(near < 0, -math.inf), -1)
    y = (p[..., None] * v[near.clamp(min=0)]).sum(2)
    (y * do).sum().backward()
    dx = torch.cat([q.grad, k.grad[None], v.grad[None]])
    loose = 4 * (math.sqrt(d) + math.sqrt(window * H) + 8) * 2 * U
    for name, a, b, n in (("y0", got["y0"], y.detach(), 2), ("dx0", got["dx0"], dx, 5)):
        b = ops.join_heads(b.numpy()[None])
        limit = loose if dtype == C.FP32 else 2 * math.sqrt(n / 3) * HALF[C.BF16]
        for lo in range(0, T, T // 10):                      # everywhere alike
            e = np.linalg.norm(a[:, :, lo:lo + T // 10] - b[:, :, lo:lo + T // 10])
            assert e <= limit * np.linalg.norm(b[:, :, lo:lo + T // 10]), (name, lo)


def test_more_heads_than_a_launch_has_groups_of_lanes_for():
    """2^28 heads of a channel in one round, 256 thousand more in the next.  Nothing turns, so y is x and dx is dy."""
    st = _rotary(C.BF16, 32767, 1, 1, 1, micro_batch=8200)
    n = 8200 * 32769
    assert n > 2 ** 28
    g = GpuStage(st, [(None, None)])
    gen_ = torch.Generator(DEV)
    gen_.manual_seed(3)
    x, dy = (torch.randint(-32768, 32768, (n,), dtype=torch.int16, device=DEV, generator=gen_) & ~0x4000 for _ in range(2))      # no infinity, no NaN
    y, dx = torch.zeros_like(x), torch.zeros_like(x)
    torch.cuda.synchronize()
    B.bapipe_stage_forward(g.h, 0, x.data_ptr(), y.data_ptr())
    B.bapipe_stage_backward(g.h, 0, dy.data_ptr(), dx.data_ptr())
    torch.cuda.synchronize()
    # as numbers: -0 cos + 0 sin is +0, the sum of two zeros of different signs
    assert all(torch.equal(a.view(torch.bfloat16), b.view(torch.bfloat16)) for a, b in ((x, y), (dy, dx)))
    assert bool(((x == y) | (x == -32768)).all()) and bool(((dy == dx) | (dy == -32768)).all())
    g.close()


def test_sums_that_the_static_workspace_does_not_hold():
    """Few key heads of many positions: the parts of their sums take more than the array.  The call is refused and the other one works."""
    st = _attention(C.BF16, 8, 1, 128, 16384, C.MASK_CAUSAL, micro_batch=1)
    xs, gs = stage_io(st)
    g = GpuStage(st, [(None, None)])
    g.forward(0, xs[0])
    with pytest.raises(B.BapipeError) as e:
        g.backward(0, gs[0], static=True)
    assert e.value.status == B.E_UNSUPPORTED
    dx = g.backward(0, gs[0])
    assert np.all(np.isfinite(dx)) and np.linalg.norm(dx) > 0
    g.close()


def test_sums_of_many_parts_and_tiles():
    """16384 positions of 8 query heads on one key head: y and dq of some positions, dk and dv of some keys, in 64 bits.

    In the 2-norm of a head's channels: y has been through two roundings (a probability, itself), gradients through at most five (a probability,
    the output in dout . o, its own, the gradient of a score, itself), each of root mean square up to HALF / sqrt(3) and independent from
    summand to summand; twice that.  One of the eight parts that the keys' sums are taken in is a third of them, in the 2-norm."""
    H, d, T = 8, 128, 16384
    st = _attention(C.BF16, H, 1, d, T, C.MASK_CAUSAL, micro_batch=1)
    xs, gs = stage_io(st)
    got = run(st, [(None, None)], xs, gs)
    r = np.random.default_rng(4)
    some = np.unique(np.concatenate([[0, 1, 63, 64, 127, 128, 129, 8191, 8192, T - 64, T - 2, T - 1], r.integers(0, T, 24)]))
    dev = lambda a, n: torch.from_numpy(ops.split_heads(a, n)[0]).to(DEV)  # noqa: E731
    x, dy, at = dev(xs[0], H + 2), dev(gs[0], H), torch.from_numpy(some).to(DEV)
    k, v = x[H], x[H + 1]
    seen = torch.ones((T, T), dtype=torch.bool, device=DEV).tril()
    y, dq, dk, dv = [], [], torch.zeros((len(some), d), dtype=torch.float64, device=DEV), torch.zeros((len(some), d), dtype=torch.float64, device=DEV)
    for h in range(H):
        q, do = x[h], dy[h]
        p = torch.softmax((q @ k.T / math.sqrt(d)).masked_fill_(~seen, -math.inf), -1)
        o = p @ v
        less = (do * o).sum(-1, keepdim=True)
        y.append(o[at])
        dq.append((p[at] * (do[at] @ v.T - less[at])) @ k / math.sqrt(d))
        p = p[:, at].contiguous()
        dk += (p * (do @ v[at].T - less)).T @ q / math.sqrt(d)
        dv += p.T @ do
    loose = 4 * (math.sqrt(d) + math.sqrt(T) + 8) * 2 * U
    dx = ops.split_heads(got["dx0"], H + 2)[0][:, some]
    for name, a, b, n in (("y", ops.split_heads(got["y0"], H)[0][:, some], torch.stack(y), 2), ("dq", dx[:H], torch.stack(dq), 5), ("dk", dx[H], dk, 5), ("dv", dx[H + 1], dv, 5)):
        b = b.cpu().numpy()
        size = np.linalg.norm(b, axis=-1)
        if name == "dq":                                     # position 0 sees one key: nothing of its gradient is left
            a, b, size = a[:, 1:], b[:, 1:], size[:, 1:]
        off = np.linalg.norm(a - b, axis=-1) / size
        assert np.all(off <= 2 * math.sqrt(n / 3) * HALF[C.BF16] + loose), (name, float(off.max()))


# ------------------------------------------------------------------------------ profile and timing
@BOTH
def test_timing_and_profile_of_attention(dtype):
    st = attention_sublayer(dtype=dtype, heads=4, groups=2, d=32, c=32, seq=100, n_micro=2, mask=C.MASK_SPANS)
    params = gen.all_params(st)
    xs, gs = stage_io(st)
    spans = [torch.from_numpy(s).to(DEV) for s in _spans(st, "documents")]
    g = GpuStage(st, params)
    rec = B.bapipe_profile_layers(g.h, 1, 2, 6)             # before any spans were given
    assert all(r["fwd_ms"] > 0 for r in rec) and all(r["bwd_ms"] > 0 for r in rec[:5])
    B.bapipe_stage_kernel_timing(g.h, B.KC_ATTENTION)
    for m in range(2):
        B.bapipe_stage_set_spans(g.h, m, spans[m].data_ptr())
        g.forward(m, xs[m])
        g.backward(m, gs[m])
    t = B.bapipe_stage_kernel_timing_read(g.h)
    pairs = 2 * 2 * 4 * 100 * 100                            # micro-batches, samples, heads, all as if seen
    assert t["launches"] == 4 and t["total_ms"] > 0 and t["flop"] == (2 + 5) * 2 * 32 * pairs      # scores are made anew in the backward pass
    g.close()


def test_what_a_micro_batch_in_flight_holds():
    """A ROTARY in front of an ATTENTION turns the projection's output in place; in bf16 its queries and keys are kept in 16-bit floats with
    a scale for each head and position."""
    def per_micro_batch(norm, dtype):
        b = C._Builder()
        b.conv(64, 512, 1, src=-1)
        b.rotary(4, 2, 64, norm=norm)
        b.attention(4, 2, 64)
        b.conv(256, 64, 1)
        g = GpuStage(_stage(b.layers, dtype, (64, 1024, 1)), [(None, None)] * 4)
        per = B.bapipe_stage_stash_bytes(g.h)[0]
        g.close()
        return per
    rows, es = 2 * 1024, 2
    base = rows * (64 + 512 + 256) * es + rows * 256 + rows * 4 * 4       # x, projection, attention's output and eight more bits of it, logarithms of its sums
    halves = rows * 6 * 64 * 2 + rows * 6 * 4
    assert per_micro_batch(0, C.BF16) == per_micro_batch(1, C.BF16) == base + halves       # the norms' input, the values with it, is the projection
    assert per_micro_batch(0, C.FP32) == rows * (64 + 512 + 256) * 4 + rows * 4 * 4
    assert per_micro_batch(1, C.FP32) == rows * (64 + 2 * 512 + 256) * 4 + rows * 4 * 4     # what was turned as well
