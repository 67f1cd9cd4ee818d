"""What a user has the layers of a transformer's feed-forward sublayer do: mini-batches of stages made of them.

One pass is one mini-batch as a pipeline worker runs it: M forward and M backward passes in 1F1B order, then the weight
update.  What comes back: the stage's output of every micro-batch, the gradient handed to the previous stage, the accumulated
weight gradients in the stage's storage type (as they go to the other replicas of the stage), and the updated master weights.

Stages, per position of a (channels, sequence, 1) tensor:
    layernorm   LAYERNORM
    dropout     DROPOUT
    gated       GATED: activation(x Wg' + bg) * (x Wu' + bu)
    sublayer    x + DROPOUT(CONV 1x1(GATED(LAYERNORM(x))))
"""
import math

import numpy as np
import torch

own = False

LR = 2e-5
EPS = 1e-5
SIGMOID, SILU, GELU, RELU = range(4)


# ---------------------------------------------------------------------------------------------- cases
def _case(name, kind, cin, cout, seq, micro_batch, n_micro=1, in_flight=1, dtype="bf16", act=SILU, p=0.0, bias=0):
    """cin: channels of the stage input; cout: units of the gated layer (0 where there is none)."""
    return dict(name=name, kind=kind, cin=cin, cout=cout, seq=seq, micro_batch=micro_batch, n_micro=n_micro,
                in_flight=in_flight, dtype=dtype, act=act, p=p, bias=bias)


def listed():
    return [
        # one position in flight: nothing but latency
        _case("layer norm token", "layernorm", 1024, 0, 1, 1),
        # between the LSTM layers of the GNMT stage that the repository is configured for
        _case("layer norm gnmt", "layernorm", 1024, 0, 50, 64, n_micro=8, in_flight=3),
        # wide model, long sequences: the HBM's rate
        _case("layer norm wide", "layernorm", 8192, 0, 2048, 8, n_micro=2, in_flight=2),
        # a float stage of odd width and ragged length
        _case("layer norm odd fp32", "layernorm", 1003, 0, 77, 13, n_micro=3, in_flight=2, dtype="fp32"),
        # dropout as GNMT is trained with, between its LSTM layers
        _case("dropout gnmt", "dropout", 1024, 0, 50, 64, n_micro=8, in_flight=3, p=0.2),
        # residual dropout of a wide model
        _case("dropout wide", "dropout", 4096, 0, 4096, 8, p=0.1),
        # one row of weights' worth of work: a single token streams both matrices
        _case("gated token", "gated", 2048, 5632, 1, 1),
        # feed-forward block of a large model, 8192 positions
        _case("gated large", "gated", 4096, 11008, 2048, 4, act=SILU),
        # widths that no vector load fits, ragged rows, biases
        _case("gated odd", "gated", 500, 1333, 77, 13, act=GELU, bias=1),
        # a float stage
        _case("gated fp32", "gated", 768, 2048, 128, 8, n_micro=2, in_flight=2, dtype="fp32", act=GELU, bias=1),
        # the whole sublayer: short sequences in many micro-batches, and a large one
        _case("sublayer small", "sublayer", 512, 1408, 64, 2, n_micro=8, in_flight=4, p=0.1),
        _case("sublayer", "sublayer", 2048, 5632, 1024, 4, n_micro=4, in_flight=2, p=0.1),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    flops, nbytes = (max(work(c)[k] for c in listed()) for k in ("flops", "bytes"))
    while True:
        kind = rng.choice(["layernorm", "dropout", "gated", "gated", "sublayer"])
        dtype = "bf16" if kind == "sublayer" else rng.choice(["bf16", "bf16", "bf16", "fp32"])
        case = dict(kind=kind, cin=_log_int(rng, 1, 16384) if kind in ("layernorm", "dropout") else _log_int(rng, 16, 8192),
                    cout=0, seq=_log_int(rng, 1, 4096), micro_batch=_log_int(rng, 1, 64), n_micro=rng.randint(1, 6),
                    in_flight=rng.randint(1, 3), dtype=dtype, act=rng.choice([SIGMOID, SILU, SILU, GELU, RELU]),
                    p=round(rng.uniform(0.02, 0.6), 3) if kind in ("dropout", "sublayer") else 0.0, bias=rng.randint(0, 1))
        if kind in ("gated", "sublayer"):
            case["cout"] = _log_int(rng, 16, 16384)
            # models are built of round widths, mostly; the 1x1 convolution behind a gated layer wants them
            if kind == "sublayer" or rng.random() < 0.75:
                to = rng.choice([8, 16, 64, 128])
                case["cin"], case["cout"] = (max(to, v // to * to) for v in (case["cin"], case["cout"]))
        # a tensor of a stage stays below 2 GiB: here the gated layer's two projections
        if case["micro_batch"] * case["seq"] * max(2 * case["cout"], case["cin"]) * 4 >= 2 ** 31:
            continue
        w = work(case)
        if w["flops"] <= (flops if dtype == "bf16" else flops / 8) and w["bytes"] <= nbytes:
            return case


# ---------------------------------------------------------------------------------------------- inputs
def _torch_dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _shapes(case):
    """Names and shapes of the parameters, in the order of the layers that hold them: weight, bias or None."""
    c, f = case["cin"], case["cout"]
    norm = [("gamma", (c,)), ("beta", (c,))]
    gated = [("w", (2 * f, c))] + ([("b", (2 * f,))] if case["bias"] else [])
    down = [("w2", (c, f))] + ([("b2", (c,))] if case["bias"] else [])
    return {"layernorm": norm, "dropout": [], "gated": gated, "sublayer": norm + gated + down}[case["kind"]]


def _uniform(shape, bound, g):
    return (torch.rand(shape, device="cuda", generator=g) * 2 - 1) * bound


class _Program:
    """What a worker holds: the tensors that its neighbours fill, the parameters (float masters on values that the storage
    type holds) and, where the framework runs, the stage's handle and the tensors that it fills."""

    def __init__(self, case, seed):
        self.handle = None
        self.case = case
        g = torch.Generator("cuda")
        g.manual_seed(int(seed))
        c, dtype = case["cin"], _torch_dtype(case)
        shape = (case["n_micro"], case["micro_batch"], case["seq"], 1, c)
        rows = shape[0] * shape[1] * shape[2]
        # a residual stream: channels of different sizes, a few of them large, and an offset
        size = torch.exp(torch.randn(c, device="cuda", generator=g) * 0.5)
        shift = torch.randn(c, device="cuda", generator=g) * 0.3
        self.x = (torch.randn(shape, device="cuda", generator=g) * size + shift).to(dtype)
        if case["kind"] == "gated":                              # what a norm hands on
            self.x = torch.randn(shape, device="cuda", generator=g).to(dtype)
        out = shape[:-1] + (case["cout"],) if case["kind"] == "gated" else shape
        self.dy = (torch.randn(out, device="cuda", generator=g) / math.sqrt(rows)).to(dtype)
        self.p = np.float32(case["p"])
        self.seed = int(seed) * 0x9E3779B97F4A7C15 % (1 << 64)  # of the masks
        self.mini_batch = 0
        self.params = {}
        for name, s in _shapes(case):
            if name == "gamma":
                v = 1 + 0.2 * torch.randn(s, device="cuda", generator=g)
            elif len(s) == 1:
                v = 0.1 * torch.randn(s, device="cuda", generator=g)
            else:
                v = _uniform(s, math.sqrt(3.0 / s[1]), g)
            self.params[name] = v.to(dtype).float()

    def __del__(self):
        if self.handle is not None:
            self.library.bapipe_stage_destroy(self.handle)
            self.handle = None


def prepare(case, seed):
    s = _Program(case, seed)
    if own:
        _create(s)
    return s


# ---------------------------------------------------------------------------------------------- the framework's calls
def _layer(kind, cin=0, cout=0, k=0, stride=0, bias=0, src0=-1, src1=-1, eps=0.0):
    return dict(kind=kind, cin=cin, cout=cout, kh=k, kw=k, stride=stride, pad=0, has_bias=bias, fuse_relu=0, src0=src0, src1=src1, eps=eps)


def _create(s):
    from paper_2012_12544_amd import binding as B
    case, c, f, p = s.case, s.case["cin"], s.case["cout"], float(s.p)
    s.library = B
    gate = {SIGMOID: B.GATE_SIGMOID, SILU: B.GATE_SILU, GELU: B.GATE_GELU, RELU: B.GATE_RELU}[case["act"]]
    norm = _layer(B.LAYERNORM, c, c, bias=1, eps=EPS)
    gated = dict(_layer(B.GATED, c, f, bias=case["bias"]), kh=gate)
    drop = _layer(B.DROPOUT, eps=p)
    layers = {"layernorm": [norm], "dropout": [drop], "gated": [gated],
              "sublayer": [norm, dict(gated, src0=0), _layer(B.CONV2D, f, c, k=1, stride=1, bias=case["bias"], src0=1),
                           dict(drop, src0=2), _layer(B.ADD, src0=3, src1=-1)]}[case["kind"]]
    stage = dict(dtype=B.BF16 if case["dtype"] == "bf16" else B.FP32, in_c=c, in_h=case["seq"], in_w=1,
                 stage_index=9 - case["in_flight"], n_stages=8, need_input_grad=1)
    s.memory = B.TorchAllocator("cuda:0")
    opts = B.make_opts(stage, io_layout=B.NHWC, stream=torch.cuda.current_stream().cuda_stream, allocator=s.memory)
    M = case["n_micro"]
    s.handle = B.bapipe_stage_create(layers, case["micro_batch"], M, opts)
    # The first block that a stage asks for holds its parameters: the float masters of all layers in order, every vector
    # padded to 256 bytes, then the gradient accumulators in the same order.
    ptr, block = next(iter(s.memory.live.items()))
    with_params = {"layernorm": [0], "dropout": [], "gated": [0], "sublayer": [0, 1, 2]}[case["kind"]]
    names = [n for n, _ in _shapes(case)]
    pairs, s.at, at = [], {}, 0
    for n in names:
        pairs.append([n]) if n in ("gamma", "w", "w2") else pairs[-1].append(n)
        s.at[n] = at
        at += (s.params[n].numel() + 63) // 64 * 64
    for layer, pair in zip(with_params, pairs):
        B.bapipe_stage_set_params(s.handle, layer, s.params[pair[0]].cpu().numpy(), s.params[pair[1]].cpu().numpy() if len(pair) > 1 else None)
    start = ptr - block.data_ptr()
    s.masters = block[start:start + 4 * at].view(torch.float32)
    s.accumulators = block[start + 4 * at:start + 8 * at].view(torch.float32)
    s.y, s.dx = torch.empty_like(s.dy), torch.empty_like(s.x)
    if case["kind"] in ("dropout", "sublayer"):
        B.bapipe_stage_set_dropout(s.handle, s.seed, 0)
    W = min(M, B.bapipe_stage_stash_bytes(s.handle)[1])
    s.order = [("F", m) for m in range(W)]
    for m in range(M - W):
        s.order += [("B", m), ("F", m + W)]
    s.order += [("B", m) for m in range(M - W, M)]


def _run_own(s):
    B = s.library
    for what, m in s.order:
        if what == "F":
            B.bapipe_stage_forward(s.handle, m, s.x[m].data_ptr(), s.y[m].data_ptr())
        else:
            B.bapipe_stage_backward(s.handle, m, s.dy[m].data_ptr(), s.dx[m].data_ptr())
    out = {"y": s.y, "dx": s.dx}
    if s.params:
        grads = s.accumulators.to(_torch_dtype(s.case), copy=True)          # the update clears them
    B.bapipe_stage_step(s.handle, LR)
    for n, v in s.params.items():
        at = s.at[n]
        out["d" + n] = grads[at:at + v.numel()].view(v.shape)
        out[n] = s.masters[at:at + v.numel()].view(v.shape)
    return out


# ---------------------------------------------------------------------------------------------- the plain form
def _keep(case, seed, mini_batch, p, layer):
    """Truth values [M][rows][channels]: the element's word of Philox4x32-10 is not below 2^32 p.  Key: the seed.  Counter:
    element / 4, layer + 65536 (stage - 1), micro-batch, mini-batch; the element's word is its index modulo 4."""
    M, n = case["n_micro"], case["micro_batch"] * case["seq"] * case["cin"]
    low = 0xFFFFFFFF
    c0 = torch.arange((n + 3) // 4, device="cuda", dtype=torch.int64).expand(M, -1)
    c1 = torch.full_like(c0, layer + 65536 * (8 - case["in_flight"]))
    c2 = torch.arange(M, device="cuda", dtype=torch.int64)[:, None].expand_as(c0)
    c3 = torch.full_like(c0, mini_batch)
    k0, k1 = seed & low, seed >> 32
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57                  # modulo 2^64: the bits are those of the unsigned products
        c0, c1, c2, c3 = ((b >> 32) & low) ^ c1 ^ k0, b & low, ((a >> 32) & low) ^ c3 ^ k1, a & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    words = torch.stack([c0, c1, c2, c3], -1).view(M, -1)[:, :n]
    return (words >= min(int(float(p) * 4294967296.0 + 0.5), low)).view(M, -1, case["cin"])


def _activation(act, g):
    """act(g) and its derivative."""
    if act == RELU:
        on = (g > 0).to(g.dtype)
        return g * on, on
    if act == GELU:
        cdf = 0.5 * (1 + torch.erf(g * math.sqrt(0.5)))
        return g * cdf, cdf + g * torch.exp(-0.5 * g * g) * (1 / math.sqrt(2 * math.pi))
    sig = 1 / (1 + torch.exp(-g))
    if act == SIGMOID:
        return sig, sig * (1 - sig)
    return g * sig, sig * (1 + g * (1 - sig))


def _run_plain(s):
    case, P, dtype = s.case, s.params, _torch_dtype(s.case)
    kind, c = case["kind"], case["cin"]
    x, dy = s.x.float().view(case["n_micro"], -1, c), s.dy.float()
    d = dy.view(case["n_micro"], -1, dy.shape[-1])
    used = {n: v.to(dtype).float() if v.dim() > 1 else v for n, v in P.items()}
    grads = {}
    keep, scale = None, float(np.float32(1.0 / (1.0 - float(s.p))))
    if kind in ("dropout", "sublayer"):
        keep = _keep(case, s.seed, s.mini_batch, s.p, 0 if kind == "dropout" else 3)
    # forward
    h = x
    if kind in ("layernorm", "sublayer"):
        centred = x - x.mean(-1, keepdim=True)
        r = torch.rsqrt((centred * centred).mean(-1, keepdim=True) + EPS)
        xhat = centred * r
        h = xhat * used["gamma"] + used["beta"]
    if kind in ("gated", "sublayer"):
        rows = h.reshape(-1, c)
        both = rows @ used["w"].t()
        if case["bias"]:
            both = both + used["b"]
        g, u = both[:, :case["cout"]], both[:, case["cout"]:]
        a, da = _activation(case["act"], g)
        h = a * u
    if kind == "sublayer":
        hidden = h
        h = hidden @ used["w2"].t()
        if case["bias"]:
            h = h + used["b2"]
        h = h.view(x.shape)
    if keep is not None:
        h = torch.where(keep, h * scale, torch.zeros_like(h))
    if kind == "sublayer":
        h = x + h
    y = h.to(dtype).view(s.dy.shape)
    # backward
    if keep is not None:
        d = torch.where(keep, d * scale, torch.zeros_like(d))
    if kind == "sublayer":
        d = d.reshape(-1, c)
        grads["w2"] = d.t() @ hidden
        if case["bias"]:
            grads["b2"] = d.sum(0)
        d = d @ used["w2"]
    if kind in ("gated", "sublayer"):
        d = d.reshape(-1, case["cout"])
        d = torch.cat([d * u * da, d * a], 1)
        grads["w"] = d.t() @ rows
        if case["bias"]:
            grads["b"] = d.sum(0)
        d = (d @ used["w"]).view(x.shape)
    if kind in ("layernorm", "sublayer"):
        grads["gamma"], grads["beta"] = (d * xhat).sum((0, 1)), d.sum((0, 1))
        d = d * used["gamma"]
        d = r * (d - d.mean(-1, keepdim=True) - xhat * (d * xhat).mean(-1, keepdim=True))
    if kind == "sublayer":
        d = d + dy.view(x.shape)
    out = {"y": y, "dx": d.to(dtype).view(s.x.shape)}
    # the update
    for n, v in P.items():
        out["d" + n] = grads[n].to(dtype)
        out[n] = v.sub_(grads[n], alpha=LR)
    s.mini_batch += 1
    return out


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---------------------------------------------------------------------------------------------- work and exact values
def work(case):
    """Multiply-adds of the products (forward, input gradient, weight gradient), and the boundary tensors and parameters, each
    once: x, y, dy, dx; masters read and written, gradients written."""
    c, f, es = case["cin"], case["cout"], 2 if case["dtype"] == "bf16" else 4
    rows = case["n_micro"] * case["micro_batch"] * case["seq"]
    out = f if case["kind"] == "gated" else c
    weights = {"gated": 2, "sublayer": 3}.get(case["kind"], 0) * c * f
    params = sum(math.prod(s) for _, s in _shapes(case))
    return {"bytes": 2 * rows * (c + out) * es + params * (8 + es), "flops": 6 * rows * weights + (20 * rows * c if not weights else 0)}


def _bits(case, seed, p, layer):
    """The mask of the first mini-batch, with products of 32-bit words put together from halves."""
    M, n = case["n_micro"], case["micro_batch"] * case["seq"] * case["cin"]
    half, low = 0xFFFF, 0xFFFFFFFF

    def product(v, m):
        lo, hi = (v & half) * m, (v >> 16) * m                  # below 2^48
        total = hi + (lo >> 16)
        return (total >> 16) & low, ((total & half) << 16) | (lo & half)

    def rounds(at, micro):
        c = [at, torch.full_like(at, layer + 65536 * (8 - case["in_flight"])), torch.full_like(at, micro), torch.zeros_like(at)]
        for r in range(10):
            (h0, l0), (h2, l2) = product(c[0], 0xD2511F53), product(c[2], 0xCD9E8D57)
            key = ((seed & low) + r * 0x9E3779B9) & low, ((seed >> 32) + r * 0xBB67AE85) & low
            c = [h2 ^ c[1] ^ key[0], l2, h0 ^ c[3] ^ key[1], l0]
        return torch.stack(c, 1).reshape(-1)

    at = torch.arange(-(-n // 4), device="cuda")
    words = torch.stack([rounds(at, m)[:n] for m in range(M)])
    return words.double() / 2.0 ** 32 >= min(round(float(p) * 2.0 ** 32), low) / 2.0 ** 32


def exact(case, seed):
    if work(case)["flops"] > 5e12:
        return None
    s = _Program({**case}, seed)
    x = s.x.double().requires_grad_()
    P = {n: v.double().requires_grad_() for n, v in s.params.items()}
    F = torch.nn.functional
    h, kind, f = x, case["kind"], case["cout"]
    if kind in ("layernorm", "sublayer"):
        h = F.layer_norm(h, (case["cin"],), P["gamma"], P["beta"], EPS)
    if kind in ("gated", "sublayer"):
        act = {SIGMOID: torch.sigmoid, SILU: F.silu, GELU: F.gelu, RELU: F.relu}[case["act"]]
        bias = P["b"] if case["bias"] else torch.zeros(2 * f, device="cuda", dtype=torch.float64)
        h = act(F.linear(h, P["w"][:f], bias[:f])) * F.linear(h, P["w"][f:], bias[f:])
    if kind == "sublayer":
        h = F.linear(h, P["w2"], P["b2"] if case["bias"] else None)
    if kind in ("dropout", "sublayer"):
        h = h * _bits(case, s.seed, s.p, 0 if kind == "dropout" else 3).view(x.shape) / (1.0 - float(s.p))
    if kind == "sublayer":
        h = h + x
    given = torch.autograd.grad(h, [x] + list(P.values()), s.dy.double())
    out = {"y": h.detach(), "dx": given[0]}
    for (n, v), g in zip(P.items(), given[1:]):
        out["d" + n] = g
        out[n] = v.detach() - LR * g
    return out
