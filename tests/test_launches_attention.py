"""What rotary positions and attention launch and keep, asked without a GPU: tests/launch_recorder.c takes the place of the runtime."""
import ctypes as ct
import json
import os
import re
import shutil
import subprocess
import sys

import pytest

from oracle.stage import one_f_one_b_order
from paper_2012_12544_amd import binding as B
from stage_inputs import configs as C
from test_launches import SOMEWHERE, STREAMS

HERE = os.path.dirname(os.path.abspath(__file__))


def _record(recorder, library, cases):
    """In a process of its own, for each case: bytes of a micro-batch in flight, the blocks that the stage asked its allocator for, the status
    of the pass that refused, and (kernel, integers among its template arguments, blocks) of every launch of a mini-batch."""
    rec = ct.CDLL(recorder, mode=ct.RTLD_GLOBAL)
    rec.recorder_launch.restype = ct.c_char_p
    B.LIB_PATH = library
    out = []
    for case in cases:
        blocks = []

        def alloc(nbytes, ctx):
            blocks.append((SOMEWHERE + (sum(n for _, n in blocks) + 4095) // 4096 * 4096 + 4096 * len(blocks), nbytes))
            return blocks[-1][0]

        b = C._Builder()
        for kind, args, kw in case["layers"]:
            getattr(b, kind)(*args, **kw)
        st = C._stage("recorded", b.layers, case["dtype"], tuple(case["input"]), case["micro_batch"], 1, 1, 1, 1, 0, "xavier")
        o = B.make_opts(st, io_layout=B.NHWC, stream=STREAMS["own"])
        o.mem.alloc, o.mem.free = B.ALLOC_FN(alloc), B.FREE_FN(lambda ptr, ctx: None)
        h = B.bapipe_stage_create(b.layers, case["micro_batch"], 1, o)
        rec.recorder_clear()
        status = 0
        backward = B.bapipe_stage_backward_static if case.get("static") else B.bapipe_stage_backward
        try:
            for what, m in one_f_one_b_order(1, 1):
                if what == "F":
                    if any(L["kind"] == C.ATTENTION and L["stride"] == C.MASK_SPANS for L in b.layers):
                        B.bapipe_stage_set_spans(h, m, SOMEWHERE >> 5)
                    B.bapipe_stage_forward(h, m, SOMEWHERE >> 1, SOMEWHERE >> 2)
                else:
                    backward(h, m, SOMEWHERE >> 3, (SOMEWHERE >> 4) + case.get("dx", 0))
        except B.BapipeError as e:
            status = e.status
        launches = []
        for i in range(rec.recorder_launches()):
            grid, stream, tickets, lds = (ct.c_uint * 3)(), ct.c_size_t(), ct.c_size_t(), ct.c_size_t()
            name = rec.recorder_launch(i, grid, ct.byref(stream), ct.byref(tickets), ct.byref(lds)).decode()
            m = re.search(r"\d(k_attention_[a-z]+|k_rotary(?:_[a-z]+)?)", name)
            if m:
                launches.append((m.group(1), [int(a) for a in re.findall(r"L[ib](\d+)E", name[m.end():])], list(grid)))
        out.append(dict(per_micro_batch=B.bapipe_stage_stash_bytes(h)[0], blocks=blocks, status=status, launches=launches))
        B.bapipe_stage_destroy(h)
    return out


@pytest.fixture(scope="module")
def record(tmp_path_factory):
    if shutil.which("gcc") is None:
        pytest.skip("needs gcc")
    B.load()
    so = str(tmp_path_factory.mktemp("recorder") / "recorder.so")
    subprocess.check_call(["gcc", "-O1", "-std=c11", "-shared", "-fPIC", "-Wall", "-o", so, os.path.join(HERE, "launch_recorder.c")])

    def run(cases):
        r = subprocess.run([sys.executable, os.path.abspath(__file__), so, B.LIB_PATH], input=json.dumps(cases), capture_output=True, text=True, timeout=120,
                           env=dict(os.environ, PYTHONPATH=os.pathsep.join([os.path.dirname(HERE), HERE])))
        assert r.returncode == 0, r.stderr[-2000:]
        return json.loads(r.stdout)
    return run


def _case(layers, dtype, c, seq, micro_batch=1, static=False):
    layers = [(layers[0][0], layers[0][1], dict(layers[0][2], src=-1))] + layers[1:]
    return dict(layers=layers, dtype=dtype, input=[c, seq, 1], micro_batch=micro_batch, static=static)


# Integers among the template arguments: of the attention kernels DP, VEC, EXTRA, HALF, KS, of k_rotary V, C, L, K, PAIRS, NORM, BACK, FLOATS
ATTENTION = ("k_attention_fwd", "k_attention_dq", "k_attention_dkv")
HALF, ROTARY_LANES, ROTARY_HEADS, ROTARY_FLOATS = 3, 2, 3, 7


def _up(n):
    return (n + 255) // 256 * 256


@pytest.mark.parametrize("norm", [0, 1])
@pytest.mark.parametrize("dtype", [C.FP32, C.BF16])
@pytest.mark.parametrize("heads,groups,d", [(12, 2, 64), (4, 2, 128), (2, 1, 256), (14, 1, 64)])
def test_an_attention_of_other_heads_than_the_rotary_in_front(record, dtype, norm, heads, groups, d):
    """Both divide 1024 channels, the ROTARY into 8 / 4 heads of 64.  Nothing of one's layout is handed to the other: all channels are stored in
    the storage type, and the gradients come back in it."""
    rows, es = 2 * 40, 4 if dtype == C.FP32 else 2

    def case(h, g, w):
        return _case([("rotary", [8, 4, 64], dict(norm=norm)), ("attention", [h, g, w], {})], dtype, 1024, 40, micro_batch=2)

    same, other = record([case(8, 4, 64), case(heads, groups, d)])
    at = {name: (args, grid) for name, args, grid in other["launches"]}
    assert all(at[name][0][HALF] == 0 for name in ATTENTION), other["launches"]
    turns = [(args, grid) for name, args, grid in other["launches"] if name == "k_rotary"]
    assert len(turns) == 2 and turns[0][0][ROTARY_FLOATS] == turns[1][0][ROTARY_FLOATS] == 0
    for args, grid in turns:                                 # value heads too, a head to a group of lanes (few rows)
        assert args[ROTARY_HEADS] == 1 and grid[0] == -(-rows * 16 // (256 // args[ROTARY_LANES])), turns
    out = rows * heads * d
    kept = _up(rows * 1024 * es) * (1 + norm) + _up(out * es) + _up(2 * heads * 40 * 4) + (_up(out) if dtype == C.BF16 else 0)
    assert other["per_micro_batch"] == kept
    # of the same heads: 16-bit floats in a bf16 stage
    assert all(args[HALF] == (dtype == C.BF16) for name, args, _ in same["launches"] if name in ATTENTION)


@pytest.mark.parametrize("d", [12, 20, 100, 8, 64])
@pytest.mark.parametrize("dx", [0, 2, 4, 8])
def test_the_sums_of_all_splits_are_stored_in_no_wider_pieces_than_dx_allows(record, d, dx):
    """Heads of 12, 20 or 100 bf16 are no whole number of 16 bytes, so dx may lie at any element: four of them at once only where that is a
    multiple of 8 bytes.  (dx of the others passes through the stage's own tensor.)"""
    case = _case([("attention", [4, 1, d], {})], C.BF16, 6 * d, 1100)
    got, = record([dict(case, dx=dx)])
    join, = [args for name, args, _ in got["launches"] if name == "k_attention_join"]
    assert join == [1 if d % 8 and dx % 8 else 4]


def _blocks_a_unit(bf16, d, extra):
    """Of k_attention_dkv, by its launch bounds; float heads of up to 64 channels fit twice by their registers."""
    if not bf16:
        return 2 if d <= 64 else 1
    extra = extra or d % 8 != 0                              # element by element there is one kernel, which knows caps and slopes
    width = next(w for w in ((64, 128, 256) if d % 8 else (32, 64, 96, 128, 192, 256)) if d <= w)
    return 2 if 2 * width <= (192 if extra else 256) else 1


@pytest.mark.parametrize("dtype", [C.FP32, C.BF16])
@pytest.mark.parametrize("rotary", [0, 1])
@pytest.mark.parametrize("bias", [0, 8])
def test_parts_of_the_keys_sums_are_no_more_than_fit_beside_each_other(record, dtype, rotary, bias):
    """Without a mask all blocks take the same time: those that start in a second round leave the units idle behind it.  The blocks of heads that
    are taken in two halves of their columns count twice, and so do those of two waves to 32 rows."""
    cases = []
    for d in (30, 64, 80, 96, 100, 104, 128, 160, 192, 200, 208, 256):
        for heads, groups, seq, micro_batch in ((8, 1, 2048, 1), (4, 2, 1024, 2), (12, 12, 700, 1), (16, 2, 520, 3)):
            layers = [("rotary", [heads, groups, d], {})] * rotary + [("attention", [heads, groups, d, C.MASK_NONE, 0.0, bias], {})]
            cases.append((d, _case(layers, dtype, (heads + 2 * groups) * d, seq, micro_batch)))
    parts = 0
    for (d, case), got in zip(cases, record([c for _, c in cases])):
        (args, grid), = [(args, grid) for name, args, grid in got["launches"] if name == "k_attention_dkv"]
        if not any(name == "k_attention_join" for name, *_ in got["launches"]):
            continue
        parts += 1
        assert grid[0] <= 256 * _blocks_a_unit(dtype == C.BF16, d, bias), (case, args, grid)
    assert parts >= 20


def test_wide_heads_behind_a_rotary_run_on_the_static_workspace(record):
    """Their columns are taken in halves, so eight parts of the keys' sums fill the units: 32 MiB."""
    case = _case([("rotary", [8, 1, 256], {}), ("attention", [8, 1, 256, C.MASK_NONE], {})], C.BF16, 2560, 2048, static=True)
    got, = record([case])
    assert got["status"] == 0 and 32 << 20 <= got["blocks"][4][1] < 33 << 20


def test_launches_stay_below_two_to_the_32_threads(record):
    """The most heads of one channel that 2 GiB hold, each for itself; many short sequences, as many blocks as an attention is taken with."""
    cases = [_case([("rotary", [32767, 1, 1], {})], C.BF16, 32769, 1, micro_batch=32767),
             _case([("attention", [256, 1, 4], {})], C.BF16, 1032, 1, micro_batch=65535)]
    for case, got in zip(cases, record(cases)):
        assert got["status"] == 0 and len(got["launches"]) >= 2
        assert all(256 * grid[0] < 1 << 32 for _, _, grid in got["launches"]), got["launches"]


if __name__ == "__main__":
    print(json.dumps(_record(sys.argv[1], sys.argv[2], json.load(sys.stdin))))
