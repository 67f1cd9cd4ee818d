"""The workspace of layer norm and gated layer, asked without a GPU: tests/launch_recorder.c takes the place of the runtime."""
import ctypes as ct
import json
import os
import shutil
import subprocess
import sys

import pytest

import test_launches
from paper_2012_12544_amd import binding as B

HERE = os.path.dirname(os.path.abspath(__file__))
STATIC = 64 << 20


def _record(recorder, library, cases):
    """In a process of its own: test_launches' record of a mini-batch, and (first byte, bytes) of the partial sums of every reduction."""
    out = []
    for case in cases:
        got, = test_launches._record(recorder, library, [case])
        rec, parts = ct.CDLL(recorder), []
        for i in range(rec.recorder_count()):
            first, nbytes = ct.c_size_t(), ct.c_size_t()
            rec.recorder_get(i, ct.byref(first), ct.byref(nbytes))
            parts.append((first.value, nbytes.value))
        out.append(dict(got, parts=parts))
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


def _case(layers, c, rows, streams=1, static=False, n_micro=1):
    first = layers[0]
    return dict(call="mini_batch", layers=[(first[0], [first[1][0], dict(first[1][1], src=-1)])] + layers[1:], input=[c, rows, 1], micro_batch=1,
                n_micro=n_micro, in_flight=n_micro, streams=streams, static=static)


def _gated(c, units):
    return [("gated", [[c, units], {}])]


def _sublayer(c, units):
    return [("layernorm", [[c], {}])] + _gated(c, units) + [("conv", [[units, c, 1], {}]), ("dropout", [[0.1], {}])]


def _layernorm_partials(got, c):
    """Bytes of the column sums that the blocks of the backward pass leave; a lone block adds its own."""
    grids = [(name, grid) for name, _, grid, *_ in got["launches"]]
    blocks = [grid[1] if name == "k_layernorm_columns" else grid[0] if grid[0] > 1 else 0 for name, grid in grids if name in ("k_layernorm_bwd", "k_layernorm_columns")]
    assert len(blocks) == 1, grids
    return blocks[0] * 8 * c


@pytest.mark.parametrize("c", [8, 100, 512, 1024, 3000, 8192, 12000, 16384, 16385, 20000, 33000])
def test_layer_norm_asks_for_the_sums_that_its_blocks_leave(record, c):
    cases = [_case([("layernorm", [[c], {}])], c, rows, streams=streams) for rows in (1, 40, 64, 65, 500, 512, 4096, 16384, 20000) for streams in (1, 3)]
    for case, got in zip(cases, record(cases)):
        need, room = _layernorm_partials(got, c), got["blocks"][4][1]
        assert need <= room <= max(need, 256), (case, need, room)


@pytest.mark.parametrize("layers,c,rows", [
    (_gated(4096, 11008), 4096, 8192), (_sublayer(4096, 11008), 4096, 8192), (_sublayer(2048, 5632), 2048, 4096),
    ([("layernorm", [[20000], {}])], 20000, 4096), ([("layernorm", [[33000], {}])], 33000, 12000),
])
def test_large_stages_run_on_the_static_workspace(record, layers, c, rows):
    """They split no product that would leave partial sums of more than it holds."""
    got, = record([_case(layers, c, rows, static=True)])
    assert got["rc"] == 0 and got["blocks"][4][1] <= STATIC


def test_a_stage_whose_split_product_needs_more_is_refused(record):
    """dw of 8192 x 1024 from 16384 rows is formed in two splits of 33.6 MB."""
    layers, c, rows = _gated(1024, 4096), 1024, 16384
    got, = record([_case(layers, c, rows)])
    assert got["blocks"][4][1] == 2 * 4 * (8192 * 1024 + 8192) > STATIC
    with pytest.raises(AssertionError, match="E_UNSUPPORTED: backward_static"):
        record([_case(layers, c, rows, static=True)])


@pytest.mark.parametrize("streams", [1, 3])
def test_partial_sums_stay_in_the_workspace(record, streams):
    """Of weight gradients on their own plan, of those that share launches, and of products of any sizes."""
    cases = [_case(make(c, units), c, rows, streams=streams, n_micro=2)
             for make in (_gated, _sublayer) for c, units in ((64, 128), (128, 1600), (512, 1408), (1024, 4096), (2048, 5632))
             for rows in (1, 33, 130, 1024, 4096)]
    asked = 0
    for case, got in zip(cases, record(cases)):
        work = [got["blocks"][4]] + [b for b in got["blocks"][6:] if b[1] == got["blocks"][4][1]]
        for first, nbytes in got["parts"]:
            assert any(at <= first and first + nbytes <= at + n for at, n in work), (case, first, nbytes, got["blocks"])
            asked += 1
    assert asked >= 20


if __name__ == "__main__":
    print(json.dumps(_record(sys.argv[1], sys.argv[2], json.load(sys.stdin))))
