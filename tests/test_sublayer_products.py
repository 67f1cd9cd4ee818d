"""What layer norm, gated layer and dropout refuse, and their products, asked without a GPU: nothing is launched."""
import ctypes as ct

import pytest

from paper_2012_12544_amd import binding as B
from stage_inputs import configs as C
from test_oracle_sublayer import _status

SOMEWHERE = ct.c_void_p(1 << 40)          # an address; nothing is read or written there
INVALID = 1                               # hipErrorInvalidValue


def test_the_projections_gradients_are_not_made_from_a_filter_in_panels():
    f = B.load()._ZN6bapipe13gated_projectEiPKvS1_bPKfPvS4_iiiP12ihipStream_t
    args = [SOMEWHERE, SOMEWHERE, ct.c_bool(True), SOMEWHERE, SOMEWHERE, None, ct.c_int(2060), ct.c_int(64), ct.c_int(1600), None]
    assert f(ct.c_int(0), *args) == INVALID


class _GatherConv(ct.Structure):
    _fields_ = [(f, ct.c_int) for f in "N Hi Wi Ci Ho Wo Co R S s_out s_in pad_h pad_w beside by_norm wt_panels".split()]


def _rows(rows, ci, co, beside=0, panels=0):
    return _GatherConv(rows, 1, 1, ci, 1, 1, co, 1, 1, 1, 1, 0, 0, beside, 0, panels)


def _parts(g):
    """Float sums of a product whose result is left as such."""
    f = B.load()._ZN6bapipe30conv_gather_mfma_raw_workspaceERKNS_10GatherConvE
    f.restype = ct.c_size_t
    n = f(ct.byref(g))
    assert n % (g.N * g.Co * 4) == 0
    return n // (g.N * g.Co * 4)


def test_float_sums_are_as_many_on_every_stream_and_from_every_layout():
    """Their number is asked for when a stage is created, without further streams and before the filters' layout is known."""
    split = 0
    for rows in (1, 8, 33, 64, 65, 200, 500, 1000, 2048, 4096, 16384, 40000):
        for ci, co in ((64, 64), (512, 64), (1024, 256), (2816, 512), (512, 1024), (4096, 4096), (6144, 2048), (11264, 2048), (22016, 4096), (28288, 64)):
            n = {_parts(_rows(rows, ci, co, beside, panels)) for beside in (0, 1) for panels in (0, 1)}
            assert len(n) == 1, (rows, ci, co, n)
            split += max(n) > 1
    assert split >= 10                        # otherwise nothing was asked


def test_another_number_of_float_sums_than_there_is_room_for_is_refused():
    f = B.load()._ZN6bapipe20conv_gather_mfma_rawEPKvS1_RKNS_10GatherConvEPfPiP12ihipStream_ti
    g, splits = _rows(64, 22016, 4096), ct.c_int()
    n = _parts(g)
    assert n > 1
    for expected in (1, n - 1, n + 1):
        assert f(SOMEWHERE, SOMEWHERE, ct.byref(g), SOMEWHERE, ct.byref(splits), None, ct.c_int(expected)) == (0 if expected == n else INVALID)


@pytest.mark.parametrize("method,args", [("layernorm", (32,)), ("gated", (32, 8)), ("dropout", (0.5,))])
@pytest.mark.parametrize("between", ["relu", "sum", "norm", "relu, sum"])
def test_what_is_made_of_a_flattened_map_element_by_element_is_refused(method, args, between):
    """Its elements still lie in the map's order; behind a LINEAR layer they are in order again."""
    def layers(flattened, linear=False):
        b = C._Builder()
        c = 8 if flattened else 32
        t = b.dropout(0.1, src=-1) if flattened else b.layernorm(c, src=-1)
        t = b.flatten(src=t)
        if "relu" in between:
            t = b.relu(src=t)
        if "sum" in between:
            t = b.addl(b.linear(32, 32, src=t), t, relu=0)
        if between == "norm":
            t = b.bn(32, src=t)
        if linear:
            b.linear(32, 32, src=t)
        getattr(b, method)(*args)
        return b.layers

    assert _status(layers(True), shape=(8, 4, 1)) == B.E_UNSUPPORTED
    assert _status(layers(True, linear=True), shape=(8, 4, 1)) == B.E_OOM
    assert _status(layers(False), shape=(32, 1, 1)) == B.E_OOM
