"""Calls of layer norm, gated layer and dropout beyond those of test_gpu_sublayer.py."""
import numpy as np
import pytest

from gpu_harness import GpuStage, compare_minibatch, stage_io
from paper_2012_12544_amd import binding as B
from stage_inputs import configs as C
from stage_inputs import gen
from test_gpu_sublayer import _rows
from test_oracle_sublayer import sublayer

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------ positions folded into the batch
MANY = [dict(c=64, units=1600, micro_batch=2060), dict(c=96, units=1608, micro_batch=2050, act=C.GATE_GELU),
        dict(c=32, units=1600, micro_batch=2060, bias=0),       # one panel: the same order as rows
        dict(c=40, units=1608, micro_batch=2050),               # no panels
        dict(c=128, units=3200, micro_batch=1000, act=C.GATE_SIGMOID), dict(c=64, units=1604, micro_batch=2060)]


@pytest.mark.parametrize("kw", MANY)
def test_sublayer_of_many_maps_of_one_pixel(kw):
    """A 1x1 convolution of single pixels keeps its filters in panels, which the products that fill the chip meet as well."""
    compare_minibatch(sublayer(seq=1, n_micro=1, stage_index=1, n_stages=1, **kw))


@pytest.mark.parametrize("kw", MANY)
def test_positions_in_the_batch_or_in_a_sequence_are_the_same(kw):
    """(C, 1, 1) x rows and (C, rows, 1) x 1 are the same elements in the same order: two mini-batches, with the update between them."""
    rows = kw["micro_batch"]
    folded = sublayer(seq=1, n_micro=2, stage_index=1, n_stages=1, **kw)
    along = sublayer(seq=rows, n_micro=2, stage_index=1, n_stages=1, **dict(kw, micro_batch=1))
    params = gen.all_params(folded, perturb=True)
    xs, gs = stage_io(folded)
    out = []
    for st in (folded, along):
        to = lambda a: np.ascontiguousarray(a if st is folded else a[:, :, 0, 0].T[None, :, :, None])  # noqa: E731
        g, got = GpuStage(st, params), []
        for _ in range(2):
            for m in range(2):
                got += [_rows(g.forward(m, to(xs[m]))), _rows(g.backward(m, to(gs[m])))]
            got += [a for i, (w, _) in enumerate(params) if w is not None for a in g.grads(i) if a is not None]
            B.bapipe_stage_step(g.h, 0.05)
        g.close()
        out.append(got)
    for a, b in zip(*out):
        assert np.array_equal(a, b) and np.any(a)
