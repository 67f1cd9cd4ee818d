"""What the products of layer norm and gated layer refuse, asked without a GPU: nothing is launched."""
import ctypes as ct

from paper_2012_12544_amd import binding as B

SOMEWHERE = ct.c_void_p(1 << 40)          # an address; nothing is read or written there
INVALID = 1                               # hipErrorInvalidValue


def test_the_projections_gradients_are_not_made_from_a_filter_in_panels():
    f = B.load()._ZN6bapipe13gated_projectEiPKvS1_bPKfPvS4_iiiP12ihipStream_t
    args = [SOMEWHERE, SOMEWHERE, ct.c_bool(True), SOMEWHERE, SOMEWHERE, None, ct.c_int(2060), ct.c_int(64), ct.c_int(1600), None]
    assert f(ct.c_int(0), *args) == INVALID
