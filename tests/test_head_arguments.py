"""What the head's operators take and refuse, without a GPU: the library's checks come before any launch."""
import ctypes as C

import pytest

import paper_2008_12336_amd as G
from tests import head_model as H
from tests.test_head_host import mat, refused


@pytest.mark.parametrize("x, w", [(True, True), (True, False), (False, True), (False, False)])
@pytest.mark.parametrize("act", [H.NONE, H.GELU])
def test_the_bias_gradient_alone(x, w, act):
    """x and w may be given where only db is asked for, whatever their columns: the call gets as far as db's memory."""
    lib = G.lib()
    dy, z = mat(cols=8), mat(cols=8)
    xs, ws = mat(cols=16), mat(rows=8, cols=16, data=0x1000)
    args = [C.byref(dy), C.byref(xs) if x else None, C.byref(ws) if w else None, C.byref(z) if act else None, act, None, None, 0x2000,
            None, 0, None]
    text = "w is not memory" if w else "db is not memory"
    refused(lib.gosh_linear_backward(*args), text)
    if x:
        args[2] = C.byref(mat(cols=15))
        refused(lib.gosh_linear_backward(*args), "w is 0 x 15: must be 8 x 16")
