"""What the head's operators take and refuse, without a GPU: the library's checks come before any launch."""
import copy
import ctypes as C
import pickle

import pytest
import torch

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


def test_an_8_bit_form_follows_its_tensors():
    """What a call sees of a Packed8 are the tensors that it holds then, also after they were replaced or moved."""
    p = G.Packed8(6, 70, torch.bfloat16, "cpu")
    p.q = torch.zeros(6, 96, dtype=torch.int8)[:, 5:85]
    p.exps = torch.zeros(6, 9, dtype=torch.uint8)[:, :4]
    m = G.binding._mat(p, "q")
    assert (m.data, m.exps) == (p.q.data_ptr(), p.exps.data_ptr())
    assert (m.rows, m.cols, m.ld, m.ld_exps, m.type, m.packed) == (6, 70, 96, 9, G.GOSH_BF16, 1)
    one = G.Packed8(1, 33, torch.float16, "cpu")  # the stride of a single row says nothing
    one.q, one.exps = torch.zeros(33, 1, dtype=torch.int8).t(), torch.zeros(2, 1, dtype=torch.uint8).t()
    m = G.binding._mat(one, "q")
    assert m.ld >= 33 and m.ld_exps >= 2


@pytest.mark.parametrize("q, exps", [
    ((6, 69), (6, 3)), ((6, 70), (6, 2)), ((5, 70), (6, 3)), ((6, 70), (7, 3)), ((420,), (6, 3)), ((6, 70), (18,)),
])
def test_an_8_bit_form_of_another_shape(q, exps):
    p = G.Packed8(6, 70, torch.float32, "cpu")
    p.q, p.exps = torch.zeros(q, dtype=torch.int8), torch.zeros(exps, dtype=torch.uint8)
    with pytest.raises(TypeError, match="rows of at least"):
        G.binding._mat(p, "q")


def test_an_8_bit_form_of_other_types_or_strides():
    p = G.Packed8(6, 70, torch.float32, "cpu")
    p.q = p.q.view(torch.uint8)
    with pytest.raises(TypeError, match="int8"):
        G.binding._mat(p, "q")
    p.q = torch.zeros(70, 6, dtype=torch.int8).t()
    with pytest.raises(TypeError, match="contiguous"):
        G.binding._mat(p, "q")


def test_an_8_bit_form_is_copied_and_pickled():
    p = G.Packed8(3, 40, torch.float16, "cpu")
    p.q.fill_(5), p.exps.fill_(7)
    for c in (copy.deepcopy(p), pickle.loads(pickle.dumps(p))):
        assert torch.equal(c.q, p.q) and torch.equal(c.exps, p.exps) and (c.rows, c.cols, c.dtype) == (3, 40, torch.float16)
        assert G.binding._mat(c, "q").data == c.q.data_ptr() != p.q.data_ptr()


def test_workspaces_of_what_is_refused():
    """Sizes, types and activations that a call refuses have no workspace, however large: nothing overflows."""
    most = 2 ** 31 - 2
    for rows in (-1, most + 1, 2 ** 62, 2 ** 63 - 1):
        assert G.gosh_layer_norm_workspace(rows, 64) == 0
        assert G.gosh_linear_backward_workspace(rows, 64, 64, G.GOSH_BF16, H.GELU) == 0
    for type_, act in ((-1, H.NONE), (3, H.NONE), (G.GOSH_F32, -1), (G.GOSH_F32, 4)):
        assert G.gosh_linear_backward_workspace(10, 64, 64, type_, act) == 0
    assert G.gosh_layer_norm_workspace(most, 65536) == 1024 * 2 * 65536 * 4
    assert G.gosh_linear_backward_workspace(most, 65536, 65536, G.GOSH_F32, H.SILU) > most * 65536 * 4 + 65536 * 65536 * 4
