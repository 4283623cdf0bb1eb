"""The head's operators without a GPU: refusals that need no device, sizes of workspaces, and the gradients that the
GPU tests compare with, against differences."""
import ctypes as C

import pytest
import torch

import paper_2008_12336_amd as G
from tests import head_model as H


def mat(rows=0, cols=8, ld=None, type_=G.GOSH_F32, packed=0, data=None, exps=None, ld_exps=1):
    return G.gosh_mat(data, exps, rows, cols if ld is None else ld, ld_exps, cols, type_, packed)


def refused(rc, text):
    assert rc == -1
    assert text in G.gosh_last_error(), G.gosh_last_error()


@pytest.mark.parametrize("bad, text", [
    (dict(type_=3), "gosh_type"), (dict(type_=-1), "gosh_type"), (dict(packed=2), "packed"), (dict(rows=-1), "rows"),
    (dict(rows=2 ** 31 - 1), "rows"), (dict(cols=0), "cols"), (dict(cols=65537), "cols"), (dict(ld=7), "ld"),
    (dict(ld=G.GOSH_MAT_MAX_LD + 1), "ld"), (dict(rows=1), "data is null"), (dict(rows=1, data=0x1002), "aligned"),
    (dict(packed=1), "must not be packed"),
])
def test_a_matrix_that_is_none(bad, text):
    lib = G.lib()
    fine = mat()
    refused(lib.gosh_linear(C.byref(mat(**bad)), C.byref(fine), None, 0, None, C.byref(fine), None, None, None), text)
    refused(lib.gosh_layer_norm(C.byref(mat(**bad)), None, None, 1e-5, C.byref(fine), None, None, None, None, None), text)
    refused(lib.gosh_layer_norm_backward(C.byref(mat(**bad)), C.byref(fine), None, None, None, None, None, None, None, None, 0, None), text)
    refused(lib.gosh_linear_backward(C.byref(mat(**bad)), C.byref(fine), None, None, 0, None, None, None, None, 0, None), text)
    refused(lib.gosh_pack8(C.byref(mat(**bad)), C.byref(fine), None), text)


def test_null_and_unpacked():
    lib = G.lib()
    m = mat()
    refused(lib.gosh_linear(None, C.byref(m), None, 0, None, C.byref(m), None, None, None), "x is null")
    refused(lib.gosh_linear(C.byref(m), None, None, 0, None, C.byref(m), None, None, None), "w is null")
    refused(lib.gosh_pack8(C.byref(m), C.byref(m), None), "q must be packed")
    refused(lib.gosh_unpack8(None, C.byref(m), None), "q is null")
    refused(lib.gosh_layer_norm(C.byref(m), None, None, 1e-5, C.byref(m), None, None, C.byref(m), None, None), "xhat8 must be packed")
    refused(lib.gosh_layer_norm(C.byref(m), None, None, float("nan"), C.byref(m), None, None, None, None, None), "eps")
    refused(lib.gosh_layer_norm(C.byref(m), None, None, 1e-5, C.byref(m), None, None, None, None, None), "gamma is null")
    refused(lib.gosh_linear(C.byref(m), C.byref(m), None, 0, None, C.byref(m), None, None, None), "w: rows")
    q = mat(rows=1, cols=40, packed=1, data=0x1000, exps=None)
    refused(lib.gosh_unpack8(C.byref(q), C.byref(mat(cols=40)), None), "q")


def test_workspaces():
    assert G.gosh_layer_norm_workspace(0, 64) == 0 and G.gosh_layer_norm_workspace(10, 0) == 0
    assert G.gosh_layer_norm_workspace(1, 64) == 2 * 64 * 4
    assert G.gosh_layer_norm_workspace(1 << 30, 64) <= 1 << 20
    assert G.gosh_linear_backward_workspace(0, 64, 64, G.GOSH_BF16, H.GELU) == 0
    assert G.gosh_linear_backward_workspace(10, 0, 64, G.GOSH_BF16, H.GELU) == 0
    rows, k, n = 65536, 512, 2048
    none = G.gosh_linear_backward_workspace(rows, k, n, G.GOSH_BF16, H.NONE)
    assert G.gosh_linear_backward_workspace(rows, k, n, G.GOSH_BF16, H.GELU) == none + rows * n * 2
    assert none < 96 << 20


def test_packed_of_another_kind():
    with pytest.raises(TypeError):
        G.Packed8(3, 4, torch.float64, "cpu")
    p = G.Packed8(3, 33, torch.bfloat16, "cpu")
    assert p.q.shape == (3, 48) and p.exps.shape == (3, 2)


@pytest.mark.parametrize("kind", [H.NONE, H.RELU, H.GELU, H.SILU])
def test_gradient_of_the_linear_layer_against_differences(kind):
    """Central differences of 64-bit values: off by the third derivative times h^2 and rounding over h, 1e-8 here."""
    g = torch.Generator().manual_seed(kind)
    r = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)  # noqa: E731
    x, w, b, dy = r(5, 4), r(3, 4), r(3), r(5, 3)
    z = x @ w.t() + b
    assert (z.abs() > 1e-3).all()  # away from relu's corner
    (dx, dw, db), _ = H.linear_backward(dy, x, w, z, kind, torch.float32)
    h = 1e-5
    for t, grad in ((x, dx), (w, dw), (b, db)):
        for i in range(t.numel()):
            old = t.view(-1)[i].item()
            sums = []
            for s in (h, -h):
                t.view(-1)[i] = old + s
                sums.append((H.linear(x, w, b, kind, None)[0] * dy).sum().item())
            t.view(-1)[i] = old
            assert abs((sums[0] - sums[1]) / (2 * h) - grad.view(-1)[i].item()) < 1e-7


def test_gradient_of_the_layer_norm_against_differences():
    g = torch.Generator().manual_seed(9)
    r = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)  # noqa: E731
    x, gamma, beta, dy, eps = r(4, 6), r(6), r(6), r(4, 6), 1e-3
    (_, _, rstd, xhat), _ = H.norm(x, gamma, beta, eps)
    (dx, dgamma, dbeta), _ = H.norm_backward(dy, xhat, gamma, rstd, None, torch.zeros_like(x))
    h = 1e-5
    for t, grad in ((x, dx), (gamma, dgamma), (beta, dbeta)):
        for i in range(t.numel()):
            old = t.view(-1)[i].item()
            sums = []
            for s in (h, -h):
                t.view(-1)[i] = old + s
                sums.append((H.norm(x, gamma, beta, eps)[0][0] * dy).sum().item())
            t.view(-1)[i] = old
            assert abs((sums[0] - sums[1]) / (2 * h) - grad.view(-1)[i].item()) < 1e-7
