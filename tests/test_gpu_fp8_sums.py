"""Sums of products in 8-bit floating point, of whole numbers that 32 bits hold: large products that cancel beside small ones."""
import pytest
import torch

import paper_2008_12336_amd as G
from tests import head_model as H
from tests import step_model as S
from tests.test_gpu_fp8 import values
from tests.test_gpu_head import DEV, gen, within

pytestmark = pytest.mark.gpu


def cancelling(rows, k, seed):
    """(rows x k, k): of eight neighbours two are 256 in magnitude and of opposite signs in the second factor; the others' products are
    1 each.  The sum along k is the number of those, whichever order and however many at once: all of it fits 24 bits."""
    g = torch.Generator().manual_seed(seed)
    a, b = torch.ones(rows, k), torch.ones(k)
    for at in range(0, k - 7, 8):
        i, j = torch.randperm(8, generator=g)[:2].tolist()
        a[:, at + i], a[:, at + j] = 256.0, 256.0
        b[at + i], b[at + j] = 256.0, -256.0
    return a.to(DEV), b.to(DEV), float(6 * (k // 8) + k % 8)


def forms(x, tall=1):
    p, t = G.PackedFp8(*x.shape, tall, DEV), G.PackedFp8(x.shape[1], x.shape[0], tall, DEV)
    G.gosh_pack_fp8(x, p, t)
    return p, t


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32], ids=["bf16", "f16", "f32"])
@pytest.mark.parametrize("rows, k, n", [(1, 512, 2048), (5, 40, 3), (32, 1024, 96), (64, 256, 64), (512, 256, 1024)])
def test_layers_of_few_results_lose_nothing(rows, k, n, dtype):
    x, w, want = cancelling(rows, k, k)
    w8 = forms(w.repeat(n, 1), 128)[0]
    for given in (x.to(dtype), None):  # put into 8 bits in the product's launch, or before
        x8 = forms(x)[0]
        y, z = (torch.zeros(rows, n, dtype=dtype, device=DEV) for _ in range(2))
        G.gosh_linear_fp8(given, x8, w8, y, z=z)
        assert (y == torch.tensor(want).to(dtype).to(DEV)).all() and torch.equal(y, z)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32], ids=["bf16", "f16", "f32"])
@pytest.mark.parametrize("rows, k, n", [(40, 24, 128), (256, 64, 512), (512, 256, 1024)])
def test_gradients_of_few_results_lose_nothing(rows, k, n, dtype):
    dy, w, of_x = cancelling(rows, n, 1)  # along the layer's results
    wt = forms(w[:, None].repeat(1, k), 128)[1]
    dx = torch.zeros(rows, k, dtype=dtype, device=DEV)
    G.gosh_linear_fp8_backward(dy.to(dtype), None, wt, None, H.NONE, dx=dx)
    assert (dx == torch.tensor(of_x).to(dtype).to(DEV)).all()
    dy, x, of_w = cancelling(n, rows, 2)  # along the rows
    xt = forms(x[:, None].repeat(1, k))[1]
    dw = torch.zeros(n, k, dtype=dtype, device=DEV)
    G.gosh_linear_fp8_backward(dy.t().contiguous().to(dtype), xt, None, None, H.NONE, dw=dw)
    assert (dw == torch.tensor(of_w).to(dtype).to(DEV)).all()


@pytest.mark.parametrize("rows, k, n", [(9000, 520, 1030), (700, 2048, 130), (33000, 264, 520)])
def test_exact_sums_of_bfloat16_results_on_request(rows, k, n):
    """In tiles of every kind: dx and the results of the layer; dw split along the rows or not, in either type."""
    t = torch.bfloat16
    x, w, want = cancelling(rows, k, k)
    y = torch.zeros(rows, n, dtype=t, device=DEV)
    for given in (x.to(t), None):
        G.gosh_linear_fp8(given, forms(x)[0], forms(w.repeat(n, 1), 128)[0], y, act=H.RELU, exact=True)
        assert (y == torch.tensor(want).to(t).to(DEV)).all()
        y.zero_()
        G.gosh_linear_fp8(given, forms(x)[0], forms(w.repeat(n, 1), 128)[0], y, exact=True)
        assert (y == torch.tensor(want).to(t).to(DEV)).all()
    dy, v, of_x = cancelling(rows, n, 1)
    dx = torch.zeros(rows, k, dtype=t, device=DEV)
    G.gosh_linear_fp8_backward(dy.to(t), None, forms(v[:, None].repeat(1, k), 128)[1], None, H.NONE, dx=dx, exact=True)
    assert (dx == torch.tensor(of_x).to(t).to(DEV)).all()
    dy, u, of_w = cancelling(n, rows, 2)
    xt = forms(u[:, None].repeat(1, k))[1]
    for kind in (t, torch.float32):
        dw = torch.zeros(n, k, dtype=kind, device=DEV)
        G.gosh_linear_fp8_backward(dy.t().contiguous().to(t), xt, None, None, H.NONE, dw=dw, exact=True)
        assert (dw == torch.tensor(of_w).to(kind).to(DEV)).all()


@pytest.mark.parametrize("rows, k, n", [(300, 97, 131), (9000, 520, 1030), (2000, 2000, 3000)])
def test_exact_layers_have_the_bounds_of_32_bits(rows, k, n):
    """Those of step_model.py without what the matrix cores cut off, and as f16 and f32 results are by themselves."""
    rnd, t = gen(rows), torch.bfloat16
    x, w, b, dy = rnd(rows, k) * torch.exp(rnd(rows, 1)), rnd(n, k) / k ** 0.5, 0.3 * rnd(n), 0.1 * rnd(rows, n)
    (x8, xt), (w8, wt) = forms(x.to(t)), forms(w.to(t), 128)
    y, z, dx, dw = (torch.zeros(*s, dtype=t, device=DEV) for s in ((rows, n), (rows, n), (rows, k), (n, k)))
    db = torch.zeros(n, device=DEV)
    G.gosh_linear_fp8(None, x8, w8, y, bias=b, act=H.GELU, z=z, exact=True)
    wy, wz, ey, ez = S.linear_fp8(values(x8), values(w8), b.double(), H.GELU, None, torch.float32)
    within(y, wy, H.rounded(ey, wy, t), "y")
    within(z, wz, H.rounded(ez, wz, t), "z")
    G.gosh_linear_fp8_backward(dy.to(t), xt, wt, z, H.GELU, dx=dx, dw=dw, db=db, exact=True)
    want, bound = S.linear_fp8_backward(dy.to(t).double(), values(xt), values(wt).t(), z.double(), H.GELU, torch.float32, torch.float32)
    within(dx, want[0], H.rounded(bound[0], want[0], t), "dx")
    within(dw, want[1], H.rounded(bound[1], want[1], t), "dw")
    within(db, want[2], H.rounded(bound[2], want[2], torch.float32), "db")
    for other in (torch.float16, torch.float32):  # they are exact anyway
        out = [torch.zeros(rows, n, dtype=other, device=DEV) for _ in range(2)]
        for o, e in zip(out, (False, True)):
            G.gosh_linear_fp8(None, x8, w8, o, bias=b, act=H.GELU, exact=e)
        assert torch.equal(*out)
