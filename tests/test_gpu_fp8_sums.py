"""Sums of products in 8-bit floating point, of whole numbers that 32 bits hold: large products that cancel beside small ones."""
import pytest
import torch

import paper_2008_12336_amd as G
from tests import head_model as H
from tests.test_gpu_head import DEV

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
