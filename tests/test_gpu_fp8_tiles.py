"""Products in 8-bit floating point in the tiles that no other test takes, which tests/test_fp8_plans.py holds these shapes to: forward
passes and dx in tiles of 64, and in tiles of 256 whose results fit the caches, results past the caches with a packed z, dw in tiles of 256
whose splits begin off multiples of four blocks, and dw in tiles of 256 that is not split."""
import math

import pytest
import torch

import paper_2008_12336_amd as G
from tests import head_model as H
from tests import step_model as S
from tests.test_gpu_fp8 import packed, values
from tests.test_gpu_head import DEV, beside, gen, view, within

pytestmark = pytest.mark.gpu
T = torch.bfloat16

LARGE = (33000, 520, 1030)     # rows, in, out: y in tiles of 256, under 256 MB; dw in tiles of 256, 16 splits of 17 blocks
LARGE_DX = (33000, 1030, 520)  # dx in tiles of 256
PAST = (65281, 140, 2056)      # y in tiles of 256, over 256 MB
WHOLE_DW = (300, 8192, 4096)   # dw in tiles of 256, in one piece
SMALL = (1500, 130, 1030)      # y in tiles of 64, exact or not
SMALL_DX = (1500, 1030, 130)   # dx in tiles of 64


@pytest.mark.parametrize("kind", [H.NONE, H.GELU, H.SILU])
def test_large_tiles_under_the_size_of_the_caches(kind):
    rows, k, n = LARGE
    rnd = gen(kind)
    x8, w8, b = packed(rnd(rows, k).to(T)), packed(rnd(n, k) / math.sqrt(k), 128), 0.3 * rnd(n)
    a, w = values(x8), values(w8)
    for pad, use_r, how in ((0, False, None), (8, True, "z"), (3, False, "z8"), (0, True, "z8")):
        r, _ = view(rnd(rows, n), T, pad, pad)
        y, ymem = view(torch.zeros(rows, n, device=DEV), T, pad, pad)
        z, zmem = view(torch.zeros(rows, n, device=DEV), T, pad, pad)
        z8 = G.Packed8(rows, n, T, DEV)
        G.gosh_linear_fp8(None, x8, w8, y, bias=b, act=kind, residual=r if use_r else None, z={None: None, "z": z, "z8": z8}[how])
        wy, wz, ey, ez = S.linear_fp8(a, w, b.double(), kind, r.double() if use_r else None, T)
        within(y, wy, H.rounded(ey, wy, T), f"y, {how}")
        if how == "z":
            within(z, wz, H.rounded(ez, wz, T), "z")
        if how == "z8":
            in_8_bits(z8, wz, ez)
        beside(y, ymem)
        beside(z, zmem)


def in_8_bits(z8, z, ez):
    """Half a unit, 1/127 of the group's largest or less, as the layers of 16 bits are held to."""
    got = z8.q[:, :z8.cols].double() * torch.exp2(z8.exps.double().repeat_interleave(32, dim=1)[:, :z8.cols] - 127)
    within(got, z, ez + H.group_most(z.abs() + ez) / 127 * (1 + 1e-6) + 2.0 ** -127, "z8")


@pytest.mark.parametrize("kind", [H.GELU, H.RELU])
def test_results_past_the_caches_with_a_packed_z(kind):
    rows, k, n = PAST
    rnd = gen(7)
    x8, w8, b = packed(rnd(rows, k).to(T)), packed(rnd(n, k) / math.sqrt(k), 128), 0.3 * rnd(n)
    y, ymem = view(torch.zeros(rows, n, device=DEV), T, 8, 8)
    z8 = G.Packed8(rows, n, T, DEV)
    G.gosh_linear_fp8(None, x8, w8, y, bias=b, act=kind, z=z8)
    wy, wz, ey, ez = S.linear_fp8(values(x8), values(w8), b.double(), kind, None, T)
    within(y, wy, H.rounded(ey, wy, T), "y")
    del wy, ey
    in_8_bits(z8, wz, ez)
    alone = torch.empty_like(y)
    G.gosh_linear_fp8(None, x8, w8, alone, bias=b, act=kind)
    assert torch.equal(alone, y)
    beside(y, ymem)  # writes over y


@pytest.mark.parametrize("exact", [False, True])
@pytest.mark.parametrize("dtype, of_dw", [(T, T), (T, torch.float32), (torch.float16, torch.float16), (torch.float32, torch.float32)],
                         ids=["bf16", "bf16-f32", "f16", "f32"])
@pytest.mark.parametrize("shape", [LARGE, LARGE_DX, WHOLE_DW, SMALL, SMALL_DX], ids=lambda s: "x".join(map(str, s)))
def test_gradients_in_large_tiles(shape, dtype, of_dw, exact):
    rows, k, n = shape
    rnd = gen(rows + k)
    dy, xt, wt = (0.1 * rnd(rows, n)).to(dtype), G.PackedFp8(k, rows, 1, DEV), G.PackedFp8(k, n, 128, DEV)
    G.gosh_pack_fp8(rnd(rows, k).to(dtype), None, xt)
    G.gosh_pack_fp8((rnd(n, k) / math.sqrt(k)).to(dtype), None, wt)
    dx, xmem = view(torch.zeros(rows, k, device=DEV), dtype, 3, 1)
    dw, wmem = view(torch.zeros(n, k, device=DEV), of_dw, 3, 1)
    db = torch.empty(n, device=DEV)
    G.gosh_linear_fp8_backward(dy, xt, wt, None, H.NONE, dx=dx, dw=dw, db=db, exact=exact)
    rounds = (torch.float32, torch.float32) if exact else (dtype, of_dw)  # whether the matrix cores cut products off
    want, bound = S.linear_fp8_backward(dy.double(), values(xt), values(wt).t(), None, H.NONE, *rounds)
    within(dx, want[0], H.rounded(bound[0], want[0], dtype), "dx")
    within(dw, want[1], H.rounded(bound[1], want[1], of_dw), "dw")
    within(db, want[2], H.rounded(bound[2], want[2], torch.float32), "db")
    beside(dx, xmem)
    beside(dw, wmem)


@pytest.mark.parametrize("exact", [False, True])
@pytest.mark.parametrize("dtype", [T, torch.float16, torch.float32], ids=["bf16", "f16", "f32"])
def test_small_tiles(dtype, exact):
    rows, k, n = SMALL
    rnd = gen(4)
    x8, w8, b = packed(rnd(rows, k).to(dtype)), packed(rnd(n, k) / math.sqrt(k), 128), 0.3 * rnd(n)
    for kind, pad in ((H.NONE, 0), (H.RELU, 3), (H.SILU, 8)):
        y, ymem = view(torch.zeros(rows, n, device=DEV), dtype, pad, pad)
        z, zmem = view(torch.zeros(rows, n, device=DEV), dtype, pad, pad)
        G.gosh_linear_fp8(None, x8, w8, y, bias=b, act=kind, z=z, exact=exact)
        wy, wz, ey, ez = S.linear_fp8(values(x8), values(w8), b.double(), kind, None, torch.float32 if exact else dtype)
        within(y, wy, H.rounded(ey, wy, dtype), f"y, activation {kind}")
        within(z, wz, H.rounded(ez, wz, dtype), f"z, activation {kind}")
        beside(y, ymem)
        beside(z, zmem)
