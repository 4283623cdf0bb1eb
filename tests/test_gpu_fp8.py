"""gosh_pack_fp8, gosh_unpack_fp8, gosh_linear_fp8 and its gradient against 64-bit arithmetic with the bounds of
step_model.py: every type, odd sizes and strides, rows of one and none, both kinds of blocks, what is not finite, memory
beside the outputs, other streams, captured graphs, offsets past 32 bits."""
import math

import pytest
import torch

import paper_2008_12336_amd as G
from tests import head_model as H
from tests import step_model as S
from tests.test_gpu_head import DEV, MARK, NAMES, beside, gen, types, view, within

pytestmark = pytest.mark.gpu


def values(p):
    """What a PackedFp8 stands for, and that its padding is zero."""
    assert (p.q.view(torch.uint8)[:, p.cols:-(-p.cols // 128) * 128] == 0).all()
    return S.fp8_values(p.q, p.exps, p.rows, p.cols, p.block_rows)


def packed(x, tall=1):
    p = G.PackedFp8(x.shape[0], x.shape[1], tall, DEV)
    G.gosh_pack_fp8(x, p)
    return p


SIZES = [(1, 1, 0, 0), (1, 130, 0, 0), (3, 31, 0, 1), (128, 128, 0, 0), (129, 257, 3, 1), (200, 64, 0, 0), (70, 520, 8, 8), (300, 127, 1, 0)]


@types
@pytest.mark.parametrize("tall", [1, 128])
@pytest.mark.parametrize("shape", SIZES, ids=lambda s: "x".join(map(str, s)))
def test_eight_bits_entry_by_entry(shape, tall, dtype):
    rows, k, pad, off = shape
    rnd = gen(rows * 3 + k)
    v = rnd(rows, k) * torch.exp2(torch.round(5 * rnd(rows, 1)))
    top = torch.finfo(dtype).max
    edge = [0.0, -0.0, top, -top, torch.finfo(dtype).tiny, math.inf, -math.inf, math.nan, 448.0, 449.0, 464.0, 2.0 ** -9, 2.0 ** -10,
            3 * 2.0 ** -10, 17.0, 19.0, -21.0]
    if rows * k > 100:
        for i, e in enumerate(edge):
            v[(7 * i) % rows, (5 * i) % k] = e
    if rows > 20:
        v[15] = 0
        v[16] *= 1e-38 if dtype != torch.float16 else 1e-6
    x, _ = view(v, dtype, pad, off)
    for which in ("q", "qt", "both"):
        q = G.PackedFp8(rows, k, tall, DEV) if which != "qt" else None
        qt = G.PackedFp8(k, rows, tall, DEV) if which != "q" else None
        for p in (q, qt):
            if p is not None:
                p.q.view(torch.uint8).fill_(99), p.exps.fill_(99)
        G.gosh_pack_fp8(x, q, qt)
        for p, source in ((q, x), (qt, x.t())):
            if p is None:
                continue
            code, exps, value = S.fp8(source.double().cpu(), tall)
            assert torch.equal(p.exps[:, :exps.shape[1]].cpu().long(), exps), which
            got = p.q.view(torch.uint8).cpu().long()
            nan = code % 128 == 127
            assert torch.equal(got % 128 == 127, nan)
            assert torch.equal(torch.where(nan, torch.zeros_like(got), got), torch.where(nan, torch.zeros_like(code), code)), which
            assert (p.exps[:, exps.shape[1]:] == 99).all()
            back = torch.float32 if which == "both" else dtype
            out, mem = view(torch.zeros(p.rows, p.cols, device=DEV), back, pad, off)
            G.gosh_unpack_fp8(p, out)
            want = value.to(torch.float32).to(back).to(torch.float64) if back != torch.float16 else value.to(torch.float16).double()
            assert torch.equal(torch.nan_to_num(out.double().cpu(), nan=123.25), torch.nan_to_num(want, nan=123.25))
            beside(out, mem)


def test_blocks_that_another_owner_gave():
    """q and exps that were replaced: rows further apart, blocks of a larger matrix."""
    rnd = gen(2)
    x = rnd(140, 200)
    p = G.PackedFp8(140, 200, 128, DEV)
    p.q = torch.full((140, 384), 99, dtype=torch.uint8, device=DEV).view(torch.float8_e4m3fn)[:, 128:]
    p.exps = torch.full((2, 12), 99, dtype=torch.uint8, device=DEV)[:, 4:8]
    G.gosh_pack_fp8(x, p)
    assert torch.equal(S.fp8_values(p.q, p.exps, 140, 200, 128).cpu(), S.fp8(x.double().cpu(), 128)[2])
    y = torch.empty(140, 140, device=DEV)
    G.gosh_linear_fp8(x, G.PackedFp8(140, 200, 1, DEV), p, y)
    a, w = S.fp8(x.double().cpu(), 1)[2].to(DEV), S.fp8(x.double().cpu(), 128)[2].to(DEV)
    wy, _, ey, _ = S.linear_fp8(a, w, None, H.NONE, None, torch.float32)
    within(y, wy, H.rounded(ey, wy, torch.float32), "y")


SHAPES = [  # rows, in, out, padding of the rows, entries off the start of memory
    (1, 1, 1, 0, 0), (1, 512, 2048, 0, 0), (2, 37, 5, 3, 1), (7, 130, 33, 0, 1), (8, 64, 257, 1, 0), (9, 8, 1, 0, 0), (33, 3, 40, 5, 3),
    (64, 64, 64, 0, 0), (129, 260, 130, 0, 0), (200, 17, 517, 2, 1), (300, 1024, 96, 8, 8), (1000, 132, 31, 0, 0), (20000, 72, 260, 0, 0),
    (5000, 300, 1500, 0, 0), (31, 2000, 70, 0, 0), (90, 97, 1844, 0, 0), (257, 2050, 129, 0, 0),
]


@types
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_linear(shape, dtype):
    rows, k, n, pad, off = shape
    rnd = gen(rows * 31 + k)
    x, _ = view(rnd(rows, k) * torch.exp(rnd(rows, 1)), dtype, pad, off)
    b, r = 0.3 * rnd(n), view(rnd(rows, n), dtype, pad, off)[0]
    for kind, tall in ((H.NONE, 1), (H.RELU, 128), (H.GELU, 128), (H.SILU, 1)):
        w8 = packed((rnd(n, k) / math.sqrt(k)).to(dtype), tall)
        w = values(w8)
        use_b, use_r = kind != H.RELU, kind in (H.NONE, H.GELU)
        x8 = G.PackedFp8(rows, k, 1, DEV)
        y, ymem = view(torch.zeros(rows, n, device=DEV), dtype, pad, off)
        z, zmem = view(torch.zeros(rows, n, device=DEV), dtype, pad, off)
        G.gosh_linear_fp8(x, x8, w8, y, bias=b if use_b else None, act=kind, residual=r if use_r else None, z=z if kind != H.SILU else None)
        a = values(x8)
        alone = packed(x)
        assert torch.equal(x8.q.view(torch.uint8), alone.q.view(torch.uint8)) and torch.equal(x8.exps, alone.exps)
        wy, wz, ey, ez = S.linear_fp8(a, w, b.double() if use_b else None, kind, r.double() if use_r else None, dtype)
        within(y, wy, H.rounded(ey, wy, dtype), f"y, activation {kind}")
        if kind != H.SILU:
            within(z, wz, H.rounded(ez, wz, dtype), f"z, activation {kind}")
        again = r.clone() if use_r else torch.empty_like(r)
        G.gosh_linear_fp8(None, x8, w8, again, bias=b if use_b else None, act=kind, residual=again if use_r else None)
        assert torch.equal(again, y)  # from x8, in place of the residual, and the same bits
        z8 = G.Packed8(rows, n, dtype, DEV)
        G.gosh_linear_fp8(None, x8, w8, again, bias=b if use_b else None, act=kind, z=z8)
        stood = H.values(z8.q[:, :n].cpu(), z8.exps.cpu()).to(DEV)
        within(stood, wz, ez + H.group_most(wz.abs() + ez) / 127 * (1 + 1e-6) + 2.0 ** (-25 if dtype == torch.float16 else -127), "z8")
        beside(y, ymem)
        if kind != H.SILU:
            beside(z, zmem)


@types
@pytest.mark.parametrize("shape", [s for s in SHAPES if s[0] * s[1] * s[2] < 1e9], ids=lambda s: "x".join(map(str, s)))
def test_linear_backward(shape, dtype):
    rows, k, n, pad, off = shape
    rnd = gen(rows * 37 + n)
    x = rnd(rows, k).to(dtype)
    xt = G.PackedFp8(k, rows, 1, DEV)
    G.gosh_pack_fp8(x, None, xt)
    dy, _ = view(0.1 * rnd(rows, n) * torch.exp(rnd(rows, 1)), dtype, pad, off)
    z, _ = view(2 * rnd(rows, n), dtype, pad, off)
    z8 = G.Packed8(rows, n, dtype, DEV)
    G.gosh_pack8(z, z8)
    for kind, zz, tall in ((H.NONE, None, 128), (H.RELU, z, 1), (H.GELU, z8, 128), (H.SILU, z, 128)):
        wt = G.PackedFp8(k, n, tall, DEV)
        G.gosh_pack_fp8((rnd(n, k) / math.sqrt(k)).to(dtype), None, wt)
        dx, xmem = view(torch.zeros(rows, k, device=DEV), dtype, pad, off)
        wide = kind in (H.NONE, H.GELU)  # dw in 32 bits
        dw, wmem = view(torch.zeros(n, k, device=DEV), torch.float32 if wide else dtype, pad, off)
        db = torch.full((n,), MARK, device=DEV)
        G.gosh_linear_fp8_backward(dy, xt, wt, zz, kind, dx=dx, dw=dw, db=db)
        open_ = (H.values(zz.q[:, :n].cpu(), zz.exps.cpu()).to(DEV) if isinstance(zz, G.Packed8) else None if zz is None else zz.double())
        want, bounds = S.linear_fp8_backward(dy.double(), values(xt), values(wt).t(), open_, kind, dtype, dw.dtype)
        within(dx, want[0], H.rounded(bounds[0], want[0], dtype), f"dx, activation {kind}")
        within(dw, want[1], H.rounded(bounds[1], want[1], dw.dtype), f"dw, activation {kind}")
        within(db, want[2], H.rounded(bounds[2], want[2], torch.float32), f"db, activation {kind}")
        one, again = torch.empty_like(dw), torch.empty_like(db)
        G.gosh_linear_fp8_backward(dy, xt, None, zz, kind, dw=one, db=again)  # each by itself, and the same bits again
        assert torch.equal(one, dw) and torch.equal(again, db)
        alone = torch.empty_like(dx)
        G.gosh_linear_fp8_backward(dy, None, wt, zz, kind, dx=alone)
        assert torch.equal(alone, dx)
        beside(dx, xmem)
        beside(dw, wmem)


@types
@pytest.mark.parametrize("shape", [(20011, 512, 1024, 0, 0), (70001, 300, 520, 3, 1), (3000, 4000, 700, 0, 0)], ids=lambda s: "x".join(map(str, s)))
def test_many_rows(shape, dtype):
    """Every size of tiles, more of them than the device holds at once, and sums that are split."""
    test_linear(shape, dtype)
    test_linear_backward(shape, dtype)


@types
@pytest.mark.parametrize("pad", [0, 8])
def test_results_larger_than_the_caches(pad, dtype):
    rows, k, n = 65281, 140, 2056
    rnd = gen(rows + pad)
    x8, w8 = packed(rnd(rows, k).to(dtype)), packed(rnd(n, k) / math.sqrt(k), 128)
    a, w, b, r = values(x8), values(w8), 0.3 * rnd(n), view(rnd(rows, n), dtype, pad, pad)[0]
    for kind, use_r, use_z in ((H.GELU, False, True), (H.SILU, True, False), (H.RELU, True, True), (H.NONE, False, False)):
        y, ymem = view(torch.zeros(rows, n, device=DEV), dtype, pad, pad)
        z, zmem = view(torch.zeros(rows, n, device=DEV), dtype, pad, pad)
        G.gosh_linear_fp8(None, x8, w8, y, bias=b, act=kind, residual=r if use_r else None, z=z if use_z else None)
        wy, wz, ey, ez = S.linear_fp8(a, w, b.double(), kind, r.double() if use_r else None, dtype)
        within(y, wy, H.rounded(ey, wy, dtype), f"y, activation {kind}")
        if use_z:
            within(z, wz, H.rounded(ez, wz, dtype), f"z, activation {kind}")
        again = r.clone()
        G.gosh_linear_fp8(None, x8, w8, again, bias=b, act=kind, residual=again if use_r else None)  # in place, and the same bits
        assert torch.equal(again, y)
        beside(y, ymem)
        beside(z, zmem)


@pytest.mark.parametrize("rows", [3, 200, 9000])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_units_far_apart(rows, dtype):
    """Powers of two come out of both operands as they are: rows scaled by 2^100 against weights scaled by 2^-100, and down to where
    results have no digits left."""
    rnd = gen(rows)
    k, n = 260, 40
    x, w = rnd(rows, k).to(dtype), rnd(n, k).to(dtype)
    out = []
    for up, down in ((0, 0), (100, -100), (-60, 60), (-100, 90)):
        x8, w8 = packed(x * 2.0 ** up), packed(w * 2.0 ** down, 128)
        y = torch.empty(rows, n, dtype=dtype, device=DEV)
        G.gosh_linear_fp8(None, x8, w8, y)
        out.append(y.double() * 2.0 ** -(up + down))
    assert all(torch.equal(y, out[0]) for y in out[1:])
    y = torch.empty(rows, n, dtype=dtype, device=DEV)
    G.gosh_linear_fp8(None, packed(x * 2.0 ** -120), packed(w * 2.0 ** -120, 128), y)
    assert (y.abs() <= 2.0 ** -126).all()
    G.gosh_linear_fp8(None, packed(x * 2.0 ** 100), packed(w * 2.0 ** 100, 128), y)
    # every product is beyond the largest number, of either sign: infinities that cancel are NaN
    assert not torch.isfinite(y[out[0] != 0]).any()


@types
def test_rows_of_none(dtype):
    e = lambda n: torch.empty(0, n, dtype=dtype, device=DEV)  # noqa: E731
    w8, wt = G.PackedFp8(5, 7, 128, DEV), G.PackedFp8(7, 5, 128, DEV)
    x8, xt = G.PackedFp8(0, 7, 1, DEV), G.PackedFp8(7, 0, 1, DEV)
    G.gosh_pack_fp8(torch.ones(5, 7, device=DEV), w8, wt)
    G.gosh_pack_fp8(e(7), x8, xt)
    G.gosh_unpack_fp8(x8, e(7))
    G.gosh_linear_fp8(e(7), x8, w8, e(5), act=H.GELU, z=e(5))
    dw, db = torch.full((5, 7), MARK, device=DEV).to(dtype), torch.full((5,), MARK, device=DEV)
    G.gosh_linear_fp8_backward(e(5), xt, wt, e(5), H.GELU, dx=e(7), dw=dw, db=db)
    assert (dw == 0).all() and (db == 0).all()


@types
@pytest.mark.parametrize("rows", [5, 300])
def test_what_is_not_finite_stays_in_its_rows(rows, dtype):
    """A row of x that holds NaN or an infinity gives NaN, all of it, and no other row; an entry of dy reaches its row of dx
    and its row of dw."""
    rnd = gen(rows)
    k, n = 170, 45
    x = rnd(rows, k).to(dtype)
    x[2, 169], x[4, 0] = math.nan, math.inf
    y = torch.empty(rows, n, device=DEV, dtype=dtype)
    x8, xt = G.PackedFp8(rows, k, 1, DEV), G.PackedFp8(k, rows, 1, DEV)
    w8, wt = G.PackedFp8(n, k, 128, DEV), G.PackedFp8(k, n, 128, DEV)
    G.gosh_pack_fp8(rnd(n, k).to(dtype), w8, wt)
    G.gosh_linear_fp8(x, x8, w8, y)
    fine = torch.ones(rows, dtype=torch.bool, device=DEV)
    fine[2] = fine[4] = False
    assert torch.isfinite(y[fine]).all() and torch.isnan(y[~fine]).all()
    dy = rnd(rows, n).to(dtype)
    dy[1, 44] = math.nan
    G.gosh_pack_fp8(rnd(rows, k).to(dtype), None, xt)
    dx, dw = torch.empty_like(x), torch.empty(n, k, device=DEV)
    G.gosh_linear_fp8_backward(dy, xt, wt, None, dx=dx, dw=dw)
    assert torch.isnan(dx[1]).all() and torch.isnan(dw[44]).all()
    fine[:] = True
    fine[1] = False
    assert torch.isfinite(dx[fine]).all() and torch.isfinite(dw[:44]).all()


def test_the_bias_gradient_against_differences():
    """sum(dy * y) in 64 bits of the results in 32, with one bias a little up and down."""
    rnd = gen(9)
    rows, k, n, h = 40, 60, 30, 2.0 ** -6
    x, b, dy = rnd(rows, k), rnd(n), rnd(rows, n)
    x8, w8, xt = G.PackedFp8(rows, k, 1, DEV), packed(rnd(n, k) / 8, 128), G.PackedFp8(k, rows, 1, DEV)
    G.gosh_pack_fp8(x, x8, xt)
    y, z, db, dw = torch.empty(rows, n, device=DEV), torch.empty(rows, n, device=DEV), torch.empty(n, device=DEV), torch.empty(n, k, device=DEV)
    for kind in (H.GELU, H.SILU):
        G.gosh_linear_fp8(None, x8, w8, y, bias=b, act=kind, z=z)
        G.gosh_linear_fp8_backward(dy, xt, None, z, kind, dw=dw, db=db)
        ends = []
        for s in (1, -1):
            out = torch.empty_like(y)
            G.gosh_linear_fp8(None, x8, w8, out, bias=b + s * h, act=kind)
            ends.append((dy.double() * out.double()).sum(dim=0))
        slope = (ends[0] - ends[1]) / (2 * h)
        # third derivatives of both are below 3, each y is off by 2^-20 of its magnitude at most
        bound = dy.double().abs().sum(dim=0) * (h * h / 6 * 3) + (dy.double().abs() * (1 + y.double().abs())).sum(dim=0) * 2.0 ** -20 / h
        within(db, slope, bound + 1e-5 * slope.abs(), f"db, activation {kind}")


def _training(rows, k, n, t, rnd):
    f = lambda *s, dtype=t: torch.empty(*s, dtype=dtype, device=DEV)  # noqa: E731
    return dict(x8=G.PackedFp8(rows, k, 1, DEV), xt=G.PackedFp8(k, rows, 1, DEV), w8=G.PackedFp8(n, k, 128, DEV),
                wt=G.PackedFp8(k, n, 128, DEV), y=f(rows, n), z=f(rows, n), dx=f(rows, k), dw=f(n, k), db=f(n, dtype=torch.float32))


def _step(o, x, w, b, dy, work=None, stream=None):
    G.gosh_pack_fp8(w, o["w8"], o["wt"], stream=stream)
    G.gosh_pack_fp8(x, o["x8"], o["xt"], stream=stream)
    G.gosh_linear_fp8(None, o["x8"], o["w8"], o["y"], bias=b, act=H.GELU, z=o["z"], stream=stream)
    G.gosh_linear_fp8_backward(dy, o["xt"], o["wt"], o["z"], H.GELU, dx=o["dx"], dw=o["dw"], db=o["db"], workspace=work, stream=stream)


def test_a_stream_of_its_own():
    rnd = gen(4)
    rows, k, n, t = 3000, 256, 512, torch.bfloat16
    x, w, b, dy = rnd(rows, k).to(t), (rnd(n, k) / 16).to(t), rnd(n), rnd(rows, n).to(t)
    want = _training(rows, k, n, t, rnd)
    _step(want, x, w, b, dy)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for how in (side, side.cuda_stream):
        got = _training(rows, k, n, t, rnd)
        late = torch.zeros_like(x)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            for _ in range(20):
                late.add_(1).sub_(1)
            late.copy_(x)
        _step(got, late, w, b, dy, stream=how)
        side.synchronize()
        assert all(torch.equal(got[name], want[name]) for name in ("y", "z", "dx", "dw", "db"))


@pytest.mark.parametrize("rows", [5, 700, 9000])
def test_a_captured_graph(rows):
    rnd = gen(5)
    k, n, t = 200, 320, torch.bfloat16
    x, w, b, dy = rnd(rows, k).to(t), (rnd(n, k) / 16).to(t), rnd(n), rnd(rows, n).to(t)
    work = torch.empty(G.gosh_linear_fp8_backward_workspace(rows, k, n), dtype=torch.uint8, device=DEV)
    held, eager = _training(rows, k, n, t, rnd), _training(rows, k, n, t, rnd)
    _step(held, x, w, b, dy, work)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        _step(held, x, w, b, dy, work)
    for turn in range(4):
        x.copy_(rnd(rows, k))
        dy.copy_(rnd(rows, n))
        work.fill_(255)  # nothing is kept in it
        graph.replay()
        torch.cuda.synchronize()
        _step(eager, x, w, b, dy)
        torch.cuda.synchronize()
        for name in ("y", "z", "dx", "dw", "db"):
            assert torch.equal(held[name], eager[name]), (turn, name)


def test_offsets_past_32_bits():
    """A matrix of more than 2^31 entries: its first and last rows, there and back, and through a layer."""
    t, k = torch.bfloat16, 512
    rows = (1 << 32) // k + 77
    x = torch.zeros(rows, k, dtype=t, device=DEV)
    ends = torch.cat((torch.arange(40), torch.arange(rows - 40, rows))).to(DEV)
    rnd = gen(6)
    x[ends] = rnd(80, k).to(t)
    p = G.PackedFp8(rows, k, 1, DEV)
    G.gosh_pack_fp8(x, p)
    want = S.fp8(x[ends].double().cpu(), 1)[2].to(DEV)
    y = torch.empty_like(x)
    G.gosh_unpack_fp8(p, y)
    assert torch.equal(y[ends].double(), want) and (y[100:200] == 0).all()
    del y
    w8 = packed(rnd(k, k) / 16, 128)
    y = torch.empty(rows, k, dtype=t, device=DEV)
    G.gosh_linear_fp8(None, p, w8, y)
    wy, _, ey, _ = S.linear_fp8(want, values(w8), None, H.NONE, None, t)
    within(y[ends], wy, H.rounded(ey, wy, t), "linear layer at the ends")
    with pytest.raises(G.GoshError, match="cols = 8388685"):  # rows of a transposed form are shorter
        G.gosh_pack_fp8(x, None, G.PackedFp8(1, rows, 1, DEV))
    x = x[77:]
    turned = G.PackedFp8(k, rows - 77, 1, DEV)
    G.gosh_pack_fp8(x, None, turned)
    back = S.fp8_values(turned.q[:, -128:], turned.exps[:, (rows - 78) // 128:(rows - 78) // 128 + 1], k, 128, 1)
    assert torch.equal(back, S.fp8(x[-128:].double().t().contiguous(), 1)[2])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=["bf16", "f16"])
def test_gradients_with_offsets_past_32_bits(dtype):
    """The most rows that dw takes but for a piece of the last block; operands, workspace and dx are all longer than 2^32 bytes."""
    rows, k, n, last = (1 << 23) - 51, 520, 524, 77
    x, dy = torch.zeros(rows, k, dtype=dtype, device=DEV), torch.zeros(rows, n, dtype=dtype, device=DEV)
    ends = torch.cat((torch.arange(128), torch.arange(rows - last, rows))).to(DEV)
    rnd = gen(16)
    x[ends], dy[ends] = rnd(128 + last, k).to(dtype), (0.1 * rnd(128 + last, n)).to(dtype)
    xt, wt = G.PackedFp8(k, rows, 1, DEV), G.PackedFp8(k, n, 128, DEV)
    G.gosh_pack_fp8(x, None, xt)
    G.gosh_pack_fp8((rnd(n, k) / math.sqrt(k)).to(dtype), None, wt)
    few = G.PackedFp8(k, 128 + last, 1, DEV)
    G.gosh_pack_fp8(x[ends], None, few)
    del x
    dx, dw, db = torch.full((rows, k), MARK, dtype=dtype, device=DEV), torch.empty(n, k, device=DEV), torch.empty(n, device=DEV)
    G.gosh_linear_fp8_backward(dy, xt, wt, None, H.NONE, dx=dx, dw=dw, db=db)
    want, bounds = S.linear_fp8_backward(dy[ends].double(), values(few), values(wt).t(), None, H.NONE, dtype, dw.dtype)
    within(dx[ends], want[0], H.rounded(bounds[0], want[0], dtype), "dx at the ends")
    within(dw, want[1], H.rounded(bounds[1], want[1], dw.dtype), "dw")
    within(db, want[2], H.rounded(bounds[2], want[2], torch.float32), "db")
    for i in range(128, rows - last, 1 << 20):  # rows of zeros
        assert not dx[i:min(i + (1 << 20), rows - last)].any()


def test_refusals_on_the_device():
    x, y = torch.zeros(64, 32, device=DEV), torch.zeros(64, 16, device=DEV)
    x8, w8 = G.PackedFp8(64, 32, 1, DEV), G.PackedFp8(16, 32, 128, DEV)
    xt, wt = G.PackedFp8(32, 64, 1, DEV), G.PackedFp8(32, 16, 128, DEV)
    with pytest.raises(G.GoshError, match="x is 64 x 31: must be 64 x 32"):
        G.gosh_linear_fp8(x[:, :31], x8, w8, y)
    with pytest.raises(G.GoshError, match="y is"):
        G.gosh_linear_fp8(x, x8, w8, y[:, :15])
    with pytest.raises(G.GoshError, match="type"):
        G.gosh_linear_fp8(x, x8, w8, y, residual=y.bfloat16())
    with pytest.raises(G.GoshError, match="x is not memory"):
        G.gosh_linear_fp8(x.cpu(), x8, w8, y)
    with pytest.raises(G.GoshError, match="x8: block_rows"):
        G.gosh_linear_fp8(x, G.PackedFp8(64, 32, 128, DEV), w8, y)
    with pytest.raises(G.GoshError, match="must be the same"):
        G.gosh_pack_fp8(x, x8, G.PackedFp8(32, 64, 128, DEV))
    with pytest.raises(G.GoshError, match="qt is 64 x 32: must be 32 x 64"):
        G.gosh_pack_fp8(x, None, x8)
    with pytest.raises(TypeError):
        G.gosh_linear_fp8(x, x8, y, y)
    with pytest.raises(G.GoshError, match="act"):
        G.gosh_linear_fp8(x, x8, w8, y, act=4)
    with pytest.raises(G.GoshError, match="z is null"):
        G.gosh_linear_fp8_backward(y, xt, wt, None, H.GELU, dx=torch.empty_like(x))
    with pytest.raises(G.GoshError, match="xt is null"):
        G.gosh_linear_fp8_backward(y, None, wt, None, dw=torch.empty(16, 32, device=DEV))
    with pytest.raises(G.GoshError, match="gosh_linear_backward gives db"):
        G.gosh_linear_fp8_backward(y, xt, wt, None, db=torch.empty(16, device=DEV))
    with pytest.raises(G.GoshError, match="workspace"):
        G.gosh_linear_fp8_backward(y, xt, wt, y, H.GELU, dx=torch.empty_like(x), workspace=torch.empty(64, dtype=torch.uint8, device=DEV))
    short = G.PackedFp8(16, 32, 1, DEV)
    short.q = torch.zeros(1, 128, dtype=torch.uint8, device=DEV).view(torch.float8_e4m3fn).expand(16, 128)
    with pytest.raises(G.GoshError, match="ld"):
        G.gosh_linear_fp8(x, x8, short, y)
    torch.cuda.synchronize()
