"""gosh_linear, gosh_layer_norm, the 8-bit form and their gradients against 64-bit arithmetic, with bounds derived in
head_model.py: every type, odd sizes and strides, views that start off alignment, rows of one and none, memory beside the
outputs, in-place use, what is not finite, other streams, captured graphs and offsets past 32 bits."""
import math

import pytest
import torch

import paper_2008_12336_amd as G
from tests import head_model as H

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
NAMES = {torch.float32: "f32", torch.bfloat16: "bf16", torch.float16: "f16"}
MARK = 77.0


def types(fn):
    return pytest.mark.parametrize("dtype", H.TYPES, ids=lambda t: NAMES[t])(fn)


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return lambda *shape: torch.randn(*shape, generator=g, device=DEV)


def view(values, dtype, pad, off):
    """A matrix with `values` inside memory full of MARK: rows `pad` entries apart from each other, `off` from the start."""
    rows, cols = values.shape
    memory = torch.full((off + (rows + 1) * (cols + pad) + 8,), MARK, device=DEV).to(dtype)
    m = memory[off:off + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    m.copy_(values)
    return m, memory


def beside(m, memory):
    """Memory beside the matrix holds MARK still."""
    m.fill_(MARK)
    assert (memory == MARK).all()


def within(got, want, bound, what):
    got, want, bound = got.double(), want.double(), bound.double()
    assert torch.isfinite(got).all(), what
    over = ((got - want).abs() - bound).max().item() if got.numel() else -1
    ratio = ((got - want).abs() / bound.clamp(min=1e-300)).max().item() if got.numel() else 0
    print(f"{what}: largest error {ratio:.3f} of its bound", flush=True)
    assert over <= 0, (what, ratio)


def packed_within(p, want, bound, what):
    """An 8-bit form of values known to `bound`: half a unit off, and a unit is under 2/127 of the group's largest."""
    got = H.values(p.q[:, :p.cols].cpu(), p.exps.cpu()).to(want.device)
    most = H.group_most(want.abs() + bound)
    within(got, want, bound + most / 127 * (1 + 1e-6) + 2.0 ** (-25 if p.dtype == torch.float16 else -127), what)


SHAPES = [  # rows, in, out, padding of the rows, entries off the start of memory
    (1, 1, 1, 0, 0), (1, 512, 2048, 0, 0), (2, 37, 5, 3, 1), (7, 130, 33, 0, 1), (8, 64, 257, 1, 0), (9, 8, 1, 0, 0),
    (33, 3, 40, 5, 3), (64, 64, 64, 0, 0), (129, 260, 130, 0, 0), (200, 17, 517, 2, 1), (300, 1024, 96, 8, 8),
    (1000, 132, 31, 0, 0), (20000, 72, 260, 0, 0), (16391, 128, 384, 0, 0), (33001, 64, 264, 0, 0),
    (90, 97, 1844, 0, 0),
]


@types
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_linear(shape, dtype):
    rows, k, n, pad, off = shape
    rnd = gen(rows * 31 + k)
    x, _ = view(rnd(rows, k), dtype, pad, off)
    w, _ = view(rnd(n, k) / math.sqrt(k), dtype, pad, off)
    b, r = 0.3 * rnd(n), view(rnd(rows, n), dtype, pad, off)[0]
    for kind in (H.NONE, H.RELU, H.GELU, H.SILU):
        use_b, use_r = kind != H.RELU, kind in (H.NONE, H.GELU)
        y, ymem = view(torch.zeros(rows, n, device=DEV), dtype, pad, off)
        z, zmem = view(torch.zeros(rows, n, device=DEV), dtype, pad, off)
        G.gosh_linear(x, w, y, bias=b if use_b else None, act=kind, residual=r if use_r else None,
                      z=z if kind != H.SILU else None)
        wy, wz, ey, ez = H.linear(x.double(), w.double(), b.double() if use_b else None, kind, r.double() if use_r else None)
        within(y, wy, H.rounded(ey, wy, dtype), f"y, activation {kind}")
        if kind != H.SILU:
            within(z, wz, H.rounded(ez, wz, dtype), f"z, activation {kind}")
        beside(y, ymem)
        if kind != H.SILU:
            beside(z, zmem)
    # 8-bit outputs
    y, ymem = view(torch.zeros(rows, n, device=DEV), dtype, pad, off)
    z8, y8 = G.Packed8(rows, n, dtype, DEV), G.Packed8(rows, n, dtype, DEV)
    for p in (z8, y8):
        p.q.fill_(99), p.exps.fill_(99)
    G.gosh_linear(x, w, y, bias=b, act=H.SILU, residual=r, z=z8, y8=y8)
    wy, wz, ey, ez = H.linear(x.double(), w.double(), b.double(), H.SILU, r.double())
    within(y, wy, H.rounded(ey, wy, dtype), "y beside 8-bit outputs")
    packed_within(z8, wz, ez, "z8")
    packed_within(y8, wy, ey, "y8")
    for p in (z8, y8):
        assert (p.q[:, n:] == 99).all()
    beside(y, ymem)


@types
@pytest.mark.parametrize("shape", [s for s in SHAPES if s[0] * s[1] * s[2] < 3e8], ids=lambda s: "x".join(map(str, s)))
def test_linear_backward(shape, dtype):
    rows, k, n, pad, off = shape
    rnd = gen(rows * 37 + n)
    x, _ = view(rnd(rows, k), dtype, pad, off)
    w, _ = view(rnd(n, k) / math.sqrt(k), dtype, pad, off)
    dy, _ = view(0.1 * rnd(rows, n), dtype, pad, off)
    z, _ = view(2 * rnd(rows, n), dtype, pad, off)
    z8, x8 = G.Packed8(rows, n, dtype, DEV), G.Packed8(rows, k, dtype, DEV)
    G.gosh_pack8(z, z8)
    G.gosh_pack8(x, x8)
    for kind, zz, xx in ((H.NONE, None, x), (H.RELU, z, x8), (H.GELU, z8, x), (H.SILU, z8, x8), (H.SILU, z, x)):
        dx, xmem = view(torch.zeros(rows, k, device=DEV), dtype, pad, off)
        wide = kind in (H.NONE, H.GELU)  # dw in 32 bits
        dw, wmem = view(torch.zeros(n, k, device=DEV), torch.float32 if wide else dtype, pad, off)
        db = torch.full((n,), MARK, device=DEV)
        G.gosh_linear_backward(dy, xx, w, zz, kind, dx=dx, dw=dw, db=db)
        open_ = lambda m: (H.values(m.q[:, :m.cols].cpu(), m.exps.cpu()).to(DEV) if isinstance(m, G.Packed8)  # noqa: E731
                           else None if m is None else m.double())
        want, bounds = H.linear_backward(dy.double(), open_(xx), w.double(), open_(zz), kind, dtype)
        within(dx, want[0], H.rounded(bounds[0], want[0], dtype), f"dx, activation {kind}")
        within(dw, want[1], H.rounded(bounds[1], want[1], dw.dtype), f"dw, activation {kind}")
        within(db, want[2], H.rounded(bounds[2], want[2], torch.float32), f"db, activation {kind}")
        one, again = torch.empty_like(dw), torch.empty_like(db)
        G.gosh_linear_backward(dy, xx, None, zz, kind, dw=one, db=again)  # each by itself, and the same bits again
        assert torch.equal(one, dw) and torch.equal(again, db)
        alone = torch.empty_like(dx)
        G.gosh_linear_backward(dy, None, w, zz, kind, dx=alone)
        assert torch.equal(alone, dx)
        beside(dx, xmem)
        beside(dw, wmem)


@types
@pytest.mark.parametrize("shape", [(20011, 512, 1024, 0, 0), (20011, 512, 1024, 8, 1)], ids=["aligned", "not"])
def test_many_rows(shape, dtype):
    """Largest tiles, more of them than the device holds at once, and sums that are split."""
    test_linear(shape, dtype)
    test_linear_backward(shape, dtype)


@types
@pytest.mark.parametrize("pad", [0, 8])
def test_results_larger_than_the_caches(pad, dtype):
    rows, k, n = 65281, 40, 2056
    rnd = gen(rows + pad)
    x, _ = view(rnd(rows, k), dtype, pad, pad)
    w, _ = view(rnd(n, k) / math.sqrt(k), dtype, pad, pad)
    b, r = 0.3 * rnd(n), view(rnd(rows, n), dtype, pad, pad)[0]
    for kind, use_r in ((H.GELU, False), (H.SILU, True), (H.RELU, True), (H.NONE, False)):
        y, ymem = view(torch.zeros(rows, n, device=DEV), dtype, pad, pad)
        G.gosh_linear(x, w, y, bias=b, act=kind, residual=r if use_r else None)
        wy, _, ey, _ = H.linear(x.double(), w.double(), b.double(), kind, r.double() if use_r else None)
        within(y, wy, H.rounded(ey, wy, dtype), f"y, activation {kind}")
        again = r.clone()
        G.gosh_linear(x, w, again, bias=b, act=kind, residual=again if use_r else None)  # in place, and the same bits
        assert torch.equal(again, y)
        beside(y, ymem)


NORMS = [  # rows, cols, padding, off the start
    (1, 1, 0, 0), (1, 128, 0, 0), (5, 2, 1, 1), (64, 8, 0, 0), (63, 31, 0, 1), (100, 33, 2, 0), (1000, 96, 0, 0),
    (257, 128, 8, 8), (70, 501, 0, 0), (33, 512, 0, 3), (20, 1000, 1, 0), (9, 2048, 0, 0), (5, 2049, 0, 1), (6, 4100, 0, 0),
    (3, 8192, 0, 0), (4, 8200, 0, 0), (2, 9001, 3, 1), (70001, 64, 0, 0),
]


@types
@pytest.mark.parametrize("shape", NORMS, ids=lambda s: "x".join(map(str, s)))
def test_layer_norm_and_its_gradient(shape, dtype):
    rows, k, pad, off = shape
    rnd = gen(rows * 41 + k)
    eps = 1e-5
    x, _ = view(rnd(rows, k) * torch.exp(rnd(rows, 1)) + rnd(rows, 1), dtype, pad, off)
    gamma, beta = 1 + 0.3 * rnd(k), 0.2 * rnd(k)
    y, ymem = view(torch.zeros(rows, k, device=DEV), dtype, pad, off)
    mean, rstd = torch.full((rows,), MARK, device=DEV), torch.full((rows,), MARK, device=DEV)
    xhat8, y8 = G.Packed8(rows, k, dtype, DEV), G.Packed8(rows, k, dtype, DEV)
    G.gosh_layer_norm(x, gamma, beta, y, mean=mean, rstd=rstd, eps=eps, xhat8=xhat8, y8=y8)
    want, bound = H.norm(x.double(), gamma.double(), beta.double(), eps)
    within(y, want[0], H.rounded(bound[0], want[0], dtype), "y")
    within(mean, want[1], H.rounded(bound[1], want[1], torch.float32), "mean")
    within(rstd, want[2], H.rounded(bound[2], want[2], torch.float32), "rstd")
    packed_within(xhat8, want[3], bound[3], "xhat8")
    packed_within(y8, want[0], bound[0], "y8")
    beside(y, ymem)
    y2 = x.clone()
    G.gosh_layer_norm(y2, gamma, beta, y2, eps=eps)  # in place, nothing else
    within(y2, want[0], H.rounded(bound[0], want[0], dtype), "y in place")

    dy, _ = view(0.1 * rnd(rows, k), dtype, pad, off)
    add, _ = view(0.1 * rnd(rows, k), dtype, pad, off)
    stood_for = H.values(xhat8.q[:, :k].cpu(), xhat8.exps.cpu()).to(DEV)
    m64, r64 = mean.double(), rstd.double()
    xhat = (x.double() - m64[:, None]) * r64[:, None]
    off32 = H.F32 * ((x.double().abs() + m64.abs()[:, None]) * r64[:, None] + xhat.abs())
    for name, from_, mm, hat, ehat, a in (("x", x, mean, xhat, off32, add), ("xhat8", xhat8, None, stood_for, torch.zeros_like(xhat), None)):
        dx, xmem = view(torch.zeros(rows, k, device=DEV), dtype, pad, off)
        dgamma, dbeta = torch.full((k,), MARK, device=DEV), torch.full((k,), MARK, device=DEV)
        G.gosh_layer_norm_backward(dy, from_, gamma, mm, rstd, dx, dgamma=dgamma, dbeta=dbeta, add=a)
        want, bound = H.norm_backward(dy.double(), hat, gamma.double(), r64, None if a is None else a.double(), ehat)
        within(dx, want[0], H.rounded(bound[0], want[0], dtype), f"dx from {name}")
        within(dgamma, want[1], H.rounded(bound[1], want[1], torch.float32), f"dgamma from {name}")
        within(dbeta, want[2], H.rounded(bound[2], want[2], torch.float32), f"dbeta from {name}")
        g2, b2, into = torch.empty_like(dgamma), torch.empty_like(dbeta), dy.clone()
        G.gosh_layer_norm_backward(into, from_, gamma, mm, rstd, into, dgamma=g2, dbeta=b2, add=a)  # dx over dy
        assert torch.equal(into, dx) and torch.equal(g2, dgamma) and torch.equal(b2, dbeta)
        if a is not None:
            into = a.clone()
            G.gosh_layer_norm_backward(dy, from_, gamma, mm, rstd, into, add=into)  # dx over add, no sums
            assert torch.equal(into, dx)
        G.gosh_layer_norm_backward(dy, from_, gamma, mm, rstd, None, dgamma=g2, dbeta=b2)  # the sums alone
        assert torch.equal(g2, dgamma) and torch.equal(b2, dbeta)
        beside(dx, xmem)


@types
@pytest.mark.parametrize("shape", [(1, 1, 0, 0), (3, 31, 0, 1), (40, 32, 0, 0), (17, 33, 3, 1), (64, 200, 0, 0)],
                         ids=lambda s: "x".join(map(str, s)))
def test_eight_bits_entry_by_entry(shape, dtype):
    rows, k, pad, off = shape
    rnd = gen(rows + k)
    v = rnd(rows, k) * torch.exp2(torch.round(6 * rnd(rows, 1)))
    top = torch.finfo(dtype).max
    edge = [0.0, top, -top, torch.finfo(dtype).tiny, math.inf, -math.inf, math.nan, 127.0, 127.5, -128.0, 0.5, 1.5, 2.5]
    for i, e in enumerate(edge):
        if rows > 3:
            v[i % rows, (5 * i) % k] = e
    if rows > 20:
        v[15] = 0
        v[16] *= 1e-38 if dtype != torch.float16 else 1e-6
    x, _ = view(v, dtype, pad, off)
    p = G.Packed8(rows, k, dtype, DEV)
    p.q.fill_(99)
    G.gosh_pack8(x, p)
    q, exps = H.eight_bits(x.double().cpu(), dtype)
    assert torch.equal(p.exps.cpu().long(), exps)
    assert torch.equal(p.q[:, :k].cpu().long(), q)
    assert (p.q[:, k:] == 99).all()
    out, mem = view(torch.zeros(rows, k, device=DEV), dtype, pad, off)
    G.gosh_unpack8(p, out)
    want = H.values(q, exps)
    assert torch.equal(torch.nan_to_num(out.double().cpu(), nan=123.25), torch.nan_to_num(want, nan=123.25))
    beside(out, mem)


@types
def test_rows_of_none(dtype):
    e = lambda n, t=dtype: torch.empty(0, n, dtype=t, device=DEV)  # noqa: E731
    w, b = torch.randn(5, 7, device=DEV).to(dtype), torch.randn(5, device=DEV)
    G.gosh_linear(e(7), w, e(5), bias=b, act=H.GELU, z=G.Packed8(0, 5, dtype, DEV))
    dw, db = torch.full((5, 7), MARK, device=DEV).to(dtype), torch.full((5,), MARK, device=DEV)
    G.gosh_linear_backward(e(5), e(7), w, e(5), H.GELU, dx=e(7), dw=dw, db=db)
    assert (dw == 0).all() and (db == 0).all()
    g = torch.ones(7, device=DEV)
    G.gosh_layer_norm(e(7), g, g, e(7), mean=torch.empty(0, device=DEV), rstd=torch.empty(0, device=DEV))
    dg, dn = torch.full((7,), MARK, device=DEV), torch.full((7,), MARK, device=DEV)
    s = torch.empty(0, device=DEV)
    G.gosh_layer_norm_backward(e(7), e(7), g, s, s, e(7), dgamma=dg, dbeta=dn)
    assert (dg == 0).all() and (dn == 0).all()
    G.gosh_pack8(e(7), G.Packed8(0, 7, dtype, DEV))


@types
@pytest.mark.parametrize("rows", [5, 300])
def test_what_is_not_finite_stays_in_its_rows(rows, dtype):
    """A row of x that holds NaN or an infinity spoils its own results, all of them, and no others; padding of the tiles
    does not multiply what lies beside the operands."""
    rnd = gen(rows)
    k, n = 70, 45
    x, _ = view(rnd(rows, k), dtype, 3, 1)
    x[2, 69], x[4, 0] = math.nan, math.inf
    w, memory = view(rnd(n, k), dtype, 3, 1)
    memory[:1] = math.nan
    hole = memory[1:1 + n * (k + 3)].view(n, k + 3)[:, k:]
    hole.fill_(math.nan)
    y, z8 = torch.empty(rows, n, device=DEV, dtype=dtype), G.Packed8(rows, n, dtype, DEV)
    G.gosh_linear(x, w, y, act=H.RELU, z=z8)
    fine = torch.ones(rows, dtype=torch.bool, device=DEV)
    fine[2] = fine[4] = False
    assert torch.isfinite(y[fine]).all()
    assert torch.isnan(y[2]).all()
    assert (z8.exps[2] == 255).all() and (z8.exps[4] == 255).all() and (z8.exps[fine] != 255).all()
    if dtype != torch.float32:  # relu of an infinity of either sign
        assert torch.equal(y[4] != 0, w[:, 0] > 0) and torch.isinf(y[4][w[:, 0] > 0]).all()
    dx = torch.empty(rows, n, dtype=dtype, device=DEV)
    g = torch.ones(n, device=DEV)
    mean, rstd = torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)
    G.gosh_layer_norm(y, g, g, dx, mean=mean, rstd=rstd)
    assert torch.isfinite(dx[fine]).all() and torch.isnan(dx[2]).all()


def test_rows_of_equal_entries():
    """No variance: xhat is 0 with eps and everything stays finite; gradients are those of rstd = 1 / sqrt(eps)."""
    x = torch.full((6, 40), 3.25, device=DEV)
    g, b = torch.full((40,), 2.0, device=DEV), torch.full((40,), 0.5, device=DEV)
    y, mean, rstd = torch.empty_like(x), torch.empty(6, device=DEV), torch.empty(6, device=DEV)
    G.gosh_layer_norm(x, g, b, y, mean=mean, rstd=rstd, eps=1e-5)
    assert (y == 0.5).all() and (mean == 3.25).all()
    assert torch.allclose(rstd, torch.full_like(rstd, 1e-5 ** -0.5), rtol=1e-6)
    dx = torch.empty_like(x)
    G.gosh_layer_norm_backward(torch.ones_like(x), x, g, mean, rstd, dx)
    assert (dx.abs() <= 40 * 2.0 ** -24 * 2 * 1e-5 ** -0.5).all()


@types
def test_in_place_residual(dtype):
    rnd = gen(3)
    for rows in (3, 150):
        x, w, r = rnd(rows, 40).to(dtype), rnd(50, 40).to(dtype), rnd(rows, 50).to(dtype)
        y = torch.empty_like(r)
        G.gosh_linear(x, w, y, act=H.SILU, residual=r)
        G.gosh_linear(x, w, r, act=H.SILU, residual=r)
        assert torch.equal(y, r)


def test_a_stream_of_its_own():
    """Work queued on another stream before the call is waited for, and the binding's workspace belongs to that stream."""
    rnd = gen(4)
    x, w, dy, z = rnd(4096, 256), rnd(512, 256), rnd(4096, 512), rnd(4096, 512)
    want = [torch.empty_like(x), torch.empty_like(w), torch.empty(512, device=DEV)]
    G.gosh_linear_backward(dy, x, w, z, H.GELU, dx=want[0], dw=want[1], db=want[2])
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for how in (side, side.cuda_stream):
        got = [torch.zeros_like(t) for t in want]
        late = torch.zeros_like(dy)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            for _ in range(20):
                late.add_(1).sub_(1)
            late.copy_(dy)
        G.gosh_linear_backward(late, x, w, z, H.GELU, dx=got[0], dw=got[1], db=got[2], stream=how)
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_a_captured_graph():
    """A step of layer norm, linear layer and both gradients, captured, replayed on changing inputs between eager calls."""
    rnd = gen(5)
    rows, k, n, t = 700, 96, 160, torch.bfloat16
    x, w, dy = rnd(rows, k).to(t), (rnd(n, k) / 10).to(t), rnd(rows, n).to(t)
    gamma, beta, bias = 1 + 0.1 * rnd(k), 0.1 * rnd(k), 0.1 * rnd(n)
    work = torch.empty(max(G.gosh_linear_backward_workspace(rows, k, n, G.GOSH_BF16, H.GELU),
                           G.gosh_layer_norm_workspace(rows, k)), dtype=torch.uint8, device=DEV)

    def buffers():
        f = lambda *s: torch.empty(*s, device=DEV)  # noqa: E731
        return dict(h=torch.empty_like(x), rstd=f(rows), y=torch.empty_like(dy), dh=torch.empty_like(x), dx=torch.empty_like(x),
                    dw=f(n, k), db=f(n), dg=f(k), dn=f(k), xhat8=G.Packed8(rows, k, t, DEV), h8=G.Packed8(rows, k, t, DEV),
                    z8=G.Packed8(rows, n, t, DEV))

    def step(o):
        G.gosh_layer_norm(x, gamma, beta, o["h"], rstd=o["rstd"], xhat8=o["xhat8"], y8=o["h8"])
        G.gosh_linear(o["h"], w, o["y"], bias=bias, act=H.GELU, z=o["z8"])
        G.gosh_linear_backward(dy, o["h8"], w, o["z8"], H.GELU, dx=o["dh"], dw=o["dw"], db=o["db"], workspace=work)
        G.gosh_layer_norm_backward(o["dh"], o["xhat8"], gamma, None, o["rstd"], o["dx"], dgamma=o["dg"], dbeta=o["dn"], workspace=work)

    held, eager = buffers(), buffers()
    step(held)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(held)
    for turn in range(4):
        x.copy_(rnd(rows, k))
        dy.copy_(rnd(rows, n))
        graph.replay()
        torch.cuda.synchronize()
        step(eager)
        torch.cuda.synchronize()
        for name in ("y", "dx", "dw", "db", "dg", "dn"):
            assert torch.equal(held[name], eager[name]), (turn, name)


def test_offsets_past_32_bits():
    """Matrices of more than 2^31 entries: their first and last rows, and a gradient that sums over all of them."""
    t, k = torch.bfloat16, 64
    rows = (1 << 31) // k + 77
    x = torch.zeros(rows, k, dtype=t, device=DEV)
    ends = torch.cat((torch.arange(40), torch.arange(rows - 40, rows))).to(DEV)
    rnd = gen(6)
    x[ends] = rnd(80, k).to(t)
    gamma, beta = 1 + 0.1 * rnd(k), 0.1 * rnd(k)
    y = torch.empty_like(x)
    mean, rstd = torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)
    G.gosh_layer_norm(x, gamma, beta, y, mean=mean, rstd=rstd)
    want, bound = H.norm(x[ends].double(), gamma.double(), beta.double(), 1e-5)
    within(y[ends], want[0], H.rounded(bound[0], want[0], t), "layer norm at the ends")
    p = G.Packed8(rows, k, t, DEV)
    G.gosh_pack8(x, p)
    y.zero_()
    G.gosh_unpack8(p, y)
    q, exps = H.eight_bits(x[ends].double().cpu(), t)
    assert torch.equal(y[ends].double().cpu(), H.values(q, exps))
    w = (rnd(k, k) / 8).to(t)
    G.gosh_linear(x, w, y)
    wy, _, ey, _ = H.linear(x[ends].double(), w.double(), None, H.NONE, None)
    within(y[ends], wy, H.rounded(ey, wy, t), "linear layer at the ends")
    # dy = y of which only the ends are not zero: dw is theirs alone
    dw, db = torch.empty(k, k, device=DEV), torch.empty(k, device=DEV)
    for from_ in (x, p):
        G.gosh_linear_backward(y, from_, w, None, H.NONE, dw=dw, db=db)
        at = x[ends].double() if from_ is x else H.values(q, exps).to(DEV)
        want, bound = H.linear_backward(y[ends].double(), at, w.double(), None, H.NONE, t)
        within(dw, want[1], H.rounded(bound[1], want[1], torch.float32), "dw over all rows")
        within(db, want[2], H.rounded(bound[2], want[2], torch.float32), "db over all rows")


def test_refusals_on_the_device():
    """What the runtime knows of the memory: spans that run past their allocation, host memory."""
    x, w, y = torch.zeros(64, 32, device=DEV), torch.zeros(16, 32, device=DEV), torch.zeros(64, 16, device=DEV)
    with pytest.raises(G.GoshError, match="w is 16 x 32: must be 16 x 31"):
        G.gosh_linear(x[:, :31], w, y)
    with pytest.raises(G.GoshError, match="y is"):
        G.gosh_linear(x, w, y[:, :15])
    with pytest.raises(G.GoshError, match="type"):
        G.gosh_linear(x, w.bfloat16(), y)
    with pytest.raises(G.GoshError, match="x is not memory"):
        G.gosh_linear(x.cpu(), w, y)
    with pytest.raises(G.GoshError, match="ld"):
        G.gosh_linear(x[:1].expand(64, 32), w, y)
    with pytest.raises(TypeError):
        G.gosh_linear(x.t(), w, y)
    with pytest.raises(TypeError):
        G.gosh_linear(x.double(), w, y)
    with pytest.raises(TypeError):
        G.gosh_linear(x, w, y, bias=torch.zeros(15, device=DEV))
    with pytest.raises(G.GoshError, match="act"):
        G.gosh_linear(x, w, y, act=4)
    with pytest.raises(G.GoshError, match="z is null"):
        G.gosh_linear_backward(y, x, w, None, H.GELU, dx=torch.empty_like(x))
    with pytest.raises(G.GoshError, match="workspace"):
        G.gosh_linear_backward(y, x, w, y, H.GELU, dx=torch.empty_like(x), workspace=torch.empty(64, dtype=torch.uint8, device=DEV))
    with pytest.raises(G.GoshError, match="must not be packed"):
        G.gosh_linear(G.Packed8(64, 32, torch.float32, DEV), w, y)
    s = torch.zeros(64, device=DEV)
    with pytest.raises(G.GoshError, match="mean is null"):
        G.gosh_layer_norm_backward(x, x, s[:32], None, s, torch.empty_like(x))
    with pytest.raises(G.GoshError, match="both or neither"):
        G.gosh_layer_norm_backward(x, x, s[:32], s, s, torch.empty_like(x), dgamma=torch.empty(32, device=DEV))
    with pytest.raises(G.GoshError, match="eps"):
        G.gosh_layer_norm(x, s[:32], s[:32], torch.empty_like(x), eps=-1.0)
    torch.cuda.synchronize()


def test_the_link_predictor_learns():
    """The example: a head trained on an embedding out of 8-bit activations tells held-out edges from other pairs."""
    from paper_2008_12336_amd.examples import link_head

    before, after, losses = link_head.train(scale=12, dim=32, steps=120, rows=8192)
    print(f"held-out AUC {before:.3f} -> {after:.3f}, loss {losses[0]:.3f} -> {losses[-1]:.3f}")
    assert after > 0.75 and after > before
    assert sum(losses[-10:]) < 0.9 * sum(losses[:10])
