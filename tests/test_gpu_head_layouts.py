"""The head's operators on matrices laid out in ways that Packed8 and ordinary tensors are not: rows as close to each other
as the entry points allow, of fewer entries than a load fetches, with bounds from head_model.py."""
import ctypes as C
import math

import pytest
import torch

import paper_2008_12336_amd as G
from tests import head_model as H
from tests.test_gpu_head import DEV, NAMES, gen, types, within

pytestmark = pytest.mark.gpu


class Eight:
    """An 8-bit form with rows `ld` bytes and their exponents `ld_exps` bytes apart, `off` bytes off the start of memory
    that holds 99 besides."""

    def __init__(self, rows, cols, dtype, ld, ld_exps, off=0):
        groups = -(-cols // 32)
        self.cols = cols
        self.bytes = torch.full((off + (rows - 1) * ld + cols + 8,), 99, dtype=torch.int8, device=DEV)
        self.units = torch.full((off + (rows - 1) * ld_exps + groups + 8,), 99, dtype=torch.uint8, device=DEV)
        self.q = torch.as_strided(self.bytes, (rows, cols), (ld, 1), off)
        self.exps = torch.as_strided(self.units, (rows, groups), (ld_exps, 1), off)
        kind = {torch.float32: G.GOSH_F32, torch.bfloat16: G.GOSH_BF16, torch.float16: G.GOSH_F16}[dtype]
        self.mat = G.gosh_mat(self.q.data_ptr(), self.exps.data_ptr(), rows, ld, ld_exps, cols, kind, 1)

    def values(self):
        return H.values(self.q.cpu(), self.exps.cpu()).to(DEV)

    def beside(self):
        """Memory beside the matrix holds 99 still."""
        self.q.fill_(99), self.exps.fill_(99)
        assert (self.bytes == 99).all() and (self.units == 99).all()


def mat(t):
    """A tensor's view, whatever its strides."""
    kind = {torch.float32: G.GOSH_F32, torch.bfloat16: G.GOSH_BF16, torch.float16: G.GOSH_F16}[t.dtype]
    return G.gosh_mat(t.data_ptr(), None, t.shape[0], t.stride(0), 0, t.shape[1], kind, 0)


def check(rc):
    assert rc == 0, G.gosh_last_error()


def pack(x, p):
    check(G.lib().gosh_pack8(C.byref(mat(x)), C.byref(p.mat), torch.cuda.current_stream().cuda_stream))


def backward(dy, x, w, dx, dw, db):
    """The gradient of a layer without an activation; x: a view."""
    kind = mat(dy).type
    n = G.gosh_linear_backward_workspace(dy.shape[0], w.shape[1], w.shape[0], kind, H.NONE)
    work = torch.empty(n, dtype=torch.uint8, device=DEV)
    check(G.lib().gosh_linear_backward(C.byref(mat(dy)), C.byref(x), C.byref(mat(w)), None, H.NONE,
                                       None if dx is None else C.byref(mat(dx)), C.byref(mat(dw)), db.data_ptr(),
                                       work.data_ptr(), n, torch.cuda.current_stream().cuda_stream))


@types
@pytest.mark.parametrize("rows", [33, 34, 35, 65, 66, 67, 129, 577])
def test_gradient_of_few_columns_without_padding(rows, dtype):
    """Rows of fewer bytes than a load, in matrices that end with them: what a load reaches past its row lies in the rows
    after it, of which the last step of the sum may hold one.  Bounds as in test_linear_backward."""
    for k, n, more in ((1, 1, 0), (1, 5, 1), (1, 64, 2), (2, 3, 0), (2, 8, 1), (3, 1, 0), (5, 7, 0), (7, 2, 0), (6, 4, 1)):
        rnd = gen(rows * 64 + k * 8 + n)
        x, w, dy = rnd(rows, k).to(dtype), rnd(n, k).to(dtype), (0.1 * rnd(rows, n)).to(dtype)
        p = Eight(rows, k, dtype, k + more, 1)
        pack(x, p)
        for name, view, open_ in (("x", mat(x), x.double()), ("packed x", p.mat, p.values())):
            want, bounds = H.linear_backward(dy.double(), open_, w.double(), None, H.NONE, dtype)
            for with_dx in (True, False):
                dx = torch.empty(rows, k, dtype=dtype, device=DEV) if with_dx else None
                dw, db = torch.empty(n, k, device=DEV), torch.empty(n, device=DEV)
                backward(dy, view, w, dx, dw, db)
                what = f"{rows} x {k} -> {n}, {name} with rows {view.ld} apart, {NAMES[dtype]}"
                within(dw, want[1], H.rounded(bounds[1], want[1], torch.float32), f"dw of {what}")
                within(db, want[2], H.rounded(bounds[2], want[2], torch.float32), f"db of {what}")
                if with_dx:
                    within(dx, want[0], H.rounded(bounds[0], want[0], dtype), f"dx of {what}")
        p.beside()


@types
@pytest.mark.parametrize("rows", [0, 1, 700, 20011])
def test_the_bias_gradient_alone(rows, dtype):
    """db without dx and dw, with and without the operands that only those need; the same bits as beside them."""
    k, n = 40, 77
    rnd = gen(rows + 5)
    x, w = rnd(rows, k).to(dtype), rnd(n, k).to(dtype)
    dy, z = (0.1 * rnd(rows, n)).to(dtype), (2 * rnd(rows, n)).to(dtype)
    z8 = G.Packed8(rows, n, dtype, DEV)
    G.gosh_pack8(z, z8)
    for kind, zz in ((H.NONE, None), (H.RELU, z), (H.GELU, z8), (H.SILU, z)):
        full, dw = torch.empty(n, device=DEV), torch.empty_like(w)
        G.gosh_linear_backward(dy, x, w, zz, kind, dw=dw, db=full)
        open_ = z8 if zz is z8 else None
        z64 = z.double() if open_ is None else H.values(z8.q[:, :n].cpu(), z8.exps.cpu()).to(DEV)
        want, bounds = H.linear_backward(dy.double(), x.double(), w.double(), z64, kind, dtype)
        for xx, ww in ((x, w), (x, None), (None, w), (None, None)):
            db = torch.full((n,), 77.0, device=DEV)
            G.gosh_linear_backward(dy, xx, ww, zz, kind, db=db)
            within(db, want[2], H.rounded(bounds[2], want[2], torch.float32), f"db alone, activation {kind}")
            assert torch.equal(db, full)


def test_an_8_bit_form_that_was_moved():
    """Saved activations that went to the host and back, while other data took their place: calls use the new tensors."""
    rnd = gen(12)
    x, out = rnd(300, 70), torch.empty(300, 70, device=DEV)
    p = G.Packed8(300, 70, torch.float32, DEV)
    G.gosh_pack8(x, p)
    want = H.values(p.q[:, :70].cpu(), p.exps.cpu())
    old = p.q, p.exps
    p.q, p.exps = p.q.cpu(), p.exps.cpu()
    with pytest.raises(G.GoshError, match="not memory"):
        G.gosh_unpack8(p, out)
    p.q, p.exps = p.q.to(DEV), p.exps.to(DEV)
    old[0].fill_(1), old[1].fill_(1)
    G.gosh_unpack8(p, out)
    assert torch.equal(out.double().cpu(), want)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=lambda t: NAMES[t])
@pytest.mark.parametrize("rows", [1, 63, 64, 200, 1000, 4000])
def test_a_split_dx_of_rows_off_alignment(rows, dtype):
    """dx whose long sum is split, of aligned rows and of others, which are planned alike and stored in the same tiles."""
    k, n = 96, 2056
    rnd = gen(rows + 9)
    dy, w = (0.1 * rnd(rows, n)).to(dtype), (rnd(n, k) / math.sqrt(k)).to(dtype)
    for pad in (0, 1):
        dys, ws = torch.zeros(rows, n + pad, dtype=dtype, device=DEV)[:, :n], torch.zeros(n, k + pad, dtype=dtype, device=DEV)[:, :k]
        dys.copy_(dy), ws.copy_(w)
        dx = torch.full((rows, k), 77.0, dtype=dtype, device=DEV)
        G.gosh_linear_backward(dys, None, ws, None, H.NONE, dx=dx)
        want, bounds = H.linear_backward(dy.double(), torch.zeros(rows, k, device=DEV).double(), w.double(), None, H.NONE, dtype)
        within(dx, want[0], H.rounded(bounds[0], want[0], dtype), f"dx, rows {pad} entries apart")


@pytest.mark.parametrize("exponent", [-108, -112, -116, -120, -126, -131])
def test_small_entries_in_32_bits(exponent):
    """Entries of 32 bits down to the least ones.  From 2^-110 on the tiles' three bf16 parts hold an entry wholly; below,
    what is left is at most 2^-134, half of the least bf16 number, and the products that are left out are under 2^-8 of
    that: 1.01 * 2^-134 times the other operand.  A few rows are multiplied as they are.  The other operand is large, so
    that no result is near the end of the range."""
    k, n, least = 96, 64, 1.01 * 2.0 ** -134
    for rows in (5, 3000):
        rnd = gen(rows - exponent)
        x, w = rnd(rows, k) * 2.0 ** exponent, rnd(n, k) * 2.0 ** 40
        y = torch.empty(rows, n, device=DEV)
        G.gosh_linear(x, w, y)
        x64, w64 = x.double(), w.double()
        wy, _, ey, _ = H.linear(x64, w64, None, H.NONE, None)
        if rows > 1024:
            ey = ey + least * (x64.abs() < 2.0 ** -110).double() @ w64.abs().t()
        within(y, wy, H.rounded(ey, wy, torch.float32), f"y of {rows} rows")
        dy, big = rnd(rows, n) * 2.0 ** exponent, rnd(rows, k) * 2.0 ** 40
        dx, dw, db = torch.empty(rows, k, device=DEV), torch.empty(n, k, device=DEV), torch.empty(n, device=DEV)
        G.gosh_linear_backward(dy, big, w, None, H.NONE, dx=dx, dw=dw, db=db)
        want, bounds = H.linear_backward(dy.double(), big.double(), w64, None, H.NONE, torch.float32)
        small = least * (dy.double().abs() < 2.0 ** -110).double()
        within(dx, want[0], H.rounded(bounds[0] + small @ w64.abs(), want[0], torch.float32), f"dx of {rows} rows")
        within(dw, want[1], H.rounded(bounds[1] + small.t() @ big.double().abs(), want[1], torch.float32), f"dw of {rows} rows")
        within(db, want[2], H.rounded(bounds[2], want[2], torch.float32), f"db of {rows} rows")


@types
@pytest.mark.parametrize("rows, cols, more, more_exps, off", [(5, 33, 0, 0, 1), (130, 70, 3, 2, 5), (64, 96, 32, 5, 3), (300, 264, 1, 1, 7)])
def test_8_bit_forms_of_any_strides(rows, cols, more, more_exps, off, dtype):
    """8-bit forms whose rows, exponents and starts lie anywhere: all calls that write one give the bytes of an ordinary one
    and leave the memory beside it, and all that read one give the same bits."""
    rnd = gen(rows + cols)
    new = lambda: Eight(rows, cols, dtype, cols + more, -(-cols // 32) + more_exps, off)  # noqa: E731
    usual = lambda: G.Packed8(rows, cols, dtype, DEV)  # noqa: E731
    x, w = rnd(rows, cols).to(dtype), (rnd(cols, cols) / math.sqrt(cols)).to(dtype)
    gamma, beta = 1 + 0.1 * rnd(cols), 0.1 * rnd(cols)
    y, rstd = torch.empty_like(x), torch.empty(rows, device=DEV)
    p, forms = usual(), []

    def odd(q):
        """The Packed8 that holds an Eight's memory."""
        o = usual()
        o.q, o.exps = q.q, q.exps
        return o

    for call in (lambda q: G.gosh_pack8(x, q), lambda q: G.gosh_layer_norm(x, gamma, beta, y, rstd=rstd, xhat8=q),
                 lambda q: G.gosh_layer_norm(x, gamma, beta, y, y8=q), lambda q: G.gosh_linear(x, w, y, act=H.GELU, z=q),
                 lambda q: G.gosh_linear(x, w, y, act=H.GELU, y8=q)):
        q = new()
        call(p)
        call(odd(q))
        assert torch.equal(q.q, p.q[:, :cols]) and torch.equal(q.exps, p.exps)
        again = new()
        again.q.copy_(q.q), again.exps.copy_(q.exps)
        q.beside()
        forms.append(odd(again))
    G.gosh_layer_norm(x, gamma, beta, y, rstd=rstd, xhat8=p)
    xhat, z = forms[1], forms[3]
    usual_z = usual()
    G.gosh_linear(x, w, y, act=H.GELU, z=usual_z)
    dy = (0.1 * rnd(rows, cols)).to(dtype)
    got = []
    for hat, pre in ((xhat, z), (p, usual_z)):
        dx, dh, dw = torch.empty_like(x), torch.empty_like(x), torch.empty_like(w)
        db, dg, dn = (torch.empty(cols, device=DEV) for _ in range(3))
        G.gosh_linear_backward(dy, hat, w, pre, H.GELU, dx=dh, dw=dw, db=db)
        G.gosh_layer_norm_backward(dh, hat, gamma, None, rstd, dx, dgamma=dg, dbeta=dn)
        back = torch.empty_like(x)
        G.gosh_unpack8(pre, back)
        got.append((dx, dh, dw, db, dg, dn, back))
    assert all(torch.equal(a, b) for a, b in zip(*got))


@types
@pytest.mark.parametrize("into", H.TYPES, ids=lambda t: NAMES[t])
def test_unpacking_into_another_type(into, dtype):
    """What an 8-bit form stands for is rounded once, to the type that it is read into."""
    rnd = gen(31)
    x = (rnd(200, 75) * torch.exp2(torch.round(8 * rnd(200, 1)))).to(dtype)
    x[7, 3], x[9, 70] = math.nan, 0.0
    p = G.Packed8(200, 75, dtype, DEV)
    G.gosh_pack8(x, p)
    out = torch.empty(200, 75, dtype=into, device=DEV)
    G.gosh_unpack8(p, out)
    want = H.values(p.q[:, :75].cpu(), p.exps.cpu()).to(into)
    assert torch.equal(torch.nan_to_num(out.cpu().double(), nan=0.123, posinf=1e300, neginf=-1e300),
                       torch.nan_to_num(want.double(), nan=0.123, posinf=1e300, neginf=-1e300))


def test_a_placed_matrix_as_operand():
    """Matrices of gosh_matrix_place, which lie in several mappings, are operands as others are."""
    n, d = 1 << 16, 128
    M, _ = G.gosh_matrix_place(n, d, arena_bytes=6 << 30)
    rnd = gen(2)
    x = rnd(n, d)
    M.copy_(x)
    w, gamma, beta = rnd(48, d) / 10, 1 + 0.1 * rnd(d), 0.1 * rnd(d)
    got = []
    for m in (M, x):
        y, p = torch.empty(n, 48, device=DEV), G.Packed8(n, d, torch.float32, DEV)
        G.gosh_linear(m, w, y)
        G.gosh_pack8(m, p)
        dw = torch.empty_like(w)
        G.gosh_linear_backward(y, m, None, None, dw=dw)
        G.gosh_layer_norm(m, gamma, beta, m)
        got.append((y, p.q, p.exps, dw, m.clone()))
    torch.cuda.synchronize()
    same = [torch.equal(a, b) for a, b in zip(*got)]
    G.gosh_matrix_release(M)
    assert all(same)


@pytest.mark.parametrize("dtype, k", [(torch.bfloat16, 8), (torch.float16, 3), (torch.float32, 1)], ids=["aligned", "not", "f32"])
def test_more_rows_than_a_launch_takes(dtype, k):
    """2^28 rows are the most that one launch has tiles for: what follows is the same layer on the rows from there."""
    rows, n, edge = (1 << 28) + 777, 5, 1 << 28
    at = torch.cat((torch.arange(50), torch.arange(edge - 50, edge + 50), torch.arange(rows - 50, rows))).to(DEV)
    rnd = gen(k)
    x, r, y = (torch.zeros(rows, c, dtype=dtype, device=DEV) for c in (k, n, n))
    x[at], r[at] = rnd(at.numel(), k).to(dtype), rnd(at.numel(), n).to(dtype)
    w, b = rnd(n, k).to(dtype), rnd(n)
    z8, y8 = (G.Packed8(0, n, dtype, DEV) for _ in range(2))
    for p in (z8, y8):
        p.rows = rows
        p.q, p.exps = torch.zeros(rows, n, dtype=torch.int8, device=DEV), torch.zeros(rows, 1, dtype=torch.uint8, device=DEV)
    G.gosh_linear(x, w, y, bias=b, act=H.SILU, residual=r, z=z8, y8=y8)
    few, one, two = torch.empty(at.numel(), n, dtype=dtype, device=DEV), G.Packed8(at.numel(), n, dtype), G.Packed8(at.numel(), n, dtype)
    G.gosh_linear(x[at], w, few, bias=b, act=H.SILU, residual=r[at], z=one, y8=two)
    assert torch.equal(y[at], few)
    for p, q in ((z8, one), (y8, two)):
        assert torch.equal(p.q[at], q.q[:, :n]) and torch.equal(p.exps[at], q.exps)
    other = torch.ones(rows, dtype=torch.bool, device=DEV)
    other[at] = False
    plain = y[60]  # a row of zeros
    assert bool(((y == plain).all(dim=1) | ~other).all())
    del other, z8, y8
    dx = torch.full((rows, k), 77.0, dtype=dtype, device=DEV)
    G.gosh_linear_backward(r, None, w, None, H.NONE, dx=dx)
    want = torch.empty(at.numel(), k, dtype=dtype, device=DEV)
    G.gosh_linear_backward(r[at], None, w, None, H.NONE, dx=want)
    assert torch.equal(dx[at], want)
    assert bool((dx == 0).all(dim=1).sum() >= rows - at.numel())
