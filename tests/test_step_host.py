"""Layers in 8-bit floating point, AdamW and the softmax loss without a GPU: refusals that need no device, sizes of workspaces
and states, and the formulas that the GPU tests compare with, against differences and against torch in 64 bits."""
import copy
import ctypes as C
import math
import pickle

import pytest
import torch

import paper_2008_12336_amd as G
from tests import head_model as H
from tests import step_model as S
from tests.test_head_host import mat, refused


def fp8(rows=0, cols=128, ld=None, ld_exps=None, block_rows=1, data=None, exps=None):
    wide = max(1, -(-max(cols, 0) // 128)) * 128
    return G.gosh_fp8(data, exps, rows, cols, wide if ld is None else ld, -(-wide // 512) * 4 if ld_exps is None else ld_exps, block_rows)


@pytest.mark.parametrize("bad, text", [
    (dict(block_rows=0), "block_rows"), (dict(block_rows=64), "block_rows"), (dict(rows=-1), "rows"), (dict(rows=2 ** 31 - 1), "rows"),
    (dict(cols=-1), "cols"), (dict(cols=G.GOSH_FP8_MAX_LD + 1), "cols"), (dict(ld=0), "ld"), (dict(ld=200), "ld"),
    (dict(ld=G.GOSH_FP8_MAX_LD + 128), "ld"), (dict(ld_exps=0), "ld_exps"), (dict(ld_exps=6), "ld_exps"), (dict(cols=600, ld_exps=4), "ld_exps"),
    (dict(rows=1), "data is null"), (dict(rows=1, data=0x1000), "exps is null"), (dict(rows=1, data=0x1008, exps=0x2000), "16-byte"),
    (dict(rows=1, data=0x1000, exps=0x2002), "4-byte"), (dict(rows=1, data=0x1000, exps=0x2000), "not memory"),
])
def test_an_8_bit_matrix_that_is_none(bad, text):
    lib = G.lib()
    m, f, w = mat(cols=128), fp8(), fp8(rows=4, data=0x1000, exps=0x1000)
    b = C.byref(fp8(**bad))
    refused(lib.gosh_pack_fp8(C.byref(m), b, None, None), text)
    refused(lib.gosh_pack_fp8(C.byref(m), None, b, None), text)
    refused(lib.gosh_unpack_fp8(b, C.byref(m), None), text)
    refused(lib.gosh_linear_fp8(None, b, C.byref(w), None, 0, None, C.byref(m), None, None), text)
    refused(lib.gosh_linear_fp8(None, C.byref(f), b, None, 0, None, C.byref(m), None, None), text)
    refused(lib.gosh_linear_fp8_backward(C.byref(m), b, C.byref(f), None, 0, None, C.byref(m), None, None, 0, None), text)
    refused(lib.gosh_linear_fp8_backward(C.byref(m), None, b, None, 0, C.byref(m), None, None, None, 0, None), text)


def test_layers_in_8_bits_that_are_refused():
    lib = G.lib()
    m, f = mat(cols=128), fp8()
    refused(lib.gosh_pack_fp8(None, C.byref(f), None, None), "x is null")
    assert lib.gosh_pack_fp8(C.byref(m), None, None, None) == 0 and lib.gosh_pack_fp8(C.byref(m), C.byref(f), None, None) == 0
    refused(lib.gosh_pack_fp8(C.byref(mat(cols=127)), C.byref(f), None, None), "must be 0 x 127")
    refused(lib.gosh_pack_fp8(C.byref(m), None, C.byref(f), None), "must be 128 x 0")
    refused(lib.gosh_unpack_fp8(None, C.byref(m), None), "q is null")
    refused(lib.gosh_linear_fp8(None, None, C.byref(f), None, 0, None, C.byref(m), None, None), "x8 is null")
    refused(lib.gosh_linear_fp8(None, C.byref(f), None, None, 0, None, C.byref(m), None, None), "w is null")
    refused(lib.gosh_linear_fp8(None, C.byref(f), C.byref(f), None, 0, None, None, None, None), "y is null")
    refused(lib.gosh_linear_fp8(None, C.byref(f), C.byref(f), None, 0, None, C.byref(m), None, None), "w: rows")
    for act in (-1, 4):
        refused(lib.gosh_linear_fp8(None, C.byref(f), C.byref(f), None, act, None, C.byref(m), None, None), "act")
        refused(lib.gosh_linear_fp8_backward(C.byref(m), C.byref(f), C.byref(f), None, act, C.byref(m), None, None, None, 0, None), "act")
    refused(lib.gosh_linear_fp8_backward(C.byref(m), None, None, None, 0, None, None, 0x1000, None, 0, None), "gosh_linear_backward gives db")
    refused(lib.gosh_linear_fp8_backward(C.byref(m), None, C.byref(f), None, 0, None, C.byref(m), None, None, 0, None), "xt is null")
    refused(lib.gosh_linear_fp8_backward(C.byref(m), C.byref(f), None, None, 0, C.byref(m), None, None, None, 0, None), "wt is null")
    refused(lib.gosh_linear_fp8_backward(C.byref(m), None, C.byref(f), None, H.SILU, C.byref(m), None, None, None, 0, None), "z is null")


def test_workspaces_and_states():
    need = G.gosh_linear_fp8_backward_workspace
    assert need(0, 64, 64) == 0 and need(10, 0, 64) == 0 and need(10, 64, 65537) == 0 and need(2 ** 31, 64, 64) == 0 and need(-1, 64, 64) == 0
    assert need(1000, 64, 200) >= 1000 * 256 + 200 * 1024 + 8 * 200 * 4  # dz both ways and sums; such a dw has no parts
    assert need(2 ** 31 - 2, 65536, 65536) > 2 * (2 ** 31 - 2) * 65536
    size = G.gosh_adamw_state_bytes
    assert size(0, 8) == 0 and size(-1, 8) == 0 and size(5, 16) == 0 and size(2 ** 40 + 1, 8) == 0
    assert size(5, 32) == 32 + 20 and size(8, 32) == 64 and size(1, 8) == 16 + 16 + 16 + 1 and size(129, 8) == 144 + 144 + 16 + 2
    assert size(2 ** 40, 32) == 2 ** 43 and size(2 ** 40, 8) == 2 ** 41 + 2 ** 34


def test_optimisers_that_are_refused():
    lib = G.lib()
    out = C.c_void_p(7)

    def create(**fields):
        q = G.gosh_param(**{**dict(p=0x1000, g=0x2000, state=0x3000, copy=None, n=4, g_type=0, copy_type=1, bits=8, weight_decay=0.0), **fields})
        return lib.gosh_adamw_create(C.byref(q), 1, C.byref(out))

    for fields, text in [
        (dict(n=-1), "n ="), (dict(n=2 ** 40 + 1), "n ="), (dict(g_type=3), "g_type"), (dict(bits=16), "bits"), (dict(weight_decay=-0.1), "weight_decay"),
        (dict(weight_decay=math.nan), "weight_decay"), (dict(weight_decay=math.inf), "weight_decay"), (dict(copy=0x4000, copy_type=0), "copy_type"),
        (dict(p=None), "p is null"), (dict(p=0x1002), "4-byte"), (dict(p=0x1000), "not memory"),
    ]:
        refused(create(**fields), text)
        assert out.value is None
    refused(lib.gosh_adamw_create(None, 1, C.byref(out)), "params is null")
    refused(lib.gosh_adamw_create(None, -1, C.byref(out)), "count")
    refused(lib.gosh_adamw_create(None, 0, None), "optimiser_out is null")
    lib.gosh_adamw_free(None)
    assert lib.gosh_adamw_entries(None) == 0
    ok = dict(lr=0.1, beta1=0.9, beta2=0.99, eps=1e-8, step=1)
    for fields, text in [(dict(lr=math.inf), "lr"), (dict(beta1=1.0), "beta1"), (dict(beta2=math.nan), "beta2"), (dict(eps=-1.0), "eps"),
                         (dict(step=0), "step"), ({}, "optimiser is null")]:
        refused(lib.gosh_adamw_step(None, C.byref(G.gosh_adamw_options(**{**ok, **fields})), None), text)
    refused(lib.gosh_adamw_step(None, None, None), "options is null")
    refused(lib.gosh_adamw_save(None, None, None, 0, G.GOSH_F16, None), "type")
    refused(lib.gosh_adamw_save(None, None, None, 0, G.GOSH_F32, None), "optimiser is null")
    refused(lib.gosh_adamw_load(None, None, None, 0, None), "optimiser is null")


def test_losses_that_are_refused():
    lib = G.lib()
    m = mat()
    refused(lib.gosh_softmax_loss(None, None, 0, None, 1.0, None, None, None), "logits is null")
    refused(lib.gosh_softmax_loss(C.byref(mat(packed=1)), None, 0, None, 1.0, None, None, None), "must not be packed")
    refused(lib.gosh_softmax_loss(C.byref(m), None, 2, None, 1.0, None, None, None), "targets_are64")
    refused(lib.gosh_softmax_loss(C.byref(m), None, 0, None, 1.0, None, C.byref(mat(cols=7)), None), "dlogits is 0 x 7")
    refused(lib.gosh_softmax_loss(C.byref(m), None, 0, None, 1.0, None, C.byref(mat(type_=2)), None), "type")
    refused(lib.gosh_softmax_loss(C.byref(m), None, 0, 0x1002, 1.0, None, None, None), "weight must be 4-byte aligned")
    refused(lib.gosh_softmax_loss(C.byref(m), None, 0, None, 1.0, 0x1002, None, None), "loss must be 4-byte aligned")
    assert lib.gosh_softmax_loss(C.byref(m), None, 0, None, 1.0, None, C.byref(m), None) == 0


def test_an_8_bit_matrix_follows_its_tensors():
    p = G.PackedFp8(6, 700, 1, "cpu")
    assert p.q.shape == (6, 768) and p.exps.shape == (6, 8) and G.PackedFp8(300, 128, 128, "cpu").exps.shape == (3, 4)
    p.q = torch.zeros(6, 1024, dtype=torch.uint8).view(torch.float8_e4m3fn)[:, 128:]
    p.exps = torch.zeros(6, 16, dtype=torch.uint8)[:, 4:12]
    m = p._fp8("q")
    assert (m.data, m.exps) == (p.q.data_ptr(), p.exps.data_ptr())
    assert (m.rows, m.cols, m.ld, m.ld_exps, m.block_rows) == (6, 700, 1024, 16, 1)
    for c in (copy.deepcopy(p), pickle.loads(pickle.dumps(p))):
        assert c._fp8("q").data == c.q.data_ptr() != p.q.data_ptr()
    none = G.PackedFp8(0, 7, 1, "cpu")._fp8("q")
    assert (none.data, none.rows, none.ld, none.ld_exps) == (None, 0, 128, 4)
    empty = G.PackedFp8(7, 0, 1, "cpu")._fp8("q")
    assert (empty.data, empty.rows, empty.cols, empty.ld_exps) == (None, 7, 0, 4)
    one = G.PackedFp8(1, 128, 1, "cpu")  # the stride of a single row says nothing
    one.q, one.exps = one.q.as_strided((1, 128), (1, 1)), one.exps.as_strided((1, 4), (1, 1))
    assert (one._fp8("q").ld, one._fp8("q").ld_exps) == (128, 4)


@pytest.mark.parametrize("q, exps", [((6, 640), (6, 8)), ((6, 768), (6, 4)), ((5, 768), (6, 8)), ((6, 768), (7, 8)), ((4608,), (6, 8))])
def test_an_8_bit_matrix_of_another_shape(q, exps):
    p = G.PackedFp8(6, 700, 1, "cpu")
    p.q, p.exps = torch.zeros(q, dtype=torch.uint8).view(torch.float8_e4m3fn), torch.zeros(exps, dtype=torch.uint8)
    with pytest.raises(TypeError, match="rows of at least"):
        p._fp8("q")
    p.q = torch.zeros(6, 768, dtype=torch.int8)
    with pytest.raises(TypeError, match="float8"):
        p._fp8("q")
    with pytest.raises(ValueError):
        G.PackedFp8(6, 7, 2, "cpu")


# ---- the formulas ----------------------------------------------------------------------------------


def test_the_format():
    """The unit is the smallest at which the block's largest entry fits, and an entry is at most half a step off."""
    torch.manual_seed(1)
    x = torch.randn(150, 300, dtype=torch.float64) * torch.exp(4 * torch.randn(150, 1, dtype=torch.float64))
    for tall in (1, 128):
        code, exps, values = S.fp8(x, tall)
        unit = S.two(exps - 127).repeat_interleave(tall, dim=0)[:150].repeat_interleave(128, dim=1)[:, :300]
        assert ((values - x).abs() <= torch.maximum(2.0 ** -4 * x.abs(), 2.0 ** -10 * unit)).all()
        most = torch.nn.functional.pad(x.abs(), (0, 84, 0, -150 % tall)).reshape(-1, tall, 3, 128).amax(dim=(1, 3))
        assert (most <= 448 * S.two(exps - 127)).all() and (most > 224 * S.two(exps - 127)).all()
        assert torch.equal(S.fp8_values(code.to(torch.uint8), exps, 150, 300, tall), values)


def test_the_gradient_of_the_loss_against_differences():
    torch.manual_seed(2)
    x, target, h = torch.randn(7, 9, dtype=torch.float64), torch.tensor([0, 8, 3, -1, 2, 2, 5]), 1e-5
    weight = torch.rand(7).double() + 0.5
    x[5, 4] = -math.inf
    _, grad = S.softmax_loss(x, target, weight, 1.0)
    for c in range(9):
        if c == 4:
            continue
        up, down = x.clone(), x.clone()
        up[:, c] += h
        down[:, c] -= h
        slope = (S.softmax_loss(up, target, weight, 1.0)[0] - S.softmax_loss(down, target, weight, 1.0)[0]) / (2 * h)
        assert ((slope - grad[:, c]).abs() < 1e-8).all()
    assert (grad[3] == 0).all() and grad[5, 4] == 0


def test_the_step_against_torch():
    torch.manual_seed(3)
    p, m, v = torch.randn(50, dtype=torch.float64), torch.zeros(50, dtype=torch.float64), torch.zeros(50, dtype=torch.float64)
    other = p.clone().requires_grad_(True)
    reference = torch.optim.AdamW([other], lr=0.01, betas=(0.8, 0.95), eps=1e-6, weight_decay=0.1)
    for t in range(1, 12):
        g = torch.randn(50, dtype=torch.float64)
        other.grad = g.clone()
        reference.step()
        p, m, v = S.adamw(p, g, m, v, t, 0.01, 0.8, 0.95, 1e-6, 0.1)
    assert (p - other.detach()).abs().max() < 1e-12


@pytest.mark.parametrize("second", [False, True])
def test_the_sequence_keeps_the_mean(second):
    """An entry between two codes is rounded up in its share of the steps: over 1,000 steps to less than 3 of them."""
    bits = 5 if second else 4
    x = torch.tensor([1.0] + [0.5 + i / 137 / 16 for i in range(127)], dtype=torch.float32)
    sums = torch.zeros(128, dtype=torch.float64)
    for t in range(1, 1001):
        sums += torch.tensor(S.moment_codes(x, second, S.sequence(128, t, second))[2], dtype=torch.float64)
    assert bits in (4, 5) and ((sums / 1000 - x.double()).abs() <= 1 / 16 * 3 / 1000 + 1e-9).all()
