"""Arguments of the 8-bit layers, the loss and the optimiser that need no device to be refused, and what the binding makes of them."""
import ctypes as C

import pytest
import torch

import paper_2008_12336_amd as G
from tests.test_head_host import mat, refused
from tests.test_step_host import fp8


@pytest.mark.parametrize("act", [4 + G.GOSH_FP8_EXACT, 2 * G.GOSH_FP8_EXACT, -G.GOSH_FP8_EXACT, G.GOSH_FP8_EXACT - 1, -1])
def test_activations_beside_the_choice_of_exact_products(act):
    lib, m, f, w = G.lib(), mat(cols=128), fp8(), fp8(rows=4, data=0x1000, exps=0x1000)
    refused(lib.gosh_linear_fp8(None, C.byref(f), C.byref(f), None, act, None, C.byref(m), None, None), "act")
    refused(lib.gosh_linear_fp8_backward(C.byref(m), C.byref(f), C.byref(f), None, act, C.byref(m), None, None, None, 0, None), "act")
    refused(lib.gosh_linear(C.byref(m), C.byref(m), None, G.GOSH_FP8_EXACT, None, C.byref(m), None, None, None), "act")  # of 8 bits alone


def test_exact_products_are_an_activation_that_the_calls_take():
    lib, m, f = G.lib(), mat(cols=128), fp8()
    for act in range(4):  # refused further on, for a w without rows
        refused(lib.gosh_linear_fp8(None, C.byref(f), C.byref(f), None, act | G.GOSH_FP8_EXACT, None, C.byref(m), None, None), "w: rows")


@pytest.mark.parametrize("shape", [(0,), (5, 0), (0, 5), (3, 0, 4), (2, 3, 0)])
def test_tensors_of_no_entries_have_no_gaps(shape):
    assert G.binding._dense(torch.empty(shape))
    if len(shape) > 1:
        assert G.binding._dense(torch.empty(shape).transpose(0, 1))


@pytest.mark.parametrize("fields, text", [(dict(lr=1e39), "lr"), (dict(lr=-1e39), "lr"), (dict(eps=1e39), "eps"), (dict(eps=1e-46), "eps"),
                                          (dict(eps=5e-324), "eps")])
def test_rates_that_32_bits_do_not_hold(fields, text):
    ok = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=1)
    refused(G.lib().gosh_adamw_step(None, C.byref(G.gosh_adamw_options(**{**ok, **fields})), None), text)
    for fine in (dict(lr=3.4e38), dict(eps=0.0), dict(eps=1e-45), dict(lr=1e-300)):
        refused(G.lib().gosh_adamw_step(None, C.byref(G.gosh_adamw_options(**{**ok, **fine})), None), "optimiser is null")
