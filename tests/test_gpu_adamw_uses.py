"""gosh_adamw_* as a program may use it beside test_gpu_adamw.py: moments that are not finite and are read out, states made on a busy
stream, rates from the device with weight decay, empty tensors, steps that count themselves."""
import math

import pytest
import torch

import paper_2008_12336_amd as G
from tests import step_model as S
from tests.test_gpu_head import DEV, MARK, gen, within

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
def test_zeros_between_moments_that_are_not_finite(bits, dtype):
    sizes = [1, 127, 300, 128, 4097, 5]
    ps, gs = ([torch.ones(n, device=DEV) for n in sizes] for _ in range(2))
    for g in gs:
        g[-1] = math.nan
    opt = G.gosh_adamw_create(ps, gs, bits=bits)
    G.gosh_adamw_step(opt, lr=1e-3, step=1)
    m, v = (torch.full((G.gosh_adamw_entries(opt),), MARK, dtype=dtype, device=DEV) for _ in range(2))
    G.gosh_adamw_save(opt, m, v)
    at = 0
    for n in sizes:
        end = at + -(-n // 128) * 128
        for x in (m, v):
            assert torch.isnan(x[at + n - 1]) and (x[at + n:end] == 0).all(), n
        at = end
    assert at == m.numel()


@pytest.mark.parametrize("bits", [8, 32])
def test_states_that_a_busy_stream_clears_are_there_for_a_step_on_another(bits):
    n = 5000
    p, g, long_ = gen(1)(n), gen(2)(n), torch.zeros(1 << 28, device=DEV)
    q = p.clone()
    want = G.gosh_adamw_create([q], [g], bits=bits)
    G.gosh_adamw_step(want, lr=1e-2, step=1)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        for _ in range(60):  # 2 GB of traffic each, some 25 ms in all
            long_.add_(1)
        opt = G.gosh_adamw_create([p], [g], bits=bits)  # its states are cleared behind them
    G.gosh_adamw_step(opt, lr=1e-2, step=1)
    torch.cuda.synchronize()
    assert torch.equal(p, q) and torch.equal(opt.states[0], want.states[0]) and opt.states[0].any()


def test_steps_that_nobody_numbers():
    """They count themselves; where that cannot be, or without a rate, they are refused."""
    rnd = gen(3)
    p, g = rnd(700), rnd(700)
    q = p.clone()
    opt, other = (G.gosh_adamw_create([t], [g]) for t in (p, q))
    for step in (1, 2, 3):
        G.gosh_adamw_step(opt, lr=1e-2)
        G.gosh_adamw_step(other, lr=1e-2, step=step)
        assert torch.equal(p, q) and opt.step == step
    G.gosh_adamw_step(opt, lr=1e-2, step=10)
    G.gosh_adamw_step(opt, lr=1e-2)
    for step in (10, 11):
        G.gosh_adamw_step(other, lr=1e-2, step=step)
    assert torch.equal(p, q) and opt.step == 11
    before = p.clone()
    with pytest.raises(TypeError, match="lr or lr_dev"):
        G.gosh_adamw_step(opt)
    with pytest.raises(TypeError, match="lr or lr_dev"):
        G.gosh_adamw_step(opt, step=12)
    m, v = (torch.ones(G.gosh_adamw_entries(opt), device=DEV) for _ in range(2))
    G.gosh_adamw_load(opt, m, v)
    given = G.gosh_adamw_create([q], [g], states=[torch.zeros(G.gosh_adamw_state_bytes(700, 32), dtype=torch.uint8, device=DEV)])
    device = G.gosh_adamw_create([q], [g])
    G.gosh_adamw_step(device, lr=0.0, steps=torch.zeros(1, dtype=torch.int64, device=DEV))
    for o in (opt, given, device):
        with pytest.raises(TypeError, match="step is needed"):
            G.gosh_adamw_step(o, lr=1e-2)
    assert torch.equal(p, before)
    G.gosh_adamw_step(opt, lr=1e-2, step=5)
    G.gosh_adamw_step(opt, lr=1e-2)
    assert opt.step == 6
    with pytest.raises(G.GoshError):  # a call that is refused counts no step
        G.gosh_adamw_step(opt, lr=math.nan)
    assert opt.step == 6


def test_tensors_of_no_entries_beside_others():
    p, g = torch.ones(9, device=DEV), torch.ones(9, device=DEV)
    none = [torch.empty(s, device=DEV) for s in ((5, 0), (0, 5), (0,), (2, 0, 3))]
    opt = G.gosh_adamw_create([none[0], p, *none[1:]], [torch.empty_like(none[0]), g, *map(torch.empty_like, none[1:])], bits=8)
    G.gosh_adamw_step(opt, lr=0.5)
    assert ((p - 0.5).abs() < 1e-6).all() and G.gosh_adamw_entries(opt) == 128


@pytest.mark.parametrize("captured", [False, True])
@pytest.mark.parametrize("bits", [8, 32])
def test_rates_from_the_device_with_weight_decay(bits, captured):
    """Each step against 64 bits from the state before it, at the rate of that moment."""
    rnd, sizes, decay, beta = gen(9), [5000, 33, 300], [0.1, 0.0, 0.3], dict(beta1=0.9, beta2=0.99)
    ps, gs = ([rnd(n) for n in sizes] for _ in range(2))
    opt = G.gosh_adamw_create(ps, gs, bits=bits, weight_decay=decay)
    lr, steps = torch.full((1,), 1.0, device=DEV), torch.zeros(1, dtype=torch.int64, device=DEV)
    flat = [torch.empty(G.gosh_adamw_entries(opt), device=DEV) for _ in range(2)]
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    if captured:
        with torch.cuda.graph(graph):
            G.gosh_adamw_step(opt, lr_dev=lr, steps=steps, **beta)
    for t, rate in enumerate((0.25, 0.03125, 0.5), 1):
        lr.fill_(rate)
        for g in gs:
            g.copy_(rnd(g.numel()))
        G.gosh_adamw_save(opt, *flat)
        before, m, v = ([x.double().clone() for x in xs] for xs in (ps, flat[:1], flat[1:]))
        torch.cuda.synchronize()
        if captured:
            graph.replay()
        else:
            G.gosh_adamw_step(opt, lr_dev=lr, steps=steps, **beta)
        torch.cuda.synchronize()
        assert int(steps) == t
        at = 0
        for p, g, b, n, d in zip(ps, gs, before, sizes, decay):
            args = (b, g.double(), m[0][at:at + n], v[0][at:at + n], t, rate, 0.9, 0.99, 1e-8, d)
            within(p, S.adamw(*args)[0], S.adamw_bound(*args), f"step {t}, {n} parameters")
            at += -(-n // 128) * 128
