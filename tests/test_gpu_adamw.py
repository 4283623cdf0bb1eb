"""gosh_adamw_* against 64-bit arithmetic with the bounds of step_model.py: moments in 8 and 32 bits (entry by entry, bit by
bit), every type of gradient, sizes of none and one, odd starts, many tensors at once, steps that are left out, the step's
number and rate on the device, captured graphs, other streams."""
import math

import pytest
import torch

import paper_2008_12336_amd as G
from tests import head_model as H
from tests import step_model as S
from tests.test_gpu_head import DEV, MARK, gen, types, within

pytestmark = pytest.mark.gpu
HYPER = dict(lr=3e-3, beta1=0.9, beta2=0.99, eps=1e-8)
SIZES = [1, 7, 127, 128, 129, 300, 0, 4095, 4096, 4097, 10001]


def tensors(sizes, dtype, rnd, off=1):
    """(flat memory, views) of parameters and of gradients: each `off` entries off the last one's end."""
    total = sum(sizes) + off * (len(sizes) + 1)
    p, g = torch.full((total,), MARK, device=DEV), torch.full((total,), MARK, device=DEV).to(dtype)
    ps, gs, at = [], [], off
    for n in sizes:
        ps.append(p[at:at + n])
        gs.append(g[at:at + n])
        ps[-1].copy_(rnd(n))
        gs[-1].copy_(torch.exp(2 * rnd(n) - 3) * rnd(n))
        at += n + off
    return p, g, ps, gs


def flat(sizes, values):
    return torch.cat([torch.nn.functional.pad(v, (0, -n % 128)) for n, v in zip(sizes, values)])


def cut(sizes, memory):
    out, at = [], 0
    for n in sizes:
        out.append(memory[at:at + n])
        at += -(-n // 128) * 128
    return out


def saved(opt, sizes):
    m, v = (torch.full((G.gosh_adamw_entries(opt),), MARK, device=DEV) for _ in range(2))
    G.gosh_adamw_save(opt, m, v)
    return cut(sizes, m), cut(sizes, v)


@types
@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("copy", [None, torch.bfloat16, torch.float16])
def test_steps(bits, copy, dtype):
    """Three steps of many tensors; each is held to 64 bits from the state before it."""
    rnd = gen(bits)
    p_memory, _, ps, gs = tensors(SIZES, dtype, rnd)
    copies = None if copy is None else [torch.zeros(n + 1, dtype=copy, device=DEV)[1:] for n in SIZES]
    decay = [0.1 * (i % 3) for i in range(len(SIZES))]
    opt = G.gosh_adamw_create(ps, gs, bits=bits, copies=copies, weight_decay=decay)
    for step in (1, 2, 3):
        before, (m0, v0) = [p.double() for p in ps], saved(opt, SIZES)
        G.gosh_adamw_step(opt, step=step, **HYPER)
        m1, v1 = saved(opt, SIZES)
        for i, n in enumerate(SIZES):
            args = (before[i], gs[i].double(), m0[i].double(), v0[i].double(), step, HYPER["lr"], HYPER["beta1"], HYPER["beta2"], HYPER["eps"], decay[i])
            want, m, v = S.adamw(*args)
            within(ps[i], want, S.adamw_bound(*args), f"step {step}, {n} parameters")
            if copy is not None:
                assert torch.equal(copies[i], ps[i].to(copy))
            m32, v32 = S.moments32(m0[i].cpu(), v0[i].cpu(), gs[i].float().cpu(), HYPER["beta1"], HYPER["beta2"])
            if bits == 32:
                assert torch.equal(m1[i].cpu(), m32) and torch.equal(v1[i].cpu(), v32)
                continue
            for got, x, second in ((m1[i], m32, False), (v1[i], v32, True)):
                values = S.moment_codes(x, second, S.sequence(n, step, second))[2]
                assert torch.equal(got.double().cpu(), torch.tensor(values, dtype=torch.float64)), (n, second)
    inside = torch.zeros_like(p_memory, dtype=torch.bool)
    at = 1
    for n in SIZES:
        inside[at:at + n] = True
        at += n + 1
    assert (p_memory[~inside] == MARK).all()


def test_the_layout_of_a_state():
    """Codes and exponents lie where the header says, and are those of the formulas; zeros begin."""
    n = 300
    rnd = gen(2)
    m = rnd(n) * torch.exp(4 * rnd(n))
    v = (rnd(n) * torch.exp(6 * rnd(n))) ** 2
    m[130:140], v[5:9] = 0.0, 0.0
    m[7], v[200] = -0.0, 1e-30
    p, g = torch.zeros(n, device=DEV), torch.zeros(n, device=DEV)
    opt = G.gosh_adamw_create([p], [g], bits=8)
    assert opt.states[0].numel() == G.gosh_adamw_state_bytes(n, 8) == 304 + 304 + 16 + 3 and (opt.states[0] == 0).all()
    a, b = saved(opt, [n])
    assert (a[0] == 0).all() and (b[0] == 0).all()
    G.gosh_adamw_load(opt, flat([n], [m]), flat([n], [v]))
    s = opt.states[0].cpu().tolist()
    for x, second, codes_at, exps_at in ((m, False, 0, 608), (v, True, 304, 624)):
        codes, exps, values = S.moment_codes(x.cpu(), second, None)
        assert s[codes_at:codes_at + n] == codes and s[exps_at:exps_at + 3] == exps
        got = saved(opt, [n])[second][0]
        assert torch.equal(got.double().cpu(), torch.tensor(values, dtype=torch.float64))
    half = [torch.empty(G.gosh_adamw_entries(opt), dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    G.gosh_adamw_save(opt, *half)  # exact in 16 bits
    assert torch.equal(half[0][:n].float(), saved(opt, [n])[0][0]) and torch.equal(half[1][:n].float(), saved(opt, [n])[1][0])
    assert (half[0][n:] == 0).all()


def test_moments_that_are_not_finite():
    """They spoil their block of 128, and no other; an entry beyond the largest number of the format counts as one."""
    n = 400
    p, g = torch.ones(n, device=DEV), torch.full((n,), 0.5, device=DEV)
    g[3], g[200] = math.nan, 1e30  # v of the second is infinite
    opt = G.gosh_adamw_create([p], [g], bits=8)
    G.gosh_adamw_step(opt, step=1, **HYPER)
    (m,), (v,) = saved(opt, [n])
    assert torch.isnan(m[:128]).all() and torch.isfinite(m[128:]).all()
    assert torch.isnan(v[:256]).all() and torch.isfinite(v[256:]).all()
    assert torch.isnan(p[3]) and torch.isfinite(p[:3]).all() and torch.isfinite(p[4:]).all()


def test_a_second_moment_shrinks():
    """Without gradients v shrinks by a thousandth a step, much less than the format's steps of a sixteenth to an eighth: its
    mean over the entries follows beta2^t, and every entry has moved."""
    n, steps = 4096, 400
    p, g = torch.zeros(n, device=DEV), torch.zeros(n, device=DEV)
    opt = G.gosh_adamw_create([p], [g], bits=8)
    v = torch.exp(gen(4)(n))
    G.gosh_adamw_load(opt, torch.ones(n, device=DEV), v)
    v = saved(opt, [n])[1][0].double()
    for t in range(1, steps + 1):
        G.gosh_adamw_step(opt, lr=0.0, step=t, beta1=0.999, beta2=0.999)
    m1, v1 = saved(opt, [n])
    want = 0.999 ** steps
    # an entry's rounding is at most a step, an eighth of it, and the last one alone is not made up for: the mean over 4,096
    # entries at different places of the sequence ends well within a step of one of them
    assert abs(float(v1[0].double().sum() / v.sum()) / want - 1) < 0.125 / 4
    assert abs(float(m1[0].double().mean()) / want - 1) < 0.125 / 4
    assert (v1[0].double() < v).float().mean() > 0.99


@pytest.mark.parametrize("bits", [8, 32])
def test_many_steps_find_the_minimum(bits):
    """A quadratic with curvatures over two orders of magnitude."""
    n = 1000
    rnd = gen(5)
    goal, curve = rnd(n), torch.exp(0.7 * rnd(n))
    p, g = torch.zeros(n, device=DEV), torch.zeros(n, device=DEV)
    opt = G.gosh_adamw_create([p], [g], bits=bits)
    for t in range(1, 601):
        torch.mul(curve, p - goal, out=g)
        G.gosh_adamw_step(opt, lr=0.05 * (1 - t / 601), step=t)
    # the rate has fallen to 1e-4: nothing is further from its goal than a few of its last steps
    assert (p - goal).abs().max() < 0.05


def test_against_torch_in_64_bits():
    rnd = gen(6)
    n = 700
    start, g = rnd(n), torch.zeros(n, device=DEV)
    p = start.clone()
    other = start.double().requires_grad_(True)
    reference = torch.optim.AdamW([other], lr=HYPER["lr"], betas=(0.9, 0.99), eps=1e-8, weight_decay=0.05)
    opt = G.gosh_adamw_create([p], [g], bits=32, weight_decay=0.05)
    for t in range(1, 21):
        g.copy_(rnd(n))
        other.grad = g.double()
        reference.step()
        G.gosh_adamw_step(opt, step=t, **HYPER)
    # 20 steps of at most lr each, moments to 20 * 4 roundings of 2^-24 of their terms; terms that cancel count by |g| <= 5
    assert (p.double() - other).abs().max() < 20 * (4 * H.F32 * 4 + HYPER["lr"] * 2.0 ** -16)


def test_number_rate_and_scale_on_the_device():
    rnd = gen(7)
    for bits in (8, 32):
        _, _, ps, gs = tensors([5000, 33], torch.float32, rnd)
        qs, hs = [p.clone() for p in ps], [0.125 * g for g in gs]
        opt, same = G.gosh_adamw_create(ps, gs, bits=bits), G.gosh_adamw_create(qs, hs, bits=bits)
        steps, lr, scale = torch.zeros(1, dtype=torch.int64, device=DEV), torch.full((1,), 3e-3, device=DEV), torch.full((1,), 0.125, device=DEV)
        for t in (1, 2, 3):
            before = [q.clone() for q in qs]
            G.gosh_adamw_step(opt, lr_dev=lr, scale=scale, steps=steps, beta1=0.9, beta2=0.99)
            G.gosh_adamw_step(same, step=t, **HYPER)
            assert int(steps) == t
            for a, b in zip(saved(opt, [5000, 33]), saved(same, [5000, 33])):
                assert all(torch.equal(x, y) for x, y in zip(a, b))
            for p, q, was in zip(ps, qs, before):
                # the corrections are off by 2^-21 there, which an update of at most 10 lr shows, and each p is rounded
                assert ((p - q).abs() <= 3 * 10 * HYPER["lr"] * 2.0 ** -20 + 3 * 2 * H.F32 * (p.abs() + 1e-2)).all()
        # a step that is left out
        kept = [t.clone() for t in ps + opt.states + same.states]
        for bad in (math.inf, math.nan, -math.inf):
            scale.fill_(bad)
            G.gosh_adamw_step(opt, lr_dev=lr, scale=scale, steps=steps)
        assert int(steps) == 3 and all(torch.equal(a, b) for a, b in zip(kept, ps + opt.states + same.states))


@pytest.mark.parametrize("bits", [8, 32])
def test_a_step_whose_number_passes_32_bits(bits):
    """beta^t is 0 there: a rate from the device gives the same bits as one from the host, and the number of steps too."""
    rnd = gen(8)
    _, _, ps, gs = tensors([3000, 7], torch.float32, rnd)
    lr, steps = torch.full((1,), HYPER["lr"], device=DEV), torch.full((1,), (1 << 32) - 1, dtype=torch.int64, device=DEV)
    rest = {k: v for k, v in HYPER.items() if k != "lr"}
    got = []
    for how in (dict(lr=HYPER["lr"], step=1 << 32), dict(lr_dev=lr, step=1 << 32), dict(lr_dev=lr, steps=steps)):
        qs = [p.clone() for p in ps]
        opt = G.gosh_adamw_create(qs, gs, bits=bits)
        G.gosh_adamw_step(opt, **how, **rest)
        got.append(qs + opt.states)
    assert int(steps) == 1 << 32 and all(torch.isfinite(q).all() for q in got[0][:2])
    assert all(torch.equal(a, b) for other in got[1:] for a, b in zip(got[0], other))


@pytest.mark.parametrize("bits", [8, 32])
def test_a_captured_graph_and_a_stream(bits):
    rnd = gen(11)
    _, _, ps, gs = tensors([9000, 5, 128], torch.bfloat16, rnd)
    qs = [p.clone() for p in ps]
    copies = [torch.zeros(p.numel(), dtype=torch.float16, device=DEV) for p in ps]
    opt, eager = G.gosh_adamw_create(ps, gs, bits=bits, copies=copies), G.gosh_adamw_create(qs, gs, bits=bits)
    steps, count = torch.zeros(1, dtype=torch.int64, device=DEV), torch.zeros(1, dtype=torch.int64, device=DEV)
    lr = torch.full((1,), 1e-2, device=DEV)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        G.gosh_adamw_step(opt, lr_dev=lr, steps=steps)
    for turn in range(4):
        for g in gs:
            g.copy_(rnd(g.numel()))
        lr.mul_(0.5)
        torch.cuda.synchronize()
        graph.replay()
        G.gosh_adamw_step(eager, lr_dev=lr, steps=count, stream=side)
        torch.cuda.synchronize()
        assert int(steps) == int(count) == turn + 1
        assert all(torch.equal(p, q) for p, q in zip(ps, qs)) and all(torch.equal(a, b) for a, b in zip(opt.states, eager.states))
        assert all(torch.equal(c, p.half()) for c, p in zip(copies, ps))


def test_many_tensors():
    rnd = gen(12)
    sizes = [1 + (i * 37) % 500 for i in range(1500)]
    _, _, ps, gs = tensors(sizes, torch.float16, rnd, off=2)
    before = [p.double() for p in ps]
    opt = G.gosh_adamw_create(ps, gs, bits=8, weight_decay=0.01)
    G.gosh_adamw_step(opt, step=1, **HYPER)
    for p, g, b in zip(ps[::50], gs[::50], before[::50]):
        args = (b, g.double(), torch.zeros_like(b), torch.zeros_like(b), 1, HYPER["lr"], 0.9, 0.99, 1e-8, 0.01)
        assert ((p.double() - S.adamw(*args)[0]).abs() <= S.adamw_bound(*args)).all()
    opt.free()
    opt.free()
    with G.gosh_adamw_create([], []) as none:
        G.gosh_adamw_step(none, lr=1.0)
        assert G.gosh_adamw_entries(none) == 0


def test_parameters_of_any_shape():
    """Memory without gaps, in any order of dimensions; the gradient's strides are the parameter's."""
    w = torch.randn(8, 6, 5, device=DEV).permute(2, 0, 1)
    g = torch.randn(8, 6, 5, device=DEV).permute(2, 0, 1)
    want = (w - HYPER["lr"] * torch.sign(g)).clone()
    opt = G.gosh_adamw_create([w], [g], bits=32)
    G.gosh_adamw_step(opt, step=1, **HYPER)
    assert torch.allclose(w, want, atol=1e-5)
    for p, q in ((w, g.contiguous()), (torch.zeros(4, 8, device=DEV)[:, ::2], torch.zeros(4, 8, device=DEV)[:, ::2])):
        with pytest.raises(TypeError):
            G.gosh_adamw_create([p], [q])


def test_offsets_past_32_bits():
    n = (1 << 31) + 5000
    ends = torch.cat((torch.arange(300), torch.arange(n - 300, n))).to(DEV)
    p, g = torch.zeros(n, device=DEV), torch.zeros(n, dtype=torch.bfloat16, device=DEV)
    p[ends] = gen(1)(600)
    g[ends] = gen(2)(600).bfloat16()
    before = p[ends].double()
    opt = G.gosh_adamw_create([p], [g], bits=8)
    G.gosh_adamw_step(opt, step=1, **HYPER)
    args = (before, g[ends].double(), torch.zeros_like(before), torch.zeros_like(before), 1, HYPER["lr"], 0.9, 0.99, 1e-8, 0.0)
    within(p[ends], S.adamw(*args)[0], S.adamw_bound(*args), "parameters at the ends")
    m, v = (torch.empty(G.gosh_adamw_entries(opt), dtype=torch.bfloat16, device=DEV) for _ in range(2))
    G.gosh_adamw_save(opt, m, v)
    assert ((m[ends].double() - 0.1 * g[ends].double()).abs() <= 0.125 * 0.1 * g[ends].double().abs() + 4 * 2.0 ** -17).all()


def test_refusals_on_the_device():
    p, g = torch.zeros(100, device=DEV), torch.zeros(100, device=DEV)
    for args, text in [
        (([p, p], [g, g]), "overlap"), (([p[:60], p[50:]], [g[:60], g[50:]]), "overlap"), (([p], [p]), "gradients overlap"),
        (([p.cpu()], [g]), "p is not memory"),
    ]:
        with pytest.raises(G.GoshError, match=text):
            G.gosh_adamw_create(*args)
    with pytest.raises(TypeError):
        G.gosh_adamw_create([p], [g[:99]])
    with pytest.raises(TypeError):
        G.gosh_adamw_create([p.half()], [g])
    with pytest.raises(ValueError):
        G.gosh_adamw_create([p], [g, g])
    with pytest.raises(TypeError):
        G.gosh_adamw_create([p], [g], states=[torch.zeros(10, dtype=torch.uint8, device=DEV)])
    opt = G.gosh_adamw_create([p], [g])
    for bad, text in ((dict(beta1=1.0), "beta1"), (dict(beta2=-0.1), "beta2"), (dict(eps=-1.0), "eps"), (dict(step=0), "step"),
                      (dict(lr=math.nan), "lr")):
        with pytest.raises(G.GoshError, match=text):
            G.gosh_adamw_step(opt, **{**dict(lr=0.1, step=1), **bad})
    with pytest.raises(G.GoshError, match="scale is not memory"):
        G.gosh_adamw_step(opt, lr=0.1, scale=torch.zeros(1))
    with pytest.raises(G.GoshError, match="the moments take 128"):
        G.gosh_adamw_save(opt, torch.zeros(100, device=DEV), torch.zeros(100, device=DEV))
    with pytest.raises(G.GoshError, match="type"):
        G.gosh_adamw_save(opt, torch.zeros(128, device=DEV).half(), torch.zeros(128, device=DEV).half())
    with pytest.raises(TypeError):
        G.gosh_adamw_load(opt, torch.zeros(128, device=DEV).bfloat16(), torch.zeros(128, device=DEV).bfloat16())
    opt.free()
    with pytest.raises(G.GoshError, match="optimiser is null"):
        G.gosh_adamw_step(opt, lr=0.1)
    torch.cuda.synchronize()
    assert (p == 0).all()
