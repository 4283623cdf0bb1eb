"""gosh_softmax_loss against 64-bit arithmetic with the bounds of step_model.py: every type, from one class to the most,
odd strides, rows without a target or with nothing left, masks, wrong targets, in-place use, other streams, graphs."""
import math

import pytest
import torch

import paper_2008_12336_amd as G
from tests import head_model as H
from tests import step_model as S
from tests.test_gpu_head import DEV, MARK, beside, gen, types, view, within

pytestmark = pytest.mark.gpu

SHAPES = [  # rows, classes, padding of the rows, entries off the start
    (1, 1, 0, 0), (1, 47, 0, 0), (5, 2, 1, 1), (300, 9, 0, 0), (7, 16, 3, 0), (1000, 33, 0, 1), (100, 64, 0, 0), (70, 100, 2, 3), (513, 250, 0, 0),
    (9, 257, 0, 0), (40, 513, 1, 0), (11, 1000, 0, 0), (6, 1025, 7, 1), (8, 2049, 0, 0), (3, 4096, 0, 0), (5, 5001, 0, 0), (2, 8193, 1, 1),
    (3, 16385, 0, 0), (2, 20000, 0, 0), (2, 12001, 1, 0), (2, 25000, 0, 1), (2, 33001, 5, 0), (2, 65536, 0, 0), (70001, 12, 0, 0),
]


@types
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_loss_and_gradient(shape, dtype):
    rows, classes, pad, off = shape
    rnd = gen(rows * 7 + classes)
    v = 3 * rnd(rows, classes) + 5 * rnd(rows, 1)
    g = torch.Generator(device=DEV).manual_seed(rows + classes)
    target = torch.randint(classes, (rows,), generator=g, device=DEV)
    if classes > 2:
        v[torch.rand(rows, classes, generator=g, device=DEV) < 0.1] = -math.inf
        v[torch.arange(rows, device=DEV), target] = 0.5
    if rows > 4:
        target[1] = -1
        v[2] = -math.inf       # nothing left
        v[3] = torch.finfo(dtype).min  # all of the lowest value: every class as likely
        v[4, :] = -60.0 if dtype != torch.float16 else -30.0
        v[4, target[4]] = 60.0 if dtype != torch.float16 else 30.0
    x, _ = view(v, dtype, pad, off)
    for weight, scale, kind in ((None, 1.0, torch.int32), (torch.rand(rows, generator=g, device=DEV) + 0.1, 0.37, torch.int64)):
        d, mem = view(torch.zeros(rows, classes, device=DEV), dtype, pad, off)
        loss = torch.full((rows,), MARK, device=DEV)
        t = target.to(kind)
        G.gosh_softmax_loss(x, t, loss, d, weight=weight, scale=scale)
        want, grad = S.softmax_loss(x.double(), target, weight, scale)
        el, eg = S.softmax_loss_bound(x.double(), target, weight, scale)
        within(loss, want, el + H.F32 * want.abs(), "loss")
        within(d, grad, H.rounded(eg, grad, dtype), "gradient")
        if rows > 4:
            assert loss[1] == loss[2] == 0 and (d[1] == 0).all() and (d[2] == 0).all()
        alone = torch.empty_like(loss)
        G.gosh_softmax_loss(x, t, alone, weight=weight)
        assert torch.equal(alone, loss)
        into = x.clone()
        G.gosh_softmax_loss(into, t, alone, into, weight=weight, scale=scale)  # over the logits
        assert torch.equal(into, d)
        beside(d, mem)


@types
def test_a_class_that_was_taken_out(dtype):
    """A target whose logit is -infinity: the loss is infinite, the gradient still softmax minus one there."""
    x = torch.tensor([[0.0, -math.inf, 1.0], [math.nan, 0.0, 1.0], [math.inf, 0.0, 1.0], [1.0, 2.0, 3.0], [math.nan, -math.inf, -math.inf]],
                     device=DEV).to(dtype)
    target = torch.tensor([1, 1, 0, 3, 1], dtype=torch.int32, device=DEV)
    loss, d = torch.zeros(5, device=DEV), torch.zeros_like(x)
    G.gosh_softmax_loss(x, target, loss, d)
    assert loss[0] == math.inf and torch.isnan(loss[1:]).all()
    e = math.e
    assert torch.allclose(d[0].double(), torch.tensor([1 / (1 + e), -1.0, e / (1 + e)], dtype=torch.float64, device=DEV), atol=2 * H.HALF[dtype])
    assert torch.isnan(d[1:]).all()
    # not where the row does not count
    G.gosh_softmax_loss(x, torch.full_like(target, -7), loss, d)
    assert (loss == 0).all() and (d == 0).all()
    G.gosh_softmax_loss(x, target, loss, d, weight=torch.zeros(5, device=DEV))
    assert (loss == 0).all() and (d == 0).all()


def test_the_gradient_against_differences():
    """Losses in 32 bits of logits a little up and down, class by class."""
    rnd = gen(3)
    rows, classes, h = 6, 11, 2.0 ** -7
    x = 2 * rnd(rows, classes)
    target = torch.tensor([0, 3, 10, 5, -1, 2], dtype=torch.int32, device=DEV)
    loss, d = torch.empty(rows, device=DEV), torch.empty_like(x)
    weight = torch.rand(rows, device=DEV) + 0.5
    G.gosh_softmax_loss(x, target, loss, d, weight=weight)
    for c in range(classes):
        ends = []
        for s in (1, -1):
            moved, l = x.clone(), torch.empty_like(loss)
            moved[:, c] += s * h
            G.gosh_softmax_loss(moved, target, l, weight=weight)
            ends.append(l.double())
        # the third derivative of log-sum-exp is below 1, losses are off by 2^-20 of 1 and their size
        bound = 1.5 * (h * h / 6 + 2.0 ** -20 * (1 + loss.double().abs()) / h) + 1e-6
        within(d[:, c], (ends[0] - ends[1]) / (2 * h), bound, f"class {c}")


def test_a_stream_and_a_graph():
    rnd = gen(8)
    rows, classes, t = 5000, 300, torch.bfloat16
    x = rnd(rows, classes).to(t)
    target = torch.randint(classes, (rows,), device=DEV)
    loss, d = torch.zeros(rows, device=DEV), torch.zeros_like(x)
    want = torch.zeros_like(loss), torch.zeros_like(x)
    side = torch.cuda.Stream()
    late = torch.zeros_like(x)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        for _ in range(20):
            late.add_(1).sub_(1)
        late.copy_(x)
    G.gosh_softmax_loss(late, target, loss, d, stream=side)
    side.synchronize()
    G.gosh_softmax_loss(x, target, *want)
    assert torch.equal(loss, want[0]) and torch.equal(d, want[1])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        G.gosh_softmax_loss(x, target, loss, d, scale=0.5)
    for turn in range(3):
        x.copy_(rnd(rows, classes))
        target.copy_(torch.randint(classes, (rows,), device=DEV))
        graph.replay()
        torch.cuda.synchronize()
        G.gosh_softmax_loss(x, target, *want, scale=0.5)
        torch.cuda.synchronize()
        assert torch.equal(loss, want[0]) and torch.equal(d, want[1]), turn


def test_offsets_past_32_bits_and_rows_of_none():
    t, classes = torch.bfloat16, 1024
    rows = (1 << 31) // classes + 5
    x = torch.zeros(rows, classes, dtype=t, device=DEV)
    ends = torch.cat((torch.arange(4), torch.arange(rows - 4, rows))).to(DEV)
    x[ends] = gen(1)(8, classes).to(t)
    target = torch.full((rows,), 7, device=DEV)
    loss = torch.zeros(rows, device=DEV)
    G.gosh_softmax_loss(x, target, loss, x, scale=2.0)
    y = gen(1)(8, classes).to(t)
    want, grad = S.softmax_loss(y.double(), target[ends], None, 2.0)
    el, eg = S.softmax_loss_bound(y.double(), target[ends], None, 2.0)
    within(loss[ends], want, el + H.F32 * want.abs(), "loss at the ends")
    within(x[ends], grad, H.rounded(eg, grad, t), "gradient at the ends")
    none = torch.empty(0, 5, device=DEV)
    G.gosh_softmax_loss(none, torch.empty(0, dtype=torch.int32, device=DEV), torch.empty(0, device=DEV), none)


def test_refusals_on_the_device():
    x, t, l = torch.zeros(8, 5, device=DEV), torch.zeros(8, dtype=torch.int32, device=DEV), torch.zeros(8, device=DEV)
    with pytest.raises(TypeError):
        G.gosh_softmax_loss(x, t[:7], l)
    with pytest.raises(TypeError):
        G.gosh_softmax_loss(x, t.to(torch.int16), l)
    with pytest.raises(TypeError):
        G.gosh_softmax_loss(x, t, l[:7])
    with pytest.raises(G.GoshError, match="dlogits is 8 x 4"):
        G.gosh_softmax_loss(x, t, l, x[:, :4])
    with pytest.raises(G.GoshError, match="type"):
        G.gosh_softmax_loss(x, t, l, x.bfloat16())
    with pytest.raises(G.GoshError, match="targets is not memory"):
        G.gosh_softmax_loss(x, t.cpu(), l)
    torch.cuda.synchronize()
