"""A training step of a classifier of rows (two layers in 8-bit floating point, softmax loss, AdamW with 8-bit moments and 16-bit
copies of the weights), as a program runs it: each part against 64 bits from what the part before gave it, the same bits
from a captured graph as from eager calls, and two optimisers at once."""
import pytest
import torch

import paper_2008_12336_amd as G
from tests import head_model as H
from tests import step_model as S
from tests.test_gpu_fp8 import values
from tests.test_gpu_head import DEV, gen, within

pytestmark = pytest.mark.gpu
T = torch.bfloat16


class Classifier:
    def __init__(self, rows, k, wide, classes, seed=1):
        rnd = gen(seed)
        self.rows, self.classes = rows, classes
        self.params = [rnd(wide, k) / k ** 0.5, 0.1 * rnd(wide), rnd(classes, wide) / wide ** 0.5, 0.1 * rnd(classes)]
        self.grads = [torch.zeros_like(p) for p in self.params]
        self.copies = [p.to(T) if p.dim() == 2 else None for p in self.params]
        self.opt = G.gosh_adamw_create(self.params, self.grads, bits=8, copies=self.copies, weight_decay=[0.01, 0, 0.01, 0])
        self.steps = torch.zeros(1, dtype=torch.int64, device=DEV)
        new = lambda *s, dtype=T: torch.zeros(*s, dtype=dtype, device=DEV)  # noqa: E731
        self.z, self.a, self.logits = new(rows, wide), new(rows, wide), new(rows, classes)
        self.dlogits, self.da, self.loss = new(rows, classes), new(rows, wide), new(rows, dtype=torch.float32)
        self.layers = [dict(x8=G.PackedFp8(rows, i), xt=G.PackedFp8(i, rows), w8=G.PackedFp8(o, i, 128), wt=G.PackedFp8(i, o, 128))
                       for o, i in ((wide, k), (classes, wide))]
        self.work = torch.empty(max(G.gosh_linear_fp8_backward_workspace(rows, k, wide),
                                    G.gosh_linear_fp8_backward_workspace(rows, wide, classes)), dtype=torch.uint8, device=DEV)

    def step(self, x, target):
        one, two = self.layers
        for layer, w in ((one, self.copies[0]), (two, self.copies[2])):
            G.gosh_pack_fp8(w, layer["w8"], layer["wt"])
        G.gosh_pack_fp8(x, one["x8"], one["xt"])
        G.gosh_linear_fp8(None, one["x8"], one["w8"], self.a, bias=self.params[1], act=H.GELU, z=self.z)
        G.gosh_pack_fp8(self.a, two["x8"], two["xt"])
        G.gosh_linear_fp8(None, two["x8"], two["w8"], self.logits, bias=self.params[3])
        G.gosh_softmax_loss(self.logits, target, self.loss, self.dlogits, scale=1 / self.rows)
        g = self.grads
        G.gosh_linear_fp8_backward(self.dlogits, two["xt"], two["wt"], None, dx=self.da, dw=g[2], db=g[3], workspace=self.work)
        G.gosh_linear_fp8_backward(self.da, one["xt"], None, self.z, H.GELU, dw=g[0], db=g[1], workspace=self.work)
        G.gosh_adamw_step(self.opt, lr=1e-2, steps=self.steps)


def batch(rows, k, classes, seed):
    rnd = gen(seed)
    target = torch.randint(classes, (rows,), generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV)
    target[::17] = -1
    return rnd(rows, k).to(T), target


@pytest.mark.parametrize("rows, k, wide, classes", [(300, 100, 130, 10), (5000, 128, 512, 47), (20000, 256, 1024, 300)])
def test_a_step_part_by_part(rows, k, wide, classes):
    c = Classifier(rows, k, wide, classes)
    x, target = batch(rows, k, classes, 3)
    for _ in range(2):
        before = [p.double() for p in c.params]
        moments = [torch.empty(G.gosh_adamw_entries(c.opt), device=DEV) for _ in range(2)]
        G.gosh_adamw_save(c.opt, *moments)
        w1, w2 = c.copies[0].double(), c.copies[2].double()
        c.step(x, target)
        one, two = c.layers
        assert torch.equal(values(one["w8"]), S.fp8(w1, 128)[2]) and torch.equal(values(two["wt"]), S.fp8(w2, 128)[2].t())
        y, z, ey, ez = S.linear_fp8(values(one["x8"]), values(one["w8"]), before[1], H.GELU, None, T)
        within(c.a, y, H.rounded(ey, y, T), "a")
        within(c.z, z, H.rounded(ez, z, T), "z")
        assert torch.equal(values(two["x8"]), S.fp8(c.a.double(), 1)[2])
        y, _, ey, _ = S.linear_fp8(values(two["x8"]), values(two["w8"]), before[3], H.NONE, None, T)
        within(c.logits, y, H.rounded(ey, y, T), "logits")
        loss, grad = S.softmax_loss(c.logits.double(), target, None, 1 / rows)
        el, eg = S.softmax_loss_bound(c.logits.double(), target, None, 1 / rows)
        within(c.loss, loss, el + H.F32 * loss.abs(), "loss")
        within(c.dlogits, grad, H.rounded(eg, grad, T), "gradient of the logits")
        for layer, dy, zz, act, dx, dw, db, w in ((two, c.dlogits, None, H.NONE, c.da, c.grads[2], c.grads[3], values(two["wt"]).t()),
                                                  (one, c.da, c.z, H.GELU, None, c.grads[0], c.grads[1], values(one["wt"]).t())):
            want, bound = S.linear_fp8_backward(dy.double(), values(layer["xt"]), w, None if zz is None else zz.double(), act, T, torch.float32)
            if dx is not None:
                within(dx, want[0], H.rounded(bound[0], want[0], T), "dx")
            within(dw, want[1], H.rounded(bound[1], want[1], torch.float32), "dw")
            within(db, want[2], H.rounded(bound[2], want[2], torch.float32), "db")
        at = 0
        t = int(c.steps)
        for p, g, b, decay, copy in zip(c.params, c.grads, before, (0.01, 0, 0.01, 0), c.copies):
            n = p.numel()
            args = (b.reshape(-1), g.double().reshape(-1), moments[0][at:at + n].double(), moments[1][at:at + n].double(), t, 1e-2, 0.9, 0.999, 1e-8, decay)
            within(p.reshape(-1), S.adamw(*args)[0], S.adamw_bound(*args), "parameters")
            assert copy is None or torch.equal(copy, p.to(T))
            at += -(-n // 128) * 128


@pytest.mark.parametrize("rows, k, wide, classes", [(300, 100, 130, 10), (9000, 128, 512, 47)])
def test_a_step_in_a_graph(rows, k, wide, classes):
    held, eager = Classifier(rows, k, wide, classes), Classifier(rows, k, wide, classes)
    x, target = batch(rows, k, classes, 4)
    held.step(x, target)
    eager.step(x, target)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held.step(x, target)
    for turn in range(5):
        a, b = batch(rows, k, classes, 10 + turn)
        x.copy_(a)
        target.copy_(b)
        held.work.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        eager.step(x, target)
        torch.cuda.synchronize()
        assert int(held.steps) == int(eager.steps) == turn + 2
        for name, p, q in zip("w1 b1 w2 b2".split(), held.params, eager.params):
            assert torch.equal(p, q), (turn, name)
        assert torch.equal(held.loss, eager.loss) and all(torch.equal(p, q) for p, q in zip(held.opt.states, eager.opt.states))


def test_two_at_once():
    """Two classifiers on two streams, their calls in turns: the same bits as one after the other."""
    want = [Classifier(3000, 128, 256, 20, seed) for seed in (1, 2)]
    got = [Classifier(3000, 128, 256, 20, seed) for seed in (1, 2)]
    data = [batch(3000, 128, 20, seed) for seed in (5, 6)]
    for c, d in zip(want, data):
        for _ in range(3):
            c.step(*d)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in got]
    for _ in range(3):
        for c, d, s in zip(got, data, streams):
            with torch.cuda.stream(s):
                c.step(*d)
    torch.cuda.synchronize()
    for c, d in zip(got, want):
        assert all(torch.equal(p, q) for p, q in zip(c.params + c.opt.states, d.params + d.opt.states))


def test_the_link_predictor_runs_on_the_optimiser():
    """The example's gradients are those of its loss, and its weights' copies follow the parameters."""
    from paper_2008_12336_amd.examples.link_head import LinkHead

    rows, dim = 500, 32
    head = LinkHead(dim, rows)
    x = gen(1)(rows, dim).to(head.dtype)
    target = (torch.arange(rows, device=DEV) % 2).float()
    opt = head.optimiser()
    p = {n: v.double().requires_grad_(True) for n, v in head.params.items()}
    xx = x.double()
    h = (xx - xx.mean(1, keepdim=True)) / torch.sqrt(xx.var(1, unbiased=False, keepdim=True) + 1e-5) * p["gamma"] + p["beta"]
    o = H.act(h @ p["w1"].t() + p["b1"], H.GELU) @ p["w2"].t() + p["b2"] + xx
    logits = (o @ p["w3"].t() + p["b3"])[:, 0]
    torch.nn.functional.binary_cross_entropy_with_logits(logits, target.double()).backward()
    s = head.forward(x, head.copies).float()
    head.backward(((torch.sigmoid(s) - target) / rows).to(head.dtype), head.copies)
    for n, v in p.items():
        # activations and weights of 8 bits each (2^-8 of theirs) and of the 8-bit forms (2^-7): a few per cent of a gradient's size
        assert (head.grads[n].double() - v.grad).norm() <= 0.05 * v.grad.norm(), n
    before = {n: v.clone() for n, v in head.params.items()}
    G.gosh_adamw_step(opt, lr=1e-3, step=1)
    for n, v in head.params.items():
        moved = head.grads[n] != 0
        assert ((v - before[n]).abs() <= 1.001e-3 + 2.0 ** -23 * before[n].abs()).all() and (v[moved] != before[n][moved]).float().mean() > 0.99, n
        assert n not in head.copies or torch.equal(head.copies[n], v.to(head.dtype))
