"""gosh_softmax_loss whose gradient lies in the memory of its logits: over them, beside them, or refused."""
import pytest
import torch

import paper_2008_12336_amd as G
from tests.test_gpu_head import DEV, gen

pytestmark = pytest.mark.gpu


def parts(memory, at, rows, cols, ld):
    return torch.as_strided(memory, (rows, cols), (ld, 1), at)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("rows, cols, first, second", [
    (50, 7, (0, 16), (7, 16)), (50, 7, (7, 16), (0, 16)), (50, 7, (3, 20), (10, 20)), (50, 8, (8, 16), (0, 16)),  # side by side
    (50, 8, (0, 16), (24, 16)), (50, 8, (0, 8), (400, 8)), (1, 9, (0, 9), (9, 30)), (50, 7, (5, 16), (5, 16)), (1, 9, (4, 9), (4, 30)),
])
def test_beside_or_over_the_logits(rows, cols, first, second, dtype):
    memory = torch.zeros(4096, dtype=dtype, device=DEV)
    x, target = gen(1)(rows, cols).to(dtype), torch.arange(rows, device=DEV) % cols
    want, loss, other = torch.empty_like(x), torch.empty(rows, device=DEV), torch.empty(rows, device=DEV)
    G.gosh_softmax_loss(x, target, loss, want)
    logits, d = parts(memory, first[0], rows, cols, first[1]), parts(memory, second[0], rows, cols, second[1])
    logits.copy_(x)
    G.gosh_softmax_loss(logits, target, other, d)
    assert torch.equal(d, want) and torch.equal(other, loss)
    assert first == second or rows == 1 and first[0] == second[0] or torch.equal(logits, x)


@pytest.mark.parametrize("rows, cols, first, second", [
    (50, 7, (0, 16), (6, 16)), (50, 7, (6, 16), (0, 16)), (50, 7, (0, 16), (10, 16)), (50, 8, (0, 8), (8, 8)), (50, 8, (0, 8), (392, 8)),
    (50, 8, (8, 8), (0, 8)), (50, 8, (0, 8), (0, 9)), (50, 8, (0, 8), (100, 9)), (1, 9, (0, 9), (8, 9)), (1, 9, (5, 9), (1, 40)),
])
def test_across_the_logits_is_refused(rows, cols, first, second):
    memory = torch.ones(4096, device=DEV)
    target, loss = torch.zeros(rows, dtype=torch.int32, device=DEV), torch.full((rows,), 3.0, device=DEV)
    with pytest.raises(G.GoshError, match="dlogits overlaps logits"):
        G.gosh_softmax_loss(parts(memory, first[0], rows, cols, first[1]), target, loss, parts(memory, second[0], rows, cols, second[1]))
    torch.cuda.synchronize()
    assert (memory == 1).all() and (loss == 3).all()
