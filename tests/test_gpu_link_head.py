"""The link predictor's head beside its training loop: parameters that something else changes, every type."""
import pytest
import torch

from tests.test_gpu_head import DEV, gen

pytestmark = pytest.mark.gpu


def test_scores_are_those_of_the_parameters_of_that_moment():
    from paper_2008_12336_amd.examples.link_head import LinkHead

    head, x = LinkHead(32, 64), gen(1)(100, 32).to(torch.bfloat16)
    other = LinkHead(32, 64, seed=5)
    assert not torch.equal(head.score(x), other.score(x))
    for name, p in head.params.items():  # a checkpoint
        p.copy_(other.params[name])
    assert torch.equal(head.score(x), other.score(x))
    assert all(torch.equal(w, head.params[name].to(torch.bfloat16)) for name, w in head.weights().items())
    head.optimiser()  # its copies begin as the parameters are now
    assert all(torch.equal(head.copies[name], w) for name, w in head.weights().items())
    for p in head.params.values():
        p.zero_()
    head.params["b3"].fill_(2.5)
    assert (head.score(x) == 2.5).all()
