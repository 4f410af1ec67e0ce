"""State of Mx4MoELayer between a step and its training calls: what they read has been written by the step that they belong to, or is given.
No GPU needed: the context here records its calls."""
import pytest
import torch

from paper_2603_19172_amd import binding as B
from paper_2603_19172_amd.layer import Mx4MoELayer

T, H, F, E, k = 6, 64, 32, 8, 2


class Calls:
    def __init__(self):
        self.seen = []

    def route_scored(self, logits, k, idx, w, **kw):
        idx.copy_(logits.topk(k, dim=1).indices)

    def moe_ffn_mx4(self, x, idx, w, table, F, y, **kw):
        return y

    def route_balance(self, logits, idx, coef, counts, mean, loss, **kw):
        counts[:E] = torch.bincount(idx.reshape(-1).long(), minlength=E)
        counts[E] = len(idx)
        self.seen.append(("balance", idx.clone()))
        return counts, mean, loss

    def route_scored_backward(self, logits, idx, counts, coef, **kw):
        self.seen.append(("backward", idx.clone(), None if counts is None else counts.clone()))
        return torch.zeros_like(logits)


class Experts:
    table = None

    def __init__(self, F=F):
        self.E, self.H, self.F = E, H, F


@pytest.fixture
def layer():
    return Mx4MoELayer(Calls(), T, H, F, E, k, device="cpu")


def logits(seed):
    return torch.randn((T, E), generator=torch.Generator().manual_seed(seed))


def step(layer, l):
    return layer.step(torch.zeros((T, H), dtype=torch.bfloat16), Experts(), logits=l)


def counted(l):
    return torch.bincount(l.topk(k, dim=1).indices.reshape(-1), minlength=E).to(torch.int32)


def test_nothing_before_the_first_step(layer):
    l, dw = logits(1), torch.zeros((T, k))
    for call in (lambda: layer.balance(l, 0.1), lambda: layer.backward(l, dw), lambda: layer.backward(l, dw, coef=0.1), lambda: layer.backward(l, None, coef=0.1)):
        with pytest.raises(RuntimeError, match="step"):
            call()
    assert layer.ctx.seen == []


def test_counts_are_the_last_steps(layer):
    l, dw = logits(1), torch.zeros((T, k))
    step(layer, l)
    layer.backward(l, dw)                                      # the weights' gradient alone needs no counts
    with pytest.raises(RuntimeError, match="balance"):
        layer.backward(l, dw, coef=0.1)
    layer.balance(l, 0.1)
    for _ in range(2):
        layer.backward(l, dw, coef=0.1)
        assert torch.equal(layer.ctx.seen[-1][2][:E], counted(l))
    # another step: the counts there are its predecessor's
    l2 = logits(2)
    step(layer, l2)
    with pytest.raises(RuntimeError, match="balance"):
        layer.backward(l2, dw, coef=0.1)
    layer.balance(l2, 0.1)
    layer.backward(l2, dw, coef=0.1)
    assert torch.equal(layer.ctx.seen[-1][2][:E], counted(l2))


def test_a_step_that_is_refused_changes_nothing(layer):
    l, dw = logits(1), torch.zeros((T, k))
    step(layer, l)
    layer.balance(l, 0.1)
    with pytest.raises(ValueError, match="other experts"):
        layer.step(torch.zeros((T, H)), Experts(F + 1), logits=l)
    layer.backward(l, dw, coef=0.1)


def test_a_step_that_fails_on_its_way_leaves_no_routing(layer):
    l = logits(1)
    step(layer, l)
    layer.balance(l, 0.1)
    layer.ctx.route_scored = None
    with pytest.raises(TypeError):
        step(layer, logits(2))
    with pytest.raises(RuntimeError, match="step"):
        layer.balance(l, 0.1)


def test_several_steps_before_their_gradients(layer):
    """Copies of a step's choices and counts bring its gradient after another step."""
    ls, dw, kept = [logits(s) for s in (1, 2)], torch.zeros((T, k)), []
    for l in ls:
        step(layer, l)
        counts, _, _ = layer.balance(l, 0.1)
        kept.append((layer.idx.clone(), counts.clone()))
    for l, (idx, counts) in zip(ls, kept):
        layer.backward(l, dw, coef=0.1, idx=idx, counts=counts)
        _, i, c = layer.ctx.seen[-1]
        assert torch.equal(i, l.topk(k, dim=1).indices.int()) and torch.equal(c[:E], counted(l))
    layer.backward(ls[0], dw, idx=kept[0][0])
    assert layer.ctx.seen[-1][2] is None
    with pytest.raises(ValueError, match="counts"):            # one step's choices with another's counts
        layer.backward(ls[0], dw, coef=0.1, idx=kept[0][0])
    layer.balance(ls[0], 0.1, idx=kept[0][0])                    # what self.counts hold is then not the last step's
    with pytest.raises(RuntimeError, match="balance"):
        layer.backward(ls[1], dw, coef=0.1)
    layer.backward(ls[0], dw, coef=0.1, idx=kept[0][0], counts=layer.counts)
    assert torch.equal(layer.ctx.seen[-1][2][:E], counted(ls[0]))
