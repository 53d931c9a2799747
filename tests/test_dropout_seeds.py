"""Which seeds the modules with dropout and the convolutions draw, without a GPU: drawing is host code."""
import pytest
import torch
import torch.utils.checkpoint

import token_reference as ref
from paper_2106_06998_amd.dropout import XDropout
from paper_2106_06998_amd.layer import _Seeds
from paper_2106_06998_amd.norm import XRMSNorm

X = torch.empty(0)


def _make():
    return [XDropout(0.5), XRMSNorm(8, p=0.5), XDropout(0.5, base_seed=3), XRMSNorm(8, p=0.5, base_seed=4)]


def test_modules_that_share_a_step_do_not_share_masks():
    """seed + step is what a mask goes by: seeds next to each other would give a layer the mask that its neighbour had a replay before"""
    layers = _make() * 3
    seeds = [m._next_seed(X) for m in layers]
    assert len(set(seeds)) == len(seeds) and all(0 <= s < 2 ** 63 for s in seeds)
    assert min(b - a for a, b in zip(sorted(seeds), sorted(seeds)[1:])) > 1 << 32          # (of 12 among 2^63 values: chance 2^-24)
    for a, b in zip(seeds, seeds[1:]):
        assert not (ref.kept(a, 32768, 0, 256, step=1) == ref.kept(b, 32768, 0, 256, step=0)).all()
        assert not (ref.kept(a, 32768, 0, 256, step=0) == ref.kept(b, 32768, 0, 256, step=1)).all()


def test_seeds_follow_the_generator():
    """torch's CPU generator rules them: a seed that is set, and a state that is saved and put back, give the same seeds again"""
    draw = lambda: [m._next_seed(X) for m in _make()]
    torch.manual_seed(5)
    first = draw()
    state = torch.get_rng_state()
    second = draw()
    assert not set(first) & set(second)
    torch.set_rng_state(state)
    assert draw() == second
    torch.manual_seed(5)
    assert draw() == first
    torch.manual_seed(6)
    assert not set(draw()) & set(first)
    # modules of other base seeds draw others from the same state
    seeds = []
    for base in range(4):
        torch.manual_seed(5)
        seeds.append(XDropout(0.5, base_seed=base)._next_seed(X))
    assert len(set(seeds)) == 4


@pytest.mark.parametrize("reentrant", [False, True])
def test_a_checkpoint_draws_its_seeds_again(reentrant):
    layers, drawn = _make(), []

    def part(x):
        drawn.append([m._next_seed(X) for m in layers])
        return x.sin()

    x = torch.ones(4, requires_grad=True)
    torch.utils.checkpoint.checkpoint(part, torch.utils.checkpoint.checkpoint(part, x, use_reentrant=reentrant), use_reentrant=reentrant).sum().backward()
    assert len(drawn) == 4 and drawn[0] != drawn[1] and drawn[2:] == drawn[1::-1]


def test_convolutions_draw_from_the_generator_too():
    torch.manual_seed(5)
    first = [next(_Seeds()) for _ in range(4)]
    assert len(set(first)) == 4 and all(0 <= s < 2 ** 63 for s in first)
    torch.manual_seed(5)
    assert [next(_Seeds()) for _ in range(4)] == first
