"""Which seeds the modules with dropout draw, without a GPU: `_next_seed` is host code."""
import pytest
import torch

import token_reference as ref
from paper_2106_06998_amd.dropout import XDropout
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
