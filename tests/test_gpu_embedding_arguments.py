"""Arguments of the embedding's gradient that name something else than they seem to: shapes and padding rows."""
import pytest
import torch

import token_reference as ref
from paper_2106_06998_amd import embedding as E

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_gradients_of_another_shape_are_refused():
    """as many places in another order would be added to other rows"""
    idx = torch.randint(0, 6, (2, 3), generator=torch.Generator().manual_seed(1)).to(DEV)
    dy = torch.randn(2, 3, 4, device=DEV)
    for wrong in (dy.transpose(0, 1), dy.view(3, 2, 4), dy.view(1, 6, 4), dy.view(6, 4), dy.view(2, 3, 2, 2)):
        for call in (lambda g: E.embedding_backward(g, idx, 6), lambda g: E.embedding_backward(g.contiguous(), idx.int(), 6)):
            with pytest.raises(RuntimeError, match="shape"):
                call(wrong)
    want, off = ref.embedding_gradient(dy, idx, 6, 1.0)
    ref.close(E.embedding_backward(dy, idx, 6), want, off)


def test_padding_rows_count_from_the_end():
    """as of embedding() and XEmbedding: -1 is the last row"""
    idx = torch.arange(6, device=DEV).repeat(3)
    dy = torch.randn(18, 4, device=DEV)
    for row in range(-6, 6):
        got = E.embedding_backward(dy, idx, 6, 1.0, row)
        want, off = ref.embedding_gradient(dy, idx, 6, 1.0, row % 6)
        ref.close(got, want, off)
        assert bool((got[row] == 0).all()) and int((got == 0).all(1).sum()) == 1
    assert not bool((E.embedding_backward(dy, idx, 6) == 0).any())
    for row in (6, -7, 2 ** 40, -2 ** 40):
        with pytest.raises(RuntimeError):
            E.embedding_backward(dy, idx, 6, 1.0, row)
