"""Layer normalisation with a bias and no weight: the bias' gradient is a sum in fp32, rounded once to the bias' own type."""
import pytest
import torch

from paper_2106_06998_amd import norm
from test_gpu_norm import DEV, TD, say

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("shape,axis", [((700, 37), -1), ((5, 19, 13, 11), 1)])
@pytest.mark.parametrize("own", [False, True])
def test_gradient_of_a_bias_without_a_weight(shape, axis, dtype, own):
    """own: a bias of the activations' type."""
    say("layer norm, bias only", shape, axis, dtype, own)
    gen = torch.Generator().manual_seed(7)
    x, dy = (torch.randn(shape, generator=gen).to(TD[dtype]) for _ in range(2))
    C = shape[axis]
    b = torch.randn(C, generator=gen).to(TD[dtype] if own else torch.float32)
    xd, bd = x.to(DEV).requires_grad_(True), b.to(DEV).requires_grad_(True)
    norm.layer_norm(xd, None, bd, 1e-5, axis).backward(dy.to(DEV))
    torch.cuda.synchronize()
    others = [i for i in range(x.dim()) if i != axis % x.dim()]
    want, weight = dy.double().sum(others), dy.double().abs().sum(others)
    # fp32 sums of n terms, at worst n / 64 one after the other (64 rows of threads), and the rounding to the bias' type
    n = x.numel() // C
    u = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -9, torch.float16: 2.0 ** -12}[b.dtype]
    assert bd.grad.dtype == b.dtype
    assert bool(((bd.grad.cpu().double() - want).abs() <= (n / 64 + 16) * 2.0 ** -24 * weight + 2 * u * want.abs()).all())


def test_a_sum_beyond_the_range_of_fp16():
    x, dy = torch.randn(9000, 24).half(), torch.full((9000, 24), 30.0).half()
    b = torch.zeros(24, device=DEV, requires_grad=True)
    say("layer norm, bias only, sums of 270000")
    norm.layer_norm(x.to(DEV), None, b).backward(dy.to(DEV))
    torch.cuda.synchronize()
    assert torch.equal(b.grad.cpu(), torch.full((24,), 270000.0))


def test_the_type_of_the_parameters_gradients_can_be_said():
    x, dy = torch.randn(300, 24).half().to(DEV), torch.randn(300, 24).half().to(DEV)
    y, mean, rstd = norm.layer_norm_forward(x)
    half = norm.layer_norm_backward(dy, x, mean, rstd)
    full = norm.layer_norm_backward(dy, x, mean, rstd, param_dtype=torch.float32)
    torch.cuda.synchronize()
    assert half[1].dtype == half[2].dtype == torch.float16 and full[1].dtype == full[2].dtype == torch.float32
    assert torch.equal(half[0], full[0]) and torch.equal(half[1], full[1].half()) and torch.equal(half[2], full[2].half())
    with pytest.raises(RuntimeError, match="float32 or of the input's type"):
        norm.layer_norm_backward(dy, x, mean, rstd, param_dtype=torch.bfloat16)
