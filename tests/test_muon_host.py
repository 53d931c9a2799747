"""Host side of the Muon step of 64-bit parameters and of the optimiser, without a GPU."""
import ctypes

import pytest
import torch

from paper_2106_06998_amd import binding as xb
from paper_2106_06998_amd import optim

ONE = ctypes.c_void_p(4096)          # never dereferenced: validation fails first


def test_parameters_of_64_bits():
    assert ctypes.sizeof(xb.xconv_muon_args64) == 32 and xb.xconv_muon_args64.nesterov.offset == 24
    L, args = xb.lib(), xb.make_orth_args()
    items = xb.make_orth_items([(4, 4, 4096, 4096, 4096)])
    step = lambda mu, ws=ONE, n=1: L.xconv_muon_step64(items, n, ctypes.byref(args), mu, ws, 1 << 30, None)
    assert step(None) == xb.XCONV_EINVAL
    good = ctypes.byref(xb.xconv_muon_args64(0.1, 0.9, 0.0, 1))
    assert step(good, ws=None) == xb.XCONV_EINVAL and step(good, n=0) == xb.XCONV_OK
    for bad in (float("nan"), float("inf"), 1e300):          # (1e300 is no float)
        for k in range(3):
            v = [0.1, 0.9, 0.0]
            v[k] = bad
            assert step(ctypes.byref(xb.xconv_muon_args64(*v, 1))) == xb.XCONV_EINVAL, (bad, k)


def trained(dtype, momentum_buffer):
    """A parameter and an optimiser that holds `momentum_buffer` for it, as after a step."""
    p = torch.nn.Parameter(torch.zeros(momentum_buffer.shape, dtype=dtype))
    opt = optim.Muon([p], lr=0.1)
    opt.state[p]["momentum_buffer"] = momentum_buffer.clone()
    return p, opt


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
def test_momenta_survive_a_checkpoint(dtype, tmp_path):
    m = torch.randn(3, 5) * 1e-3
    _, opt = trained(dtype, m)
    torch.save(opt.state_dict(), tmp_path / "opt.pt")
    for state in (opt.state_dict(), torch.load(tmp_path / "opt.pt", weights_only=True)):
        q, new = trained(dtype, torch.ones(3, 5))
        seen = []
        new.register_load_state_dict_post_hook(lambda o: seen.append(o.state[q]["momentum_buffer"].dtype))
        new.load_state_dict(state)
        got = new.state[q]["momentum_buffer"]
        assert got.dtype == torch.float32 and torch.equal(got, m) and seen == [torch.float32]


def test_checkpoints_with_several_groups_missing_and_changed_state():
    a, b, c = (torch.nn.Parameter(torch.zeros(4, 3, dtype=torch.bfloat16)) for _ in range(3))
    opt = optim.Muon([{"params": [a, b]}, {"params": [c], "lr": 0.5}])
    m = {p: torch.randn(4, 3) for p in (b, c)}              # (the first parameter has not been stepped)
    for p, t in m.items():
        opt.state[p]["momentum_buffer"] = t.clone()
    x, y, z = (torch.nn.Parameter(torch.zeros(4, 3, dtype=torch.bfloat16)) for _ in range(3))
    new = optim.Muon([{"params": [x, y]}, {"params": [z]}])
    # what a hook makes of the checkpoint is what is loaded
    def doubled(o, state):
        return {"param_groups": state["param_groups"], "state": {k: {n: 2 * t for n, t in v.items()} for k, v in state["state"].items()}}
    hook = new.register_load_state_dict_pre_hook(doubled)
    new.load_state_dict(opt.state_dict())
    assert "momentum_buffer" not in new.state.get(x, {}) and new.param_groups[1]["lr"] == 0.5
    assert torch.equal(new.state[y]["momentum_buffer"], 2 * m[b]) and torch.equal(new.state[z]["momentum_buffer"], 2 * m[c])
    hook.remove()
    new.load_state_dict(opt.state_dict())
    assert torch.equal(new.state[y]["momentum_buffer"], m[b])
    # a momentum that an earlier checkpoint holds in 16 bits comes back as floats
    old = opt.state_dict()
    old["state"][1]["momentum_buffer"] = old["state"][1]["momentum_buffer"].bfloat16()
    new.load_state_dict(old)
    assert new.state[y]["momentum_buffer"].dtype == torch.float32 and torch.equal(new.state[y]["momentum_buffer"], m[b].bfloat16().float())
    with pytest.raises(ValueError):
        new.load_state_dict(optim.Muon([torch.nn.Parameter(torch.zeros(2, 2))]).state_dict())


def weight(*shape):
    return torch.nn.Parameter(torch.zeros(*shape))


def test_every_group_is_checked_not_only_the_defaults():
    for kw in ({"lr": -1}, {"lr": float("nan")}, {"momentum": 2.0}, {"weight_decay": -1}, {"steps": -1}, {"steps": 1.5}, {"coefficients": (1, 2)}, {"eps": -1.0}):
        with pytest.raises(ValueError, match="Muon"):
            optim.Muon([{"params": [weight(3, 4)]}, {"params": [weight(3, 4)], **kw}])
        opt = optim.Muon([weight(3, 4)])
        with pytest.raises(ValueError, match="Muon"):
            opt.add_param_group({"params": [weight(3, 4)], **kw})
        assert len(opt.param_groups) == 1          # nothing is left of what was refused
    with pytest.raises(ValueError, match="two and more axes"):
        opt.add_param_group({"params": weight(3)})
    with pytest.raises(ValueError, match="two and more axes"):
        opt.add_param_group({"params": iter([weight(3, 3), weight(3)])})
    assert len(opt.param_groups) == 1
    opt.add_param_group({"params": iter([weight(3, 3)]), "steps": 3.0, "coefficients": [1.5, -0.5, 0.0]})
    assert opt.param_groups[1]["steps"] == 3 and isinstance(opt.param_groups[1]["steps"], int) and opt.param_groups[1]["coefficients"] == (1.5, -0.5, 0.0)
    opt.step()
