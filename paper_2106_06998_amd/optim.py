"""Orthogonalised weight updates: what the (estimated) weight gradients of the layers are used for.

`orthogonalize` brings the singular values of a matrix near one by a few Newton-Schulz products; `muon_step`
updates the momenta and the weights of any number of layers with it in one call; `Muon` is the optimiser.  A
convolution's weight [C_out, C_in, kH, kW] counts as the matrix [C_out, C_in*kH*kW].  All matrices of a call share
their launches (xconv_orth / xconv_muon_step)."""
import torch

from .layer import _DTYPE, _glue, _raw_stream

COEFFICIENTS = (3.4445, -4.7750, 2.0315)


def _check_tensor(t, where):
    if not isinstance(t, torch.Tensor):
        raise TypeError("%s: tensors are expected, got %s" % (where, type(t).__name__))
    if not t.is_cuda:
        raise RuntimeError("%s: runs on the GPU only (tensor on %s)" % (where, t.device))
    if t.dtype not in _DTYPE:
        raise RuntimeError("%s: storage type %s is not supported (float32, bfloat16, float16)" % (where, t.dtype))


def orthogonalize(G, steps=5, coefficients=COEFFICIENTS, eps=1e-7):
    """X_steps of X_0 = G / max(|G|_F, eps), X <- a X + (b A + c A A) X with A = X X^T, in the type and shape of G;
    a list of matrices gives a list."""
    one = isinstance(G, torch.Tensor)
    many = [G] if one else list(G)
    if not many:
        return []
    for t in many:
        _check_tensor(t, "orthogonalize")
    a, b, c = coefficients
    out = _glue().orthogonalize(many, steps, a, b, c, eps, _raw_stream(many[0]))
    return out[0] if one else out


def muon_step(weights, grads, momenta, lr, momentum=0.95, weight_decay=0.0, nesterov=True, steps=5, coefficients=COEFFICIENTS, eps=1e-7):
    """One step for every weight, in place: M <- M + (1 - momentum)(G - M), U = G + momentum (M - G) or M,
    W <- (1 - lr weight_decay) W - lr sqrt(max(1, rows/cols)) orthogonalize(U).  Momenta are float32.  Weights and
    momenta share no memory with each other or with a gradient."""
    if not weights:
        if grads or momenta:
            raise ValueError("muon_step: as many gradients and momenta as weights are expected")
        return
    _check_tensor(weights[0], "muon_step")
    a, b, c = coefficients
    _glue().muon_step(weights, grads, momenta, lr, momentum, weight_decay, nesterov, steps, a, b, c, eps, _raw_stream(weights[0]))


class Muon(torch.optim.Optimizer):
    """Stochastic gradient descent with momentum whose updates are orthogonalised, for parameters of two and more
    axes (weights of convolutions and linear layers; give norms and biases to another optimiser)."""

    def __init__(self, params, lr=0.02, momentum=0.95, weight_decay=0.0, nesterov=True, steps=5, coefficients=COEFFICIENTS, eps=1e-7):
        options = dict(lr=lr, momentum=momentum, weight_decay=weight_decay, nesterov=nesterov, steps=steps, coefficients=coefficients, eps=eps)
        self._check_options(options)
        super().__init__(params, options)

    @staticmethod
    def _check_options(group):
        if not group["lr"] >= 0 or not 0 <= group["momentum"] <= 1 or not group["weight_decay"] >= 0 or not group["eps"] >= 0:
            raise ValueError("Muon: lr, weight_decay and eps must not be negative, momentum lies in [0, 1]")
        if int(group["steps"]) != group["steps"] or group["steps"] < 0 or len(group["coefficients"]) != 3:
            raise ValueError("Muon: steps is a count, coefficients are three numbers")
        group["steps"], group["coefficients"] = int(group["steps"]), tuple(group["coefficients"])

    def add_param_group(self, param_group):
        super().add_param_group(param_group)
        group = self.param_groups[-1]
        try:
            self._check_options(group)
            for p in group["params"]:
                if p.dim() < 2:
                    raise ValueError("Muon: parameters of two and more axes only, got one of shape %s" % (tuple(p.shape),))
        except ValueError:
            self.param_groups.pop()
            raise

    def load_state_dict(self, state_dict):
        """As of any optimiser, but that the momenta stay float32 whatever the parameters' type: torch brings floating state to the
        type of its parameter, which drops digits that a checkpoint holds."""
        # what is loaded is known after the other hooks, and is put right before theirs
        loaded = {}
        hooks = [self.register_load_state_dict_pre_hook(lambda _, state: loaded.update(state)),
                 self.register_load_state_dict_post_hook(lambda _: self._restore_momenta(loaded), prepend=True)]
        try:
            super().load_state_dict(state_dict)
        finally:
            for h in hooks:
                h.remove()

    def _restore_momenta(self, loaded):
        keys = [k for group in loaded["param_groups"] for k in group["params"]]
        params = [p for group in self.param_groups for p in group["params"]]
        for key, p in zip(keys, params):
            m = loaded["state"].get(key, {}).get("momentum_buffer")
            if m is not None:
                self.state[p]["momentum_buffer"] = m.to(device=p.device, dtype=torch.float32)

    @torch.no_grad()
    def step(self, closure=None):
        loss = None
        if closure is not None:
            with torch.enable_grad():
                loss = closure()
        for group in self.param_groups:
            by_device = {}
            for p in group["params"]:
                if p.grad is None:
                    continue
                if p.grad.is_sparse:
                    raise RuntimeError("Muon: sparse gradients are not supported")
                state = self.state[p]
                if "momentum_buffer" not in state:
                    state["momentum_buffer"] = torch.zeros_like(p, dtype=torch.float32)
                w, g, m = by_device.setdefault(p.device, ([], [], []))
                w.append(p)
                g.append(p.grad)
                m.append(state["momentum_buffer"])
            for w, g, m in by_device.values():
                muon_step(w, g, m, group["lr"], group["momentum"], group["weight_decay"], group["nesterov"], group["steps"],
                          group["coefficients"], group["eps"])
        return loss
