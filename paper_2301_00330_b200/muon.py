"""Orthogonalised updates on the library's kernels (include/gf_train.h): `newton_schulz` for a matrix or a
batch of them, and `Muon`, the optimiser built on it.

Only marshalling happens here: grouping parameters of one shape into one library call, descriptors
and workspaces.
"""
from __future__ import annotations

import math

import torch

from . import binding as B
from .norm import _dense

_PRECISION = {"f16": B.GF_NS_F16, "f32": B.GF_NS_F32}


def newton_schulz(G: torch.Tensor, steps: int = 5, eps: float = 1e-7, precision: str | None = None, coeffs=None,
                  out_dtype: torch.dtype | None = None) -> torch.Tensor:
    """Newton-Schulz iterates of G [..., rows, cols] (float32 or bfloat16), of G's dtype or `out_dtype`.

    precision: "f16" (products of fp16 operands, fp32 sums) or "f32" (operands as pairs); by default
    "f32" for float32 results and "f16" for bfloat16 ones.  coeffs: (a, b, c) for each step.  The result is not
    connected to G for autograd."""
    if not G.is_cuda:
        raise RuntimeError("newton_schulz needs a CUDA tensor: there is no CPU path")
    if G.dim() < 2:
        raise ValueError("newton_schulz needs a matrix or a batch of matrices")
    out_dtype = G.dtype if out_dtype is None else out_dtype
    if precision is None:
        precision = "f32" if out_dtype == torch.float32 else "f16"
    if precision not in _PRECISION:
        raise ValueError("precision is 'f16', 'f32' or None")
    rows, cols = G.shape[-2:]
    G = _dense(G.detach())
    O = torch.empty(G.shape, dtype=out_dtype, device=G.device)
    batch = math.prod(G.shape[:-2])
    desc = B.make_ns_desc(batch, rows, cols, in_dtype=G.dtype, out_dtype=out_dtype, precision=_PRECISION[precision], steps=steps, eps=eps)
    with torch.cuda.device(G.device):
        ws = torch.empty(B.gf_newton_schulz_workspace_bytes(desc), dtype=torch.uint8, device=G.device)
        B.gf_newton_schulz(desc, G, O, ws, None, coeffs, torch.cuda.current_stream(G.device))
    return O


class Muon(torch.optim.Optimizer):
    """Muon for matrices and convolution kernels [C_out, C_in / groups, KH, KW] (flattened to
    [C_out, C_in / groups * KH * KW]); vectors belong to another optimiser.

    The momentum is M <- momentum M + (1 - momentum) g, the update NS(u) with u the Nesterov
    combination or M, times lr * 0.2 * sqrt(max(rows, cols)), so that its entries have the size of
    an Adam update and learning rates carry over; weight_decay is decoupled.

    A parameter whose attribute `filtered_taps` is true has gradients with one value for all taps of a
    kernel -- the weights of FilteredConv2d with r >= 2 -- and its update then costs the products of
    [C_out, C_in / groups] alone; the result is the same.  This reads each gradient at its first tap: whatever
    else is added to such a gradient (an L2 term in the loss, another use of the weight) has to have one value
    for all taps too, or the parameter's attribute, or `filtered_taps` here, is set to False.  Using the weight
    with r = 1 does that by itself, for good; the momentum is spread over the taps then.  Parameters of one
    shape and kind go through one call of the library."""

    def __init__(self, params, lr: float = 1e-3, momentum: float = 0.95, nesterov: bool = True, weight_decay: float = 0.0,
                 steps: int = 5, eps: float = 1e-7, precision: str | None = None,
                 filtered_taps: bool = True):
        super().__init__(params, dict(lr=lr, momentum=momentum, nesterov=nesterov, weight_decay=weight_decay, steps=steps, eps=eps,
                                      precision=precision, filtered_taps=filtered_taps))
        self._workspaces = {}

    def add_param_group(self, param_group):
        """As torch's; settings and parameters are checked for every group, those of the constructor among them."""
        if not isinstance(param_group["params"], torch.Tensor):
            param_group["params"] = list(param_group["params"])      # (a generator can be read once)
        params = param_group["params"]
        for p in [params] if isinstance(params, torch.Tensor) else params:
            p = p[1] if isinstance(p, tuple) else p                  # named parameters
            if isinstance(p, torch.Tensor) and p.dim() not in (2, 4):
                raise ValueError(f"Muon takes matrices and convolution kernels, got a parameter of shape {tuple(p.shape)}")
        given = {**self.defaults, **param_group}
        if given["lr"] < 0 or not 0 <= given["momentum"] < 1 or given["weight_decay"] < 0:
            raise ValueError("lr >= 0, 0 <= momentum < 1 and weight_decay >= 0 expected")
        if given["precision"] is not None and given["precision"] not in _PRECISION:
            raise ValueError("precision is 'f16', 'f32' or None")
        super().add_param_group(param_group)

    def __setstate__(self, state):      # of a copy, or of one that was pickled: a base class without the workspaces
        super().__setstate__(state)
        self.__dict__.setdefault("_workspaces", {})

    def load_state_dict(self, state_dict):
        # torch casts a state to the dtype of its parameter; the momentum is kept in 32 bits whatever that is, and so it is
        # taken from the state as it was given (after the hooks that may change it)
        given = {}
        last = self.register_load_state_dict_pre_hook(lambda _, d: given.update(d))
        try:
            super().load_state_dict(state_dict)
        finally:
            last.remove()
        ids = [i for group in given["param_groups"] for i in group["params"]]
        for i, p in zip(ids, [p for group in self.param_groups for p in group["params"]]):
            momentum = given["state"].get(i, {}).get("momentum")
            if momentum is not None:
                self.state[p]["momentum"] = momentum.to(device=p.device, dtype=torch.float32, copy=True)

    def _workspace(self, device, nbytes: int) -> torch.Tensor:
        # one per device and stream: calls on one stream follow one another
        key = device, torch.cuda.current_stream(device).cuda_stream
        ws = self._workspaces.get(key)
        if ws is None or ws.numel() < nbytes:
            ws = self._workspaces[key] = torch.empty(nbytes, dtype=torch.uint8, device=device)
        return ws

    def _momentum(self, p, rows: int, cols: int) -> torch.Tensor:
        state = self.state[p]
        m = state.get("momentum")
        if m is None:
            m = torch.zeros((rows, cols), dtype=torch.float32, device=p.device)
        elif m.shape != (rows, cols):      # kept while the gradients had one value for all taps, which they no longer have
            m = m.repeat_interleave(cols // m.shape[1], 1)
        state["momentum"] = m = m.to(torch.float32).contiguous()      # (itself, unless someone else put it there)
        return m

    @torch.no_grad()
    def step(self, closure=None):
        loss = None
        if closure is not None:
            with torch.enable_grad():
                loss = closure()
        # what one call takes is gathered and checked first, for all groups: a step that is refused has changed nothing
        calls = []
        for group in self.param_groups:
            alike = {}
            for p in group["params"]:
                if p.grad is None or p.numel() == 0:
                    continue
                if not p.is_cuda:
                    raise RuntimeError("Muon needs CUDA parameters: there is no CPU path")
                if not p.is_contiguous():
                    raise ValueError("Muon updates parameters in place: they have to be contiguous")
                if p.grad.layout != torch.strided:
                    raise TypeError("Muon takes dense gradients")
                rows, taps = p.shape[0], math.prod(p.shape[2:])
                uniform = taps if group["filtered_taps"] and getattr(p, "filtered_taps", False) else 1
                cols = p.numel() // rows // uniform
                m = self.state[p].get("momentum") if p in self.state else None
                if m is not None and m.shape != (rows, cols) and not (
                        group["filtered_taps"] and uniform == 1 and taps > 1 and m.shape == (rows, cols // taps)):
                    raise ValueError(f"a momentum of shape {(rows, cols)} expected, got {tuple(m.shape)}: was it kept with another "
                                     "setting of filtered_taps?")
                alike.setdefault((p.device, rows, cols, uniform, p.grad.dtype, p.dtype), []).append(p)
            for (device, rows, cols, taps, gdt, wdt), ps in alike.items():
                precision = group["precision"] or ("f32" if wdt == torch.float32 else "f16")
                desc = B.make_muon_desc(len(ps), rows, cols, taps, grad_dtype=gdt, weight_dtype=wdt, precision=_PRECISION[precision],
                                        steps=group["steps"], nesterov=group["nesterov"], eps=group["eps"],
                                        momentum=group["momentum"], lr=group["lr"], weight_decay=group["weight_decay"],
                                        scale=0.2 * math.sqrt(max(rows, cols * taps)))
                with torch.cuda.device(device):
                    calls.append((device, desc, ps, B.gf_muon_workspace_bytes(desc)))
        for device, desc, ps, nbytes in calls:
            momenta = [self._momentum(p, desc.rows, desc.cols) for p in ps]
            with torch.cuda.device(device):
                grads = [p.grad.contiguous() for p in ps]
                B.gf_muon_step(desc, grads, momenta, ps, momenta, ps, self._workspace(device, nbytes), None, None,
                               torch.cuda.current_stream(device))
            # the library writes through addresses, which autograd does not see: a graph that saved a weight before has to know
            torch.autograd.graph.increment_version(ps)
        return loss
