"""The optimizer's side of a training step: AdamW over a model's tensors.

An AdamW holds the states of a list of device tensors and the plan by which
one launch updates all of them (nsd_adamw_step).  It reads gradients where the
gradient calls write them: the `grads` given at construction are caller
buffers that are overwritten step by step.
"""
from __future__ import annotations

import torch

from . import nsd


def _flat(t, what, device, n=None, dtypes=None):
    if not t.is_cuda or not t.is_contiguous():
        raise ValueError(f"{what}: not a contiguous device tensor")
    if t.device != device:
        raise ValueError(f"{what}: on {t.device}, the first tensor on {device}")
    if n is not None and t.numel() != n:
        raise ValueError(f"{what}: {t.numel()} values for {n}")
    if dtypes is not None and t.dtype not in dtypes:
        raise ValueError(f"{what}: {t.dtype}")
    return t


class AdamW:
    """params: fp32 or bf16 tensors, updated in place; grads: as many, fp32 or
    bf16.  masters: the fp32 copies of bf16 weights (a list that may hold None),
    or True to make them from the weights now.  state_bits: 32, or 8 for
    states in 8-bit floats with a scale per nsd.ADAMW_BLOCK values.
    weight_decay: one number, or one per tensor.  m, v, m_scale, v_scale and
    step continue a run: its state tensors (updated in place) and the number
    of steps done; without them the states start at zero."""

    def __init__(self, params, grads, lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8,
                 weight_decay=0.01, state_bits=32, masters=None, m=None, v=None, m_scale=None,
                 v_scale=None, step=0, stream=None):
        self.params, self.grads = list(params), list(grads)
        count = len(self.params)
        if state_bits not in (8, 32):
            raise ValueError(f"states of {state_bits} bits (8 or 32)")
        decay = list(weight_decay) if isinstance(weight_decay, (list, tuple)) \
            else [weight_decay] * count
        for x, what in ((self.grads, "gradients"), (decay, "weight decays")):
            if len(x) != count:
                raise ValueError(f"{len(x)} {what} for {count} tensors")
        floats = (torch.float32, torch.bfloat16)
        if masters is True:
            masters = [p.float() if p.dtype == torch.bfloat16 else None for p in self.params]
        self.masters = list(masters) if masters is not None else [None] * count
        T_m = torch.float32 if state_bits == 32 else torch.float8_e4m3fn
        T_v = torch.float32 if state_bits == 32 else torch.float8_e5m2

        def states(given, dtype, per):
            if given is not None:
                if len(given) != count:
                    raise ValueError(f"{len(given)} states for {count} tensors")
                return list(given)
            return [torch.zeros(-(-p.numel() // per), dtype=torch.uint8 if dtype.itemsize == 1
                                else dtype, device=p.device).view(dtype) for p in self.params]

        self.m, self.v = states(m, T_m, 1), states(v, T_v, 1)
        scales = state_bits == 8
        block = nsd.ADAMW_BLOCK
        self.m_scale = states(m_scale, torch.float32, block) if scales else [None] * count
        self.v_scale = states(v_scale, torch.float32, block) if scales else [None] * count
        self.records = []
        for i, p in enumerate(self.params):
            n = p.numel()
            dev = self.params[0].device
            _flat(p, f"tensor {i}", dev, dtypes=floats)
            _flat(self.grads[i], f"gradient {i}", dev, n, floats)
            _flat(self.m[i], f"first moment {i}", dev, n, (T_m,))
            _flat(self.v[i], f"second moment {i}", dev, n, (T_v,))
            if self.masters[i] is not None:
                _flat(self.masters[i], f"copy {i}", dev, n, (torch.float32,))
            if scales:
                for s in (self.m_scale[i], self.v_scale[i]):
                    _flat(s, f"scales {i}", dev, -(-n // block), (torch.float32,))
            t = [p, self.masters[i], self.grads[i], self.m[i], self.v[i], self.m_scale[i],
                 self.v_scale[i]]
            self.records.append(nsd.nsd_adamw_tensor(
                n, *(None if x is None else x.data_ptr() for x in t), nsd.dtype_of(p),
                nsd.dtype_of(self.grads[i]), decay[i]))
        table = torch.empty(nsd.nsd_adamw_plan_size(self.records), dtype=torch.uint8,
                            device=self.params[0].device if count else "cuda")
        self.plan = nsd.nsd_adamw_plan_build(self.records, state_bits, table, stream)
        self.t = step
        self.hyper = nsd.nsd_adamw(lr, beta1, beta2, eps, step, None, None, None)

    def step(self, lr=None, grad_scale=None, step_dev=None, lr_dev=None, stream=None):
        """One step.  lr changes the rate from now on; grad_scale (a device fp32
        scalar) multiplies every gradient.  step_dev (device int32, the number
        of this step) and lr_dev (device fp32) are read when the step runs: with
        them a captured graph counts its replays.  The count is then the caller's:
        `t`, the steps done, is not advanced, and has to be set before steps
        without step_dev or a checkpoint of it.  A refused step changes nothing."""
        last = self.hyper
        t = self.t + 1 if step_dev is None else self.t
        h = nsd.nsd_adamw(last.lr if lr is None else lr, last.beta1, last.beta2, last.eps, t,
                          *(None if x is None else x.data_ptr()
                            for x in (step_dev, lr_dev, grad_scale)))
        nsd.nsd_adamw_step(self.plan, h, stream)
        self.t, self.hyper = t, h
