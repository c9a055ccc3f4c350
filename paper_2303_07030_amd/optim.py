"""The optimizer's side of a training step: the norm of all gradients, and AdamW
over a model's tensors.

Both read gradients where the gradient calls write them: the `grads` given at
construction are caller buffers that are overwritten step by step.  A GradNorm
measures them (nsd_grad_norm) and holds the factor that clips them; an AdamW
holds the states of a list of device tensors and the plan by which one launch
updates all of them (nsd_adamw_step).
"""
from __future__ import annotations

import math

import torch

from . import nsd
from .operand import _allocate_on


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


class GradNorm:
    """The norm of a list of fp32 or bf16 gradients and the factor that clips it to
    max_norm.  order: 2, or math.inf for the largest magnitude.  measure() leaves
    on the device `norm` (fp64, one value), `norms` (fp64, one for each tensor) and
    `scale` (fp32, one value): what AdamW.step takes as grad_scale, or what clip()
    multiplies the gradients by."""

    def __init__(self, grads, max_norm=math.inf, order=2, stream=None):
        if order not in (2, math.inf):
            raise ValueError(f"norm of order {order} (2 or math.inf)")
        self.grads = list(grads)
        dev = self.grads[0].device if self.grads else torch.device("cuda")
        for i, g in enumerate(self.grads):
            _flat(g, f"gradient {i}", dev, dtypes=(torch.float32, torch.bfloat16))
        records = [nsd.nsd_grad_tensor(g.numel(), g.data_ptr(), nsd.dtype_of(g))
                   for g in self.grads]
        self.max_norm, self.order = max_norm, order
        with _allocate_on(stream, dev):
            # (filled before the plan is built, which waits for its stream: a measure on any
            # stream comes later)
            self.norm = torch.zeros(1, dtype=torch.float64, device=dev)
            self.norms = torch.zeros(len(records), dtype=torch.float64, device=dev)
            self.scale = torch.ones(1, device=dev)
            table = torch.empty(nsd.nsd_grad_plan_size(records), dtype=torch.uint8, device=dev)
            self.plan = nsd.nsd_grad_plan_build(records, table, stream)
            self.ws = torch.empty(nsd.nsd_grad_norm_workspace_size(self.plan), dtype=torch.uint8,
                                  device=dev)

    def measure(self, grad_scale=None, stream=None):
        """The norms of grad_scale (a device fp32 scalar but `scale` itself, or None)
        times the gradients; `scale` holds grad_scale as a factor."""
        if grad_scale is not None:
            _flat(grad_scale, "grad_scale", self.scale.device, 1, (torch.float32,))
        h = nsd.nsd_clip(self.max_norm, 2 if self.order == 2 else 0,
                         None if grad_scale is None else grad_scale.data_ptr())
        nsd.nsd_grad_norm(self.plan, h, self.norm, self.scale, self.norms, self.ws, stream)

    def clip(self, stream=None):
        """Every gradient times `scale`, in place."""
        nsd.nsd_grad_clip(self.plan, self.scale, stream)


class AdamW:
    """params: fp32 or bf16 tensors, updated in place; grads: as many, fp32 or
    bf16.  masters: the fp32 copies of bf16 weights (a list that may hold None),
    or True to make them from the weights now.  state_bits: 32, or 8 for
    states in 8-bit floats with a scale per nsd.ADAMW_BLOCK values.
    weight_decay: one number, or one per tensor.  m, v, m_scale, v_scale and
    step continue a run: its state tensors (updated in place) and the number
    of steps done; without them the states start at zero.  max_norm: every step
    measures the gradients first (`grad_norm`, a GradNorm) and clips what it takes
    of them; the gradients themselves stay."""

    def __init__(self, params, grads, lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8,
                 weight_decay=0.01, state_bits=32, masters=None, m=None, v=None, m_scale=None,
                 v_scale=None, step=0, stream=None, max_norm=None):
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
        if stream is not None and count:  # the states' first values were filled on the current one
            torch.cuda.current_stream(dev).synchronize()
        self.plan = nsd.nsd_adamw_plan_build(self.records, state_bits, table, stream)
        self.grad_norm = None if max_norm is None else GradNorm(self.grads, max_norm,
                                                                stream=stream)
        self.t = step
        self.hyper = nsd.nsd_adamw(lr, beta1, beta2, eps, step, None, None, None)

    def step(self, lr=None, grad_scale=None, step_dev=None, lr_dev=None, stream=None):
        """One step.  lr changes the rate from now on; grad_scale (a device fp32
        scalar) multiplies every gradient.  step_dev (device int32, the number
        of this step) and lr_dev (device fp32) are read when the step runs: with
        them a captured graph counts its replays.  The count is then the caller's:
        `t`, the steps done, is not advanced, and has to be set before steps
        without step_dev or a checkpoint of it.  A refused step changes nothing but
        what `grad_norm` measured."""
        if self.grad_norm is not None:
            self.grad_norm.measure(grad_scale, stream)
            grad_scale = self.grad_norm.scale
        last = self.hyper
        t = self.t + 1 if step_dev is None else self.t
        h = nsd.nsd_adamw(last.lr if lr is None else lr, last.beta1, last.beta2, last.eps, t,
                          *(None if x is None else x.data_ptr()
                            for x in (step_dev, lr_dev, grad_scale)))
        nsd.nsd_adamw_step(self.plan, h, stream)
        self.t, self.hyper = t, h
