"""AdamW over many tensors by one call of libtopk.so (topk_adamw_step in include/topk_attention.h).

Moments in 32 bits, or in 8 (e4m3 floats with a scale for every 256 elements, the second moment held
as its root, stochastic rounding): 2 bytes a parameter in place of 8.  Parameters in fp32, or in
bf16 with or without a 32-bit master.
"""
from __future__ import annotations

from operator import attrgetter, is_

import numpy as np
import torch

from . import topk as T

BLOCK = 256  # elements that share the scale of an 8-bit moment
_TENSOR = np.dtype([(n, np.uint64) for n in ("param", "grad", "master", "m", "v", "m_scale", "v_scale")]
                   + [("n", np.int64), ("index", np.int64), ("lr", np.float64), ("weight_decay", np.float64)])


_ADDRESS, _NUMEL, _CONTIGUOUS, _DEVICE = (
    torch.Tensor.data_ptr, torch.Tensor.numel, torch.Tensor.is_contiguous, torch.Tensor.get_device)
_DTYPE = attrgetter("dtype")


class AdamW:
    """params: tensors, or dicts {"params": [...], "lr": .., "weight_decay": ..} (groups).  All share a dtype
    (float32 or bfloat16) and are contiguous tensors, on the current CUDA device when a step is taken.

    state_bits: 32 or 8.  masters: None, True (32-bit masters are made of bf16 parameters), or a
    list of fp32 tensors to use as masters.  state: buffers of an earlier optimizer (as state_dict
    returns them) to continue with; they are used as they are, not copied.

    Not a torch.optim.Optimizer.  A step's number goes to the kernel by value: a CUDA graph repeats the one it captured."""

    def __init__(self, params, lr: float = 1e-3, betas=(0.9, 0.999), eps: float = 1e-8, weight_decay: float = 0.01,
                 state_bits: int = 32, seed: int = 0, masters=None, state=None):
        params = list(params)
        groups = params if params and isinstance(params[0], dict) else [{"params": params}]
        self.param_groups = [{"lr": lr, "weight_decay": weight_decay, **g, "params": list(g["params"])} for g in groups]
        self.params = [p for g in self.param_groups for p in g["params"]]
        if not self.params:
            raise ValueError("no parameters")
        if state_bits not in (8, 32):
            raise ValueError("state_bits must be 8 or 32")
        self.dtype, self.device = self.params[0].dtype, self.params[0].device
        self._param_code = T._dtype_code(self.params[0])
        for p in self.params:
            if p.dtype != self.dtype or p.device != self.device or not p.is_contiguous():
                raise ValueError("parameters must be contiguous and share a dtype and a device")
        self.betas, self.eps, self.state_bits, self.seed = tuple(betas), eps, state_bits, int(seed)
        # every tensor's moments start a block of their own in flat buffers
        self._n = [p.numel() for p in self.params]
        at = np.concatenate(([0], np.cumsum([-(-n // BLOCK) * BLOCK for n in self._n]))).astype(np.int64)
        total = int(at[-1])
        self.state = self._new_state(total) if state is None else self._adopt(state, total)
        if masters is True:
            masters = [p.detach().float() for p in self.params]
        if masters is not None:
            masters = list(masters)
            if self.dtype != torch.bfloat16:
                raise ValueError("masters go with bfloat16 parameters")
            if len(masters) != len(self.params) or any(
                    m.dtype != torch.float32 or m.numel() != n or m.device != self.device or not m.is_contiguous()
                    for m, n in zip(masters, self._n)):
                raise ValueError("masters must be contiguous float32 tensors of the parameters' sizes")
        self.masters = masters
        self._table = np.zeros(len(self.params), _TENSOR)
        t, s = self._table, self.state
        t["n"], t["index"] = self._n, at[:-1]
        if masters is not None:
            t["master"] = [m.data_ptr() for m in masters]
        if state_bits == 32:
            t["m"], t["v"] = (s[k].data_ptr() + 4 * at[:-1] for k in ("exp_avg", "exp_avg_sq"))
        else:
            t["m"], t["v"] = (s[k].data_ptr() + at[:-1] for k in ("exp_avg", "exp_avg_root"))
            t["m_scale"], t["v_scale"] = (s[k].data_ptr() + 4 * (at[:-1] // BLOCK) for k in ("exp_avg_scale", "exp_avg_root_scale"))
        self._names = tuple(k for k in s if k != "step")
        self._held = self._buffers_now()  # the table has their addresses
        self._address = self._table.ctypes.data
        self._index, self._options = {self.params[0].get_device()}, None
        self._step = T.lib().topk_adamw_step

    def _buffers_now(self):
        return [*(self.masters or ()), *map(self.state.get, self._names)]

    def _buffers(self, total: int):
        if self.state_bits == 32:
            return {k: (total, torch.float32) for k in ("exp_avg", "exp_avg_sq")}
        return {"exp_avg": (total, torch.float8_e4m3fn), "exp_avg_scale": (total // BLOCK, torch.float32),
                "exp_avg_root": (total, torch.float8_e4m3fn), "exp_avg_root_scale": (total // BLOCK, torch.float32)}

    def _new_state(self, total: int):
        return {"step": 0, **{k: torch.zeros(n, dtype=dt, device=self.device) for k, (n, dt) in self._buffers(total).items()}}

    def _adopt(self, state, total: int):
        for k, (n, dt) in self._buffers(total).items():
            t = state.get(k)
            if t is None or t.dtype != dt or t.numel() != n or t.device != self.device or not t.is_contiguous():
                raise ValueError(f"state {k} must be a contiguous {dt} tensor of {n} elements")
        return {"step": int(state.get("step", 0)), **{k: state[k] for k in self._buffers(total)}}

    def step(self, grads=None, grad_scale=None, stream=None) -> None:
        """One step with the parameters' .grad (or `grads`, one for each parameter; None skips it).
        grad_scale: a float32 CUDA tensor of one element that multiplies the gradients.  If it is not finite nothing is
        updated, but state["step"], which the host counts without waiting for the GPU, goes on; a caller that finds the scale
        not finite takes the step back (opt.state["step"] -= 1), or the bias corrections run ahead of the moments."""
        if grads is None:
            grads = [p.grad for p in self.params]
        elif len(grads) != len(self.params):
            raise ValueError("one gradient for each parameter")
        table, given, params = self._table, [g for g in grads if g is not None], self.params
        if not given:
            return
        # a parameter's data can have been replaced since the last step (Module.to, p.data = ..)
        if (set(map(_DTYPE, params)) != {self.dtype} or set(map(_DEVICE, params)) != self._index or list(map(_NUMEL, params)) != self._n
                or not all(map(_CONTIGUOUS, params))):
            raise ValueError("the parameters are no longer of the dtype, sizes and device that the optimizer was made for")
        sizes = self._n if len(given) == len(grads) else [n for g, n in zip(grads, self._n) if g is not None]
        gdt = given[0].dtype
        if (set(map(_DTYPE, given)) != {gdt} or set(map(_DEVICE, given)) != self._index or not all(map(_CONTIGUOUS, given))
                or list(map(_NUMEL, given)) != sizes):
            raise ValueError("gradients must be contiguous, of the parameters' sizes and device, and of one dtype")
        if gdt not in (torch.float32, torch.bfloat16):
            raise TypeError("gradients must be float32 or bfloat16")
        held = self._buffers_now()
        if len(held) != len(self._held) or not all(map(is_, held, self._held)):
            raise ValueError("the state's buffers or the masters were replaced: load_state_dict copies into them")
        if grad_scale is not None and (grad_scale.dtype != torch.float32 or grad_scale.numel() != 1
                                       or grad_scale.device != self.device):
            raise ValueError("grad_scale must be one float32 element on the parameters' device")
        T._on_gpu("parameters", params[0])
        table["param"] = list(map(_ADDRESS, params))
        options = [(g["lr"], g["weight_decay"], len(g["params"])) for g in self.param_groups]
        if options != self._options:
            k = 0
            for lr, wd, n in options:
                table["lr"][k:k + n], table["weight_decay"][k:k + n] = lr, wd
                k += n
            self._options = options
        address, count = self._address, len(table)
        if len(given) == len(grads):
            table["grad"] = list(map(_ADDRESS, given))
        else:  # parameters without a gradient are left alone
            table = table[[g is not None for g in grads]]
            table["grad"] = list(map(_ADDRESS, given))
            address, count = table.ctypes.data, len(table)
        rc = self._step(address, count, self._param_code, T.TOPK_F32 if gdt == torch.float32 else T.TOPK_BF16, self.state_bits,
                        self.betas[0], self.betas[1], self.eps, self.state["step"] + 1, T._ptr(grad_scale),
                        self.seed & 0xFFFFFFFF, T._stream(stream))
        T._check(rc, "topk_adamw_step")
        whole = len(given) == len(grads)
        for changed in (params, self.masters):
            if changed is not None:
                T._changed(*(changed if whole else [t for t, g in zip(changed, grads) if g is not None]))
        T._changed(*held[0 if self.masters is None else len(self.masters):])
        self.state["step"] += 1

    def zero_grad(self, set_to_none: bool = True) -> None:
        for p in self.params:
            if set_to_none:
                p.grad = None
            elif p.grad is not None:
                p.grad.zero_()

    def moments(self, i: int):
        """(m, v) of parameter i as fp32 tensors of its shape: the values that the state stands for."""
        n, at = self._n[i], int(self._table["index"][i])
        s, shape = self.state, self.params[i].shape
        if self.state_bits == 32:
            return s["exp_avg"][at:at + n].view(shape).clone(), s["exp_avg_sq"][at:at + n].view(shape).clone()
        stop = at + -(-n // BLOCK) * BLOCK
        m, r = ((s[k][at:stop].float().view(-1, BLOCK) * s[k + "_scale"][at // BLOCK:stop // BLOCK, None]).view(-1)[:n].view(shape)
                for k in ("exp_avg", "exp_avg_root"))
        return m, r * r

    def state_dict(self):
        """The state's own buffers, the masters, the step and the groups' options."""
        return {"state": dict(self.state), "masters": self.masters, "betas": self.betas, "eps": self.eps, "seed": self.seed,
                "state_bits": self.state_bits,
                "param_groups": [{k: v for k, v in g.items() if k != "params"} for g in self.param_groups]}

    def load_state_dict(self, d) -> None:
        """Copies a state_dict of an optimizer over the same parameters into this one's buffers."""
        if d["state_bits"] != self.state_bits or (d["masters"] is None) != (self.masters is None):
            raise ValueError("the state is of another kind of optimizer")
        if len(d["param_groups"]) != len(self.param_groups):
            raise ValueError("the state has other parameter groups")
        for k, t in self.state.items():
            if k != "step":
                if d["state"][k].shape != t.shape:
                    raise ValueError(f"state {k} has another size")
        for k, t in self.state.items():
            if k != "step":
                t.copy_(d["state"][k])
        self.state["step"] = int(d["state"]["step"])
        if self.masters is not None:
            for a, b in zip(self.masters, d["masters"]):
                a.copy_(b)
        self.betas, self.eps, self.seed = tuple(d["betas"]), d["eps"], d["seed"]
        for g, new in zip(self.param_groups, d["param_groups"]):
            g.update(new)
