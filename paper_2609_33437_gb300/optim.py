"""The optimizer's update on ordinary steps: one AdamW step over many tensors in one launch, moments in 32 bits or in 8
(include/smat.h, "AdamW").

    moments = Moments(params, bits=8)
    adamw(params, grads, moments, step=t, lr=1e-4)            params and moments in place

`AdamW` is a torch.optim.Optimizer around it. Parameters are contiguous CUDA tensors of one dtype per call (float32 or
bfloat16), gradients of one dtype. Argument marshalling only: the step runs in the library's kernel, on the current stream or
the one given. On simulated-loss steps `PeriodicSmat.optimizer_step` takes an AdamW of 32 bits into the gradient map's pass.
"""

import ctypes
import operator
import struct
from typing import Dict, List, Optional, Sequence, Union

import torch

from . import linear as L
from . import smat as S

GROUP = 256

_ADAMW = struct.Struct("@10P6dqQ4i")
_numel, _contiguous, _get_device, _data_ptr = (torch.Tensor.numel, torch.Tensor.is_contiguous, torch.Tensor.get_device,
                                               torch.Tensor.data_ptr)
_dtype = operator.attrgetter("dtype")


class Moments:
    """The moments of a list of tensors, zeros at first. Tensor k's lie at starts[k] .. starts[k] + sizes[k] - 1 of each buffer;
    starts are multiples of 256.

    bits 32: m1 and m2, float32. bits 8: m1 and r = sqrt(m2) as bytes q1 and q2, and a power of two for every 256 of them, e1
    and e2; two bytes an element where 32 bits take eight."""

    def __init__(self, params: Sequence[torch.Tensor], bits: int = 32):
        params = list(params)
        if bits not in (8, 32):
            raise ValueError("bits: 8 or 32")
        if not params:
            raise ValueError("params: at least one tensor")
        self.bits, self.device = bits, params[0].device
        if any(p.device != self.device for p in params):
            raise ValueError("params: on one device")
        self.sizes: List[int] = [p.numel() for p in params]
        self.starts: List[int] = []
        at = 0
        for n in self.sizes:
            self.starts.append(at)
            at += -(-n // GROUP) * GROUP
        self.places = at
        if bits == 8 and at >= 1 << 32:
            raise ValueError(f"8 bits: {at} places, 2^32 and more are not numbered")
        kw = dict(device=self.device)
        if bits == 8:
            self._buffers = {"q1": torch.zeros(at, dtype=torch.uint8, **kw),
                             "e1": torch.ones(at // GROUP, dtype=torch.uint8, **kw),
                             "q2": torch.zeros(at, dtype=torch.uint8, **kw),
                             "e2": torch.ones(at // GROUP, dtype=torch.uint8, **kw)}
        else:
            self._buffers = {"m1": torch.zeros(at, dtype=torch.float32, **kw), "m2": torch.zeros(at, dtype=torch.float32, **kw)}
        # what a call hands over of the list
        self._numels = struct.pack(f"{len(self.sizes)}q", *self.sizes)
        self._pointers = f"{len(self.sizes)}P"

    def buffers(self) -> Dict[str, torch.Tensor]:
        """The buffers by name: m1 and m2, or q1, e1, q2 and e2. They may be read and written (a checkpoint), and moved away and
        back: a step takes them where they lie then, and refuses them elsewhere or in another form."""
        return dict(self._buffers)

    def _addresses(self):
        """(m1, m2, 0, 0) or (q1, q2, e1, e2), where they lie now: whoever was handed a buffer may have given it other storage."""
        out = []
        index = self.device.index if self.device.index is not None else -1
        for name in ("q1", "q2", "e1", "e2") if self.bits == 8 else ("m1", "m2"):
            t = self._buffers[name]
            count = self.places // GROUP if name[0] == "e" else self.places
            dtype = torch.uint8 if self.bits == 8 else torch.float32
            if t.dtype is not dtype or _numel(t) != count or _get_device(t) != index or not _contiguous(t):
                raise ValueError(f"moments: {name} must be contiguous {dtype} of {count} elements on {self.device}, as it was made")
            out.append(_data_ptr(t))
        return out if self.bits == 8 else (*out, 0, 0)

    def values(self, stream: Optional[torch.cuda.Stream] = None):
        """(m1, m2) for 32 bits, the buffers themselves; (m1, r) in bfloat16, which holds what 8 bits stand for exactly."""
        b = self._buffers
        if self.bits == 32:
            return b["m1"], b["m2"]
        if stream is not None:
            return L._on(stream, self.values)
        q1, q2, e1, e2 = self._addresses()
        m1, r = (torch.empty(self.places, dtype=torch.bfloat16, device=self.device) for _ in range(2))
        L._call("smat_adamw_values", self.device, q1, e1, q2, e2, m1.data_ptr(), r.data_ptr(), self.places)
        return m1, r

    def views(self, name: str) -> List[torch.Tensor]:
        """A buffer of 32 bits by tensors, each flat."""
        b = self._buffers[name]
        return [b[a:a + n] for a, n in zip(self.starts, self.sizes)]

    def nbytes(self) -> int:
        return sum(t.numel() * t.element_size() for t in self._buffers.values())


def _addresses(name: str, ts: Sequence[Optional[torch.Tensor]], sizes: Sequence[int], index: int, optional: bool):
    """(their addresses, their dtype): contiguous tensors of one dtype and these sizes on the device. A None: 0."""
    try:  # whole lists by functions in C: 24 tensors 4 us, one by one 6.5
        dts = set(map(_dtype, ts))
        if (len(dts) == 1 and list(map(_numel, ts)) == sizes and all(map(_contiguous, ts))
                and set(map(_get_device, ts)) == {index}):
            return list(map(_data_ptr, ts)), dts.pop()
    except (TypeError, AttributeError):  # something else than a tensor among them
        pass
    first = next((t for t in ts if t is not None), None)
    if first is None:
        return [0] * len(ts), None
    dt, out = first.dtype, []
    for t, n in zip(ts, sizes):
        if t is None and optional:
            out.append(0)
            continue
        if t.dtype is not dt or _numel(t) != n or _get_device(t) != index or not _contiguous(t):
            raise ValueError(f"{name}[{len(out)}]: must be contiguous {dt} of {n} elements on cuda:{index}")
        out.append(_data_ptr(t))
    return out, dt


def _one(name: str, v, dtype, device):
    """(number, address) of a number, or of a tensor that holds one."""
    if not isinstance(v, torch.Tensor):
        return v, 0
    if v.dtype is not dtype or v.device != device or v.numel() != 1:
        raise ValueError(f"{name}: must be a number, or one {dtype} on {device}")
    return 0, v.data_ptr()


def adamw(params: Sequence[torch.Tensor], grads: Sequence[Optional[torch.Tensor]], moments: Moments,
          step: Union[int, torch.Tensor], lr: Union[float, torch.Tensor] = 1e-3, beta1: float = 0.9, beta2: float = 0.999,
          eps: float = 1e-8, weight_decay: float = 0.01, scale: Union[float, torch.Tensor] = 1.0, seed: int = 0,
          stream: Optional[torch.cuda.Stream] = None) -> None:
    """One AdamW step of params and moments, in place. A tensor whose gradient is None is left as it is.

    step: t, from 1 on. scale: what gradients are multiplied with first (one over a loss scale, a clipping factor). seed: of the
    roundings to 8 bits. step (int64), lr and scale (float32) may be tensors of one element on the device: a captured call then
    goes on with what they hold at each replay."""
    if stream is not None:
        return L._on(stream, adamw, params, grads, moments, step, lr, beta1, beta2, eps, weight_decay, scale, seed)
    args, _ = _arguments(params, grads, moments, step, lr, beta1, beta2, eps, weight_decay, scale, seed)
    L._call("smat_adamw_step", moments.device, args)


def _arguments(params, grads, moments, step, lr, beta1, beta2, eps, weight_decay, scale, seed):
    """(what smat_adamw_step takes, the arrays that have to live until it returns)"""
    n = len(moments.sizes)
    if len(params) != n or len(grads) != n:
        raise ValueError(f"{len(params)} params and {len(grads)} grads for moments of {n}")
    device = moments.device
    index = device.index
    if index is None:
        raise ValueError("params: must be CUDA tensors")
    pp, pdt = _addresses("params", params, moments.sizes, index, False)
    gp, gdt = _addresses("grads", grads, moments.sizes, index, True)
    code = S.dtype_code(pdt)
    t, step_at = _one("step", step, torch.int64, device)
    rate, lr_at = _one("lr", lr, torch.float32, device)
    by, scale_at = _one("scale", scale, torch.float32, device)
    arrays = ctypes.create_string_buffer(struct.pack(moments._pointers, *pp) + struct.pack(moments._pointers, *gp) + moments._numels)
    at = ctypes.addressof(arrays)
    args = _ADAMW.pack(at, at + 8 * n, at + 16 * n, *moments._addresses(), scale_at, lr_at, step_at, by, rate, beta1, beta2, eps,
                       weight_decay, t, seed & 0xFFFFFFFFFFFFFFFF, n, code, code if gdt is None else S.dtype_code(gdt),
                       moments.bits)
    return args, arrays


def _check(args: bytes, device) -> None:
    """Raises what the step would."""
    if device.index != L._current_device():
        with torch.cuda.device(device):
            return _check(args, device)
    st = L._function("smat_adamw_check")[1](args)
    if st:
        S.check("smat_adamw_check", st)


class AdamW(torch.optim.Optimizer):
    """AdamW whose step is one launch for every group of parameters of one dtype (gradients then share one dtype, and every
    parameter without one is left as it is). bits 8 keeps two bytes of moments per element; with 32 the moments are fp32
    whatever the parameters' type. The group's hyperparameters are those of torch.optim.AdamW, and so are the step counts, one for
    each parameter, which its gradients count (parameters of one count are one launch); `steps` counts the calls. In a captured
    graph use `adamw` with a step on the device."""

    def __init__(self, params, lr: float = 1e-3, betas=(0.9, 0.999), eps: float = 1e-8, weight_decay: float = 0.01, bits: int = 32,
                 seed: int = 0):
        if bits not in (8, 32):
            raise ValueError("bits: 8 or 32")
        self.bits, self.seed, self.steps = bits, int(seed), 0
        self._lists, self.counts = None, []
        super().__init__(params, dict(lr=lr, betas=tuple(betas), eps=eps, weight_decay=weight_decay))

    def __getstate__(self):
        """For copies and pickles, which torch.optim.Optimizer makes of its own fields alone."""
        return {**super().__getstate__(), "bits": self.bits, "seed": self.seed, "steps": self.steps, "counts": self.counts,
                "_lists": self._lists}

    def add_param_group(self, group):
        super().add_param_group(group)
        if self._lists is not None:  # further lists: those that are there keep their place
            try:
                self._lay_out(self.param_groups[-1])
            except Exception:
                self.param_groups.pop()
                raise

    def _lay_out(self, group):
        lists = []
        for dt in dict.fromkeys(p.dtype for p in group["params"]):
            ps = [p for p in group["params"] if p.dtype is dt]
            lists.append((group, ps, Moments(ps, self.bits)))
        self._lists += lists
        self.counts += [[0] * len(ps) for _, ps, _ in lists]

    def lists(self):
        """[(group, parameters of one dtype, their Moments)], laid out at the first step; `counts` holds their step counts."""
        if self._lists is None:
            self._lists = []
            try:
                for group in self.param_groups:
                    self._lay_out(group)
            except Exception:
                self._lists, self.counts = None, []
                raise
        return self._lists

    @torch.no_grad()
    def step(self, closure=None, scale: Union[float, torch.Tensor] = 1.0):
        """One step; scale: see adamw. What is refused leaves every parameter, moment and count as it was."""
        loss = None
        if closure is not None:
            with torch.enable_grad():
                loss = closure()
        calls = []
        for k, (group, ps, moments) in enumerate(self.lists()):
            beta1, beta2 = group["betas"]
            grads = [p.grad if p.grad is None or p.grad.is_contiguous() else p.grad.contiguous() for p in ps]
            counts = self.counts[k]
            there = {c for c, g in zip(counts, grads) if g is not None}
            for t in there:
                gs = grads if len(there) == 1 else [g if c == t else None for c, g in zip(counts, grads)]
                args = _arguments(ps, gs, moments, t + 1, group["lr"], beta1, beta2, group["eps"], group["weight_decay"], scale,
                                  self.seed + k)
                calls.append((moments.device, args, ps, gs, counts))
        if len(calls) > 1:  # all of them before the first moves anything
            for device, args, *_ in calls:
                _check(args[0], device)
        for device, args, ps, gs, counts in calls:
            L._call("smat_adamw_step", device, args[0])
            moved = [i for i, g in enumerate(gs) if g is not None]
            # what a graph saved of those that moved is no longer what it saved
            torch.autograd.graph.increment_version([ps[i] for i in moved])
            for i in moved:
                counts[i] += 1
        self.steps += 1
        return loss

    def state_dict(self):
        """The step counts, the moments' buffers list by list, and the groups' hyperparameters."""
        lists = self.lists()
        return {"steps": self.steps, "counts": [list(c) for c in self.counts], "bits": self.bits, "seed": self.seed,
                "moments": [dict(sizes=list(m.sizes), **m.buffers()) for _, _, m in lists],
                "param_groups": [{k: v for k, v in g.items() if k != "params"} for g in self.param_groups]}

    def load_state_dict(self, state_dict):
        """What does not fit is refused before anything is taken."""
        lists = self.lists()
        saved = state_dict["moments"]
        if state_dict["bits"] != self.bits or [m["sizes"] for m in saved] != [m.sizes for _, _, m in lists]:
            raise ValueError("the state is of other parameters, or of moments in other bits")
        if len(state_dict["param_groups"]) != len(self.param_groups):
            raise ValueError("the state is of other parameter groups")
        steps, seed = int(state_dict["steps"]), int(state_dict["seed"])
        # (a state of before there were counts: one for all)
        counts = [[int(c) for c in cs] for cs in state_dict.get("counts", [[steps] * len(ps) for _, ps, _ in lists])]
        if [len(c) for c in counts] != [len(ps) for _, ps, _ in lists]:
            raise ValueError("the state's step counts are of other parameters")
        for (_, _, m), there in zip(lists, saved):
            for name, t in m.buffers().items():
                if name not in there or there[name].shape != t.shape or there[name].dtype is not t.dtype:
                    raise ValueError(f"the state's {name} is missing or of another form")
        self.steps, self.seed, self.counts = steps, seed, counts
        for (_, _, m), there in zip(lists, saved):
            for name, t in m.buffers().items():
                t.copy_(there[name])
        for group, there in zip(self.param_groups, state_dict["param_groups"]):
            group.update(there)
