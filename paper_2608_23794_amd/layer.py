"""A MoCE layer held on the GPU, driven through the C ABI.

``MoceLayer`` owns the device copies of a layer's parameters (support rows,
selected logits, gate parameters), prepares the supports once with
``moce_support_prepare`` and then forwards batches with ``moce_forward`` or
the individual ``moce_pool`` / ``moce_gate`` / ``moce_mix`` calls.
``ProjectLayer`` is a dense projection beside it (``moce_project`` and its
backward), and ``gradient_norm`` / ``clip_gradients`` take the global norm of
the gradients of both (``moce_gradient_norm`` / ``moce_gradient_clip``).  Torch
provides device memory and the current stream; every step of the layer runs in
libmoce's HIP kernels.
"""
from __future__ import annotations

import contextlib
import math
import operator
from typing import Optional

import numpy as np
import torch

from . import binding as mb

_DT = {"f32": mb.MOCE_F32, "bf16": mb.MOCE_BF16}
_LAYOUT = {"nchw": mb.MOCE_NCHW, "nhwc": mb.MOCE_NHWC}
_TORCH_DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def _dev(a, dtype, device) -> torch.Tensor:
    return torch.as_tensor(np.ascontiguousarray(a), dtype=dtype).to(device)


class MoceLayer:
    def __init__(self, C: int, E: int, k: int, H: int, W: int, dtype: str, layout: str,
                 s: np.ndarray, w: np.ndarray, gate: str = "softplus", a=None, c=None,
                 W1=None, b1=None, w2=None, b2: float = 0.0, tau_min: float = 0.2, tau_max: float = 6.0,
                 device: str = "cuda", allow_invalid: bool = False):
        self.C, self.E, self.k, self.H, self.W = C, E, k, H, W
        self.R = E - 1
        self.dtype, self.layout, self.device = dtype, layout, device
        i32, f32 = torch.int32, torch.float32
        R = self.R
        self.s = _dev(np.asarray(s, np.int32).reshape(R, k), i32, device)
        self.w = _dev(np.asarray(w, np.float32).reshape(R, k), f32, device)
        self.s_c = torch.empty((R, k), dtype=i32, device=device)
        self.w_c = torch.empty((R, k), dtype=f32, device=device)
        self.covered = torch.empty(C, dtype=torch.uint8, device=device)
        self.U = torch.empty(C, dtype=i32, device=device)
        self.info = torch.empty(2, dtype=i32, device=device)
        self._keep = []
        if gate == "softplus":
            self.a = _dev(np.asarray(a, np.float32).reshape(R, k), f32, device)
            self.c = _dev(np.asarray(c, np.float32).reshape(R), f32, device)
            self.gate = mb.make_gate(mb.MOCE_GATE_SOFTPLUS_LINEAR, a=self.a, c=self.c)
        elif gate == "mlp":
            self.W1 = _dev(np.asarray(W1, np.float32).reshape(k, k), f32, device)
            self.b1 = _dev(np.asarray(b1, np.float32).reshape(k), f32, device)
            self.w2 = _dev(np.asarray(w2, np.float32).reshape(k), f32, device)
            self.gate = mb.make_gate(mb.MOCE_GATE_MLP_SIGMOID, W1=self.W1, b1=self.b1, w2=self.w2,
                                     b2=float(b2), tau_min=float(tau_min), tau_max=float(tau_max))
        else:
            raise ValueError(gate)
        self.status, self.nU, self.bad_expert = self.prepare(check=False)
        # A failed preparation leaves s_c and U unspecified (channels may lie
        # outside [0, C)), and the kernels do not validate indices.  Such a
        # layer is only kept for inspecting the status (allow_invalid=True),
        # and every entry method below refuses to run on it.
        if self.status != 0 and not allow_invalid:
            raise mb.MoceError("moce_support_prepare", self.status, f"(first bad expert {self.bad_expert})")

    # -- construction helpers ------------------------------------------------
    @classmethod
    def from_workload(cls, wl, params: dict, layout: Optional[str] = None, gate: str = "softplus",
                      device: str = "cuda") -> "MoceLayer":
        return cls(wl.C, wl.E, wl.k, wl.H, wl.W, wl.dtype, layout or wl.layouts[0], params["s"], params["w"],
                   gate=gate, a=params.get("a"), c=params.get("c"), W1=params.get("W1"),
                   b1=params.get("b1"), w2=params.get("w2"), b2=float(params.get("b2", 0.0)),
                   tau_min=float(params.get("tau_min", 0.2)), tau_max=float(params.get("tau_max", 6.0)),
                   device=device)

    def desc(self, B: int) -> mb.moce_desc:
        return mb.make_desc(B, self.C, self.H, self.W, self.E, self.k, _DT[self.dtype], _LAYOUT[self.layout])

    @property
    def torch_dtype(self):
        return _TORCH_DT[self.dtype]

    def y_shape(self, B: int):
        return (B, self.E, self.H, self.W) if self.layout == "nchw" else (B, self.H, self.W, self.E)

    def _stream(self):
        return torch.cuda.current_stream(self.device)

    def _ready(self):
        if self.status != 0:
            raise mb.MoceError("MoceLayer", self.status, "(support preparation failed; the layer cannot run)")

    # -- the C ABI -------------------------------------------------------------
    def prepare(self, check: bool = True):
        return mb.moce_support_prepare(self.desc(1), self.s, self.w, self.s_c, self.w_c, self.covered, self.U,
                                       self.info, self._stream(), check=check)

    def pool(self, x: torch.Tensor, d: Optional[torch.Tensor] = None) -> torch.Tensor:
        self._ready()
        B = x.shape[0]
        if d is None:
            d = torch.empty((B, self.C), dtype=torch.float32, device=self.device)
        mb.moce_pool(self.desc(B), x, d, self._stream())
        return d

    def gate_tau(self, d: torch.Tensor, with_alpha: bool = True):
        self._ready()
        B = d.shape[0]
        tau = torch.empty((B, self.R), dtype=torch.float32, device=self.device)
        alpha = torch.empty((B, self.R, self.k), dtype=torch.float32, device=self.device) if with_alpha else None
        mb.moce_gate(self.desc(B), d, self.s_c, self.w_c, self.gate, tau, alpha, self._stream())
        return tau, alpha

    def gate_mix(self, x: torch.Tensor, d: torch.Tensor, y: Optional[torch.Tensor] = None) -> torch.Tensor:
        """moce_gate_mix: temperatures, coefficients and mixing in one kernel from the pooled d."""
        self._ready()
        B = x.shape[0]
        if y is None:
            y = torch.empty(self.y_shape(B), dtype=x.dtype, device=self.device)
        mb.moce_gate_mix(self.desc(B), x, d, self.s_c, self.w_c, self.gate, self.U if self.nU else None, self.nU,
                         y, self._stream())
        return y

    def mix(self, x: torch.Tensor, alpha: torch.Tensor, y: Optional[torch.Tensor] = None) -> torch.Tensor:
        self._ready()
        B = x.shape[0]
        if y is None:
            y = torch.empty(self.y_shape(B), dtype=x.dtype, device=self.device)
        mb.moce_mix(self.desc(B), x, self.s_c, alpha, self.U if self.nU else None, self.nU, y, self._stream())
        return y

    def workspace_bytes(self, B: int) -> int:
        return mb.moce_forward_workspace_bytes(self.desc(B))

    def new_workspace(self, B: int) -> torch.Tensor:
        return torch.empty(max(self.workspace_bytes(B), 1), dtype=torch.uint8, device=self.device)

    def forward(self, x: torch.Tensor, y: Optional[torch.Tensor] = None,
                ws: Optional[torch.Tensor] = None, epilogue=None) -> torch.Tensor:
        """moce_forward, or with epilogue = (scale, shift, relu) moce_forward_ex (scale and shift: device
        float32 [E] or both None)."""
        self._ready()
        B = x.shape[0]
        if y is None:
            y = torch.empty(self.y_shape(B), dtype=x.dtype, device=self.device)
        if ws is None:
            ws = self.new_workspace(B)
        if epilogue is None:
            mb.moce_forward(self.desc(B), x, self.s_c, self.w_c, self.gate, self.U if self.nU else None, self.nU,
                            y, ws, ws.numel(), self._stream())
        else:
            scale, shift, relu = epilogue
            ep = mb.make_epilogue(scale, shift, relu)
            mb.moce_forward_ex(self.desc(B), x, self.s_c, self.w_c, self.gate, self.U if self.nU else None,
                               self.nU, ep, y, ws, ws.numel(), self._stream())
        return y

    # -- backward --------------------------------------------------------------
    def backward_workspace_bytes(self, B: int) -> int:
        return mb.moce_backward_workspace_bytes(self.desc(B), self.gate.kind)

    def new_backward_workspace(self, B: int) -> torch.Tensor:
        n = self.backward_workspace_bytes(B)
        if n == 0:
            raise mb.MoceError("moce_backward_workspace_bytes", -10, "(shape beyond the backward's limits)")
        return torch.empty(n, dtype=torch.uint8, device=self.device)

    def backward(self, x: torch.Tensor, dy: torch.Tensor, dx: Optional[torch.Tensor] = None,
                 ws: Optional[torch.Tensor] = None) -> dict:
        """moce_backward: dx, dw [E-1][k] (prepared rows) and the gate's parameter gradients."""
        self._ready()
        B = x.shape[0]
        f32, dev = torch.float32, self.device
        if dx is None:
            dx = torch.empty_like(x)
        if ws is None:
            ws = self.new_backward_workspace(B)
        R, k = self.R, self.k
        out = {"dx": dx, "dw": torch.empty((R, k), dtype=f32, device=dev)}
        if self.gate.kind == mb.MOCE_GATE_SOFTPLUS_LINEAR:
            out["da"] = torch.empty((R, k), dtype=f32, device=dev)
            out["dc"] = torch.empty(max(R, 1), dtype=f32, device=dev)
            grads = mb.make_gate_grads(da=out["da"], dc=out["dc"])
        else:
            out["dW1"] = torch.empty((k, k), dtype=f32, device=dev)
            out["db1"] = torch.empty(k, dtype=f32, device=dev)
            out["dw2"] = torch.empty(k, dtype=f32, device=dev)
            out["db2"] = torch.empty(1, dtype=f32, device=dev)
            grads = mb.make_gate_grads(dW1=out["dW1"], db1=out["db1"], dw2=out["dw2"], db2=out["db2"])
        mb.moce_backward(self.desc(B), x, dy, self.s_c, self.w_c, self.gate, dx, out["dw"], grads, ws, ws.numel(),
                         self._stream())
        return out

    def logit_backward(self, L: torch.Tensor, dw: Optional[torch.Tensor], eps: float, lam: float):
        """moce_logit_backward over the full logits L [E-1][C]: (loss, dL)."""
        R, C = self.R, self.C
        n = mb.moce_logit_backward_workspace_bytes(R, C)
        ws = torch.empty(max(n, 1), dtype=torch.uint8, device=self.device)
        loss = torch.empty(1, dtype=torch.float32, device=self.device)
        dL = torch.empty((R, C), dtype=torch.float32, device=self.device)
        mb.moce_logit_backward(R, C, self.k, L, self.s_c if dw is not None else None, dw, eps, lam, loss, dL, ws, n,
                               self._stream())
        return loss, dL


class DynamicMoceLayer:
    """The layer with input-conditioned supports (Sec. 4.5 Eq. 11): device
    copies of the full routing logits, the router and the gate, and the
    library's dynamic forward over them."""

    def __init__(self, C: int, E: int, k: int, H: int, W: int, dtype: str, layout: str, L, Wh, bh, v, q,
                 gate: str = "softplus", a=None, c=None, W1=None, b1=None, w2=None, b2: float = 0.0,
                 tau_min: float = 0.2, tau_max: float = 6.0, device: str = "cuda"):
        self.C, self.E, self.k, self.H, self.W = C, E, k, H, W
        self.R = R = E - 1
        self.dtype, self.layout, self.device = dtype, layout, device
        f32 = torch.float32
        self.dd = int(np.asarray(Wh).shape[0])
        self.L = _dev(np.asarray(L, np.float32).reshape(R, C), f32, device)
        self.Wh = _dev(np.asarray(Wh, np.float32).reshape(self.dd, C), f32, device)
        self.bh = _dev(np.asarray(bh, np.float32).reshape(self.dd), f32, device)
        self.v = _dev(np.asarray(v, np.float32).reshape(C, self.dd), f32, device)
        self.q = _dev(np.asarray(q, np.float32).reshape(R, self.dd), f32, device)
        self.router = mb.make_router(self.dd, self.Wh, self.bh, self.v, self.q)
        if gate == "softplus":
            self.a = _dev(np.asarray(a, np.float32).reshape(R, k), f32, device)
            self.c = _dev(np.asarray(c, np.float32).reshape(R), f32, device)
            self.gate = mb.make_gate(mb.MOCE_GATE_SOFTPLUS_LINEAR, a=self.a, c=self.c)
        elif gate == "mlp":
            self.W1 = _dev(np.asarray(W1, np.float32).reshape(k, k), f32, device)
            self.b1 = _dev(np.asarray(b1, np.float32).reshape(k), f32, device)
            self.w2 = _dev(np.asarray(w2, np.float32).reshape(k), f32, device)
            self.gate = mb.make_gate(mb.MOCE_GATE_MLP_SIGMOID, W1=self.W1, b1=self.b1, w2=self.w2,
                                     b2=float(b2), tau_min=float(tau_min), tau_max=float(tau_max))
        else:
            raise ValueError(gate)

    @classmethod
    def from_workload(cls, wl, params: dict, router: dict, layout: Optional[str] = None, gate: str = "softplus",
                      device: str = "cuda") -> "DynamicMoceLayer":
        return cls(wl.C, wl.E, wl.k, wl.H, wl.W, wl.dtype, layout or wl.layouts[0], router["L"], router["Wh"],
                   router["bh"], router["v"], router["q"], gate=gate, a=params.get("a"), c=params.get("c"),
                   W1=params.get("W1"), b1=params.get("b1"), w2=params.get("w2"), b2=float(params.get("b2", 0.0)),
                   tau_min=float(params.get("tau_min", 0.2)), tau_max=float(params.get("tau_max", 6.0)),
                   device=device)

    def desc(self, B: int) -> mb.moce_desc:
        return mb.make_desc(B, self.C, self.H, self.W, self.E, self.k, _DT[self.dtype], _LAYOUT[self.layout])

    def y_shape(self, B: int):
        return (B, self.E, self.H, self.W) if self.layout == "nchw" else (B, self.H, self.W, self.E)

    def workspace_bytes(self, B: int) -> int:
        return mb.moce_forward_dynamic_workspace_bytes(self.desc(B), self.dd)

    def new_workspace(self, B: int) -> torch.Tensor:
        return torch.empty(max(self.workspace_bytes(B), 1), dtype=torch.uint8, device=self.device)

    def forward(self, x: torch.Tensor, y: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None,
                S_out: Optional[torch.Tensor] = None) -> torch.Tensor:
        B = x.shape[0]
        if y is None:
            y = torch.empty(self.y_shape(B), dtype=x.dtype, device=self.device)
        if ws is None:
            ws = self.new_workspace(B)
        mb.moce_forward_dynamic(self.desc(B), x, self.L, self.router, self.gate, y, S_out, ws, ws.numel(),
                                torch.cuda.current_stream())
        return y


_ACT = {"none": mb.MOCE_ACT_NONE, "relu": mb.MOCE_ACT_RELU, "gelu": mb.MOCE_ACT_GELU, "silu": mb.MOCE_ACT_SILU}
_DTYPE_OF = {torch.float32: mb.MOCE_F32, torch.bfloat16: mb.MOCE_BF16}


def _on(device):
    """The device as the current one, which the library launches on."""
    return torch.cuda.device(device) if torch.cuda.current_device() != device.index else contextlib.nullcontext()


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
    lambda index: torch.cuda.current_stream(index).cuda_stream)


def _need(name: str, t: torch.Tensor, shape, dtype, device):
    """Raises unless t is a contiguous tensor of this shape, type and device: the library sees only its address."""
    if t.shape != shape or t.dtype != dtype or t.device != device or not t.is_contiguous():
        raise ValueError(f"{name} has to be a contiguous {dtype} tensor of shape {tuple(shape)} on {device}, got "
                         f"{t.dtype} {tuple(t.shape)} on {t.device}{'' if t.is_contiguous() else ', strided'}")


def _given_workspace(ws: torch.Tensor, device):
    if ws.device != device or not ws.is_contiguous():
        raise ValueError(f"the workspace has to be a contiguous tensor on {device}, got one on {ws.device}")
    return ws, ws.numel() * ws.element_size()


class ProjectLayer:
    """A dense pointwise projection: y = act(scale x W^T + shift + residual) over the channels.

    weight: [O, C], float32 or bfloat16, on the GPU; scale and shift: float32 [O] or None; act: "none", "relu",
    "gelu" or "silu".  x: [B, C, H, W] for layout "nchw"; [..., C] for "nhwc" (images, tokens or rows).  The layer
    keeps the tensors it is given: updating them in place updates the layer."""

    def __init__(self, weight: torch.Tensor, scale: Optional[torch.Tensor] = None,
                 shift: Optional[torch.Tensor] = None, act: str = "none", layout: str = "nhwc"):
        if act not in _ACT or layout not in _LAYOUT:
            raise ValueError(f"act {act!r}, layout {layout!r}")
        if weight.dim() != 2 or weight.dtype not in _DTYPE_OF or not weight.is_cuda:
            raise ValueError(f"weight has to be a float32 or bfloat16 [O, C] tensor on the GPU, got {weight.dtype} "
                             f"{tuple(weight.shape)} on {weight.device}")
        if weight.numel() == 0:
            raise ValueError(f"weight has to have outputs and channels, got {tuple(weight.shape)}")
        self.O, self.C = weight.shape
        self.dtype, self.device = weight.dtype, weight.device
        _need("weight", weight, weight.shape, self.dtype, self.device)
        for name, t in (("scale", scale), ("shift", shift)):
            if t is not None:
                _need(name, t, (self.O,), torch.float32, self.device)
        self.weight, self.scale, self.shift, self.act, self.layout = weight, scale, shift, act, layout

    def y_shape(self, x_shape):
        if self.layout == "nchw":
            return (x_shape[0], self.O) + tuple(x_shape[2:])
        return tuple(x_shape[:-1]) + (self.O,)

    def desc(self, x_shape) -> mb.moce_project_desc:
        """The call's descriptor for an x of this shape."""
        s = x_shape
        if self.layout == "nchw":
            if len(s) != 4 or s[1] != self.C:
                raise ValueError(f"x has to be [B, {self.C}, H, W], got {tuple(s)}")
            B, H, W = s[0], s[2], s[3]
        else:
            if len(s) < 2 or s[-1] != self.C:
                raise ValueError(f"x has to be [..., {self.C}], got {tuple(s)}")
            B, H, W = math.prod(s[:-1]), 1, 1      # rows of channels, however they are grouped
        return mb.moce_project_desc(B, self.C, H, W, self.O, _DTYPE_OF[self.dtype], _LAYOUT[self.layout],
                                    _ACT[self.act], 0)

    def workspace_bytes(self, x_shape) -> int:
        return mb.moce_project_workspace_bytes(self.desc(x_shape))

    def backward_workspace_bytes(self, x_shape) -> int:
        return mb.moce_project_backward_workspace_bytes(self.desc(x_shape))

    def _workspace(self, n: int, ws: Optional[torch.Tensor]):
        if ws is not None:
            return _given_workspace(ws, self.device)
        return (torch.empty(n, dtype=torch.uint8, device=self.device) if n else None), n

    def forward(self, x: torch.Tensor, residual: Optional[torch.Tensor] = None, y: Optional[torch.Tensor] = None,
                z: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None) -> torch.Tensor:
        """moce_project.  z, where given, receives the pre-activation that the backward needs."""
        desc, shape = self.desc(x.shape), self.y_shape(x.shape)
        _need("x", x, x.shape, self.dtype, self.device)
        if y is None:
            y = torch.empty(shape, dtype=self.dtype, device=self.device)
        for name, t in (("residual", residual), ("y", y), ("z", z)):
            if t is not None:
                _need(name, t, shape, self.dtype, self.device)
        if x.numel() == 0:
            return y
        with _on(self.device):
            ws, n = self._workspace(mb.moce_project_workspace_bytes(desc), ws)
            mb.moce_project(desc, x, self.weight, self.scale, self.shift, residual, y, z, ws, n,
                            _raw_stream(self.device.index))
        return y

    def backward(self, x: torch.Tensor, dy: torch.Tensor, z: Optional[torch.Tensor] = None, residual: bool = False,
                 dx: Optional[torch.Tensor] = None, ws: Optional[torch.Tensor] = None) -> dict:
        """moce_project_backward: dx, dweight, dscale and dshift where the layer has them, and with residual=True
        dresidual.  The scale of a "gelu" or "silu" layer takes a second call over the dz of the first: dweight and
        dscale then come from sums over dz as it is, not scaled before its rounding."""
        desc, shape = self.desc(x.shape), self.y_shape(x.shape)
        f32, dev = torch.float32, self.device
        _need("x", x, x.shape, self.dtype, dev)
        _need("dy", dy, shape, self.dtype, dev)
        if self.act != "none":
            if z is None:
                raise ValueError(f"the backward of {self.act!r} needs the pre-activation z")
            _need("z", z, shape, self.dtype, dev)
        if dx is None:
            dx = torch.empty_like(x)
        _need("dx", dx, x.shape, self.dtype, dev)
        out = {"dx": dx, "dweight": torch.empty_like(self.weight)}
        if self.scale is not None:
            out["dscale"] = torch.empty(self.O, dtype=f32, device=dev)
        if self.shift is not None:
            out["dshift"] = torch.empty(self.O, dtype=f32, device=dev)
        if residual:
            out["dresidual"] = torch.empty_like(dy)
        if x.numel() == 0:
            for t in out.values():
                t.zero_()
            return out
        with _on(dev):
            ws, n = self._workspace(mb.moce_project_backward_workspace_bytes(desc), ws)
            stream, first = _raw_stream(dev.index), out
            two = self.scale is not None and self.act in ("gelu", "silu")
            if two:
                first = {k: v for k, v in out.items() if k not in ("dweight", "dscale")}
                first["dresidual"] = dz = out["dresidual"] if residual else torch.empty_like(dy)
            mb.moce_project_backward(desc, x, self.weight, self.scale, z, dy, mb.make_project_grads(**first), ws, n,
                                     stream)
            if two:
                desc.act = mb.MOCE_ACT_NONE    # needs no more workspace than the activation
                mb.moce_project_backward(desc, x, self.weight, self.scale, None, dz,
                                         mb.make_project_grads(dweight=out["dweight"], dscale=out["dscale"]), ws, n,
                                         stream)
        return out


_dtype = operator.attrgetter("dtype")


def _columns(name: str, tensors):
    """Addresses, sizes and types of the tensors, a list each (hundreds of them: one pass a property is the fastest)."""
    codes = list(map(_DTYPE_OF.get, map(_dtype, tensors)))
    device = tensors[0].get_device()
    if (device < 0 or None in codes or set(map(torch.Tensor.get_device, tensors)) != {device}
            or not all(map(torch.Tensor.is_contiguous, tensors))):
        raise ValueError(f"every {name} has to be a contiguous float32 or bfloat16 tensor on one GPU, got " +
                         ", ".join(f"{t.dtype} {tuple(t.shape)} on {t.device}" for t in tensors)[:300])
    return list(map(torch.Tensor.data_ptr, tensors)), list(map(torch.Tensor.numel, tensors)), codes, device


def _gradient_call(tensors, out, ws, call):
    tensors = list(tensors)
    if not tensors:
        raise ValueError("no gradients")
    src, sizes, codes, index = _columns("gradient", tensors)
    dst = src
    if out is not None:
        out = list(out)
        if len(out) != len(tensors):
            raise ValueError(f"{len(tensors)} gradients, {len(out)} outputs")
        dst, *rest = _columns("output", out)
        if rest != [sizes, codes, index]:
            raise ValueError("an output differs from its gradient in type, size or device")
    device, n = tensors[0].device, len(tensors)
    grads = mb.make_gradients(src, dst, sizes, codes)
    norm = torch.empty(1, dtype=torch.float32, device=device)
    with _on(device):
        if ws is None:
            ws = torch.empty(mb.moce_gradient_workspace_bytes(grads, n), dtype=torch.uint8, device=device)
        call(grads, n, norm, *_given_workspace(ws, device), _raw_stream(index))
    return norm


def gradient_norm(tensors, ws: Optional[torch.Tensor] = None) -> torch.Tensor:
    """moce_gradient_norm: the 2-norm [1] over every element of a list of float32 and bfloat16 tensors."""
    return _gradient_call(tensors, None, ws, mb.moce_gradient_norm)


def clip_gradients(tensors, max_norm: float, out=None, ws: Optional[torch.Tensor] = None) -> torch.Tensor:
    """moce_gradient_clip: scales the tensors (in place, or into the tensors of `out`) so that their global norm is
    at most max_norm; returns the norm [1] before.  Nothing waits for the GPU."""
    return _gradient_call(tensors, out, ws, lambda arr, n, norm, w, nb, st: mb.moce_gradient_clip(
        arr, n, float(max_norm), norm, w, nb, st))


def to_device_x(x: np.ndarray, dtype: str, device: str = "cuda") -> torch.Tensor:
    """Uploads f32 values or bf16 bit patterns (uint16) as a float32/bfloat16 tensor."""
    if dtype == "f32":
        return torch.from_numpy(np.ascontiguousarray(x, np.float32)).to(device)
    bits = np.ascontiguousarray(x, np.uint16).view(np.int16)
    return torch.from_numpy(bits).to(device).view(torch.bfloat16)


def to_host_f64(y: torch.Tensor) -> np.ndarray:
    """Exact float64 copy of a float32 or bfloat16 device tensor."""
    return y.float().cpu().numpy().astype(np.float64)
