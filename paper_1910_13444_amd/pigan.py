"""ctypes binding of libpigan.so (argument marshalling only).

Every step of the PI-GAN hot path runs in the library's HIP kernels; this
module only checks torch tensors (device, dtype, contiguity, sizes), passes
their device pointers and the current HIP stream, and turns non-OK statuses
into exceptions.  There is no CPU fallback: without the built library every
call raises.
"""
from __future__ import annotations

import ctypes as C
import os
import re
import struct
from dataclasses import dataclass

import torch

from .configs import Workload, n_params

_HERE = os.path.dirname(os.path.abspath(__file__))
# PIGAN_LIBRARY selects another build of the same sources (the host-sanitized
# one of the CPU argument-check tests)
LIB_PATH = os.environ.get("PIGAN_LIBRARY") or os.path.join(_HERE, "libpigan.so")
HEADER = os.path.join(os.path.dirname(_HERE), "include", "pigan.h")

OK, EINVAL, ENOTSUP, EWORKSPACE, EDEVICE = 0, 1, 2, 3, 4
STATUS_NAMES = {0: "OK", 1: "EINVAL", 2: "ENOTSUP", 3: "EWORKSPACE", 4: "EDEVICE"}
DTYPES = {"fp32": 0, "bf16": 1, "fp16": 2}
TORCH_DTYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}
ACTS = {"none": 0, "tanh": 1, "relu": 2, "gelu": 3, "silu": 4}

# pigan_linear, pigan_act_args and pigan_norm, each matrix as (p, ld, gs)
LINEAR_ARGS = struct.Struct("4i3q" + "Pqq" * 7 + "3P")
ACT_ARGS = struct.Struct("4i2q" + "Pqq" * 3)
NORM_ARGS = struct.Struct("2i2qfi" + "Pqq" * 5 + "6P")
# pigan_group_norm, each field as (p, ld, ss, gs)
GROUP_NORM_ARGS = struct.Struct("3if4q" + "Pqqq" * 5 + "6P")
# pigan_tensor, pigan_tensors and pigan_adamw
TENSOR = struct.Struct("3Pqd2i")
TENSORS_ARGS = struct.Struct("2i5P")
ADAMW_ARGS = struct.Struct("2P5d3P2i")
ADAMW_WORKSPACE = 256   # PIGAN_ADAMW_WORKSPACE
STATE_BLOCK = 256       # elements of a tensor that share the scale of an 8-bit state


class PiganError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"{STATUS_NAMES.get(status, status)}: {msg}")
        self.status = status


class Mlp(C.Structure):
    _fields_ = [("n_groups", C.c_int32), ("in_dim", C.c_int32), ("n_hidden", C.c_int32), ("width", C.c_int32)]


class StepDesc(C.Structure):
    _fields_ = [("genY", Mlp), ("genU", Mlp), ("disc", Mlp),
                ("d", C.c_int32), ("n_z", C.c_int32), ("S", C.c_int32), ("P", C.c_int32),
                ("n_sY", C.c_int32), ("n_sU", C.c_int32), ("B_r", C.c_int32), ("chunk_S", C.c_int32),
                ("dt", C.c_int32), ("lambda_pde", C.c_float), ("lambda_gp", C.c_float),
                ("loss_scale", C.c_float), ("critic_only", C.c_int32)]


class TrunkDesc(C.Structure):
    _fields_ = [("trunk", Mlp), ("disc", Mlp),
                ("d", C.c_int32), ("n_z", C.c_int32), ("S", C.c_int32), ("P", C.c_int32),
                ("n_sY", C.c_int32), ("n_sU", C.c_int32), ("B_r", C.c_int32), ("chunk_S", C.c_int32),
                ("dt", C.c_int32), ("lambda_pde", C.c_float), ("loss_scale", C.c_float),
                ("lambda_gp", C.c_float), ("critic_only", C.c_int32)]


class HierDesc(C.Structure):
    _fields_ = [("genY", Mlp), ("genU", Mlp), ("disc", Mlp),
                ("d", C.c_int32), ("n_z", C.c_int32), ("S", C.c_int32), ("P", C.c_int32),
                ("n_sY", C.c_int32), ("n_sU", C.c_int32), ("B_r", C.c_int32), ("chunk_S", C.c_int32),
                ("mY", C.c_int32), ("mU", C.c_int32), ("nF", C.c_int32),
                ("dt", C.c_int32), ("lambda_pde", C.c_float), ("loss_scale", C.c_float),
                ("lambda_gp", C.c_float), ("critic_only", C.c_int32)]


class HierTrunkDesc(C.Structure):
    _fields_ = [("trunk", Mlp), ("disc", Mlp),
                ("d", C.c_int32), ("n_z", C.c_int32), ("S", C.c_int32), ("P", C.c_int32),
                ("n_sY", C.c_int32), ("n_sU", C.c_int32), ("B_r", C.c_int32), ("chunk_S", C.c_int32),
                ("mY", C.c_int32), ("mU", C.c_int32), ("nF", C.c_int32),
                ("dt", C.c_int32), ("lambda_pde", C.c_float), ("loss_scale", C.c_float),
                ("lambda_gp", C.c_float), ("critic_only", C.c_int32)]


class KernelStat(C.Structure):
    _fields_ = [("name", C.c_char * 48), ("launches", C.c_int64), ("total_ms", C.c_double),
                ("flops", C.c_double), ("bytes", C.c_double)]


_lib = None
P = C.c_void_p


def lib():
    """Open libpigan.so (raises if it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_1910_13444_amd.build`")
    L = C.CDLL(LIB_PATH)
    i32, i64, f32, f64, sz = C.c_int32, C.c_int64, C.c_float, C.c_double, C.c_size_t
    sigs = {
        "pigan_mlp_n_params": (i64, [P]),
        "pigan_gen_forward_workspace": (sz, [P, i32, i32, i32, i32, i32]),
        "pigan_gen_forward": (i32, [P, P, i32, P, P, i32, i32, i32, i32, i32, P, P, sz, P]),
        "pigan_pde_residual": (i32, [i32, i32, i64, P, P, P, f32, P, P]),
        "pigan_disc_forward_workspace": (sz, [P, i32, i32]),
        "pigan_disc_forward": (i32, [P, P, P, i32, i32, P, P, sz, P]),
        "pigan_workspace_bytes": (sz, [P]),
        "pigan_train_step_grads": (i32, [P, P, P, P, P, P, P, P, P, f32, P, P, P, P, P, P, P, P, sz, P]),
        "pigan_train_step_grads_gp": (i32, [P, P, P, P, P, P, P, P, P, f32, P, P, P, P, P, P, P, P, P, P, sz, P]),
        "pigan_train_step_grads_noalloc": (i32, [P, P, P, P, P, P, P, P, P, f32, P, P, P, P, P, P, P, P]),
        "pigan_adam_update": (i32, [i64, P, P, P, P, f32, f32, f32, f32, i32, P, P]),
        "pigan_hier_workspace_bytes": (sz, [P]),
        "pigan_hier_step_grads": (i32, [P, P, P, P, P, P, P, P, P, f32, P, P, P, P, P, P, P, P, P, P, P, sz, P]),
        "pigan_hier_step_grads_gp": (i32, [P, P, P, P, P, P, P, P, P, f32, P, P, P, P, P, P, P, P, P, P, P, P, P, sz,
                                           P]),
        "pigan_hier_trunk_workspace_bytes": (sz, [P]),
        "pigan_hier_trunk_step_grads": (i32, [P, P, P, P, P, P, P, P, f32, P, P, P, P, P, P, P, P, P, P, sz, P]),
        "pigan_hier_trunk_step_grads_gp": (i32, [P, P, P, P, P, P, P, P, f32, P, P, P, P, P, P, P, P, P, P, P, P, sz,
                                                 P]),
        "pigan_trunk_param_count": (i64, [P]),
        "pigan_trunk_workspace_bytes": (sz, [P]),
        "pigan_trunk_step_grads": (i32, [P, P, P, P, P, P, P, P, f32, P, P, P, P, P, P, P, sz, P]),
        "pigan_trunk_step_grads_gp": (i32, [P, P, P, P, P, P, P, P, f32, P, P, P, P, P, P, P, P, P, sz, P]),
        "pigan_linear_forward_workspace": (sz, [P]),
        "pigan_linear_forward": (i32, [P, P, sz, P]),
        "pigan_linear_backward_workspace": (sz, [P]),
        "pigan_linear_backward": (i32, [P, P, sz, P]),
        "pigan_act_backward": (i32, [P, P]),
        "pigan_layer_norm_forward": (i32, [P, P]),
        "pigan_layer_norm_backward_workspace": (sz, [P]),
        "pigan_layer_norm_backward": (i32, [P, P, sz, P]),
        "pigan_group_norm_forward_workspace": (sz, [P]),
        "pigan_group_norm_forward": (i32, [P, P, sz, P]),
        "pigan_group_norm_backward_workspace": (sz, [P]),
        "pigan_group_norm_backward": (i32, [P, P, sz, P]),
        "pigan_tensors_states": (i64, [P]),
        "pigan_tensors_table_bytes": (sz, [P]),
        "pigan_tensors_table": (i32, [P, P, sz]),
        "pigan_grad_norm_workspace": (sz, [P]),
        "pigan_grad_norm": (i32, [P, P, f64, f64, P, P, P, P, sz, P]),
        "pigan_adamw_update": (i32, [P, P, sz, P]),
        "pigan_state_values": (i32, [i64, P, P, P, P, P, P, P]),
        "pigan_last_error": (C.c_char_p, []),
        "pigan_profile_enable": (i32, [i32]),
        "pigan_profile_read": (i32, [P, i32, P]),
    }
    for name, (res, args) in sigs.items():
        fn = getattr(L, name)
        fn.restype = res
        fn.argtypes = args
    _lib = L
    return L


def declared_symbols() -> list[str]:
    """Function names declared in include/pigan.h."""
    txt = open(HEADER).read()
    txt = re.sub(r"/\*.*?\*/", "", txt, flags=re.S)
    return sorted(set(re.findall(r"\b(pigan_[a-z0-9_]+)\s*\(", txt)))


def _check(status: int):
    if status != OK:
        raise PiganError(status, lib().pigan_last_error().decode())


def _ptr(t: torch.Tensor | None, name: str, numel: int | None = None, dtype=torch.float32):
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if t.dtype != dtype:
        raise ValueError(f"{name} must be {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if numel is not None and t.numel() != numel:
        raise ValueError(f"{name} has {t.numel()} elements, expected {numel}")
    return C.c_void_p(t.data_ptr())


def _stream():
    return C.c_void_p(torch.cuda.current_stream().cuda_stream)


def mlp(G: int, in_dim: int, L: int, W: int) -> Mlp:
    return Mlp(G, in_dim, L, W)


def _workspace(nbytes: int, device) -> torch.Tensor:
    return torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=device)


# ---------------------------------------------------------------------------
# entry points
# ---------------------------------------------------------------------------

def gen_forward(params: torch.Tensor, shape: tuple[int, int, int], d: int, z: torch.Tensor, x: torch.Tensor,
                order: int, dtype: str = "bf16", x_shared: bool = False, out: torch.Tensor | None = None,
                ws: torch.Tensor | None = None) -> torch.Tensor:
    """Generator jets [G, 1 + order*d, S, P] at points x ([G,S,P,d] or [G,P,d] shared)."""
    in_dim, L, W = shape
    G, S, n_z = z.shape
    Pn = x.shape[-2]
    net = Mlp(G, in_dim, L, W)
    dt = DTYPES[dtype]
    need = lib().pigan_gen_forward_workspace(C.byref(net), d, S, Pn, order, dt)
    if need == 0:  # invalid shape: let the library report why
        _check(lib().pigan_gen_forward(C.byref(net), None, d, None, None, 0, S, Pn, order, dt, None, None, 0, None))
    if out is None:
        out = torch.empty((G, 1 + order * d, S, Pn), dtype=torch.float32, device=z.device)
    if ws is None or ws.numel() < need:
        ws = _workspace(need, z.device)
    xn = G * (Pn if x_shared else S * Pn) * d
    st = lib().pigan_gen_forward(C.byref(net), _ptr(params, "params", G * n_params(in_dim, L, W)), d,
                                 _ptr(z, "z"), _ptr(x, "x", xn), int(bool(x_shared)), S, Pn, order, dt,
                                 _ptr(out, "jet", G * (1 + order * d) * S * Pn), _ptr(ws, "ws", dtype=torch.uint8),
                                 ws.numel(), _stream())
    _check(st)
    return out


def pde_residual(jetY: torch.Tensor, jetU: torch.Tensor, d: int, f: torch.Tensor | None = None,
                 f_const: float = 0.0, out: torch.Tensor | None = None) -> torch.Tensor:
    """r = -div(exp(Y) grad u) - f from jets [G,1+d,M] and [G,1+2d,M]."""
    G = jetY.shape[0]
    M = jetY[0, 0].numel()
    if out is None:
        out = torch.empty((G, M), dtype=torch.float32, device=jetY.device)
    st = lib().pigan_pde_residual(d, G, M, _ptr(jetY, "jetY", G * (1 + d) * M), _ptr(jetU, "jetU", G * (1 + 2 * d) * M),
                                  _ptr(f, "f", G * M), float(f_const), _ptr(out, "r", G * M), _stream())
    _check(st)
    return out


def disc_forward(params: torch.Tensor, shape: tuple[int, int, int], snap: torch.Tensor, dtype: str = "bf16",
                 out: torch.Tensor | None = None, ws: torch.Tensor | None = None) -> torch.Tensor:
    in_dim, L, W = shape
    G, B, n_in = snap.shape
    net = Mlp(G, in_dim, L, W)
    dt = DTYPES[dtype]
    need = lib().pigan_disc_forward_workspace(C.byref(net), B, dt)
    if need == 0:
        _check(lib().pigan_disc_forward(C.byref(net), None, None, B, dt, None, None, 0, None))
    if out is None:
        out = torch.empty((G, B), dtype=torch.float32, device=snap.device)
    if ws is None or ws.numel() < need:
        ws = _workspace(need, snap.device)
    st = lib().pigan_disc_forward(C.byref(net), _ptr(params, "params", G * n_params(in_dim, L, W)),
                                  _ptr(snap, "snap", G * B * in_dim), B, dt, _ptr(out, "score", G * B),
                                  _ptr(ws, "ws", dtype=torch.uint8), ws.numel(), _stream())
    _check(st)
    return out


def step_desc(wl: Workload, S: int | None = None, B_r: int | None = None, chunk_S: int = 0,
              dtype: str | None = None, lambda_pde: float | None = None, loss_scale: float = 1.0,
              lambda_gp: float = 0.0) -> StepDesc:
    S = wl.S if S is None else S
    B_r = wl.B_r if B_r is None else B_r
    return StepDesc(Mlp(wl.G, wl.in_dim, wl.L, wl.W), Mlp(wl.G, wl.in_dim, wl.L, wl.W),
                    Mlp(wl.G, wl.n_in, wl.L_D, wl.W_D), wl.d, wl.n_z, S, wl.P, wl.n_sY, wl.n_sU, B_r, chunk_S,
                    DTYPES[dtype or wl.dtype], wl.lambda_pde if lambda_pde is None else lambda_pde, lambda_gp,
                    loss_scale)


def workspace_bytes(desc: StepDesc) -> int:
    return int(lib().pigan_workspace_bytes(C.byref(desc)))


@dataclass
class StepOut:
    gY: torch.Tensor
    gU: torch.Tensor
    gD: torch.Tensor
    loss: torch.Tensor
    nonfinite: torch.Tensor
    gp: torch.Tensor | None = None      # [G] critic gradient penalty (included in loss[:, 0])


class TrainStep:
    """Holds the workspace and output buffers of repeated training steps.
    noalloc=True calls pigan_train_step_grads_noalloc instead: no workspace
    is allocated, the library's fixed device array serves as workspace."""

    def __init__(self, desc: StepDesc, device="cuda", noalloc: bool = False):
        self.desc = desc
        self.noalloc = noalloc
        self.device = torch.device(device)
        G = desc.genY.n_groups
        self.nY = n_params(desc.genY.in_dim, desc.genY.n_hidden, desc.genY.width)
        self.nU = n_params(desc.genU.in_dim, desc.genU.n_hidden, desc.genU.width)
        self.nD = n_params(desc.disc.in_dim, desc.disc.n_hidden, desc.disc.width)
        need = workspace_bytes(desc)
        if need == 0:
            _check(lib().pigan_train_step_grads(C.byref(desc), *([None] * 8), 0.0, *([None] * 8), 0, None))
        self.ws_bytes = need
        self.ws = None if noalloc else _workspace(need, self.device)
        f32 = dict(dtype=torch.float32, device=self.device)
        self.out = StepOut(torch.empty((G, self.nY), **f32), torch.empty((G, self.nU), **f32),
                           torch.empty((G, self.nD), **f32), torch.empty((G, 3), **f32),
                           torch.zeros((1,), dtype=torch.int32, device=self.device),
                           torch.zeros((G,), **f32) if desc.lambda_gp != 0.0 else None)

    def __call__(self, pY, pU, pD, z, xc, xsY, xsU, real, f=None, f_const=0.0, w_group=None,
                 gp_eps=None) -> StepOut:
        """gp_eps: [G, min(S, B_r)] mixing weights of the critic gradient
        penalty (required when the descriptor's lambda_gp is non-zero)."""
        d = self.desc
        G, S, Pn = d.genY.n_groups, d.S, d.P
        o = self.out
        args = [C.byref(d), _ptr(pY, "pY", G * self.nY), _ptr(pU, "pU", G * self.nU), _ptr(pD, "pD", G * self.nD),
                _ptr(z, "z", G * S * d.n_z), _ptr(xc, "xc", G * S * Pn * d.d), _ptr(xsY, "xsY", G * d.n_sY * d.d),
                _ptr(xsU, "xsU", G * d.n_sU * d.d), _ptr(f, "f", G * S * Pn), float(f_const),
                _ptr(real, "real", G * d.B_r * (d.n_sY + d.n_sU)), _ptr(w_group, "w_group", G)]
        outs = [_ptr(o.gY, "gY"), _ptr(o.gU, "gU"), _ptr(o.gD, "gD"), _ptr(o.loss, "loss")]
        tail = [_ptr(o.nonfinite, "nonfinite", 1, dtype=torch.int32), _ptr(self.ws, "ws", dtype=torch.uint8),
                self.ws_bytes, _stream()]
        if self.noalloc:
            st = lib().pigan_train_step_grads_noalloc(*args, *outs, _ptr(o.nonfinite, "nonfinite", 1,
                                                                         dtype=torch.int32), _stream())
        elif d.lambda_gp != 0.0:
            eps = _ptr(gp_eps, "gp_eps", G * min(S, d.B_r))
            st = lib().pigan_train_step_grads_gp(*args, eps, *outs, _ptr(o.gp, "gp", G), *tail)
        else:
            st = lib().pigan_train_step_grads(*args, *outs, *tail)
        _check(st)
        return o


def trunk_desc(wl: Workload, S: int | None = None, B_r: int | None = None, chunk_S: int = 0,
               dtype: str | None = None, lambda_pde: float | None = None, loss_scale: float = 1.0,
               lambda_gp: float = 0.0) -> TrunkDesc:
    S = wl.S if S is None else S
    B_r = wl.B_r if B_r is None else B_r
    return TrunkDesc(Mlp(wl.G, wl.in_dim, wl.L, wl.W), Mlp(wl.G, wl.n_in, wl.L_D, wl.W_D), wl.d, wl.n_z, S, wl.P,
                     wl.n_sY, wl.n_sU, B_r, chunk_S, DTYPES[dtype or wl.dtype],
                     wl.lambda_pde if lambda_pde is None else lambda_pde, loss_scale, lambda_gp)


def trunk_workspace_bytes(desc: TrunkDesc) -> int:
    return int(lib().pigan_trunk_workspace_bytes(C.byref(desc)))


@dataclass
class TrunkOut:
    gT: torch.Tensor
    gD: torch.Tensor
    loss: torch.Tensor
    nonfinite: torch.Tensor
    gp: torch.Tensor | None = None    # [G] gradient penalty (when lambda_gp > 0)


class TrunkStep:
    """Repeated training steps with the shared-trunk generator."""

    def __init__(self, desc: TrunkDesc, device="cuda"):
        self.desc = desc
        self.device = torch.device(device)
        G = desc.trunk.n_groups
        self.nT = int(lib().pigan_trunk_param_count(C.byref(desc.trunk)))
        self.nD = n_params(desc.disc.in_dim, desc.disc.n_hidden, desc.disc.width)
        need = trunk_workspace_bytes(desc)
        if need == 0:
            _check(lib().pigan_trunk_step_grads(C.byref(desc), *([None] * 7), 0.0, *([None] * 7), 0, None))
        self.ws_bytes = need
        self.ws = _workspace(need, self.device)
        f32 = dict(dtype=torch.float32, device=self.device)
        self.out = TrunkOut(torch.empty((G, self.nT), **f32), torch.empty((G, self.nD), **f32),
                            torch.empty((G, 3), **f32), torch.zeros((1,), dtype=torch.int32, device=self.device),
                            torch.empty((G,), **f32) if desc.lambda_gp > 0 else None)

    def __call__(self, pT, pD, z, xc, xsY, xsU, real, f=None, f_const=0.0, w_group=None, gp_eps=None) -> TrunkOut:
        d = self.desc
        G, S, Pn = d.trunk.n_groups, d.S, d.P
        o = self.out
        args = [C.byref(d), _ptr(pT, "pT", G * self.nT), _ptr(pD, "pD", G * self.nD), _ptr(z, "z", G * S * d.n_z),
                _ptr(xc, "xc", G * S * Pn * d.d), _ptr(xsY, "xsY", G * d.n_sY * d.d),
                _ptr(xsU, "xsU", G * d.n_sU * d.d), _ptr(f, "f", G * S * Pn), float(f_const),
                _ptr(real, "real", G * d.B_r * (d.n_sY + d.n_sU)), _ptr(w_group, "w_group", G)]
        tail = [_ptr(o.nonfinite, "nonfinite", 1, dtype=torch.int32), _ptr(self.ws, "ws", dtype=torch.uint8),
                self.ws_bytes, _stream()]
        if d.lambda_gp > 0:
            eps = _ptr(gp_eps, "gp_eps", G * min(S, d.B_r))
            st = lib().pigan_trunk_step_grads_gp(*args, eps, _ptr(o.gT, "gT"), _ptr(o.gD, "gD"),
                                                 _ptr(o.loss, "loss"), _ptr(o.gp, "gp", G), *tail)
        else:
            st = lib().pigan_trunk_step_grads(*args, _ptr(o.gT, "gT"), _ptr(o.gD, "gD"), _ptr(o.loss, "loss"),
                                              *tail)
        _check(st)
        return o


def hier_desc(wl: Workload, D: int, mY: int, mU: int, nF: int, S: int | None = None, B_r: int | None = None,
              chunk_S: int = 0, dtype: str | None = None, lambda_pde: float = 0.0,
              loss_scale: float = 1.0, lambda_gp: float = 0.0) -> HierDesc:
    S = wl.S if S is None else S
    B_r = wl.B_r if B_r is None else B_r
    n_in = mY + mU + nF * (1 + wl.d)
    return HierDesc(Mlp(1, wl.in_dim, wl.L, wl.W), Mlp(1, wl.in_dim, wl.L, wl.W), Mlp(D, n_in, wl.L_D, wl.W_D),
                    wl.d, wl.n_z, S, wl.P, wl.n_sY, wl.n_sU, B_r, chunk_S, mY, mU, nF, DTYPES[dtype or wl.dtype],
                    lambda_pde, loss_scale, lambda_gp)


@dataclass
class HierOut:
    gY: torch.Tensor
    gU: torch.Tensor
    gD: torch.Tensor      # [D, nD]
    loss: torch.Tensor    # [D, 3]: L_D[k], L_adv[k], L_pde
    nonfinite: torch.Tensor
    gp: torch.Tensor | None = None    # [D] every critic's gradient penalty (when lambda_gp > 0)


class HierStep:
    """Repeated domain-decomposition steps: one generator pair, D critics."""

    def __init__(self, desc: HierDesc, device="cuda"):
        self.desc = desc
        self.device = torch.device(device)
        D = desc.disc.n_groups
        self.nY = n_params(desc.genY.in_dim, desc.genY.n_hidden, desc.genY.width)
        self.nU = n_params(desc.genU.in_dim, desc.genU.n_hidden, desc.genU.width)
        self.nD = n_params(desc.disc.in_dim, desc.disc.n_hidden, desc.disc.width)
        need = int(lib().pigan_hier_workspace_bytes(C.byref(desc)))
        if need == 0:
            _check(lib().pigan_hier_step_grads(C.byref(desc), *([None] * 8), 0.0, *([None] * 10), None, 0, None))
        self.ws_bytes = need
        self.ws = _workspace(need, self.device)
        f32 = dict(dtype=torch.float32, device=self.device)
        self.out = HierOut(torch.empty((self.nY,), **f32), torch.empty((self.nU,), **f32),
                           torch.empty((D, self.nD), **f32), torch.empty((D, 3), **f32),
                           torch.zeros((1,), dtype=torch.int32, device=self.device),
                           torch.empty((D,), **f32) if desc.lambda_gp > 0 else None)

    def __call__(self, pY, pU, pD, z, xc, xsY, xsU, idxY, idxU, idxF, real, w_disc, f=None, f_const=0.0,
                 gp_eps=None) -> HierOut:
        """gp_eps: [D, min(S, B_r)] mixing weights of the critics' gradient
        penalty (required when the descriptor's lambda_gp is non-zero)."""
        d = self.desc
        D, S, Pn = d.disc.n_groups, d.S, d.P
        o = self.out
        i32 = torch.int32
        args = [C.byref(d), _ptr(pY, "pY", self.nY), _ptr(pU, "pU", self.nU), _ptr(pD, "pD", D * self.nD),
                _ptr(z, "z", S * d.n_z), _ptr(xc, "xc", S * Pn * d.d), _ptr(xsY, "xsY", d.n_sY * d.d),
                _ptr(xsU, "xsU", d.n_sU * d.d), _ptr(f, "f", S * Pn), float(f_const),
                _ptr(idxY, "idxY", D * d.mY, dtype=i32), _ptr(idxU, "idxU", D * d.mU, dtype=i32),
                _ptr(idxF, "idxF", D * d.nF, dtype=i32), _ptr(real, "real", D * d.B_r * d.disc.in_dim),
                _ptr(w_disc, "w_disc", D)]
        outs = [_ptr(o.gY, "gY"), _ptr(o.gU, "gU"), _ptr(o.gD, "gD"), _ptr(o.loss, "loss")]
        tail = [_ptr(o.nonfinite, "nonfinite", 1, dtype=i32), _ptr(self.ws, "ws", dtype=torch.uint8), self.ws_bytes,
                _stream()]
        if d.lambda_gp > 0:
            eps = _ptr(gp_eps, "gp_eps", D * min(S, d.B_r))
            st = lib().pigan_hier_step_grads_gp(*args, eps, *outs, _ptr(o.gp, "gp", D), *tail)
        else:
            st = lib().pigan_hier_step_grads(*args, *outs, *tail)
        _check(st)
        return o


def hier_trunk_desc(wl: Workload, D: int, mY: int, mU: int, nF: int, S: int | None = None,
                    B_r: int | None = None, chunk_S: int = 0, dtype: str | None = None, lambda_pde: float = 0.0,
                    loss_scale: float = 1.0, lambda_gp: float = 0.0) -> HierTrunkDesc:
    S = wl.S if S is None else S
    B_r = wl.B_r if B_r is None else B_r
    n_in = mY + mU + nF * (1 + wl.d)
    return HierTrunkDesc(Mlp(1, wl.in_dim, wl.L, wl.W), Mlp(D, n_in, wl.L_D, wl.W_D), wl.d, wl.n_z, S, wl.P,
                         wl.n_sY, wl.n_sU, B_r, chunk_S, mY, mU, nF, DTYPES[dtype or wl.dtype], lambda_pde,
                         loss_scale, lambda_gp)


@dataclass
class HierTrunkOut:
    gT: torch.Tensor
    gD: torch.Tensor      # [D, nD]
    loss: torch.Tensor    # [D, 3]: L_D[k], L_adv[k], L_pde
    nonfinite: torch.Tensor
    gp: torch.Tensor | None = None    # [D] every critic's gradient penalty (when lambda_gp > 0)


class HierTrunkStep:
    """Repeated domain-decomposition steps with the shared-trunk generator."""

    def __init__(self, desc: HierTrunkDesc, device="cuda"):
        self.desc = desc
        self.device = torch.device(device)
        D = desc.disc.n_groups
        self.nT = int(lib().pigan_trunk_param_count(C.byref(desc.trunk)))
        self.nD = n_params(desc.disc.in_dim, desc.disc.n_hidden, desc.disc.width)
        need = int(lib().pigan_hier_trunk_workspace_bytes(C.byref(desc)))
        if need == 0:
            _check(lib().pigan_hier_trunk_step_grads(C.byref(desc), *([None] * 7), 0.0, *([None] * 10), 0, None))
        self.ws_bytes = need
        self.ws = _workspace(need, self.device)
        f32 = dict(dtype=torch.float32, device=self.device)
        self.out = HierTrunkOut(torch.empty((self.nT,), **f32), torch.empty((D, self.nD), **f32),
                                torch.empty((D, 3), **f32), torch.zeros((1,), dtype=torch.int32, device=self.device),
                                torch.empty((D,), **f32) if desc.lambda_gp > 0 else None)

    def __call__(self, pT, pD, z, xc, xsY, xsU, idxY, idxU, idxF, real, w_disc, f=None, f_const=0.0,
                 gp_eps=None) -> HierTrunkOut:
        d = self.desc
        D, S, Pn = d.disc.n_groups, d.S, d.P
        o = self.out
        i32 = torch.int32
        args = [C.byref(d), _ptr(pT, "pT", self.nT), _ptr(pD, "pD", D * self.nD), _ptr(z, "z", S * d.n_z),
                _ptr(xc, "xc", S * Pn * d.d), _ptr(xsY, "xsY", d.n_sY * d.d), _ptr(xsU, "xsU", d.n_sU * d.d),
                _ptr(f, "f", S * Pn), float(f_const),
                _ptr(idxY, "idxY", D * d.mY, dtype=i32), _ptr(idxU, "idxU", D * d.mU, dtype=i32),
                _ptr(idxF, "idxF", D * d.nF, dtype=i32), _ptr(real, "real", D * d.B_r * d.disc.in_dim),
                _ptr(w_disc, "w_disc", D)]
        outs = [_ptr(o.gT, "gT"), _ptr(o.gD, "gD"), _ptr(o.loss, "loss")]
        tail = [_ptr(o.nonfinite, "nonfinite", 1, dtype=i32), _ptr(self.ws, "ws", dtype=torch.uint8), self.ws_bytes,
                _stream()]
        if d.lambda_gp > 0:
            eps = _ptr(gp_eps, "gp_eps", D * min(S, d.B_r))
            st = lib().pigan_hier_trunk_step_grads_gp(*args, eps, *outs, _ptr(o.gp, "gp", D), *tail)
        else:
            st = lib().pigan_hier_trunk_step_grads(*args, *outs, *tail)
        _check(st)
        return o


class StepGraph:
    """A step call captured once in a HIP graph (torch.cuda.CUDAGraph) and
    replayed: the same kernels on the same device buffers, launched as one
    graph (no per-kernel launch gaps).  `fn` issues the work on the current
    stream and takes no arguments (e.g. a lambda around a TrainStep call with
    fixed device tensors); it runs once eagerly on a side stream first.  The
    library's launches are all kernels (no memset or host synchronisation), so
    every replay recomputes the outputs from the current contents of the
    inputs."""

    def __init__(self, fn):
        self.fn = fn
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            fn()
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        self.graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(self.graph):
            fn()
        torch.cuda.synchronize()

    def replay(self):
        self.graph.replay()


# ---------------------------------------------------------------------------
# layers of normalised residual networks
# ---------------------------------------------------------------------------
# Matrices are [M, columns], or [G, M, columns] for G independent layers of one
# shape, of one dtype (fp32, bf16, fp16), with unit stride along the columns
# and any strides above; vectors ([columns] or [G, columns]) and parameter
# gradients are fp32.  A result given by the caller may share memory with another
# operand only where its function says so: other overlaps raise PiganError.

_NO_MAT = (0, 0, 0)


def _mat(t: torch.Tensor, name: str, like: torch.Tensor, shape) -> tuple[int, int, int]:
    """(pointer, row stride, group stride) of a matrix operand."""
    if t.dtype != like.dtype:
        raise ValueError(f"{name} must be {like.dtype}, got {t.dtype}")
    if t.shape != shape:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    if t.device != like.device:
        raise ValueError(f"{name} is on {t.device}, expected {like.device}")
    st = t.stride()
    cols = shape[-1]
    if st[-1] != 1 and cols > 1:
        raise ValueError(f"{name} must have unit stride along its columns")
    ld = st[-2] if shape[-2] > 1 else cols
    if ld < cols:
        raise ValueError(f"{name} has overlapping rows (stride {ld}, {cols} columns)")
    if len(st) == 2:
        return t.data_ptr(), ld, 0
    gs = st[0] if shape[0] > 1 else 0
    if shape[0] > 1 and gs < (shape[1] - 1) * ld + cols:
        raise ValueError(f"{name} has overlapping groups (stride {gs})")
    return t.data_ptr(), ld, gs


def _vec(t: torch.Tensor, name: str, like: torch.Tensor, shape) -> int:
    """Pointer of an fp32 vector (one per group)."""
    if t.dtype != torch.float32:
        raise ValueError(f"{name} must be torch.float32, got {t.dtype}")
    if t.shape != shape:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    if t.device != like.device or not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous and on {like.device}")
    return t.data_ptr()


def _new(shape, like: torch.Tensor) -> tuple[torch.Tensor, tuple[int, int, int]]:
    """A matrix for a result, and its operand."""
    t = torch.empty(shape, dtype=like.dtype, device=like.device)
    return t, (t.data_ptr(), shape[-1], shape[-2] * shape[-1])


def _new_vec(shape, like: torch.Tensor) -> tuple[torch.Tensor, int]:
    t = torch.empty(shape, dtype=torch.float32, device=like.device)
    return t, t.data_ptr()


def _layer_dims(x: torch.Tensor, name: str) -> tuple[int, int]:
    """(groups, dtype) of the matrix that sets a call's type and device."""
    if not x.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if x.dim() not in (2, 3):
        raise ValueError(f"{name} must be [rows, columns] or [groups, rows, columns]")
    dt = TORCH_DTYPES.get(x.dtype)
    if dt is None:
        raise ValueError(f"{name} must be fp32, bf16 or fp16, got {x.dtype}")
    return (x.shape[0] if x.dim() == 3 else 1), dt


def _result(need: bool, t: torch.Tensor | None, name: str, like: torch.Tensor, shape):
    """(tensor, operand) of a result: the caller's, a new one, or none."""
    if not need:
        return None, _NO_MAT
    return _new(shape, like) if t is None else (t, _mat(t, name, like, shape))


def _result_vec(need: bool, t: torch.Tensor | None, name: str, like: torch.Tensor, shape):
    if not need:
        return None, 0
    return _new_vec(shape, like) if t is None else (t, _vec(t, name, like, shape))


def _second_vec(need: bool, t: torch.Tensor | None, name: str, like: torch.Tensor, shape, first: torch.Tensor | None):
    """_result_vec beside a first one of its shape, which a new one is made like (the shorter call)"""
    if not need or t is not None:
        return _result_vec(need, t, name, like, shape)
    t = torch.empty_like(first)
    return t, t.data_ptr()


def _act(act: str) -> int:
    if act not in ACTS:
        raise ValueError(f"unknown activation {act!r}: one of {', '.join(ACTS)}")
    return ACTS[act]


def _call(fn, args: bytes, like: torch.Tensor, *ws):
    """One library call on the current stream of the operands' device."""
    dev = like.device
    if dev.index != torch.cuda.current_device():
        with torch.cuda.device(dev):
            return _call(fn, args, like, *ws)
    # the current stream's handle; torch.cuda.current_stream() builds an object
    # around it, which takes as long as the launch of a kernel
    st = fn(args, *ws, torch._C._cuda_getCurrentRawStream(dev.index))
    if st != OK:
        _check(st)


def _call_ws(fn, query, args: bytes, like: torch.Tensor, ws: torch.Tensor | None):
    """_call with a workspace: the caller's where it is large enough, else one
    of the stream's allocator."""
    need = query(args)
    if need > 1 and (ws is None or ws.numel() < need):
        ws = torch.empty(need, dtype=torch.uint8, device=like.device)
    if ws is not None and (ws.dtype != torch.uint8 or ws.device != like.device or not ws.is_contiguous()):
        raise ValueError(f"ws must be a contiguous torch.uint8 tensor on {like.device}")
    if ws is None:
        _call(fn, args, like, None, 0)
    else:
        _call(fn, args, like, ws.data_ptr(), ws.numel())


def linear(x: torch.Tensor, w: torch.Tensor, bias: torch.Tensor | None = None, act: str = "none",
           residual: torch.Tensor | None = None, save_pre: bool = False, out: torch.Tensor | None = None,
           pre: torch.Tensor | None = None, ws: torch.Tensor | None = None):
    """act(x w^T + bias) + residual: x [.., M, K], w [.., N, K], bias [.., N] fp32.

    With save_pre (or `pre`) the pre-activation x w^T + bias is stored too, for
    linear_backward or act_backward, and (y, pre) is returned.  `out` may be
    `residual`."""
    L = lib()
    G, dt = _layer_dims(x, "x")
    *lead, M, K = x.shape
    N = w.shape[-2] if w.dim() == x.dim() else 0
    shape, vec = (*lead, M, N), (*lead, N)
    mw = _mat(w, "w", x, (*lead, N, K))
    mx = _mat(x, "x", x, x.shape)
    out, my = _new(shape, x) if out is None else (out, _mat(out, "out", x, shape))
    if pre is not None:
        mp = _mat(pre, "pre", x, shape)
    else:
        pre, mp = _new(shape, x) if save_pre else (None, _NO_MAT)
    args = LINEAR_ARGS.pack(G, dt, _act(act), 0, M, K, N, *mx, *mw, *my, *mp,
                            *(_NO_MAT if residual is None else _mat(residual, "residual", x, shape)), *_NO_MAT,
                            *_NO_MAT, 0 if bias is None else _vec(bias, "bias", x, vec), 0, 0)
    _call_ws(L.pigan_linear_forward, L.pigan_linear_forward_workspace, args, x, ws)
    return out if pre is None else (out, pre)


def linear_backward(g: torch.Tensor, x: torch.Tensor, w: torch.Tensor, act: str = "none",
                    pre: torch.Tensor | None = None, add: torch.Tensor | None = None, need_dx: bool = True,
                    need_dw: bool = True, need_db: bool = True, dx: torch.Tensor | None = None,
                    dw: torch.Tensor | None = None, db: torch.Tensor | None = None, ws: torch.Tensor | None = None):
    """Gradients of x w^T + bias from its cotangent g [.., M, N]: (dx, dw, db).

    dx = (g w) * act'(pre) + add, where x = act(pre): the cotangent of the
    pre-activation that x was formed from (act "none": of x itself); dw = g^T x
    and db = sum of g over the rows, in fp32.  What is not needed is None.
    `dx` may be `add` or `pre`."""
    L = lib()
    G, dt = _layer_dims(g, "g")
    *lead, M, N = g.shape
    K = x.shape[-1]
    shape = (*lead, M, K)
    mx, mw = _mat(x, "x", g, shape), _mat(w, "w", g, (*lead, N, K))
    dx, mdx = _result(need_dx, dx, "dx", g, shape)
    dw, pdw = _result_vec(need_dw, dw, "dw", g, (*lead, N, K))
    db, pdb = _result_vec(need_db, db, "db", g, (*lead, N))
    args = LINEAR_ARGS.pack(G, dt, _act(act), 0, M, K, N, *mx, *mw, *_NO_MAT,
                            *(_NO_MAT if pre is None else _mat(pre, "pre", g, shape)),
                            *(_NO_MAT if add is None else _mat(add, "add", g, shape)), *_mat(g, "g", g, g.shape), *mdx, 0,
                            pdw, pdb)
    _call_ws(L.pigan_linear_backward, L.pigan_linear_backward_workspace, args, g, ws)
    return dx, dw, db


def act_backward(dy: torch.Tensor, pre: torch.Tensor, act: str, out: torch.Tensor | None = None) -> torch.Tensor:
    """dy * act'(pre): the cotangent of a pre-activation from that of its
    activation.  `out` may be `dy` or `pre`."""
    G, dt = _layer_dims(dy, "dy")
    shape = dy.shape
    md, mp = _mat(dy, "dy", dy, shape), _mat(pre, "pre", dy, shape)
    out, mo = _result(True, out, "out", dy, shape)
    args = ACT_ARGS.pack(G, dt, _act(act), 0, shape[-2], shape[-1], *md, *mp, *mo)
    _call(lib().pigan_act_backward, args, dy)
    return out


def layer_norm(x: torch.Tensor, gamma: torch.Tensor | None = None, beta: torch.Tensor | None = None,
               eps: float = 1e-5, out: torch.Tensor | None = None, mean: torch.Tensor | None = None,
               rstd: torch.Tensor | None = None):
    """(y, mean, rstd): y = (x - mean) rstd gamma + beta over the columns of
    every row, rstd = 1 / sqrt(variance + eps); mean and rstd [.., M] fp32.
    `out` may be `x`."""
    G, dt = _layer_dims(x, "x")
    shape = x.shape
    rows, cols = shape[:-1], (*shape[:-2], shape[-1])
    mx = _mat(x, "x", x, shape)
    out, mo = _result(True, out, "out", x, shape)
    mean, pm = _result_vec(True, mean, "mean", x, rows)
    rstd, pr = _result_vec(True, rstd, "rstd", x, rows)
    args = NORM_ARGS.pack(G, dt, shape[-2], shape[-1], eps, 0, *mx, *mo, *_NO_MAT, *_NO_MAT, *_NO_MAT,
                          0 if gamma is None else _vec(gamma, "gamma", x, cols),
                          0 if beta is None else _vec(beta, "beta", x, cols), pm, pr, 0, 0)
    _call(lib().pigan_layer_norm_forward, args, x)
    return out, mean, rstd


def layer_norm_backward(dy: torch.Tensor, x: torch.Tensor, mean: torch.Tensor, rstd: torch.Tensor,
                        gamma: torch.Tensor | None = None, add: torch.Tensor | None = None, need_dx: bool = True,
                        need_params: bool = True, dx: torch.Tensor | None = None, dgamma: torch.Tensor | None = None,
                        dbeta: torch.Tensor | None = None, ws: torch.Tensor | None = None):
    """Gradients of layer_norm: (dx, dgamma, dbeta), `add` (a skip's cotangent)
    added to dx.  What is not needed is None.  `dx` may be `dy` or `add`."""
    L = lib()
    G, dt = _layer_dims(dy, "dy")
    shape = dy.shape
    rows, cols = shape[:-1], (*shape[:-2], shape[-1])
    dx, mdx = _result(need_dx, dx, "dx", dy, shape)
    dgamma, pg = _result_vec(need_params, dgamma, "dgamma", dy, cols)
    dbeta, pb = _result_vec(need_params, dbeta, "dbeta", dy, cols)
    args = NORM_ARGS.pack(G, dt, shape[-2], shape[-1], 0.0, 0, *_mat(x, "x", dy, shape), *_NO_MAT,
                          *_mat(dy, "dy", dy, shape), *(_NO_MAT if add is None else _mat(add, "add", dy, shape)),
                          *mdx, 0 if gamma is None else _vec(gamma, "gamma", dy, cols), 0,
                          _vec(mean, "mean", dy, rows), _vec(rstd, "rstd", dy, rows), pg, pb)
    _call_ws(L.pigan_layer_norm_backward, L.pigan_layer_norm_backward_workspace, args, dy, ws)
    return dx, dgamma, dbeta


# ---------------------------------------------------------------------------
# group norm: fields [S, P, C] of S samples, P points and C channels, or
# [G, S, P, C] for G independent layers, with unit stride along the channels and
# any strides above
# ---------------------------------------------------------------------------
_NO_FIELD = (0, 0, 0, 0)


def _field(t: torch.Tensor, name: str, like: torch.Tensor, shape) -> tuple[int, int, int, int]:
    """(pointer, point stride, sample stride, group stride) of a field operand."""
    if t is not like:
        if t.dtype != like.dtype:
            raise ValueError(f"{name} must be {like.dtype}, got {t.dtype}")
        if t.shape != shape:
            raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
        if t.device != like.device:
            raise ValueError(f"{name} is on {t.device}, expected {like.device}")
    if t.is_contiguous():
        *_, S, P, C_ = shape
        return t.data_ptr(), C_, P * C_, S * P * C_
    st = t.stride()
    extent = shape[-1]
    if st[-1] != 1 and extent > 1:
        raise ValueError(f"{name} must have unit stride along its channels")
    out = []
    for axis, what in ((-2, "points"), (-3, "samples"), (-4, "groups")):
        if -axis > len(shape) or shape[axis] < 2:
            out.append(extent)   # not used
            continue
        if st[axis] < extent:
            raise ValueError(f"{name} has overlapping {what} (stride {st[axis]}, {extent} elements)")
        out.append(st[axis])
        extent += (shape[axis] - 1) * st[axis]
    return t.data_ptr(), *out


def _field_dims(x: torch.Tensor, name: str) -> tuple[int, int]:
    """(groups, dtype) of the field that sets a call's type and device."""
    if not x.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if x.dim() not in (3, 4):
        raise ValueError(f"{name} must be [samples, points, channels] or [groups, samples, points, channels]")
    dt = TORCH_DTYPES.get(x.dtype)
    if dt is None:
        raise ValueError(f"{name} must be fp32, bf16 or fp16, got {x.dtype}")
    return (x.shape[0] if x.dim() == 4 else 1), dt


def _new_field(need: bool, t: torch.Tensor | None, name: str, like: torch.Tensor, shape):
    """(tensor, operand) of a result: the caller's, a new one, or none."""
    if not need:
        return None, _NO_FIELD
    if t is not None:
        return t, _field(t, name, like, shape)
    t = torch.empty_like(like) if like.is_contiguous() else torch.empty(shape, dtype=like.dtype, device=like.device)
    return t, (t.data_ptr(), shape[-1], shape[-2] * shape[-1], shape[-3] * shape[-2] * shape[-1])


def group_norm(x: torch.Tensor, n: int, gamma: torch.Tensor | None = None, beta: torch.Tensor | None = None,
               act: str = "none", eps: float = 1e-5, out: torch.Tensor | None = None, mean: torch.Tensor | None = None,
               rstd: torch.Tensor | None = None, need_stats: bool = True, ws: torch.Tensor | None = None):
    """(y, mean, rstd): y = act((x - mean) rstd gamma + beta) of x [.., S, P, C],
    each of the n groups of C / n neighbouring channels normalised over its
    channels and all points of a sample, rstd = 1 / sqrt(variance + eps); gamma
    and beta [.., C], mean and rstd [.., S, n] fp32 (None without need_stats).
    `out` may be `x`."""
    L = lib()
    G, dt = _field_dims(x, "x")
    shape = x.shape
    *lead, S, P, C_ = shape
    if n < 1 or C_ % n:
        raise ValueError(f"n = {n} channel groups do not divide {C_} channels")
    chans, stats = (*lead, C_), (*lead, S, n)
    mx = _field(x, "x", x, shape)
    out, mo = _new_field(True, out, "out", x, shape)
    mean, pm = _result_vec(need_stats, mean, "mean", x, stats)
    rstd, pr = _second_vec(need_stats, rstd, "rstd", x, stats, mean)
    args = GROUP_NORM_ARGS.pack(G, dt, _act(act), eps, S, P, C_, n, *mx, *mo, *_NO_FIELD, *_NO_FIELD, *_NO_FIELD,
                                0 if gamma is None else _vec(gamma, "gamma", x, chans),
                                0 if beta is None else _vec(beta, "beta", x, chans), pm, pr, 0, 0)
    _call_ws(L.pigan_group_norm_forward, L.pigan_group_norm_forward_workspace, args, x, ws)
    return out, mean, rstd


def group_norm_backward(dy: torch.Tensor, x: torch.Tensor, mean: torch.Tensor, rstd: torch.Tensor,
                        gamma: torch.Tensor | None = None, beta: torch.Tensor | None = None, act: str = "none",
                        add: torch.Tensor | None = None, need_dx: bool = True, need_params: bool = True,
                        dx: torch.Tensor | None = None, dgamma: torch.Tensor | None = None,
                        dbeta: torch.Tensor | None = None, ws: torch.Tensor | None = None):
    """Gradients of group_norm: (dx, dgamma, dbeta), `add` (a skip's cotangent)
    added to dx.  mean and rstd [.., S, n] say how many channel groups there are.
    What is not needed is None.  `dx` may be `dy` or `add`."""
    L = lib()
    G, dt = _field_dims(dy, "dy")
    shape = dy.shape
    *lead, S, P, C_ = shape
    n = mean.shape[-1] if mean.dim() else 0
    chans, stats = (*lead, C_), (*lead, S, n)
    dx, mdx = _new_field(need_dx, dx, "dx", dy, shape)
    dgamma, pg = _result_vec(need_params, dgamma, "dgamma", dy, chans)
    dbeta, pb = _second_vec(need_params, dbeta, "dbeta", dy, chans, dgamma)
    args = GROUP_NORM_ARGS.pack(G, dt, _act(act), 0.0, S, P, C_, n, *_field(x, "x", dy, shape), *_NO_FIELD,
                                *_field(dy, "dy", dy, shape), *(_NO_FIELD if add is None else _field(add, "add", dy, shape)),
                                *mdx, 0 if gamma is None else _vec(gamma, "gamma", dy, chans),
                                0 if beta is None else _vec(beta, "beta", dy, chans), _vec(mean, "mean", dy, stats),
                                _vec(rstd, "rstd", dy, stats), pg, pb)
    _call_ws(L.pigan_group_norm_backward, L.pigan_group_norm_backward_workspace, args, dy, ws)
    return dx, dgamma, dbeta


# ---------------------------------------------------------------------------
# many tensors at once: their gradients' norm and their AdamW step
# ---------------------------------------------------------------------------

def _flat(t: torch.Tensor, name: str, i: int, dtypes, device) -> int:
    """Pointer of a contiguous device tensor."""
    if t.dtype in dtypes and t.is_cuda and t.device == device and t.is_contiguous():
        return t.data_ptr()
    name = f"{name}[{i}]"
    if not t.is_cuda or t.device != device:
        raise ValueError(f"{name} must be a device tensor, all of them on one device")
    if t.dtype not in dtypes:
        raise ValueError(f"{name} must be {' or '.join(str(d) for d in dtypes)}, got {t.dtype}")
    raise ValueError(f"{name} must be contiguous")


_F32 = (torch.float32,)
_HALVES = (torch.bfloat16, torch.float16)


def _leaf(t: torch.Tensor) -> torch.Tensor:
    return t.detach() if t.requires_grad else t


class TensorTable:
    """Where many tensors are, laid out once for the calls that take all of them:
    gradients (fp32, bf16 or fp16) alone for grad_norm, or with their fp32
    parameters, 16-bit copies (or None for single ones), weight decays (one for
    all, or one each) and states of `bits` bits for adamw_update.

    The states m and v (zero at first) are flat tensors made here, in the order of
    the parameters: fp32, or int8 and uint8 codes with m_scale and v_scale, where
    each tensor begins at a whole block of 256 (pigan.h has the format); `starts`
    are the tensors' first elements in them.  The table holds the tensors, and is
    good as long as they stay where they are: one whose memory was exchanged needs
    a new table, whose states take the values of the old one's (`new.m.copy_(old.m)`;
    v, and in 8 bits the scales, alike)."""

    def __init__(self, grads, params=None, copies=None, decay=0.0, bits: int = 0):
        self.grads = [_leaf(g) for g in grads]
        n = len(self.grads)
        if (bits == 0) != (params is None) or bits not in (0, 8, 32):
            raise ValueError("bits is 8 or 32 with params, 0 without")
        self.params = None if params is None else [_leaf(p) for p in params]
        self.copies = [None if c is None else _leaf(c) for c in copies] if copies is not None else [None] * n
        self.decay = [float(d) for d in decay] if isinstance(decay, (list, tuple)) else [float(decay)] * n
        self.bits = bits
        if not n:
            raise ValueError("no tensors")
        if params is None and copies is not None:
            raise ValueError("copies without params")
        if any(len(v) != n for v in (self.params or self.grads, self.copies, self.decay)):
            raise ValueError(f"{n} gradients need {n} parameters, copies and weight decays")
        dev = self.device = self.grads[0].device
        rows = []
        for i, (g, c, d) in enumerate(zip(self.grads, self.copies, self.decay)):
            pg, pp, pc = _flat(g, "grads", i, TORCH_DTYPES, dev), 0, 0
            if self.params is not None:
                pp = _flat(self.params[i], "params", i, _F32, dev)
                if self.params[i].shape != g.shape:
                    raise ValueError(f"grads[{i}] has shape {tuple(g.shape)}, expected {tuple(self.params[i].shape)}")
            if c is not None:
                pc = _flat(c, "copies", i, _HALVES, dev)
                if c.shape != g.shape:
                    raise ValueError(f"copies[{i}] has shape {tuple(c.shape)}, expected {tuple(g.shape)}")
            rows.append(TENSOR.pack(pp, pg, pc, g.numel(), d, TORCH_DTYPES[g.dtype], 0 if c is None else TORCH_DTYPES[c.dtype]))
        tensors = C.create_string_buffer(b"".join(rows))
        L = lib()

        def args(*states):
            return TENSORS_ARGS.pack(n, bits, C.addressof(tensors), *states)

        count = L.pigan_tensors_states(args(0, 0, 0, 0))
        if count < 0:   # let the library report why
            _check(L.pigan_tensors_table(args(0, 0, 0, 0), None, 0))
        self.m = self.v = self.m_scale = self.v_scale = None
        self.starts, at = [], 0
        for g in self.grads:
            self.starts.append(at)
            at += g.numel() if bits != 8 else -(-g.numel() // STATE_BLOCK) * STATE_BLOCK
        if bits:
            kinds = (torch.int8, torch.uint8) if bits == 8 else (torch.float32, torch.float32)
            self.m, self.v = (torch.zeros(count, dtype=k, device=dev) for k in kinds)
        if bits == 8:
            self.m_scale, self.v_scale = (torch.zeros(count // STATE_BLOCK, dtype=torch.float32, device=dev) for _ in range(2))
        full = args(*(0 if t is None else t.data_ptr() for t in (self.m, self.v, self.m_scale, self.v_scale)))
        size = L.pigan_tensors_table_bytes(full)
        self._host = (C.c_uint64 * -(-size // 8))()
        _check(L.pigan_tensors_table(full, self._host, size))
        self._device = torch.frombuffer(self._host, dtype=torch.uint8).to(dev)
        self.host_ptr, self.device_ptr = C.addressof(self._host), self._device.data_ptr()
        self._norm_ws = int(L.pigan_grad_norm_workspace(self.host_ptr))
        # results of grad_norm are made like these
        self._value, self._flag = (torch.empty((), dtype=k, device=dev) for k in (torch.float32, torch.int32))


def grad_norm(table: TensorTable, max_norm: float = float("inf"), scale: float = 1.0, ws: torch.Tensor | None = None):
    """(norm, coef, nonfinite) of all gradients of a table, on the device:
    norm = scale sqrt(sum of squares) and coef = scale min(1, max_norm / norm) in
    fp32, nonfinite int32 (1 where a gradient is infinite or NaN).  scale is 1 /
    loss scale."""
    L = lib()
    dev = table.device
    if dev.index != torch.cuda.current_device():
        with torch.cuda.device(dev):
            return grad_norm(table, max_norm, scale, ws)
    norm, coef, flag = torch.empty_like(table._value), torch.empty_like(table._value), torch.empty_like(table._flag)
    if ws is None or ws.numel() < table._norm_ws:
        ws = table._device.new_empty(table._norm_ws)
    elif ws.dtype != torch.uint8 or ws.device != dev or not ws.is_contiguous():
        raise ValueError(f"ws must be a contiguous torch.uint8 tensor on {dev}")
    st = L.pigan_grad_norm(table.host_ptr, table.device_ptr, max_norm, scale, norm.data_ptr(), coef.data_ptr(), flag.data_ptr(),
                           ws.data_ptr(), ws.numel(), torch._C._cuda_getCurrentRawStream(dev.index))
    if st != OK:
        _check(st)
    return norm, coef, flag


def _word(t: torch.Tensor | None, name: str, dtype, device) -> int:
    """Pointer of a single device value."""
    if t is None:
        return 0
    if t.dtype != dtype or t.device != device or t.numel() != 1:
        raise ValueError(f"{name} must be one {dtype} value on {device}")
    return t.data_ptr()


def adamw_update(table: TensorTable, lr: float, beta1: float, beta2: float, eps: float, t: int = 0, scale: float = 1.0,
                 coef: torch.Tensor | None = None, skip: torch.Tensor | None = None, step: torch.Tensor | None = None,
                 ws: torch.Tensor | None = None):
    """One AdamW update of every parameter of a table from its gradient times
    scale times coef (one fp32 value on the device, grad_norm's); nothing changes
    where the int32 `skip` on the device is not 0.  The count of updates, this one
    included, is t, or what the int32 `step` on the device is after the call has
    added one to it (for captured calls; a ws of ADAMW_WORKSPACE bytes goes with
    it)."""
    dev = table.device
    if step is not None and (ws is None or ws.numel() < ADAMW_WORKSPACE):
        ws = torch.empty(ADAMW_WORKSPACE, dtype=torch.uint8, device=dev)
    if ws is not None and (ws.dtype != torch.uint8 or ws.device != dev or not ws.is_contiguous()):
        raise ValueError(f"ws must be a contiguous torch.uint8 tensor on {dev}")
    args = ADAMW_ARGS.pack(table.host_ptr, table.device_ptr, lr, beta1, beta2, eps, scale,
                           _word(coef, "coef", torch.float32, dev), _word(skip, "skip", torch.int32, dev),
                           _word(step, "step", torch.int32, dev), t, 0)
    if ws is None:
        _call(lib().pigan_adamw_update, args, table._device, None, 0)
    else:
        _call(lib().pigan_adamw_update, args, table._device, ws.data_ptr(), ws.numel())


def state_values(table: TensorTable):
    """(m, v): a table's flat states as fp32 values (the states themselves where
    they are fp32)."""
    if table.bits != 8:
        return table.m, table.v
    dev = table.device
    if dev.index != torch.cuda.current_device():
        with torch.cuda.device(dev):
            return state_values(table)
    m = torch.empty_like(table.m, dtype=torch.float32)
    v = torch.empty_like(m)
    _check(lib().pigan_state_values(m.numel(), table.m.data_ptr(), table.m_scale.data_ptr(), table.v.data_ptr(),
                                    table.v_scale.data_ptr(), m.data_ptr(), v.data_ptr(),
                                    torch._C._cuda_getCurrentRawStream(dev.index)))
    return m, v


def profile_enable(on: bool = True):
    _check(lib().pigan_profile_enable(1 if on else 0))


def profile_read() -> list[dict]:
    arr = (KernelStat * 64)()
    n = C.c_int32(0)
    _check(lib().pigan_profile_read(arr, 64, C.byref(n)))
    return [dict(name=arr[i].name.decode(), launches=arr[i].launches, total_ms=arr[i].total_ms,
                 flops=arr[i].flops, bytes=arr[i].bytes) for i in range(min(n.value, 64))]
