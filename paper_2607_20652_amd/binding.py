"""ctypes binding over libdpb.so (the C ABI in include/dpb.h).

Argument marshalling only: every step of the path runs in the library's HIP
kernels.  torch supplies device memory and the current stream.  There is no
fallback: if libdpb.so is missing the first call raises.
"""
from __future__ import annotations

import contextlib
import ctypes
import operator
import os
import struct
from typing import Sequence

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
lib_path = os.path.join(_HERE, "libdpb.so")

DPB_F32, DPB_BF16 = 0, 1
EDIT_ZERO, EDIT_REPLACE, EDIT_RESCALE, EDIT_NONE = 0, 1, 2, 3
_STATUS = {0: "DPB_OK", -1: "DPB_EINVAL", -2: "DPB_EUNSUPPORTED", -3: "DPB_EHIP", -4: "DPB_ENOMEM"}
MAX_LEVELS = 8

_lib = None


class DPBError(RuntimeError):
    def __init__(self, fn: str, status: int):
        self.status = status
        super().__init__(f"{fn} failed: {_STATUS.get(status, status)}")


def load():
    """Loads libdpb.so (built by `python -m paper_2607_20652_amd.build`)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(lib_path):
        raise RuntimeError(f"{lib_path} is not built; run `python -m paper_2607_20652_amd.build`")
    lib = ctypes.CDLL(lib_path)
    i32, i64, u64, P = ctypes.c_int, ctypes.c_int64, ctypes.c_uint64, ctypes.c_void_p
    sig = {
        "dpb_status_string": (ctypes.c_char_p, [i32]),
        "dpb_hierarchy": (i32, [i32, i32, i32, i32, i32, i32, P, P, P]),
        "dpb_build_tables": (i32, [i32, i32, P, P, u64, P, P]),
        "dpb_plan_create": (i32, [P, i32, i32, i32, i32, i32, i32, u64]),
        "dpb_plan_create_ex": (i32, [P, i32, i32, P, P, P, P, u64]),
        "dpb_plan_destroy": (None, [P]),
        "dpb_plan_code_width": (i32, [P]),
        "dpb_plan_describe": (i32, [P, P, P, P, P, P, P, P]),
        "dpb_plan_tables": (i32, [P, P, P]),
        "dpb_encode": (i32, [P, P, i32, i64, P, P, P, ctypes.c_size_t, P]),
        "dpb_decode": (i32, [P, P, P, i64, P, i32, P]),
        "dpb_forward": (i32, [P, P, i32, i64, P, P, P, P, i32, P, ctypes.c_size_t, P]),
        "dpb_decode_bwd": (i32, [P, P, P, i32, i64, P, P, i32, P]),
        "dpb_decode_bwd_ex": (i32, [P, P, P, i32, i64, P, P, P, P, P, i32, P]),
        "dpb_encode_std": (i32, [P, P, i32, i64, P, P, P, P, ctypes.c_size_t, P]),
        "dpb_encode_noalloc": (i32, [P, P, i32, i64, P, P, P, P]),
        "dpb_encode_workspace_bytes": (ctypes.c_size_t, [P, i64]),
        "dpb_std_init": (i32, [P, P, P, P]),
        "dpb_std_workspace_bytes": (ctypes.c_size_t, [P]),
        "dpb_std_update": (i32, [P, P, i32, i64, P, ctypes.c_float, ctypes.c_float, P, P, P, ctypes.c_size_t, P]),
        "dpb_normalize": (i32, [P, P, i32, P, i32, P, i64, i64, P, i32, P, P]),
        "dpb_normalize_bwd": (i32, [P, P, i32, P, i32, P, i32, i64, P, i32, P, i32, i32, P]),
        "dpb_edit_codes": (i32, [P, P, P, P, P, i64, P, P, P, i64, P, P, P]),
        "dpb_variance_workspace_bytes": (ctypes.c_size_t, [P, i64]),
        "dpb_variance_loss": (i32, [P, P, P, i64, i32, P, ctypes.c_size_t, P, P, P, P]),
        "dpb_variance_grad": (i32, [P, i64, P, ctypes.c_size_t, P, P, P]),
        "dpb_attention_workspace_bytes": (ctypes.c_size_t, [P]),
        "dpb_attention_bwd_workspace_bytes": (ctypes.c_size_t, [P]),
        "dpb_attention": (i32, [P, i32] + [P] * 6 + [ctypes.c_size_t, P]),
        "dpb_attention_bwd": (i32, [P, i32] + [P] * 10 + [ctypes.c_size_t, P]),
        "dpb_attention_clear": (i32, [P, i32] + [P] * 5),
        "dpb_embedding": (i32, [i32, P, i64, i64, i32, P, i32, i64, ctypes.c_float, P, P]),
        "dpb_embedding_bwd_workspace_bytes": (ctypes.c_size_t, [i64, i32, i64]),
        "dpb_embedding_bwd": (i32, [i32, P, i64, P, i32, i64, i64, i32, ctypes.c_float, P, P, ctypes.c_size_t, P]),
        "dpb_rms_norm": (i32, [i32, P, i64, P, i64, P, i32, i64, i32, ctypes.c_float, P, P, P, P]),
        "dpb_rms_norm_bwd_workspace_bytes": (ctypes.c_size_t, [i64, i32]),
        "dpb_rms_norm_bwd": (i32, [i32, P, i64, P, i64, P, i64, P, i32, P, i64, i32, P, P, P, ctypes.c_size_t, P]),
        "dpb_cross_entropy_workspace_bytes": (ctypes.c_size_t, [P, i32]),
        "dpb_cross_entropy": (i32, [P, i32, P, i32, P, P, P, ctypes.c_size_t, P]),
        "dpb_cross_entropy_bwd_workspace_bytes": (ctypes.c_size_t, [P, i32]),
        "dpb_cross_entropy_bwd": (i32, [P, i32, P, i32] + [P] * 6 + [ctypes.c_size_t, P]),
        "dpb_adamw_blocks": (i64, [P, i32]),
        "dpb_adamw_step": (i32, [P, i32, P, P, P, P, i32, i32, i32, P, P, P, P, P, P]),
    }
    for name, (res, args) in sig.items():
        fn = getattr(lib, name)
        fn.restype = res
        fn.argtypes = args
    _lib = lib
    return lib


def _need(met: bool, what: str = "arguments of shapes or types that do not fit the call"):
    """A condition of a call, checked under python -O too: what it guards are raw pointers."""
    if not met:
        raise AssertionError(what)


def _check(fn: str, status: int):
    if status != 0:
        raise DPBError(fn, status)


def _ints(vals: Sequence[int]):
    arr = (ctypes.c_int * MAX_LEVELS)()
    for i, v in enumerate(vals):
        arr[i] = int(v)
    return arr


def hierarchy(d: int, n_bits: int, levels: int, branching: int, beam: int, k: int):
    """(level_bits, branching, active) the library derives from configuration terms."""
    nb, br, ac = _ints([]), _ints([]), _ints([])
    _check("dpb_hierarchy", load().dpb_hierarchy(d, n_bits, levels, branching, beam, k, nb, br, ac))
    return list(nb[:levels]), list(br[:levels]), list(ac[:levels])


def build_tables(d: int, level_bits: Sequence[int], branching: Sequence[int], seed: int = 0):
    """Host-only tables (masks [d], generators [sum Delta]) as Python int lists."""
    L = len(level_bits)
    masks = (ctypes.c_uint32 * d)()
    ng = max(1, sum(int(b) for b in list(branching)[1:]))
    gens = (ctypes.c_uint32 * ng)()
    _check("dpb_build_tables",
           load().dpb_build_tables(d, L, _ints(level_bits), _ints(branching), seed & (2**64 - 1), masks, gens))
    return list(masks), list(gens[: sum(int(b) for b in list(branching)[1:])])


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return DPB_F32
    if t.dtype == torch.bfloat16:
        return DPB_BF16
    raise TypeError(f"unsupported dtype {t.dtype}; use float32 or bfloat16")


def _stream(t: torch.Tensor):
    # torch.cuda.current_stream(t.device).cuda_stream without the Stream object (2 us a call)
    return torch._C._cuda_getCurrentRawStream(t.device.index)


def _elsewhere(t: torch.Tensor, name: str, device: int | None):
    """The refusal of a tensor that is not on this device (None: on any)."""
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if device is not None:
        raise ValueError(f"{name} is on device {t.get_device()}, other tensors of the call on {device}")


def _dev(t: torch.Tensor, name: str, device: int | None = None):
    if t.get_device() != device:
        _elsewhere(t, name, device)
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return ctypes.c_void_p(t.data_ptr())


class Plan:
    """A DPB hierarchy and its device tables (one plan per device)."""

    def __init__(self, d: int, n_bits: int | None = None, levels: int | None = None, branching: int | None = None,
                 beam: int | None = None, k: int | None = None, seed: int = 0, *,
                 level_bits: Sequence[int] | None = None, branchings: Sequence[int] | None = None,
                 active: Sequence[int] | None = None, generators: Sequence[int] | None = None,
                 device: torch.device | int | None = None):
        lib = load()
        self._handle = ctypes.c_void_p()
        dev = torch.device("cuda", torch.cuda.current_device()) if device is None else torch.device("cuda", device) \
            if isinstance(device, int) else torch.device(device)
        self.device = dev
        with torch.cuda.device(dev):
            if level_bits is None:
                st = lib.dpb_plan_create(ctypes.byref(self._handle), d, n_bits, levels, branching, beam, k,
                                         seed & (2**64 - 1))
                _check("dpb_plan_create", st)
            else:
                L = len(level_bits)
                g = None
                if generators is not None:
                    g = (ctypes.c_uint32 * max(1, len(generators)))(*[int(v) for v in generators])
                st = lib.dpb_plan_create_ex(ctypes.byref(self._handle), d, L, _ints(level_bits),
                                            _ints(branchings if branchings is not None else [0] * L),
                                            _ints(active), g, seed & (2**64 - 1))
                _check("dpb_plan_create_ex", st)
        self.d = d
        nb, br, ac = _ints([]), _ints([]), _ints([])
        dd, ll = ctypes.c_int(), ctypes.c_int()
        _check("dpb_plan_describe", lib.dpb_plan_describe(self._handle, ctypes.byref(dd), ctypes.byref(ll), nb, br,
                                                          ac, None, None))
        self.levels = ll.value
        self.level_bits = list(nb[: self.levels])
        self.branching = list(br[: self.levels])
        self.active = list(ac[: self.levels])
        self.k_tot = lib.dpb_plan_code_width(self._handle)

    def tables(self):
        """Host copies of the plan's masks [d] and generators (level by level)."""
        lib = load()
        masks = (ctypes.c_uint32 * self.d)()
        ng = max(1, sum(self.branching[1:]))
        gens = (ctypes.c_uint32 * ng)()
        _check("dpb_plan_tables", lib.dpb_plan_tables(self._handle, masks, gens))
        return list(masks), list(gens[: sum(self.branching[1:])])

    def close(self):
        if getattr(self, "_handle", None) and self._handle.value:
            load().dpb_plan_destroy(self._handle)
            self._handle = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def encode_workspace(plan: Plan, T: int, device) -> torch.Tensor | None:
    """Workspace for encode of T tokens, or None when the plan needs none."""
    n = int(load().dpb_encode_workspace_bytes(plan._handle, int(T)))
    return None if n == 0 else torch.empty(((n + 15) // 16) * 4, dtype=torch.float32, device=device)


def encode(plan: Plan, x: torch.Tensor, idx: torch.Tensor | None = None, coef: torch.Tensor | None = None,
           stats: torch.Tensor | None = None, workspace: torch.Tensor | None = None):
    """x [T, d] fp32/bf16 (device) -> (idx [T, k_tot] int32, coef [T, k_tot] fp32); on
    standardized scores when stats is given.  A workspace is allocated when the
    plan needs one (wide hierarchies) and none is given."""
    T = x.shape[0]
    _need(x.dim() == 2 and x.shape[1] == plan.d)
    if idx is None:
        idx = torch.empty((T, plan.k_tot), dtype=torch.int32, device=x.device)
    if coef is None:
        coef = torch.empty((T, plan.k_tot), dtype=torch.float32, device=x.device)
    if workspace is None:
        workspace = encode_workspace(plan, T, x.device)
    nbytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    if stats is None:
        _check("dpb_encode", load().dpb_encode(plan._handle, _dev(x, "x"), _dtype_code(x), T, _dev(idx, "idx"),
                                               _dev(coef, "coef"), _opt(workspace, "workspace"), nbytes,
                                               _stream(x)))
    else:
        _check("dpb_encode_std", load().dpb_encode_std(plan._handle, _dev(x, "x"), _dtype_code(x), T,
                                                       _dev(stats, "stats"), _dev(idx, "idx"), _dev(coef, "coef"),
                                                       _opt(workspace, "workspace"), nbytes, _stream(x)))
    return idx, coef


def encode_noalloc(plan: Plan, x: torch.Tensor, idx: torch.Tensor, coef: torch.Tensor,
                   stats: torch.Tensor | None = None):
    """encode (stats None) or encode_std into the given idx, coef [T, k_tot]
    through the library's allocation-free entry point (no workspace)."""
    T = x.shape[0]
    _need(x.dim() == 2 and x.shape[1] == plan.d and idx.shape == coef.shape == (T, plan.k_tot))
    _check("dpb_encode_noalloc", load().dpb_encode_noalloc(plan._handle, _dev(x, "x"), _dtype_code(x), T,
                                                           _opt(stats, "stats"), _dev(idx, "idx"),
                                                           _dev(coef, "coef"), _stream(x)))
    return idx, coef


def forward(plan: Plan, x: torch.Tensor, idx: torch.Tensor | None = None, coef: torch.Tensor | None = None,
            y: torch.Tensor | None = None, stats: torch.Tensor | None = None, out_dtype: torch.dtype | None = None,
            workspace: torch.Tensor | None = None):
    """x [T, d] -> (idx, coef, y): encode (on standardized scores when stats is
    given) and decode in one library call (dpb_forward); y [T, d] in out_dtype
    (default: the type of x)."""
    T = x.shape[0]
    _need(x.dim() == 2 and x.shape[1] == plan.d)
    if idx is None:
        idx = torch.empty((T, plan.k_tot), dtype=torch.int32, device=x.device)
    if coef is None:
        coef = torch.empty((T, plan.k_tot), dtype=torch.float32, device=x.device)
    if y is None:
        y = torch.empty((T, plan.d), dtype=out_dtype or x.dtype, device=x.device)
    if workspace is None:
        workspace = encode_workspace(plan, T, x.device)
    nbytes = 0 if workspace is None else workspace.numel() * workspace.element_size()
    _check("dpb_forward", load().dpb_forward(plan._handle, _dev(x, "x"), _dtype_code(x), T, _opt(stats, "stats"),
                                             _dev(idx, "idx"), _dev(coef, "coef"), _dev(y, "y"), _dtype_code(y),
                                             _opt(workspace, "workspace"), nbytes, _stream(x)))
    return idx, coef, y


def decode(plan: Plan, idx: torch.Tensor, coef: torch.Tensor, out_dtype: torch.dtype = torch.float32,
           y: torch.Tensor | None = None):
    """(idx, coef) [T, k_tot] -> y [T, d] in out_dtype (fp32 or bf16)."""
    T = idx.shape[0]
    _need(idx.dtype == torch.int32 and coef.dtype == torch.float32 and idx.shape == coef.shape)
    _need(idx.shape[1] == plan.k_tot)
    if y is None:
        y = torch.empty((T, plan.d), dtype=out_dtype, device=idx.device)
    _check("dpb_decode", load().dpb_decode(plan._handle, _dev(idx, "idx"), _dev(coef, "coef"), T, _dev(y, "y"),
                                           _dtype_code(y), _stream(idx)))
    return y


def decode_bwd(plan: Plan, idx: torch.Tensor, grad_y: torch.Tensor, gx_dtype: torch.dtype | None = None,
               grad_coef: torch.Tensor | None = None, grad_x: torch.Tensor | None = None):
    """(idx [T, k_tot], grad_y [T, d]) -> (grad_coef [T, k_tot] fp32, grad_x [T, d])."""
    T = idx.shape[0]
    _need(idx.dtype == torch.int32 and idx.shape[1] == plan.k_tot and grad_y.shape == (T, plan.d))
    if grad_coef is None:
        grad_coef = torch.empty((T, plan.k_tot), dtype=torch.float32, device=idx.device)
    if grad_x is None:
        grad_x = torch.empty((T, plan.d), dtype=gx_dtype or grad_y.dtype, device=idx.device)
    _check("dpb_decode_bwd", load().dpb_decode_bwd(plan._handle, _dev(idx, "idx"), _dev(grad_y, "grad_y"),
                                                   _dtype_code(grad_y), T, _dev(grad_coef, "grad_coef"),
                                                   _dev(grad_x, "grad_x"), _dtype_code(grad_x), _stream(idx)))
    return grad_coef, grad_x


def _opt(t: torch.Tensor | None, name: str, device: int | None = None):
    return None if t is None else _dev(t, name, device)


def decode_bwd_ex(plan: Plan, idx: torch.Tensor, grad_y: torch.Tensor, add_grad_coef: torch.Tensor | None = None,
                  add_grad_x: torch.Tensor | None = None, gx_dtype: torch.dtype | None = None,
                  grad_coef: torch.Tensor | None = None, grad_x: torch.Tensor | None = None,
                  stats: torch.Tensor | None = None):
    """decode_bwd plus extra terms: grad_coef = Phi^T g + add_grad_coef,
    grad_x = Phi (r * grad_coef) + add_grad_x, r from the standardization
    statistics when given (else 1); add_grad_x is in grad_x's dtype and may
    be grad_x itself."""
    T = idx.shape[0]
    _need(idx.dtype == torch.int32 and idx.shape[1] == plan.k_tot and grad_y.shape == (T, plan.d))
    if grad_coef is None:
        grad_coef = torch.empty((T, plan.k_tot), dtype=torch.float32, device=idx.device)
    if grad_x is None:
        grad_x = torch.empty((T, plan.d), dtype=gx_dtype or grad_y.dtype, device=idx.device)
    if add_grad_coef is not None:
        _need(add_grad_coef.dtype == torch.float32 and add_grad_coef.shape == (T, plan.k_tot))
    if add_grad_x is not None:
        _need(add_grad_x.dtype == grad_x.dtype and add_grad_x.shape == (T, plan.d))
    _check("dpb_decode_bwd_ex", load().dpb_decode_bwd_ex(
        plan._handle, _dev(idx, "idx"), _dev(grad_y, "grad_y"), _dtype_code(grad_y), T,
        _opt(add_grad_coef, "add_grad_coef"), _opt(add_grad_x, "add_grad_x"), _opt(stats, "stats"),
        _dev(grad_coef, "grad_coef"), _dev(grad_x, "grad_x"), _dtype_code(grad_x), _stream(idx)))
    return grad_coef, grad_x


def normalize(plan: Plan, u: torch.Tensor, ref: torch.Tensor, ref_rows: torch.Tensor | None = None,
              out_dtype: torch.dtype | None = None, y: torch.Tensor | None = None, with_norms: bool = False):
    """y = u ||ref_r|| / ||u|| per row (r = ref_rows[t] or t); optionally the
    (||ref_r||, ||u||) pairs [T, 2]."""
    T = u.shape[0]
    _need(u.shape == (T, plan.d) and ref.dim() == 2 and ref.shape[1] == plan.d)
    if ref_rows is not None:
        _need(ref_rows.dtype == torch.int32 and ref_rows.shape == (T,))
    else:
        _need(ref.shape[0] == T)
    if y is None:
        y = torch.empty((T, plan.d), dtype=out_dtype or u.dtype, device=u.device)
    norms = torch.empty((T, 2), dtype=torch.float32, device=u.device) if with_norms else None
    _check("dpb_normalize", load().dpb_normalize(
        plan._handle, _dev(u, "u"), _dtype_code(u), _dev(ref, "ref"), _dtype_code(ref), _opt(ref_rows, "ref_rows"),
        ref.shape[0], T, _dev(y, "y"), _dtype_code(y), _opt(norms, "norms"), _stream(u)))
    return (y, norms) if with_norms else y


def normalize_bwd(plan: Plan, g: torch.Tensor, u: torch.Tensor, ref: torch.Tensor,
                  gu_dtype: torch.dtype | None = None, grad_ref: torch.Tensor | None = None,
                  accumulate: bool = False, gr_dtype: torch.dtype | None = None):
    """(grad_u, grad_ref) of normalize for upstream g; grad_ref is added to
    the given buffer when accumulate is True."""
    T = u.shape[0]
    _need(g.shape == u.shape == ref.shape == (T, plan.d))
    grad_u = torch.empty((T, plan.d), dtype=gu_dtype or g.dtype, device=u.device)
    if grad_ref is None:
        _need(not accumulate)
        grad_ref = torch.empty((T, plan.d), dtype=gr_dtype or ref.dtype, device=u.device)
    _check("dpb_normalize_bwd", load().dpb_normalize_bwd(
        plan._handle, _dev(g, "g"), _dtype_code(g), _dev(u, "u"), _dtype_code(u), _dev(ref, "ref"),
        _dtype_code(ref), T, _dev(grad_u, "grad_u"), _dtype_code(grad_u), _dev(grad_ref, "grad_ref"),
        _dtype_code(grad_ref), int(bool(accumulate)), _stream(u)))
    return grad_u, grad_ref


def edit_codes(plan: Plan, idx: torch.Tensor, coef: torch.Tensor, rows: torch.Tensor, slots: torch.Tensor,
               ops: torch.Tensor, tgt_idx: torch.Tensor | None = None, tgt_coef: torch.Tensor | None = None):
    """One edited copy of source row rows[e] per edit (slot slots[e], op
    ops[e]: EDIT_ZERO, EDIT_REPLACE, EDIT_RESCALE, EDIT_NONE) -> (idx, coef) [E, k_tot]."""
    T, E = idx.shape[0], rows.shape[0]
    _need(idx.shape == coef.shape == (T, plan.k_tot) and idx.dtype == torch.int32 and coef.dtype == torch.float32)
    for t in (rows, slots, ops):
        _need(t.dtype == torch.int32 and t.shape == (E,))
    out_idx = torch.empty((E, plan.k_tot), dtype=torch.int32, device=idx.device)
    out_coef = torch.empty((E, plan.k_tot), dtype=torch.float32, device=idx.device)
    _check("dpb_edit_codes", load().dpb_edit_codes(
        plan._handle, _dev(idx, "idx"), _dev(coef, "coef"), _opt(tgt_idx, "tgt_idx"), _opt(tgt_coef, "tgt_coef"), T,
        _dev(rows, "rows"), _dev(slots, "slots"), _dev(ops, "ops"), E, _dev(out_idx, "out_idx"),
        _dev(out_coef, "out_coef"), _stream(idx)))
    return out_idx, out_coef


def variance_workspace_bytes(plan: Plan, T: int) -> int:
    return int(load().dpb_variance_workspace_bytes(plan._handle, int(T)))


def variance_workspace(plan: Plan, T: int, device) -> torch.Tensor:
    """A device buffer of dpb_variance_workspace_bytes(plan, T) bytes."""
    return torch.empty((variance_workspace_bytes(plan, T) + 15) // 16 * 4, dtype=torch.float32, device=device)


def variance_loss(plan: Plan, idx: torch.Tensor, coef: torch.Tensor, n_min: int, with_grad: bool = True,
                  workspace: torch.Tensor | None = None, grad_scale: torch.Tensor | None = None):
    """Variance auxiliary loss of a batch of codes -> (loss [] fp32, grad_coef
    [T, k_tot] fp32 or None); grad_coef is multiplied by the device scalar
    grad_scale when given."""
    T = idx.shape[0]
    _need(idx.shape == coef.shape == (T, plan.k_tot) and idx.dtype == torch.int32 and coef.dtype == torch.float32)
    if workspace is None:
        workspace = variance_workspace(plan, T, idx.device)
    loss = torch.empty((), dtype=torch.float32, device=idx.device)
    grad = torch.empty((T, plan.k_tot), dtype=torch.float32, device=idx.device) if with_grad else None
    _check("dpb_variance_loss", load().dpb_variance_loss(
        plan._handle, _dev(idx, "idx"), _dev(coef, "coef"), T, int(n_min), _dev(workspace, "workspace"),
        workspace.numel() * workspace.element_size(), _dev(loss, "loss"), _opt(grad, "grad_coef"),
        _opt(grad_scale, "grad_scale"), _stream(idx)))
    return loss, grad


def variance_grad(plan: Plan, T: int, workspace: torch.Tensor, grad_scale: torch.Tensor | None = None,
                  grad: torch.Tensor | None = None):
    """Gradient of the variance loss from what a variance_loss call over T
    tokens left in `workspace`."""
    if grad is None:
        grad = torch.empty((T, plan.k_tot), dtype=torch.float32, device=workspace.device)
    _check("dpb_variance_grad", load().dpb_variance_grad(
        plan._handle, int(T), _dev(workspace, "workspace"), workspace.numel() * workspace.element_size(),
        _dev(grad, "grad_coef"), _opt(grad_scale, "grad_scale"), _stream(workspace)))
    return grad


STD_SAMPLE = 64


def std_state(plan: Plan, device=None):
    """Fresh standardization state (stats [N, 2] = (mu, r), m2 [N]) at its
    initial value (mu 0, r 1, m2 1)."""
    device = device or plan.device
    N = 1 << plan.level_bits[-1]
    stats = torch.empty((N, 2), dtype=torch.float32, device=device)
    m2 = torch.empty((N,), dtype=torch.float32, device=device)
    _check("dpb_std_init", load().dpb_std_init(plan._handle, _dev(stats, "stats"), _dev(m2, "m2"),
                                               _stream(stats)))
    return stats, m2


def encode_std(plan: Plan, x: torch.Tensor, stats: torch.Tensor, idx: torch.Tensor | None = None,
               coef: torch.Tensor | None = None, workspace: torch.Tensor | None = None):
    """Encoder on standardized scores z = (s - mu) r -> (idx, coef = z)."""
    _need(stats.dtype == torch.float32 and stats.shape == (1 << plan.level_bits[-1], 2))
    return encode(plan, x, idx, coef, stats=stats, workspace=workspace)


def std_workspace(plan: Plan, device) -> torch.Tensor:
    n = int(load().dpb_std_workspace_bytes(plan._handle))
    return torch.empty(((n + 15) // 16) * 4, dtype=torch.float32, device=device)


def std_update(plan: Plan, x: torch.Tensor, idx: torch.Tensor, stats: torch.Tensor, m2: torch.Tensor,
               momentum: float, eps: float = 1e-6, workspace: torch.Tensor | None = None):
    """EMA update of (stats, m2) in place from the batch x and its code idx."""
    T = x.shape[0]
    _need(idx.shape == (T, plan.k_tot) and idx.dtype == torch.int32)
    if workspace is None:
        workspace = std_workspace(plan, x.device)
    _check("dpb_std_update", load().dpb_std_update(
        plan._handle, _dev(x, "x"), _dtype_code(x), T, _dev(idx, "idx"), float(momentum), float(eps),
        _dev(stats, "stats"), _dev(m2, "m2"), _dev(workspace, "workspace"),
        workspace.numel() * workspace.element_size(), _stream(x)))
    return stats, m2


# ---- training operators beside the bottleneck: attention and AdamW

def _written(tensors):
    """Tells autograd that the library wrote these of the caller's tensors, as torch's own
    in-place operations do: a graph that saved one before is an error afterwards."""
    tensors = [t for t in tensors if t is not None]
    try:
        torch.autograd.graph.increment_version(tensors)
    except RuntimeError:   # inference tensors have no versions
        torch.autograd.graph.increment_version([t for t in tensors if not t.is_inference()])


# dpb_attn and dpb_heads as bytes: several times quicker to make than ctypes
# structures, which tells in a call for one token
_ATTN = struct.Struct("=qqqqqiiiif4xQQQQ")
_HEADS = struct.Struct("=Qqqq")


_SAME_DEVICE = contextlib.nullcontext()


def _device_of(t: torch.Tensor, name: str):
    """(device, context in which it is the current one): the training operators, which have no
    plan, run on the current device, and that has to be their tensors'."""
    device = t.get_device()
    if device < 0:
        _elsewhere(t, name, None)
    return device, _SAME_DEVICE if device == torch._C._cuda_getDevice() else torch.cuda.device(device)


def _heads(t: torch.Tensor, name: str, device: int | None = None) -> bytes:
    st = t.stride()
    if t.get_device() != device:
        _elsewhere(t, name, device)
    if st[-1] != 1 and t.shape[-1] > 1:
        raise ValueError(f"{name} must be contiguous along head_dim")
    return _HEADS.pack(t.data_ptr(), st[0] if len(st) == 4 else 0, st[-3], st[-2])


def _index(t: torch.Tensor | None, n: int, name: str, device: int) -> int:
    """Address of an int32 device array of n entries, or 0."""
    if t is None:
        return 0
    if t.dtype != torch.int32 or t.shape != (n,):
        raise AssertionError(f"{name}: int32 [{n}]")
    return _dev(t, name, device).value or 0


def _attn(q, k, v, causal, scale, q_lens, k_lens, q_starts, k_starts, max_q, max_k) -> bytes:
    """The description of an attention call, its arguments checked."""
    qs, ks, device = q.shape, k.shape, q.get_device()
    packed = q_starts is not None
    _need(packed == (k_starts is not None), "packed sequences need q_starts and k_starts")
    _need(len(qs) == len(ks) == (3 if packed else 4) and v.shape == ks and ks[-1] == qs[-1])
    _need(q.dtype == k.dtype == v.dtype)
    if packed:
        _need(q_lens is None and k_lens is None and max_q is not None and max_k is not None)
        batch, q_len, k_len, q_rows, k_rows = len(q_starts) - 1, int(max_q), int(max_k), qs[0], ks[0]
        _need(batch >= 0)
    else:
        batch, q_len, k_len, q_rows, k_rows = qs[0], qs[1], ks[1], 0, 0
        _need(ks[0] == batch)
    return _ATTN.pack(batch, q_len, k_len, q_rows, k_rows, qs[-2], ks[-2], qs[-1], int(bool(causal)),
                      qs[-1] ** -0.5 if scale is None else scale, _index(q_lens, batch, "q_lens", device),
                      _index(k_lens, batch, "k_lens", device), _index(q_starts, batch + 1, "q_starts", device),
                      _index(k_starts, batch + 1, "k_starts", device))


def attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, causal: bool = False, scale: float | None = None,
              q_lens: torch.Tensor | None = None, k_lens: torch.Tensor | None = None,
              q_starts: torch.Tensor | None = None, k_starts: torch.Tensor | None = None,
              max_q: int | None = None, max_k: int | None = None, out: torch.Tensor | None = None,
              lse: torch.Tensor | None = None, workspace: torch.Tensor | None = None):
    """softmax(scale q k^T) v -> (out like q, lse fp32 [..., heads]).

    Padded: q [B, Sq, H, D], k and v [B, Sk, Hkv, D] (any order in memory), with
    lengths q_lens / k_lens int32 [B] or none; packed: q [rows, H, D], k and v
    [rows, Hkv, D] with q_starts / k_starts int32 [B + 1] and the longest sequences
    max_q / max_k.  scale defaults to 1 / sqrt(D); causal: query i sees the keys
    j <= i + k_len - q_len.  A query that sees none gets 0 and lse -inf, and so do packed
    rows of no sequence in outputs made here; in an out or lse that is given those
    rows are left as they are.  Tensors start on 16 bytes and their strides are multiples of 16
    bytes (0 too, for inputs)."""
    a = _attn(q, k, v, causal, scale, q_lens, k_lens, q_starts, k_starts, max_q, max_k)
    new_out, new_lse, given = out is None, lse is None, (out, lse)
    if out is None:
        out = torch.empty_like(q, memory_format=torch.contiguous_format)
    if lse is None:
        lse = q.new_empty(q.shape[:-1], dtype=torch.float32)
    _need(out.shape == q.shape and out.dtype == q.dtype)
    _need(lse.shape == q.shape[:-1] and lse.dtype == torch.float32)
    lib = load()
    device, here = _device_of(q, "q")
    with here:
        need = lib.dpb_attention_workspace_bytes(a)
        if need and workspace is None:
            workspace = torch.empty((need + 3) // 4, dtype=torch.float32, device=q.device)
        o, l = _heads(out, "out", device), _dev(lse, "lse", device)
        _check("dpb_attention", lib.dpb_attention(
            a, _dtype_code(q), _heads(q, "q"), _heads(k, "k", device), _heads(v, "v", device), o, l,
            _opt(workspace, "workspace", device), 0 if workspace is None else workspace.numel() * workspace.element_size(),
            _stream(q)))
        if q_starts is not None and (new_out or new_lse):
            _check("dpb_attention_clear", lib.dpb_attention_clear(
                a, _dtype_code(q), o if new_out else None, l if new_lse else None, None, None, _stream(q)))
    if not (new_out and new_lse):
        _written(given)
    return out, lse


def attention_bwd(grad_out: torch.Tensor, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, out: torch.Tensor,
                  lse: torch.Tensor, causal: bool = False, scale: float | None = None,
                  q_lens: torch.Tensor | None = None, k_lens: torch.Tensor | None = None,
                  q_starts: torch.Tensor | None = None, k_starts: torch.Tensor | None = None,
                  max_q: int | None = None, max_k: int | None = None, dq: torch.Tensor | None = None,
                  dk: torch.Tensor | None = None, dv: torch.Tensor | None = None,
                  workspace: torch.Tensor | None = None):
    """Gradients (dq, dk, dv) of attention for grad_out, from its out and lse; the
    other arguments as in the forward call.  Packed rows of no sequence are 0 in
    gradients made here and left as they are in those that are given."""
    a = _attn(q, k, v, causal, scale, q_lens, k_lens, q_starts, k_starts, max_q, max_k)
    _need(grad_out.shape == out.shape == q.shape and grad_out.dtype == out.dtype == q.dtype)
    _need(lse.shape == q.shape[:-1] and lse.dtype == torch.float32)
    new_q, new_k, new_v, given = dq is None, dk is None, dv is None, (dq, dk, dv)
    grads = []
    for x, g in ((q, dq), (k, dk), (v, dv)):
        grads.append(torch.empty_like(x, memory_format=torch.contiguous_format) if g is None else g)
        _need(grads[-1].shape == x.shape and grads[-1].dtype == x.dtype)
    lib = load()
    dq, dk, dv = grads
    device, here = _device_of(q, "q")
    with here:
        if workspace is None:
            need = lib.dpb_attention_bwd_workspace_bytes(a)
            workspace = torch.empty((need + 3) // 4, dtype=torch.float32, device=q.device)
        gq, gk, gv = _heads(dq, "dq", device), _heads(dk, "dk", device), _heads(dv, "dv", device)
        _check("dpb_attention_bwd", lib.dpb_attention_bwd(
            a, _dtype_code(q), _heads(grad_out, "grad_out", device), _heads(q, "q"), _heads(k, "k", device),
            _heads(v, "v", device), _heads(out, "out", device), _dev(lse, "lse", device), gq, gk, gv,
            _dev(workspace, "workspace", device), workspace.numel() * workspace.element_size(), _stream(q)))
        if q_starts is not None and (new_q or new_k or new_v):
            _check("dpb_attention_clear", lib.dpb_attention_clear(
                a, _dtype_code(q), gq if new_q else None, None, gk if new_k else None, gv if new_v else None, _stream(q)))
    if not (new_q and new_k and new_v):
        _written(given)
    return dq, dk, dv


ADAMW_BLOCK = 256
_DTYPE = operator.attrgetter("dtype")


class _AdamW(ctypes.Structure):
    _fields_ = [("lr", ctypes.c_double), ("beta1", ctypes.c_double), ("beta2", ctypes.c_double),
                ("eps", ctypes.c_double), ("step", ctypes.c_int64), ("seed", ctypes.c_uint32)]


def adamw_blocks(sizes: Sequence[int]) -> int:
    """Blocks of ADAMW_BLOCK elements in the states of tensors of these sizes."""
    n = len(sizes)
    return int(load().dpb_adamw_blocks((ctypes.c_int64 * n)(*sizes), n))


def adamw_state(params: Sequence[torch.Tensor], bits: int = 32, master: bool = False):
    """First states (m, v, scales, master) of adamw_step for these tensors: m and v
    fp32, or 8-bit floats with scales [blocks, 2]; master: fp32 copies of the
    tensors (or None)."""
    if bits not in (8, 32):
        raise ValueError(f"states have 8 or 32 bits, not {bits}")
    sizes = [p.numel() for p in params]
    blocks, dev = adamw_blocks(sizes), params[0].device
    m, v = (torch.zeros(blocks * ADAMW_BLOCK, dtype=torch.float32 if bits == 32 else torch.float8_e4m3fn, device=dev)
            for _ in range(2))
    scales = None if bits == 32 else torch.zeros((blocks, 2), dtype=torch.float32, device=dev)
    weights = None
    if master:
        weights, at = torch.zeros(blocks * ADAMW_BLOCK, dtype=torch.float32, device=dev), 0
        for p, n in zip(params, sizes):
            weights[at:at + n] = p.detach().reshape(-1)
            at += -(-n // ADAMW_BLOCK) * ADAMW_BLOCK
    return m, v, scales, weights


def adamw_step(params: Sequence[torch.Tensor], grads: Sequence[torch.Tensor], m: torch.Tensor, v: torch.Tensor,
               scales: torch.Tensor | None = None, master: torch.Tensor | None = None, *, step: int, lr: float,
               betas: tuple[float, float] = (0.9, 0.999), eps: float = 1e-8,
               weight_decay: float | Sequence[float] = 0.0, grad_scale: torch.Tensor | None = None, seed: int = 0):
    """One AdamW step over all params in place, with the states of adamw_state (8
    bits when scales are given).  weight_decay: one for all, or one per tensor; seed:
    of the rounding of 8-bit states, another one each step; grad_scale: a device
    scalar that multiplies the gradients.  All params have one type, all grads one;
    what is written (params and states) overlaps nothing else."""
    _adamw(params, grads, m, v, scales, master, step, lr, betas, eps, weight_decay, grad_scale, seed)()


def _adamw(params, grads, m, v, scales, master, step, lr, betas, eps, weight_decay, grad_scale, seed):
    """adamw_step with its arguments checked and nothing done yet, as a function without
    arguments (which holds the tensors' addresses: the caller keeps them alive).  A step over
    tensors of several types thus checks all before it writes any."""
    n = len(params)
    _need(len(grads) == n)
    if n == 0:
        return lambda: None
    sizes = list(map(torch.Tensor.numel, params))
    _need(list(map(torch.Tensor.numel, grads)) == sizes)
    for tensors in (params, grads):
        _need(len(set(map(_DTYPE, tensors))) == 1)
        if set(map(torch.Tensor.get_device, tensors)) != {m.get_device()} or not m.is_cuda:
            raise ValueError("params and grads must be device tensors, on the states' device")
        if not all(map(torch.Tensor.is_contiguous, tensors)):
            raise ValueError("params and grads must be contiguous")
    size_arr = struct.pack(f"={n}q", *sizes)
    lib = load()
    elems = lib.dpb_adamw_blocks(size_arr, n) * ADAMW_BLOCK
    state = torch.float32 if scales is None else torch.float8_e4m3fn
    _need(m.dtype == v.dtype == state and m.numel() >= elems and v.numel() >= elems)
    _need(scales is None or (scales.dtype == torch.float32 and scales.numel() >= elems // (ADAMW_BLOCK // 2)))
    _need(master is None or (master.dtype == torch.float32 and master.numel() >= elems))
    _need(grad_scale is None or (grad_scale.dtype == torch.float32 and grad_scale.numel() == 1))
    decay = [weight_decay] * n if isinstance(weight_decay, (int, float)) else weight_decay
    _need(len(decay) == n)
    pointers = struct.Struct(f"={n}Q")
    o = _AdamW(lr, betas[0], betas[1], eps, step, seed & 0xFFFFFFFF)
    device, here = _device_of(m, "m")
    args = (pointers.pack(*map(torch.Tensor.data_ptr, params)), pointers.pack(*map(torch.Tensor.data_ptr, grads)), size_arr,
            struct.pack(f"={n}f", *decay), _dtype_code(params[0]), _dtype_code(grads[0]), 32 if scales is None else 8,
            _dev(m, "m"), _dev(v, "v", device), _opt(scales, "scales", device), _opt(master, "master", device),
            _opt(grad_scale, "grad_scale", device))

    def call():
        with here:
            _check("dpb_adamw_step", lib.dpb_adamw_step(ctypes.byref(o), n, *args, _stream(m)))
        _written([*params, m, v, scales, master])

    return call


# ---- operators around the blocks: embedding, norm, loss over the vocabulary

_LOGITS = struct.Struct("=QQqqqqif")
LOGITS_STRIDE = 1 << 23     # bytes: rows of hidden states and vocabularies are closer than this


def _place(t: torch.Tensor | None, name: str, device: int) -> int | None:
    """Address of a tensor on this device, contiguous or not."""
    if t is None:
        return None
    if t.get_device() != device:
        _elsewhere(t, name, device)
    return t.data_ptr()


def _whole(t: torch.Tensor | None, name: str, device: int) -> int | None:
    """Address of a contiguous tensor on this device (_dev without its ctypes object: these calls are short)."""
    if t is None:
        return None
    if t.get_device() != device:
        _elsewhere(t, name, device)
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


def _rows(t: torch.Tensor, name: str):
    """(rows, stride between them) of [..., dim] as rows of dim elements, contiguous each."""
    shape = t.shape
    if len(shape) == 0:
        raise ValueError(f"{name} has no rows")
    if t.is_contiguous():
        dim = shape[-1]
        return t.numel() // dim if dim else 0, dim
    st = t.stride()
    if shape[-1] > 1 and st[-1] != 1:
        raise ValueError(f"{name} must be contiguous along its last dimension")
    # the other dimensions have to be one, in the order of memory
    n, stride = 1, shape[-1]
    for size, step in zip(reversed(shape[:-1]), reversed(st[:-1])):
        if size == 1:
            continue
        if n == 1:
            stride = step
        elif step != n * stride:
            raise ValueError(f"{name}: its rows must be evenly apart")
        n *= size
    return n, stride


def _integers(t: torch.Tensor, name: str, device: int):
    """(address, bits) of a contiguous tensor of tokens."""
    dtype = t.dtype
    if dtype != torch.int64 and dtype != torch.int32:
        raise TypeError(f"{name}: int64 or int32, not {dtype}")
    return _whole(t, name, device), 64 if dtype == torch.int64 else 32


def _space(workspace: torch.Tensor | None, need: int, like: torch.Tensor):
    """A workspace of at least `need` bytes (the caller's, if given) and its size."""
    if workspace is None:
        if not need:
            return None, 0
        workspace = torch.empty((need + 15) // 16 * 4, dtype=torch.float32, device=like.device)
    return workspace, workspace.numel() * workspace.element_size()


def embedding(tokens: torch.Tensor, table: torch.Tensor, scale: float = 1.0, out: torch.Tensor | None = None):
    """scale * table[tokens] -> [*tokens.shape, dim] of the table's type; table [vocab, dim]
    with any stride of its rows.  A token outside [0, vocab) gives a row of zeros."""
    _need(table.dim() == 2)
    vocab, dim = table.shape
    if out is None:
        out = table.new_empty((*tokens.shape, dim))
        given = None
    else:
        _need(out.shape == (*tokens.shape, dim) and out.dtype == table.dtype)
        given = out
    _need(dim >= 1, "a table of no columns")
    device, here = _device_of(table, "table")
    with here:
        at, bits = _integers(tokens, "tokens", device)
        _, stride = _rows(table, "table")
        _check("dpb_embedding", load().dpb_embedding(
            _dtype_code(table), table.data_ptr(), stride, vocab, dim, at, bits, tokens.numel(), scale,
            _whole(out, "out", device), _stream(table)))
    if given is not None:
        _written([given])
    return out


def embedding_bwd(grad_out: torch.Tensor, tokens: torch.Tensor, vocab: int, scale: float = 1.0,
                  dweight: torch.Tensor | None = None, workspace: torch.Tensor | None = None):
    """Gradient [vocab, dim] of the table for grad_out [*tokens.shape, dim] of embedding:
    scale times the sum of each row's tokens' gradients, added up in their order."""
    _need(grad_out.dim() >= 1 and grad_out.shape[:-1] == tokens.shape and grad_out.shape[-1] >= 1)
    dim, vocab, given = grad_out.shape[-1], int(vocab), dweight
    _need(vocab >= 0)
    if dweight is None:
        dweight = grad_out.new_empty((vocab, dim))
    _need(dweight.shape == (vocab, dim) and dweight.dtype == grad_out.dtype)
    lib = load()
    device, here = _device_of(grad_out, "grad_out")
    with here:
        at, bits = _integers(tokens, "tokens", device)
        n, stride = _rows(grad_out, "grad_out")
        workspace, size = _space(workspace, lib.dpb_embedding_bwd_workspace_bytes(vocab, dim, n), grad_out)
        _check("dpb_embedding_bwd", lib.dpb_embedding_bwd(
            _dtype_code(grad_out), grad_out.data_ptr(), stride, at, bits, n, vocab, dim, scale,
            _whole(dweight, "dweight", device), _whole(workspace, "workspace", device), size, _stream(grad_out)))
    if given is not None:
        _written([given])
    return dweight


def rms_norm(x: torch.Tensor, weight: torch.Tensor | None, residual: torch.Tensor | None = None, eps: float = 1e-6,
             out: torch.Tensor | None = None, total: torch.Tensor | None = None, rstd: torch.Tensor | None = None):
    """(out, total, rstd): total = x + residual in their type (x itself without a residual),
    rstd = (mean(total^2) + eps)^-1/2 over the last dimension (fp32), out = total rstd weight.

    x, residual: [..., dim], rows evenly apart; weight [dim], fp32 or bf16, or None.  out and
    total may be x or residual themselves, if those are contiguous."""
    shape = x.shape
    _need(len(shape) >= 1 and shape[-1] >= 1)
    dim = shape[-1]
    _need(residual is None or (residual.shape == shape and residual.dtype == x.dtype))
    _need(weight is None or weight.shape == (dim,))
    _need(residual is not None or total is None, "without a residual the sum is x")
    given = None if out is None and total is None and rstd is None else [out, total, rstd]
    if given is not None:
        _need(out is None or (out.shape == shape and out.dtype == x.dtype))
        _need(total is None or (total.shape == shape and total.dtype == x.dtype))
        _need(rstd is None or (rstd.shape == shape[:-1] and rstd.dtype == torch.float32))
    if out is None:   # (empty_like without a format is the quickest where it gives the same)
        out = torch.empty_like(x) if x.is_contiguous() else x.new_empty(shape)
    if residual is not None and total is None:
        total = torch.empty_like(out)
    if rstd is None:
        rstd = torch.empty(shape[:-1], dtype=torch.float32, device=x.device)
    device, here = _device_of(x, "x")
    with here:
        n, stride = _rows(x, "x")
        r_stride = 0 if residual is None else _rows(residual, "residual")[1]
        _check("dpb_rms_norm", load().dpb_rms_norm(
            _dtype_code(x), x.data_ptr(), stride, _place(residual, "residual", device), r_stride,
            _whole(weight, "weight", device), DPB_F32 if weight is None else _dtype_code(weight), n, dim, eps,
            _whole(out, "out", device), _whole(total, "total", device), _whole(rstd, "rstd", device), _stream(x)))
    if given is not None:
        _written(given)
    return out, x if residual is None else total, rstd


def rms_norm_bwd(grad_out: torch.Tensor, total: torch.Tensor, weight: torch.Tensor | None, rstd: torch.Tensor,
                 grad_total: torch.Tensor | None = None, dx: torch.Tensor | None = None,
                 dweight: torch.Tensor | None = None, workspace: torch.Tensor | None = None):
    """Gradients (dx, dweight) of rms_norm for grad_out of out and grad_total of total, from its
    total and rstd: dx is the gradient of x and of residual alike; dweight in the weight's type
    (None without one).  dx may be grad_out or grad_total itself, if that is contiguous."""
    shape = total.shape
    _need(len(shape) >= 1 and shape[-1] >= 1)
    dim = shape[-1]
    _need(grad_out.shape == shape and grad_out.dtype == total.dtype)
    _need(grad_total is None or (grad_total.shape == shape and grad_total.dtype == total.dtype))
    _need(rstd.shape == shape[:-1] and rstd.dtype == torch.float32)
    _need(weight is None or weight.shape == (dim,))
    _need(weight is not None or dweight is None)
    given = [dx, dweight]
    if dx is None:
        dx = torch.empty_like(total, memory_format=torch.contiguous_format)
    if weight is not None and dweight is None:
        dweight = torch.empty_like(weight)
    _need(dx.shape == shape and dx.dtype == total.dtype)
    _need(dweight is None or (dweight.shape == (dim,) and dweight.dtype == weight.dtype))
    lib = load()
    device, here = _device_of(total, "total")
    with here:
        n, stride = _rows(total, "total")
        g_stride = _rows(grad_out, "grad_out")[1]
        t_stride = 0 if grad_total is None else _rows(grad_total, "grad_total")[1]
        need = 0 if dweight is None else lib.dpb_rms_norm_bwd_workspace_bytes(n, dim)
        workspace, size = _space(workspace, need, total)
        _check("dpb_rms_norm_bwd", lib.dpb_rms_norm_bwd(
            _dtype_code(total), _place(grad_out, "grad_out", device), g_stride, _place(grad_total, "grad_total", device),
            t_stride, total.data_ptr(), stride, _whole(weight, "weight", device),
            DPB_F32 if weight is None else _dtype_code(weight), _whole(rstd, "rstd", device), n, dim,
            _whole(dx, "dx", device), _whole(dweight, "dweight", device), _whole(workspace, "workspace", device), size,
            _stream(total)))
    if any(t is not None for t in given):
        _written(given)
    return dx, dweight


def _logits(hidden: torch.Tensor, weight: torch.Tensor, targets: torch.Tensor, scale: float) -> tuple[bytes, int]:
    """The description of a call's logits, and its rows."""
    _need(hidden.dim() >= 1 and weight.dim() == 2 and hidden.shape[-1] == weight.shape[1] >= 1)
    _need(hidden.dtype == weight.dtype and targets.shape == hidden.shape[:-1])
    n, stride = _rows(hidden, "hidden")
    w_stride = _rows(weight, "weight")[1]
    return _LOGITS.pack(hidden.data_ptr(), weight.data_ptr(), stride, w_stride, n, weight.shape[0], weight.shape[1], scale), n


def cross_entropy(hidden: torch.Tensor, weight: torch.Tensor, targets: torch.Tensor, scale: float = 1.0,
                  loss: torch.Tensor | None = None, lse: torch.Tensor | None = None,
                  workspace: torch.Tensor | None = None):
    """(loss, lse), fp32 of the targets' shape: lse = log sum_v exp(scale <hidden, weight_v>),
    loss = lse - scale <hidden, weight_target>, 0 for a target outside [0, vocab).

    hidden [..., dim] and weight [vocab, dim] of one type, rows evenly apart and under 8 MiB from one to the
    next (rows further apart are the caller's to copy); the logits are never in memory."""
    a, n = _logits(hidden, weight, targets, scale)
    given = [loss, lse]
    if loss is None:
        loss = hidden.new_empty(targets.shape, dtype=torch.float32)
    if lse is None:
        lse = hidden.new_empty(targets.shape, dtype=torch.float32)
    _need(loss.shape == lse.shape == targets.shape and loss.dtype == lse.dtype == torch.float32)
    lib, dtype = load(), _dtype_code(hidden)
    device, here = _device_of(hidden, "hidden")
    with here:
        _place(weight, "weight", device)
        at, bits = _integers(targets, "targets", device)
        workspace, size = _space(workspace, lib.dpb_cross_entropy_workspace_bytes(a, dtype), hidden)
        _check("dpb_cross_entropy", lib.dpb_cross_entropy(
            a, dtype, at, bits, _whole(loss, "loss", device), _whole(lse, "lse", device),
            _whole(workspace, "workspace", device), size, _stream(hidden)))
    if any(t is not None for t in given):
        _written(given)
    return loss, lse


def cross_entropy_bwd(grad_loss: torch.Tensor | None, hidden: torch.Tensor, weight: torch.Tensor, targets: torch.Tensor,
                      lse: torch.Tensor, scale: float = 1.0, grad_lse: torch.Tensor | None = None,
                      dhidden: torch.Tensor | None = None, dweight: torch.Tensor | None = None,
                      workspace: torch.Tensor | None = None, hidden_grad: bool = True, weight_grad: bool = True):
    """Gradients (dhidden, dweight) of cross_entropy for grad_loss and grad_lse (fp32 of the
    targets' shape, or None for zeros) from the forward's lse.  hidden_grad, weight_grad: which of
    the two are wanted (None in the place of the other)."""
    a, n = _logits(hidden, weight, targets, scale)
    _need(lse.shape == targets.shape and lse.dtype == torch.float32)
    for g in (grad_loss, grad_lse):
        _need(g is None or (g.shape == targets.shape and g.dtype == torch.float32))
    given = [dhidden, dweight]
    if hidden_grad and dhidden is None:
        dhidden = torch.empty_like(hidden, memory_format=torch.contiguous_format)
    if weight_grad and dweight is None:
        dweight = torch.empty_like(weight, memory_format=torch.contiguous_format)
    _need((dhidden is None) != bool(hidden_grad) and (dweight is None) != bool(weight_grad))
    _need(dhidden is None or (dhidden.shape == hidden.shape and dhidden.dtype == hidden.dtype))
    _need(dweight is None or (dweight.shape == weight.shape and dweight.dtype == weight.dtype))
    lib, dtype = load(), _dtype_code(hidden)
    device, here = _device_of(hidden, "hidden")
    with here:
        _place(weight, "weight", device)
        at, bits = _integers(targets, "targets", device)
        outs = _whole(dhidden, "dhidden", device), _whole(dweight, "dweight", device)
        if n == 0:
            if dweight is not None:
                dweight.zero_()
        else:
            workspace, size = _space(workspace, lib.dpb_cross_entropy_bwd_workspace_bytes(a, dtype), hidden)
            _check("dpb_cross_entropy_bwd", lib.dpb_cross_entropy_bwd(
                a, dtype, at, bits, _whole(grad_loss, "grad_loss", device), _whole(grad_lse, "grad_lse", device),
                _whole(lse, "lse", device), *outs, _whole(workspace, "workspace", device), size, _stream(hidden)))
    if any(t is not None for t in given):
        _written(given)
    return dhidden, dweight
