"""ctypes binding of libmuloco (argument marshalling only).

Every optimizer step runs inside the CUDA library; this module only loads the
shared object, mirrors the C structs of include/muloco.h and turns torch
tensors into raw device pointers.  torch is used for device memory and streams.
There is no fallback: if the library cannot be loaded, or there is no CUDA
device, the calls raise.
"""
from __future__ import annotations

import ctypes as C
import math
import os
import struct
import weakref
from typing import List, Optional, Sequence

import numpy as np

from . import configs as _cfg

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.environ.get("MULOCO_LIBRARY", os.path.join(_HERE, "libmuloco.so"))

OK, EINVAL, ESHAPE, ENOMEM, ECUDA, ENONFINITE, ETIMEOUT, ESTATE = range(8)
STATUS_NAMES = ["OK", "EINVAL", "ESHAPE", "ENOMEM", "ECUDA", "ENONFINITE", "ETIMEOUT", "ESTATE"]
MUON, ADAMW = 0, 1
NS_BF16, NS_FP32 = 0, 1
F32, BF16 = 0, 1
DEBUG_WAIT_LIMIT_NS, DEBUG_WITHHOLD_COPY, DEBUG_CANARIES, DEBUG_CORRUPT_CANARY = 1, 2, 3, 4
PHASES = ["prologue", "ns", "adamw", "sync", "copy"]
ACTIVATIONS = {"silu": 0, "gelu": 1}
ADAMW_BLOCK = 256              # elements that share a scale in 8-bit AdamW states

EXPORTS = [
    "muloco_create", "muloco_destroy", "muloco_inner_step", "muloco_inner_step_host",
    "muloco_outer_sync", "muloco_outer_sync_host", "muloco_fragments_due", "muloco_newton_schulz",
    "muloco_quantize", "muloco_topk_sparsify", "muloco_pseudogradient", "muloco_get_state", "muloco_set_state",
    "muloco_set_timing", "muloco_get_timings", "muloco_sync_status", "muloco_last_error",
    "muloco_newton_schulz_static", "muloco_debug_set", "muloco_check_workspace",
    "muloco_shard_layout", "muloco_shard_delta", "muloco_shard_step", "muloco_shard_broadcast",
    "muloco_adamw_create", "muloco_adamw_step", "muloco_adamw_moments", "muloco_adamw_destroy",
    "muloco_qk_norm_rope", "muloco_qk_norm_rope_backward", "muloco_gated_ffn", "muloco_gated_ffn_backward",
    "muloco_debug_ffn_forms",
]


class TensorDesc(C.Structure):
    _fields_ = [("rows", C.c_int64), ("cols", C.c_int64), ("kind", C.c_int32), ("fragment", C.c_int32),
                ("wd_mult", C.c_float), ("lr_mult", C.c_float)]


class Config(C.Structure):
    _fields_ = [("K", C.c_int32), ("H", C.c_int32), ("J", C.c_int32),
                ("muon_lr", C.c_float), ("muon_beta", C.c_float), ("muon_wd", C.c_float),
                ("muon_nesterov", C.c_int32), ("ns_steps", C.c_int32),
                ("ns_a", C.c_float), ("ns_b", C.c_float), ("ns_c", C.c_float), ("ns_eps", C.c_float),
                ("ns_mode", C.c_int32), ("wd_uses_scaled_lr", C.c_int32),
                ("adam_lr", C.c_float), ("adam_beta1", C.c_float), ("adam_beta2", C.c_float),
                ("adam_eps", C.c_float), ("adam_wd", C.c_float), ("adam_bias_correction", C.c_int32),
                ("outer_lr", C.c_float), ("outer_momentum", C.c_float),
                ("quant", C.c_int32), ("quant_block", C.c_int32), ("grad_dtype", C.c_int32),
                ("quant_stages", C.c_int32), ("workspace_bytes", C.c_uint64),
                ("error_feedback", C.c_int32), ("ef_beta", C.c_float),
                ("topk_fraction", C.c_float), ("adam_state_bits", C.c_int32), ("adam_seed", C.c_uint32)]


class Buffers(C.Structure):
    _fields_ = [("theta_k", C.POINTER(C.c_void_p)), ("theta_g", C.POINTER(C.c_void_p)),
                ("outer_u", C.POINTER(C.c_void_p)), ("state1_k", C.POINTER(C.c_void_p)),
                ("state2_k", C.POINTER(C.c_void_p)), ("ef_k", C.POINTER(C.c_void_p))]


class AdamwConfig(C.Structure):
    _fields_ = [("lr", C.c_float), ("beta1", C.c_float), ("beta2", C.c_float), ("eps", C.c_float),
                ("weight_decay", C.c_float), ("bias_correction", C.c_int32), ("state_bits", C.c_int32),
                ("grad_dtype", C.c_int32), ("seed", C.c_uint32)]


class AdamwTensor(C.Structure):
    _fields_ = [("n", C.c_int64), ("theta", C.c_void_p), ("copy", C.c_void_p), ("grad", C.c_void_p),
                ("state1", C.c_void_p), ("state2", C.c_void_p), ("scale1", C.c_void_p), ("scale2", C.c_void_p),
                ("wd_mult", C.c_float), ("lr_mult", C.c_float)]


class QkNorm(C.Structure):
    _fields_ = [("tokens", C.c_int64), ("table_len", C.c_int64),
                ("heads_q", C.c_int32), ("heads_k", C.c_int32), ("head_dim", C.c_int32), ("rotary_dim", C.c_int32),
                ("dtype", C.c_int32), ("interleaved", C.c_int32), ("eps", C.c_float), ("pad", C.c_int32),
                ("gain_q", C.c_void_p), ("gain_k", C.c_void_p), ("cos", C.c_void_p), ("sin", C.c_void_p),
                ("positions", C.c_void_p), ("q", C.c_void_p), ("k", C.c_void_p),
                ("q_token_stride", C.c_int64), ("q_head_stride", C.c_int64),
                ("k_token_stride", C.c_int64), ("k_head_stride", C.c_int64)]


class Ffn(C.Structure):
    _fields_ = [("tokens", C.c_int64), ("d", C.c_int64), ("F", C.c_int64),
                ("ldx", C.c_int64), ("ldw1", C.c_int64), ("ldw3", C.c_int64), ("ldw2", C.c_int64),
                ("x", C.c_void_p), ("w1", C.c_void_p), ("w3", C.c_void_p), ("w2", C.c_void_p),
                ("activation", C.c_int32), ("pad", C.c_int32)]


# QkNorm and Ffn as bytes
_QK_PACK = struct.Struct("qqiiiiiifiQQQQQQQqqqq").pack
_FFN_PACK = struct.Struct("qqqqqqqQQQQii").pack


class MulocoError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"muloco status {STATUS_NAMES[status] if 0 <= status < 8 else status}: {msg}")
        self.status = status


_lib = None


def _load_fastcall():
    """The compiled call path of the operators (build.build_fastcall), or None where it was not built, or was for another
    torch: the methods then marshal their arguments in Python, in front of the same library."""
    import torch
    try:
        from . import _fastcall
    except ImportError:
        return None
    return _fastcall if getattr(_fastcall, "TORCH", None) == torch.__version__ else None


def load_library():
    """Load libmuloco.so from the package directory; raises if it is missing."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_2505_23725_b200.build` "
                           "(there is no CPU fallback)")
    lib = C.CDLL(LIB_PATH)
    vp, i32, i64, f32 = C.c_void_p, C.c_int32, C.c_int64, C.c_float
    lib.muloco_create.argtypes = [C.POINTER(Config), C.POINTER(TensorDesc), i32, C.POINTER(Buffers), vp,
                                  C.POINTER(vp)]
    lib.muloco_destroy.argtypes = [vp]
    lib.muloco_destroy.restype = None
    lib.muloco_inner_step.argtypes = [vp, i32, C.POINTER(vp), f32]
    lib.muloco_inner_step_host.argtypes = [vp, i32, C.POINTER(vp), f32]
    lib.muloco_outer_sync.argtypes = [vp, i32]
    lib.muloco_outer_sync_host.argtypes = [vp, i32, C.POINTER(vp)]
    lib.muloco_fragments_due.argtypes = [vp, i64, C.POINTER(i32)]
    lib.muloco_newton_schulz.argtypes = [vp, vp, i32, vp, i32, i32, i64, i64, i32]
    lib.muloco_quantize.argtypes = [vp, vp, i64, i64, i32, vp, vp, vp]
    lib.muloco_pseudogradient.argtypes = [vp, i32, vp]
    lib.muloco_topk_sparsify.argtypes = [vp, vp, i64, C.c_float, vp]
    lib.muloco_get_state.argtypes = [vp, vp, C.POINTER(C.c_size_t)]
    lib.muloco_set_state.argtypes = [vp, vp, C.c_size_t]
    lib.muloco_set_timing.argtypes = [vp, i32]
    lib.muloco_get_timings.argtypes = [vp, C.POINTER(f32), C.POINTER(i64)]
    lib.muloco_sync_status.argtypes = [vp]
    lib.muloco_last_error.argtypes = [vp]
    lib.muloco_last_error.restype = C.c_char_p
    lib.muloco_debug_set.argtypes = [vp, i32, i64]
    lib.muloco_check_workspace.argtypes = [vp]
    lib.muloco_shard_layout.argtypes = [vp, i32, i32, i32, C.POINTER(i64), C.POINTER(i64)]
    lib.muloco_shard_delta.argtypes = [vp, i32, i32, vp]
    lib.muloco_shard_step.argtypes = [vp, i32, i32, i32, vp, vp]
    lib.muloco_shard_broadcast.argtypes = [vp, i32, i32, vp]
    lib.muloco_newton_schulz_static.argtypes = [vp, vp, i32, i64, i64, vp, C.c_char_p, C.c_size_t]
    lib.muloco_adamw_create.argtypes = [vp, C.POINTER(AdamwConfig), C.POINTER(AdamwTensor), i32, C.POINTER(vp)]
    lib.muloco_adamw_step.argtypes = [vp, C.POINTER(vp), i64, f32]
    lib.muloco_adamw_moments.argtypes = [vp, vp, vp]
    lib.muloco_adamw_destroy.argtypes = [vp]
    lib.muloco_adamw_destroy.restype = None
    # the argument structs of the operators are packed bytes (_QK_PACK, _FFN_PACK): a fifth of the time of a ctypes struct
    packed = C.c_char_p
    lib.muloco_qk_norm_rope.argtypes = [vp, packed, vp, i64, i64, vp, i64, i64]
    lib.muloco_qk_norm_rope_backward.argtypes = [vp, packed, vp, i64, i64, vp, i64, i64, vp, vp, vp, vp]
    lib.muloco_gated_ffn.argtypes = [vp, packed, vp, vp, vp, vp]
    lib.muloco_gated_ffn_backward.argtypes = [vp, packed, vp, i64] + [vp] * 9
    lib.muloco_debug_ffn_forms.argtypes = [i64, i64, i64, i32, C.POINTER(i64)]
    for name in EXPORTS:
        fn = getattr(lib, name)
        if name not in ("muloco_destroy", "muloco_last_error", "muloco_adamw_destroy"):
            fn.restype = i32
    _lib = lib
    return lib


def newton_schulz_static(X, stream=None, out=None):
    """muloco_newton_schulz_static: fp32 Newton-Schulz of a small [batch, rows, cols]
    (or [rows, cols]) float32 CUDA tensor without any device allocation by the library.
    The result goes to `out` (same shape, float32, contiguous) when given; otherwise the
    output tensor is allocated here, by torch, before the call.  For callers that may
    not allocate; sizes beyond the library's fixed scratch raise MulocoError(ESHAPE)."""
    import torch
    lib = load_library()
    x = (X if X.dim() == 3 else X.unsqueeze(0)).contiguous()
    if x.dtype != torch.float32 or not x.is_cuda:
        raise ValueError("expects a float32 CUDA tensor")
    if out is None:
        o = torch.empty_like(x)
    else:
        o = out if out.dim() == 3 else out.unsqueeze(0)
        if o.shape != x.shape or o.dtype != torch.float32 or not o.is_contiguous() or o.device != x.device:
            raise ValueError("out must be a contiguous float32 tensor of X's shape on X's device")
    st = stream if stream is not None else torch.cuda.current_stream(x.device)
    err = C.create_string_buffer(256)
    with torch.cuda.device(x.device):
        rc = lib.muloco_newton_schulz_static(x.data_ptr(), o.data_ptr(), x.shape[0], x.shape[1], x.shape[2],
                                             C.c_void_p(st.cuda_stream), err, 256)
    if rc != OK:
        raise MulocoError(rc, err.value.decode())
    return o if X.dim() == 3 else o[0]


def shard_wire_bytes(stage_floats: int, world: int) -> int:
    """Bytes one rank moves per sharded sync: a reduce-scatter and an all-gather of stage_floats
    float32 values, (world - 1) / world of it each."""
    return 2 * 4 * stage_floats * (world - 1) // world


def _reduce_scatter_sum(dist, out, inp, group):
    """out <- this rank's shard of the element-wise sum of inp over the ranks."""
    if dist.get_backend(group) == "nccl":
        dist.reduce_scatter_tensor(out, inp, op=dist.ReduceOp.SUM, group=group)
    else:                                   # backends without reduce-scatter (gloo): all-reduce, keep the shard
        tmp = inp.clone()
        dist.all_reduce(tmp, op=dist.ReduceOp.SUM, group=group)
        r = dist.get_rank(group)
        out.copy_(tmp[r * out.numel():(r + 1) * out.numel()])


def sharded_outer_sync(opt, fragment: int, dist, group=None):
    """Drives the three shard calls of `opt` (a MuLoCo, or any object with shard_layout /
    shard_delta / shard_step / shard_broadcast and new_buffer) around the two collectives."""
    world, rank = dist.get_world_size(group), dist.get_rank(group)
    stage_floats, shard_floats = opt.shard_layout(fragment, world, rank)
    if stage_floats == 0:
        return 0
    with opt.stream_context():
        stage = opt.new_buffer(stage_floats)
        reduced = opt.new_buffer(shard_floats)
        theta_shard = opt.new_buffer(shard_floats)
        opt.shard_delta(fragment, world, stage)
        if world > 1:
            _reduce_scatter_sum(dist, reduced, stage, group)
        else:
            reduced = stage
        opt.shard_step(fragment, world, rank, reduced, theta_shard)
        if world > 1:
            dist.all_gather_into_tensor(stage, theta_shard, group=group)
        else:
            stage = theta_shard
        opt.shard_broadcast(fragment, world, stage)
    return shard_wire_bytes(stage_floats, world)


def make_config(w: _cfg.Workload, workspace_bytes: int = 0, ns_mode: Optional[str] = None, **over) -> Config:
    c = Config()
    c.K, c.H, c.J = w.K, w.H, w.J
    c.muon_lr, c.muon_beta, c.muon_wd = w.muon_lr, w.muon_beta, w.muon_wd
    c.muon_nesterov = int(w.muon_nesterov)
    c.ns_steps = 5
    c.ns_a, c.ns_b, c.ns_c = 3.4445, -4.7750, 2.0315
    c.ns_eps = 1e-7
    mode = ns_mode or w.ns_mode
    c.ns_mode = NS_FP32 if mode == "fp32" else NS_BF16
    c.wd_uses_scaled_lr = 1
    c.adam_lr = w.muon_lr if w.adam_lr is None else w.adam_lr
    c.adam_wd = w.muon_wd if w.adam_wd is None else w.adam_wd
    c.adam_beta1, c.adam_beta2, c.adam_eps = w.adam_beta1, w.adam_beta2, w.adam_eps
    c.adam_bias_correction = 1
    c.outer_lr, c.outer_momentum = w.outer_lr, w.outer_momentum
    c.quant = w.quant_bits
    c.quant_block = w.quant_block
    c.quant_stages = w.quant_stages
    c.error_feedback = int(w.error_feedback)
    c.ef_beta = w.ef_beta
    c.topk_fraction = w.topk_fraction
    c.adam_state_bits, c.adam_seed = w.adam_state_bits, w.adam_seed
    c.grad_dtype = BF16 if w.grad_dtype == "bf16" else F32
    c.workspace_bytes = workspace_bytes
    for k, v in over.items():
        setattr(c, k, v)
    return c


def ffn_forms(tokens: int, d: int, F: int, n_sms: int = 148):
    """muloco_debug_ffn_forms: the products of a feed-forward call of this size that run on 256 x 256 tiles, and the tiles of its
    launches on them."""
    tiles = (C.c_int64 * 4)()
    forms = load_library().muloco_debug_ffn_forms(tokens, d, F, n_sms, tiles)
    return {n for i, n in enumerate(("gate", "y", "gate_back", "dx")) if forms >> i & 1}, list(tiles)


def _ptr_table(ptrs: Sequence[int]):
    arr = (C.c_void_p * max(1, len(ptrs)))()
    for i, p in enumerate(ptrs):
        arr[i] = p
    return arr


class _Operators:
    """The operators of the training step around the optimizer, as methods of whatever owns a library
    context (self.ctx, self.lib, self.stream, self.device, self.torch, self._check).

    Work runs on the context's stream.  When the caller's current stream is another one, the context's
    stream first waits for it and it then waits for the context's, and the tensors are
    recorded on the context's stream, so inputs, results and their memory may be used as usual."""

    def _init_operators(self):
        """What every call looks up, once: device number, types, the stream's handle and the way to ask for the handle
        of the current stream without building a Stream object."""
        torch = self.torch
        self._lists = weakref.WeakSet()          # AdamW lists, which the library's context must outlive
        self._dev = self.device.index if self.device.index is not None else torch.cuda.current_device()
        self._bf16, self._f32, self._i64 = torch.bfloat16, torch.float32, torch.int64
        self._raw_stream = torch._C._cuda_getCurrentRawStream
        self._handle = self.stream.cuda_stream
        fast = _load_fastcall()
        self._fast = {}
        if fast is not None:
            for name in ("qk_norm_rope", "qk_norm_rope_backward", "gated_ffn", "gated_ffn_backward", "adamw_step",
                         "adamw_moments"):
                self._fast[name] = (getattr(fast, name), C.cast(getattr(self.lib, "muloco_" + name), C.c_void_p).value)

    def _quick(self, name, *args):
        """The compiled form of a call: its results, or None when this one has to go the long way (an argument is not as
        it should be, or the caller is on another stream)."""
        if self.ctx is None:
            raise RuntimeError("the context is closed")
        f = self._fast.get(name)
        if f is None:
            return None
        r = f[0](self.ctx.value, f[1], self._dev, self._handle, *args)
        if r.__class__ is int:
            self._check(r)
        return r

    def close(self):
        """Releases the context, and before it the AdamW lists made with it."""
        if getattr(self, "ctx", None):
            for o in list(self._lists):
                o.close()
            self.lib.muloco_destroy(self.ctx)
            self.ctx = None

    def _other_stream(self):
        """The caller's current stream when it is not the context's, else None."""
        if self._raw_stream(self._dev) == self._handle:
            return None
        return self.torch.cuda.current_stream(self.device)

    def _enter(self, cur, tensors):
        self.stream.wait_stream(cur)
        for t in tensors:
            if t is not None:
                t.record_stream(self.stream)

    def _need(self, name, t, dtype, shape, dense=False):
        """Raises unless t is a tensor of this context's device with the given type and shape (None: any
        size) whose last dimension is consecutive (dense: which is contiguous)."""
        if t.get_device() != self._dev:
            raise ValueError(f"{name} must be on {self.device} (got {t.device})")
        if t.dtype is not dtype:
            raise ValueError(f"{name} must be {dtype} (got {t.dtype})")
        if t.dim() != len(shape) or any(w is not None and w != h for w, h in zip(shape, t.shape)):
            raise ValueError(f"{name} must have shape {tuple(shape)} (got {tuple(t.shape)})")
        if dense and not t.is_contiguous():
            raise ValueError(f"{name} must be contiguous")
        if t.shape[-1] > 1 and t.stride(-1) != 1 and t.numel():
            raise ValueError(f"{name}: the entries of its last dimension must be consecutive")

    # -- norm of queries and keys with the rotation -----------------------------------------------
    def _check_qk(self, q, k, cos, sin, positions, gain_q, gain_k):
        """The checks of _qk one by one, for the message."""
        torch = self.torch
        some = q if q is not None else k
        if some is None:
            raise ValueError("q and k are both None")
        if some.dtype not in (torch.float32, torch.bfloat16):
            raise ValueError(f"q and k must be float32 or bfloat16 (got {some.dtype})")
        if some.dim() != 3:
            raise ValueError(f"q and k must be [tokens, heads, head_dim] (got {tuple(some.shape)})")
        T, _, D = some.shape
        for name, t in (("q", q), ("k", k)):
            if t is not None:
                self._need(name, t, some.dtype, (T, None, D))
        self._need("cos", cos, torch.float32, (None, None), dense=True)
        self._need("sin", sin, torch.float32, tuple(cos.shape), dense=True)
        if positions is not None:
            self._need("positions", positions, torch.int64, (T,), dense=True)
        for name, t in (("gain_q", gain_q), ("gain_k", gain_k)):
            if t is not None:
                self._need(name, t, torch.float32, (D,), dense=True)

    def _qk(self, q, k, cos, sin, positions, gain_q, gain_k, eps, interleaved):
        """The packed argument struct of a call.  The checks run every time, so they are written to be
        quick; _check_qk repeats them with a message when one fails."""
        torch, dev, f32 = self.torch, self._dev, self._f32
        some = q if q is not None else k
        if some is None or some.dim() != 3 or cos.dim() != 2:
            self._check_qk(q, k, cos, sin, positions, gain_q, gain_k)
        dt = some.dtype
        T, _, D = some.shape
        ok = (dt is self._bf16 or dt is f32) and cos.shape == sin.shape and cos.dtype is f32 and sin.dtype is f32 \
            and cos.is_contiguous() and sin.is_contiguous() and cos.get_device() == dev and sin.get_device() == dev
        hq = hk = pq = pk = qt = qh = kt = kh = pp = pgq = pgk = 0
        if q is not None:
            _, hq, d = q.shape
            qt, qh, one = q.stride()
            pq = q.data_ptr()
            ok = ok and d == D and (one == 1 or D < 2) and q.get_device() == dev
        if k is not None:
            t, hk, d = k.shape if k.dim() == 3 else (-1, 0, 0)
            kt, kh, one = k.stride() if k.dim() == 3 else (0, 0, 0)
            pk = k.data_ptr()
            ok = ok and t == T and d == D and (one == 1 or D < 2) and k.dtype is dt and k.get_device() == dev
        if positions is not None:
            pp = positions.data_ptr()
            ok = ok and positions.dtype is self._i64 and positions.shape == (T,) and positions.is_contiguous() \
                and positions.get_device() == dev
        if gain_q is not None:
            pgq = gain_q.data_ptr()
            ok = ok and gain_q.dtype is f32 and gain_q.shape == (D,) and gain_q.is_contiguous() and gain_q.get_device() == dev
        if gain_k is not None:
            pgk = gain_k.data_ptr()
            ok = ok and gain_k.dtype is f32 and gain_k.shape == (D,) and gain_k.is_contiguous() and gain_k.get_device() == dev
        if not ok:
            self._check_qk(q, k, cos, sin, positions, gain_q, gain_k)
        L, half = cos.shape
        return _QK_PACK(T, L, hq, hk, D, 2 * half, F32 if dt is f32 else BF16, 1 if interleaved else 0, eps,
                        0, pgq, pgk, cos.data_ptr(), sin.data_ptr(), pp, pq, pk, qt, qh, kt, kh)

    def qk_norm_rope(self, q, k, cos, sin, positions=None, gain_q=None, gain_k=None, eps=1e-6, interleaved=False,
                     out=None):
        """muloco_qk_norm_rope: norm and rotation of the heads of q [tokens, heads, head_dim] and k (either may be
        None).  cos and sin: float32 tables [length, rotary_dim / 2]; positions: int64 [tokens] or None
        for 0, 1, ...  Returns (q_out, k_out), new tensors in the inputs' order of dimensions unless
        `out` = (q_out, k_out) gives them."""
        if out is None:
            r = self._quick("qk_norm_rope", q, k, cos, sin, positions, gain_q, gain_k, eps, interleaved)
            if r is not None:
                return r
        empty_like = self.torch.empty_like
        a = self._qk(q, k, cos, sin, positions, gain_q, gain_k, eps, interleaved)
        if out is None:
            qo = None if q is None else empty_like(q)
            ko = None if k is None else empty_like(k)
        else:
            qo, ko = out
            for name, o, t in (("q_out", qo, q), ("k_out", ko, k)):
                if (o is None) != (t is None):
                    raise ValueError(f"{name} is given without its input, or missing")
                if o is not None:
                    self._need(name, o, t.dtype, tuple(t.shape))
        p1 = t1 = h1 = p2 = t2 = h2 = 0
        if qo is not None:
            p1 = qo.data_ptr()
            t1, h1, _ = qo.stride()
        if ko is not None:
            p2 = ko.data_ptr()
            t2, h2, _ = ko.stride()
        cur = self._other_stream()
        if cur is not None:
            self._enter(cur, (q, k, cos, sin, positions, gain_q, gain_k, qo, ko))
        st = self.lib.muloco_qk_norm_rope(self.ctx, a, p1, t1, h1, p2, t2, h2)
        if st:
            self._check(st)
        if cur is not None:
            cur.wait_stream(self.stream)
        return qo, ko

    def qk_norm_rope_backward(self, dq_out, dk_out, q, k, cos, sin, positions=None, gain_q=None, gain_k=None,
                              eps=1e-6, interleaved=False):
        """muloco_qk_norm_rope_backward: from the gradients of the results, (dq, dk, dgain_q, dgain_k)."""
        r = self._quick("qk_norm_rope_backward", dq_out, dk_out, q, k, cos, sin, positions, gain_q, gain_k, eps, interleaved)
        if r is not None:
            return r
        a = self._qk(q, k, cos, sin, positions, gain_q, gain_k, eps, interleaved)
        dev = self._dev
        for name, y, t in (("dq_out", dq_out, q), ("dk_out", dk_out, k)):
            if (y is None) != (t is None):
                raise ValueError(f"{name} is given without its input, or missing")
            if y is not None and (y.dtype is not t.dtype or y.shape != t.shape or y.get_device() != dev or y.stride(2) != 1):
                self._need(name, y, t.dtype, tuple(t.shape))
        dq = dk = gq = gk = None
        p1 = t1 = h1 = p2 = t2 = h2 = o1 = o2 = g1 = g2 = 0
        if q is not None:
            dq, gq = q.new_empty(q.shape), cos.new_empty(q.shape[2])
            p1, o1, g1 = dq_out.data_ptr(), dq.data_ptr(), gq.data_ptr()
            t1, h1, _ = dq_out.stride()
        if k is not None:
            dk, gk = k.new_empty(k.shape), cos.new_empty(k.shape[2])
            p2, o2, g2 = dk_out.data_ptr(), dk.data_ptr(), gk.data_ptr()
            t2, h2, _ = dk_out.stride()
        cur = self._other_stream()
        if cur is not None:
            self._enter(cur, (q, k, cos, sin, positions, gain_q, gain_k, dq_out, dk_out, dq, dk, gq, gk))
        st = self.lib.muloco_qk_norm_rope_backward(self.ctx, a, p1, t1, h1, p2, t2, h2, o1, o2, g1, g2)
        if st:
            self._check(st)
        if cur is not None:
            cur.wait_stream(self.stream)
        return dq, dk, gq, gk

    # -- gated feed-forward block -----------------------------------------------------------------
    def _check_ffn(self, x, w1, w3, w2):
        """The checks of _ffn one by one, for the message."""
        bf16 = self.torch.bfloat16
        self._need("x", x, bf16, (None, None))
        self._need("w1", w1, bf16, (x.shape[1], None))
        self._need("w3", w3, bf16, tuple(w1.shape))
        self._need("w2", w2, bf16, (w1.shape[1], w1.shape[0]))

    def _ffn(self, x, w1, w3, w2, activation):
        """The packed argument struct of a call (its checks as in _qk)."""
        bf16, dev = self._bf16, self._dev
        act = ACTIVATIONS.get(activation, -1)
        if act < 0:
            raise ValueError(f"activation must be one of {sorted(ACTIVATIONS)} (got {activation!r})")
        if x.dim() != 2 or w1.dim() != 2 or w3.dim() != 2 or w2.dim() != 2:
            self._check_ffn(x, w1, w3, w2)
        T, d = x.shape
        d1, F = w1.shape
        ldx, one = x.stride()
        ld1, one1 = w1.stride()
        ld3, one3 = w3.stride()
        ld2, one2 = w2.stride()
        if not (d1 == d and w3.shape == w1.shape and w2.shape == (F, d) and x.dtype is bf16 and w1.dtype is bf16
                and w3.dtype is bf16 and w2.dtype is bf16 and one == 1 and one1 == 1 and one3 == 1 and one2 == 1
                and x.get_device() == dev and w1.get_device() == dev and w3.get_device() == dev
                and w2.get_device() == dev):
            self._check_ffn(x, w1, w3, w2)
        # the row stride of a single row does not matter
        return _FFN_PACK(T, d, F, ldx if T > 1 else d, ld1, ld3, ld2, x.data_ptr(), w1.data_ptr(), w3.data_ptr(),
                         w2.data_ptr(), act, 0), T, d, F

    def gated_ffn(self, x, w1, w3, w2, activation="silu", save=True):
        """muloco_gated_ffn: y = (act(x w1) * (x w3)) w2, all bf16.  Returns (y, saved): saved = (g, u, h) is what
        the backward pass needs (None with save=False, and g and u are then not written)."""
        r = self._quick("gated_ffn", x, w1, w3, w2, ACTIVATIONS.get(activation, -1), save)
        if r is not None:
            return r
        a, T, d, F = self._ffn(x, w1, w3, w2, activation)
        y, h = x.new_empty((T, d)), x.new_empty((T, F))
        g = u = None
        pg = pu = 0
        if save:
            g, u = x.new_empty((T, F)), x.new_empty((T, F))
            pg, pu = g.data_ptr(), u.data_ptr()
        cur = self._other_stream()
        if cur is not None:
            self._enter(cur, (x, w1, w3, w2, y, h, g, u))
        st = self.lib.muloco_gated_ffn(self.ctx, a, pg, pu, h.data_ptr(), y.data_ptr())
        if st:
            self._check(st)
        if cur is not None:
            cur.wait_stream(self.stream)
        return y, ((g, u, h) if save else None)

    def gated_ffn_backward(self, dy, x, w1, w3, w2, saved, activation="silu"):
        """muloco_gated_ffn_backward: (dx, dw1, dw3, dw2), bf16, from dy and the forward pass's saved = (g, u, h)."""
        g, u, h = saved
        r = self._quick("gated_ffn_backward", dy, x, w1, w3, w2, ACTIVATIONS.get(activation, -1), g, u, h)
        if r is not None:
            return r
        bf16 = self.torch.bfloat16
        a, T, d, F = self._ffn(x, w1, w3, w2, activation)
        self._need("dy", dy, bf16, (T, d))
        for name, t in (("g", g), ("u", u), ("h", h)):
            self._need(name, t, bf16, (T, F), dense=True)
        dg, du = x.new_empty((T, F)), x.new_empty((T, F))
        dx, dw1, dw3, dw2 = x.new_empty((T, d)), x.new_empty((d, F)), x.new_empty((d, F)), x.new_empty((F, d))
        cur = self._other_stream()
        if cur is not None:
            self._enter(cur, (dy, x, w1, w3, w2, g, u, h, dg, du, dx, dw1, dw3, dw2))
        st = self.lib.muloco_gated_ffn_backward(
            self.ctx, a, dy.data_ptr(), dy.stride(0) if T > 1 else d, g.data_ptr(), u.data_ptr(), h.data_ptr(),
            dg.data_ptr(), du.data_ptr(), dx.data_ptr(), dw1.data_ptr(), dw3.data_ptr(), dw2.data_ptr())
        if st:
            self._check(st)
        if cur is not None:
            cur.wait_stream(self.stream)
        return dx, dw1, dw3, dw2


class Context(_Operators):
    """A library context without optimizer state: for the operators of the training step around the
    optimizer (and AdamW lists) on `device` and `stream` (default: the current one)."""

    def __init__(self, device="cuda:0", stream=None):
        import torch

        self.torch = torch
        self.ctx = None
        self.lib = load_library()
        if not torch.cuda.is_available():
            raise RuntimeError("no CUDA device: libmuloco has no CPU path")
        self.device = torch.device(device)
        torch.cuda.set_device(self.device)
        self.stream = stream if stream is not None else torch.cuda.current_stream(self.device)
        self._init_operators()
        cfg = make_config(_cfg.Workload("operators", K=1, H=1, J=1, tensors=[], muon_lr=0.0, muon_beta=0.0,
                                        muon_wd=0.0, outer_lr=1.0, outer_momentum=0.0))
        ctx = C.c_void_p()
        st = self.lib.muloco_create(C.byref(cfg), None, 0, None, C.c_void_p(self.stream.cuda_stream), C.byref(ctx))
        if st != OK:
            raise MulocoError(st, self.lib.muloco_last_error(None).decode())
        self.ctx = ctx

    def _check(self, st):
        if st != OK:
            raise MulocoError(st, self.lib.muloco_last_error(self.ctx).decode())

    def sync_status(self):
        """Waits for the stream; raises what the device reported since the last call."""
        self._check(self.lib.muloco_sync_status(self.ctx))

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class AdamW:
    """muloco_adamw_*: AdamW over a list of float32 tensors, one launch per step, states in 32 or 8 bits.

    `owner` is a Context or a MuLoCo.  params: contiguous float32 tensors, updated in place; grads: tensors of the
    same shapes (float32 or bf16) used by step() without arguments; copies: bf16 tensors that receive the new
    parameters in the same pass.  The states live in flat buffers, every tensor starting on a multiple
    of 256 elements: state1, state2 (float32, or int8 / uint8 codes) and scale1, scale2 (one float32 per 256 codes).
    `steps` counts the steps taken; with it, the states are all there is to save for a checkpoint."""

    def __init__(self, owner, params, grads=None, lr=1e-3, beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=0.0,
                 bias_correction=True, state_bits=32, wd_mult=None, lr_mult=None, copies=None, seed=0, grad_dtype=None):
        torch = owner.torch
        self.opt = None
        # own lists: the library's table holds the tensors' addresses
        grads, copies = (None if l is None else list(l) for l in (grads, copies))
        self.owner, self.lib, self.params, self.grads, self.copies = owner, owner.lib, list(params), grads, copies
        n = len(self.params)
        if state_bits not in (8, 32):
            raise ValueError("state_bits must be 8 or 32")
        for name, seq in (("grads", grads), ("copies", copies), ("wd_mult", wd_mult), ("lr_mult", lr_mult)):
            if seq is not None and len(seq) != n:
                raise ValueError(f"{name} must have one entry per parameter")
        if grad_dtype is None:
            grad_dtype = grads[0].dtype if grads else torch.float32
        if grad_dtype not in (torch.float32, torch.bfloat16):
            raise ValueError("gradients must be float32 or bfloat16")
        self.state_bits, self.grad_dtype = state_bits, grad_dtype
        self.numel = [p.numel() for p in self.params]
        self.offsets, off = [], 0
        for k in self.numel:
            self.offsets.append(off)
            off += -(-k // ADAMW_BLOCK) * ADAMW_BLOCK
        self.padded = off
        for i, p in enumerate(self.params):
            self._same(f"params[{i}]", p, torch.float32, p)
            if copies is not None:
                self._same(f"copies[{i}]", copies[i], torch.bfloat16, p)
        if grads is not None:
            self._check_grads(grads)
        dev = owner.device
        q8 = state_bits == 8
        self.state1 = torch.zeros(off, dtype=torch.int8 if q8 else torch.float32, device=dev)
        self.state2 = torch.zeros(off, dtype=torch.uint8 if q8 else torch.float32, device=dev)
        self.scale1 = torch.zeros(off // ADAMW_BLOCK, dtype=torch.float32, device=dev) if q8 else None
        self.scale2 = torch.zeros(off // ADAMW_BLOCK, dtype=torch.float32, device=dev) if q8 else None
        cur = owner._other_stream()
        if cur is not None:                      # the zeros above are written there
            owner._enter(cur, (self.state1, self.state2, self.scale1, self.scale2))
        self.steps = 0
        cfg = AdamwConfig(lr, beta1, beta2, eps, weight_decay, int(bias_correction), state_bits,
                          BF16 if grad_dtype == torch.bfloat16 else F32, seed)
        table = (AdamwTensor * max(1, n))()
        for i, p in enumerate(self.params):
            o, e = self.offsets[i], table[i]
            e.n, e.theta = self.numel[i], p.data_ptr()
            e.copy = copies[i].data_ptr() if copies is not None else None
            e.grad = grads[i].data_ptr() if grads is not None else None
            e.state1 = self.state1.data_ptr() + o * self.state1.element_size()
            e.state2 = self.state2.data_ptr() + o * self.state2.element_size()
            if q8:
                e.scale1 = self.scale1.data_ptr() + o // ADAMW_BLOCK * 4
                e.scale2 = self.scale2.data_ptr() + o // ADAMW_BLOCK * 4
            e.wd_mult = 1.0 if wd_mult is None else wd_mult[i]
            e.lr_mult = 1.0 if lr_mult is None else lr_mult[i]
        opt = C.c_void_p()
        owner._check(self.lib.muloco_adamw_create(owner.ctx, C.byref(cfg), table, n, C.byref(opt)))
        self.opt = opt
        owner._lists.add(self)

    def _open(self):
        """Raises when the library's list is gone: its memory and, after the owner's close(), that of the context it names."""
        if self.opt is None:
            raise RuntimeError("the AdamW list is closed (by itself or with its context)")

    def _same(self, name, t, dtype, like):
        if t.get_device() != self.owner._dev or t.dtype != dtype or t.shape != like.shape or not t.is_contiguous():
            raise ValueError(f"{name} must be a contiguous {dtype} tensor of shape {tuple(like.shape)} on {self.owner.device}")

    def _check_grads(self, grads):
        for i, (g, p) in enumerate(zip(grads, self.params)):
            self._same(f"grads[{i}]", g, self.grad_dtype, p)

    def step(self, grads=None, lr_scale: float = 1.0):
        """One step of all tensors, with the gradients named at construction or those given."""
        self._open()
        if grads is None:
            f = self.owner._fast.get("adamw_step")
            if f is not None:
                st = f[0](self.opt.value, f[1], self.owner._dev, self.owner._handle, self.steps + 1, lr_scale)
                if st is not None:
                    if st:
                        self.owner._check(st)
                    self.steps += 1
                    return
        table = None
        if grads is not None:
            if len(grads) != len(self.params):
                raise ValueError("grads must have one entry per parameter")
            self._check_grads(grads)
            table = _ptr_table([g.data_ptr() for g in grads])
        cur = self.owner._other_stream()
        if cur is not None:
            self.owner._enter(cur, (*(grads if grads is not None else self.grads or ()), *self.params,
                                    *(self.copies or ())))
        self.owner._check(self.lib.muloco_adamw_step(self.opt, table, self.steps + 1, lr_scale))
        if cur is not None:
            cur.wait_stream(self.owner.stream)
        self.steps += 1

    def moments(self):
        """(m, v) as flat float32 tensors in the layout of the states: what the codes stand for, or the
        32-bit states themselves.  Padding entries are zero."""
        if self.state_bits == 32:
            return self.state1, self.state2
        self._open()
        f = self.owner._fast.get("adamw_moments")
        if f is not None:
            r = f[0](self.opt.value, f[1], self.owner._dev, self.owner._handle, self.scale1, self.padded)
            if r.__class__ is int:
                self.owner._check(r)
            if r is not None:
                return r
        m, v = self.scale1.new_empty(self.padded), self.scale1.new_empty(self.padded)
        cur = self.owner._other_stream()
        if cur is not None:
            self.owner._enter(cur, (m, v))
        self.owner._check(self.lib.muloco_adamw_moments(self.opt, m.data_ptr(), v.data_ptr()))
        if cur is not None:
            cur.wait_stream(self.owner.stream)
        return m, v

    def close(self):
        if getattr(self, "opt", None):
            if self.owner.ctx:
                self.lib.muloco_adamw_destroy(self.opt)
            self.opt = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class MuLoCo(_Operators):
    """Owns the device state of one MuLoCo problem and forwards to the C ABI.

    State lives in flat torch buffers (one per replica / state kind) so that the
    tensors of a replica are contiguous; each tensor starts on a 256-byte
    boundary.  `self.theta_g[i]`, `self.theta_k[k][i]` ... are torch views.  With
    adam_state_bits == 8 the states of AdamW tensors are byte tensors of their own
    (2.03 bytes per element instead of 8): `self.adam_moments(k, i)` has their values.
    """

    ALIGN = 64  # elements

    def __init__(self, workload: _cfg.Workload, device="cuda:0", init: Optional[Sequence[np.ndarray]] = None,
                 workspace_bytes: int = 0, ns_mode: Optional[str] = None, stream=None, alloc_grads: bool = False,
                 init_seed: Optional[int] = None, **config_overrides):
        import torch

        self.torch = torch
        self.lib = load_library()
        if not torch.cuda.is_available():
            raise RuntimeError("no CUDA device: libmuloco has no CPU path")
        self.w = workload
        self.device = torch.device(device)
        torch.cuda.set_device(self.device)
        self.K, self.n = workload.K, len(workload.tensors)
        self.cfg = make_config(workload, workspace_bytes, ns_mode, **config_overrides)
        self.offsets = []
        off = 0
        for t in workload.tensors:
            self.offsets.append(off)
            off += (t.numel + self.ALIGN - 1) // self.ALIGN * self.ALIGN
        self.flat_numel = off
        f32 = torch.float32
        dev = self.device
        self.flat_theta_g = torch.zeros(off, dtype=f32, device=dev)
        self.flat_u = torch.zeros(off, dtype=f32, device=dev)
        self.flat_theta_k = [torch.empty(off, dtype=f32, device=dev) for _ in range(self.K)]
        # 8-bit AdamW states: bytes (codes, then scales; see the header) instead of places in flat_s1 and flat_s2
        self.state8 = self.cfg.adam_state_bits == 8
        off1, offsets1 = 0, []
        for t in workload.tensors:
            offsets1.append(off1)
            off1 += 0 if self.state8 and t.kind == _cfg.ADAMW else (t.numel + self.ALIGN - 1) // self.ALIGN * self.ALIGN
        self.flat_s1 = [torch.empty(off1, dtype=f32, device=dev) for _ in range(self.K)]
        # Adam's second moment exists for AdamW tensors only: its own compact buffer
        self.offsets2, off2 = [], 0
        for t in workload.tensors:
            self.offsets2.append(off2 if t.kind == _cfg.ADAMW and not self.state8 else None)
            if t.kind == _cfg.ADAMW and not self.state8:
                off2 += (t.numel + self.ALIGN - 1) // self.ALIGN * self.ALIGN
        self.flat_s2 = [torch.empty(off2, dtype=f32, device=dev) if off2 else None for _ in range(self.K)]
        self.flat_ef = [torch.empty(off, dtype=f32, device=dev) for _ in range(self.K)] \
            if workload.error_feedback else None
        self.ef = [self._views(b) for b in self.flat_ef] if self.flat_ef else None
        self.theta_g = self._views(self.flat_theta_g)
        self.outer_u = self._views(self.flat_u)
        self.theta_k = [self._views(b) for b in self.flat_theta_k]
        self.state1 = [[b[o:o + t.numel].view(t.rows, t.cols) if not (self.state8 and t.kind == _cfg.ADAMW) else None
                        for o, t in zip(offsets1, workload.tensors)] for b in self.flat_s1]
        self.state2 = [[b[o:o + t.numel].view(t.rows, t.cols) if (b is not None and o is not None) else None
                        for o, t in zip(self.offsets2, workload.tensors)] for b in self.flat_s2]
        if self.state8:
            for k in range(self.K):
                for i, t in enumerate(workload.tensors):
                    if t.kind == _cfg.ADAMW:
                        n = -(-t.numel // ADAMW_BLOCK) * (ADAMW_BLOCK + 4)
                        self.state1[k][i], self.state2[k][i] = (torch.empty(n, dtype=torch.uint8, device=dev) for _ in range(2))
        if init is not None:
            for i, a in enumerate(init):
                self.theta_g[i].copy_(torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(dev))
        elif init_seed is not None:
            # device-side initial weights for the large configurations: N(0, 0.02^2), gains = 1
            gen = torch.Generator(device=dev)
            gen.manual_seed(init_seed)
            self.flat_theta_g.normal_(0.0, 0.02, generator=gen)
            for i, t in enumerate(workload.tensors):
                if t.init == "ones":
                    self.theta_g[i].fill_(1.0)
        self.gdtype = torch.bfloat16 if workload.grad_dtype == "bf16" else torch.float32
        self.flat_grads = None
        self.grads = None
        self._grad_table_all = None
        if alloc_grads:
            self.alloc_grads()

        descs = (TensorDesc * max(1, self.n))()
        for i, t in enumerate(workload.tensors):
            descs[i].rows, descs[i].cols = t.rows, t.cols
            descs[i].kind = MUON if t.kind == _cfg.MUON else ADAMW
            descs[i].fragment = t.fragment
            descs[i].wd_mult = t.wd_mult
            descs[i].lr_mult = float("nan") if t.lr_mult is None else t.lr_mult
        bufs = Buffers()
        self._tables = [
            _ptr_table([self.theta_k[k][i].data_ptr() for k in range(self.K) for i in range(self.n)]),
            _ptr_table([v.data_ptr() for v in self.theta_g]),
            _ptr_table([v.data_ptr() for v in self.outer_u]),
            _ptr_table([self.state1[k][i].data_ptr() for k in range(self.K) for i in range(self.n)]),
            _ptr_table([(self.state2[k][i].data_ptr() if self.state2[k][i] is not None else 0)
                        for k in range(self.K) for i in range(self.n)]),
        ]
        bufs.theta_k, bufs.theta_g, bufs.outer_u, bufs.state1_k, bufs.state2_k = [
            C.cast(t, C.POINTER(C.c_void_p)) for t in self._tables]
        if self.ef is not None:
            self._tables.append(_ptr_table([self.ef[k][i].data_ptr() for k in range(self.K) for i in range(self.n)]))
            bufs.ef_k = C.cast(self._tables[-1], C.POINTER(C.c_void_p))
        self.stream = stream if stream is not None else torch.cuda.current_stream(dev)
        self._init_operators()
        cur = self._other_stream()
        if cur is not None:                      # the initial weights are written there
            self.stream.wait_stream(cur)
        self.ctx = C.c_void_p()
        st = self.lib.muloco_create(C.byref(self.cfg), descs, self.n, C.byref(bufs),
                                    C.c_void_p(self.stream.cuda_stream), C.byref(self.ctx))
        if st != OK:
            msg = self.lib.muloco_last_error(None).decode()
            self.ctx = None
            raise MulocoError(st, msg)

    # -- helpers --------------------------------------------------------------
    def _views(self, flat):
        return [flat[o:o + t.numel].view(t.rows, t.cols) for o, t in zip(self.offsets, self.w.tensors)]

    def alloc_grads(self):
        torch = self.torch
        self.flat_grads = [torch.zeros(self.flat_numel, dtype=self.gdtype, device=self.device)
                           for _ in range(self.K)]
        self.grads = [self._views(b) for b in self.flat_grads]
        self._grad_table_all = _ptr_table([self.grads[k][i].data_ptr() for k in range(self.K)
                                           for i in range(self.n)])

    def new_buffer(self, n: int):
        return self.torch.empty(n, dtype=self.torch.float32, device=self.device)

    def stream_context(self):
        return self.torch.cuda.stream(self.stream)

    def _check(self, st):
        if st != OK:
            raise MulocoError(st, self.lib.muloco_last_error(self.ctx).decode())

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # -- the C ABI, one method per entry point ----------------------------------
    def inner_step(self, worker: int = -1, grads=None, lr_scale: float = 1.0):
        """muloco_inner_step.  grads: list (one worker) or list of lists (all) of torch
        tensors; None uses the buffers of alloc_grads()."""
        if grads is None:
            if worker < 0:
                table = self._grad_table_all
            else:
                table = _ptr_table([self.grads[worker][i].data_ptr() for i in range(self.n)])
        elif worker < 0:
            table = _ptr_table([grads[k][i].data_ptr() for k in range(self.K) for i in range(self.n)])
        else:
            table = _ptr_table([g.data_ptr() for g in grads])
        self._check(self.lib.muloco_inner_step(self.ctx, worker, C.cast(table, C.POINTER(C.c_void_p)), lr_scale))

    def inner_step_host(self, worker: int, host_grads, lr_scale: float = 1.0):
        """muloco_inner_step_host.  host_grads: like grads, but CPU (pinned) tensors."""
        if worker < 0:
            table = _ptr_table([host_grads[k][i].data_ptr() for k in range(self.K) for i in range(self.n)])
        else:
            table = _ptr_table([g.data_ptr() for g in host_grads])
        self._check(self.lib.muloco_inner_step_host(self.ctx, worker, C.cast(table, C.POINTER(C.c_void_p)),
                                                    lr_scale))

    def outer_sync(self, fragment: int = -1):
        self._check(self.lib.muloco_outer_sync(self.ctx, fragment))

    def outer_sync_host(self, fragment: int, host_theta_g):
        table = _ptr_table([(t.data_ptr() if t is not None else 0) for t in host_theta_g])
        self._check(self.lib.muloco_outer_sync_host(self.ctx, fragment, C.cast(table, C.POINTER(C.c_void_p))))

    def fragments_due(self, step: int) -> List[int]:
        out = (C.c_int32 * max(1, self.cfg.J))()
        n = self.lib.muloco_fragments_due(self.ctx, step, out)
        if n < 0:
            raise MulocoError(EINVAL, "muloco_fragments_due")
        return [out[i] for i in range(n)]

    def newton_schulz(self, X, out_dtype=None, ns_mode: str = "bf16"):
        """muloco_newton_schulz on a [batch, rows, cols] (or [rows, cols]) CUDA tensor."""
        torch = self.torch
        x = X if X.dim() == 3 else X.unsqueeze(0)
        x = x.contiguous()
        out_dtype = out_dtype or torch.float32
        o = torch.empty(x.shape, dtype=out_dtype, device=x.device)
        dt = {torch.float32: F32, torch.bfloat16: BF16}
        self._check(self.lib.muloco_newton_schulz(self.ctx, x.data_ptr(), dt[x.dtype], o.data_ptr(), dt[out_dtype],
                                                  x.shape[0], x.shape[1], x.shape[2],
                                                  NS_FP32 if ns_mode == "fp32" else NS_BF16))
        return o if X.dim() == 3 else o[0]

    def quantize(self, psi, bits: int):
        torch = self.torch
        p = psi.contiguous().view(-1, psi.shape[-1]) if psi.dim() > 1 else psi.contiguous().view(1, -1)
        rows, cols = p.shape
        blk = self.cfg.quant_block
        codes = torch.empty((rows, cols), dtype=torch.int8, device=p.device)
        scales = torch.empty((rows, (cols + blk - 1) // blk), dtype=torch.float32, device=p.device)
        deq = torch.empty((rows, cols), dtype=torch.float32, device=p.device)
        self._check(self.lib.muloco_quantize(self.ctx, p.data_ptr(), rows, cols, bits, codes.data_ptr(),
                                             scales.data_ptr(), deq.data_ptr()))
        return codes, scales, deq

    def topk_sparsify(self, x, fraction: float):
        torch = self.torch
        xc = x.contiguous()
        out = torch.empty_like(xc)
        self._check(self.lib.muloco_topk_sparsify(self.ctx, xc.data_ptr(), xc.numel(), fraction, out.data_ptr()))
        return out

    def pseudogradient(self, tensor: int):
        torch = self.torch
        t = self.w.tensors[tensor]
        out = torch.empty((t.rows, t.cols), dtype=torch.float32, device=self.device)
        self._check(self.lib.muloco_pseudogradient(self.ctx, tensor, out.data_ptr()))
        return out

    def get_state(self) -> bytes:
        n = C.c_size_t(0)
        self._check(self.lib.muloco_get_state(self.ctx, None, C.byref(n)))
        buf = C.create_string_buffer(n.value)
        self._check(self.lib.muloco_get_state(self.ctx, buf, C.byref(n)))
        return buf.raw[:n.value]

    def set_state(self, blob: bytes):
        self._check(self.lib.muloco_set_state(self.ctx, blob, len(blob)))

    def set_timing(self, on: bool):
        self._check(self.lib.muloco_set_timing(self.ctx, int(on)))

    def get_timings(self):
        ms = (C.c_float * len(PHASES))()
        launches = C.c_int64(0)
        self._check(self.lib.muloco_get_timings(self.ctx, ms, C.byref(launches)))
        return {p: ms[i] for i, p in enumerate(PHASES)}, launches.value

    def sync_status(self):
        self._check(self.lib.muloco_sync_status(self.ctx))

    # -- worker-sharded outer sync: three library calls around the caller's two collectives --------
    def shard_layout(self, fragment: int, world: int, rank: int):
        """muloco_shard_layout -> (stage_floats, shard_floats)."""
        a, b = C.c_int64(0), C.c_int64(0)
        self._check(self.lib.muloco_shard_layout(self.ctx, fragment, world, rank, C.byref(a), C.byref(b)))
        return a.value, b.value

    def shard_delta(self, fragment: int, world: int, stage):
        self._check(self.lib.muloco_shard_delta(self.ctx, fragment, world, stage.data_ptr()))

    def shard_step(self, fragment: int, world: int, rank: int, reduced, theta_shard):
        self._check(self.lib.muloco_shard_step(self.ctx, fragment, world, rank, reduced.data_ptr(),
                                               theta_shard.data_ptr()))

    def shard_broadcast(self, fragment: int, world: int, theta_all):
        self._check(self.lib.muloco_shard_broadcast(self.ctx, fragment, world, theta_all.data_ptr()))

    def sharded_outer_sync(self, fragment: int, dist, group=None):
        """The outer synchronisation with the workers spread over the ranks of `group`
        (torch.distributed): local delta sums -> reduce-scatter -> Nesterov step on the shard ->
        all-gather -> broadcast into the local replicas.  The collectives run on this context's
        stream.  Returns the bytes this rank sent and received over the wire (the ring
        algorithm's 2 * 4 * stage_floats * (world - 1) / world)."""
        return sharded_outer_sync(self, fragment, dist, group)

    def adam_moments(self, worker: int, tensor: int):
        """(m, v) of an AdamW tensor as float32 of its shape: the states, or the values 8-bit states stand for."""
        t = self.w.tensors[tensor]
        a, b = self.state1[worker][tensor], self.state2[worker][tensor]
        if not self.state8:
            return a, b
        torch, n = self.torch, -(-t.numel // ADAMW_BLOCK) * ADAMW_BLOCK
        def values(s, dtype):
            return s[:n].view(dtype).float().view(-1, ADAMW_BLOCK) * s[n:].view(torch.float32)[:, None]
        m, r = values(a, torch.int8), values(b, torch.uint8)
        return m.view(-1)[:t.numel].view(t.rows, t.cols), r.square().view(-1)[:t.numel].view(t.rows, t.cols)

    def check_workspace(self):
        """muloco_check_workspace: raises MulocoError(ESTATE) if a workspace canary was overwritten."""
        self._check(self.lib.muloco_check_workspace(self.ctx))

    def debug_set(self, what: int, value: int):
        """muloco_debug_set (test hooks of the failure path)."""
        self._check(self.lib.muloco_debug_set(self.ctx, what, value))
