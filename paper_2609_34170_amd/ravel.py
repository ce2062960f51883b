"""Thin ctypes binding of libravel (include/ravel.h).

Argument marshalling only: every step of the rolling denoise path runs in the
HIP kernels of libravel.so.  Device buffers are torch tensors on the GPU (used
for memory and streams only); host arrays are numpy arrays.  The library must
be built first (``paper_2609_34170_amd.build.build()``); importing this module
without it raises immediately -- there is no CPU fallback.
"""

from __future__ import annotations

import contextlib
import ctypes
import os
import struct
from typing import Dict, List, Optional, Tuple

import numpy as np

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libravel.so")

F32, BF16 = 0, 1
TRANSFORMER, ANALYTIC_OT, ANALYTIC_LINEAR = 0, 1, 2
OPT_SYNC_CONTEXT, OPT_USE_GRAPH, OPT_DEBUG, OPT_PERSISTENT, OPT_FAIL_LAYERS = 1, 2, 3, 4, 5
Q_GRAPHS, Q_PERSISTENT, Q_PHASES, Q_STEPS = 1, 2, 3, 4

_STATUS = {0: "OK", -1: "E_INVALID", -2: "E_NOMEM", -3: "E_HIP", -4: "E_SHAPE", -5: "E_STATE"}


class RavelError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"{_STATUS.get(status, status)}: {msg}")
        self.status = status


class RavelConfig(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in (
        "layers", "width", "n_q_heads", "n_kv_heads", "head_dim", "mlp_dim", "horizon", "action_dim",
        "prefix_len", "n_fop", "fop_obs_dim", "fop_stride", "dtype", "model_kind")] + [
        ("delta_bias", ctypes.c_float), ("rms_eps", ctypes.c_float), ("offset_mode", ctypes.c_int32),
        ("rope_base", ctypes.c_float)]


class RavelTensor(ctypes.Structure):
    _fields_ = [("name", ctypes.c_char_p), ("dtype", ctypes.c_int32), ("rank", ctypes.c_int32),
                ("dims", ctypes.c_int64 * 4), ("data", ctypes.c_void_p)]


class KernelRecord(ctypes.Structure):
    _fields_ = [("name", ctypes.c_char * 48), ("bytes", ctypes.c_double), ("flops", ctypes.c_double),
                ("ms", ctypes.c_float)]


class RavelCache(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in (
        "n_seq", "n_kv_heads", "head_dim", "capacity", "block", "reserved")] + [
        (n, ctypes.c_void_p) for n in ("k", "v", "k_scale", "v_scale", "len", "weight")]


class RavelCacheQuery(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("dtype", "batch", "n_q_heads", "rows", "n_self", "track")] + [
        ("scale", ctypes.c_float), ("reserved", ctypes.c_int32)] + [
        (n, ctypes.c_void_p) for n in ("seq", "q", "self_k", "self_v", "out")] + [
        (n, ctypes.c_int64 * 3) for n in ("q_stride", "self_stride", "out_stride")] + [
        ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_int64)]


# RavelCacheQuery's fields in one call (filling the structure field by field costs more than a launch)
_pack_query = struct.Struct("@6ifi5P9qPq").pack


SYMBOLS = [
    "ravel_create", "ravel_destroy", "ravel_model_weight_bytes", "ravel_buffer_create",
    "ravel_buffer_destroy", "ravel_buffer_set_option", "ravel_context_acquire", "ravel_set_context",
    "ravel_step", "ravel_step_state", "ravel_set_relative_dims", "ravel_full_denoise", "ravel_train_loss",
    "ravel_fop_encode", "ravel_fop_encode_noalloc", "ravel_buffer_sync", "ravel_debug_state",
    "ravel_publish_log", "ravel_buffer_query",
    "ravel_buffer_save", "ravel_buffer_load", "ravel_profile_step", "ravel_last_error",
    "ravel_cache_append", "ravel_cache_attention_workspace", "ravel_cache_attention", "ravel_cache_evict_workspace",
    "ravel_cache_evict", "ravel_buffer_create_quantized", "ravel_context_track", "ravel_context_evict",
    "ravel_context_cache",
]

_lib = None


def load_library(path: str = LIB_PATH) -> ctypes.CDLL:
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise RuntimeError(f"{path} is missing: build it with paper_2609_34170_amd.build.build()")
    lib = ctypes.CDLL(path)
    vp, i32, i64, u64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_uint64
    sig = {
        "ravel_create": ([ctypes.POINTER(RavelConfig), ctypes.POINTER(RavelTensor), i32, ctypes.POINTER(vp)], i32),
        "ravel_destroy": ([vp], None),
        "ravel_model_weight_bytes": ([vp], i64),
        "ravel_buffer_create": ([vp, i32, u64, ctypes.POINTER(vp)], i32),
        "ravel_buffer_destroy": ([vp], None),
        "ravel_buffer_set_option": ([vp, i32, i64], i32),
        "ravel_context_acquire": ([vp, i32, ctypes.POINTER(vp), ctypes.POINTER(vp), vp], i32),
        "ravel_set_context": ([vp, i32, vp, vp, i64, vp], i32),
        "ravel_step": ([vp, vp, vp, vp], i32),
        "ravel_full_denoise": ([vp, i32, vp, vp, vp, vp], i32),
        "ravel_train_loss": ([vp, vp, vp, vp, vp, vp, vp, vp], i32),
        "ravel_set_relative_dims": ([vp, vp], i32),
        "ravel_step_state": ([vp, vp, vp, vp, vp], i32),
        "ravel_fop_encode": ([vp, vp, vp, vp], i32),
        "ravel_fop_encode_noalloc": ([vp, i32, vp, vp, vp], i32),
        "ravel_buffer_sync": ([vp], i32),
        "ravel_debug_state": ([vp, vp, vp, vp], i32),
        "ravel_publish_log": ([vp, vp, ctypes.POINTER(i32)], i32),
        "ravel_buffer_query": ([vp, i32, ctypes.POINTER(i64)], i32),
        "ravel_buffer_save": ([vp, vp, ctypes.POINTER(ctypes.c_size_t)], i32),
        "ravel_buffer_load": ([vp, vp, ctypes.c_size_t], i32),
        "ravel_profile_step": ([vp, vp, vp, vp, ctypes.POINTER(KernelRecord), ctypes.POINTER(i32)], i32),
        "ravel_last_error": ([], ctypes.c_char_p),
        "ravel_cache_append": ([ctypes.POINTER(RavelCache), i32, vp, vp, vp, i32, i32, vp, vp, i64, i64, i64, vp], i32),
        "ravel_cache_attention_workspace": ([ctypes.POINTER(RavelCache), vp, ctypes.POINTER(i64)], i32),
        "ravel_cache_attention": ([ctypes.POINTER(RavelCache), vp, vp], i32),
        "ravel_cache_evict_workspace": ([ctypes.POINTER(RavelCache), i32, i32, ctypes.POINTER(i64)], i32),
        "ravel_cache_evict": ([ctypes.POINTER(RavelCache), i32, vp, i32, i32, ctypes.POINTER(RavelCache), vp, vp, vp,
                               i64, vp], i32),
        "ravel_buffer_create_quantized": ([vp, i32, u64, i32, ctypes.POINTER(vp)], i32),
        "ravel_context_track": ([vp, i32], i32),
        "ravel_context_evict": ([vp, i32, i32, i32, vp], i32),
        "ravel_context_cache": ([vp, i32, ctypes.POINTER(RavelCache)], i32),
    }
    for name, (args, res) in sig.items():
        fn = getattr(lib, name)
        fn.argtypes = args
        fn.restype = res
    _lib = lib
    return lib


def _check(status: int):
    if status != 0:
        msg = load_library().ravel_last_error().decode(errors="replace")
        raise RavelError(status, msg)


def _ptr(x) -> Optional[int]:
    """Device/host address of a torch tensor, numpy array or raw int (None -> NULL)."""
    if x is None:
        return None
    if isinstance(x, int):
        return x
    if isinstance(x, np.ndarray):
        if not x.flags["C_CONTIGUOUS"]:
            raise ValueError("host arrays must be C-contiguous")
        return x.ctypes.data
    if hasattr(x, "data_ptr"):
        if not x.is_contiguous():
            raise ValueError("tensors must be contiguous")
        return x.data_ptr()
    raise TypeError(f"cannot take the address of {type(x)}")


def _stream(stream) -> Optional[int]:
    if stream is None:
        import torch
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def make_config(shape) -> RavelConfig:
    c = RavelConfig()
    for f, _ in RavelConfig._fields_:
        setattr(c, f, getattr(shape, f))
    return c


class Model:
    """A model on the current HIP device (ravel_create)."""

    def __init__(self, shape, weights: Dict[str, np.ndarray]):
        lib = load_library()
        self.shape = shape
        self.cfg = make_config(shape)
        keep: List[np.ndarray] = []
        arr = (RavelTensor * max(len(weights), 1))()
        for i, (name, a) in enumerate(weights.items()):
            a = np.ascontiguousarray(a, dtype=np.float32)
            keep.append(a)
            t = arr[i]
            t.name = name.encode()
            t.dtype = F32
            t.rank = a.ndim
            for d in range(a.ndim):
                t.dims[d] = a.shape[d]
            t.data = a.ctypes.data
        h = ctypes.c_void_p()
        _check(lib.ravel_create(ctypes.byref(self.cfg), arr, len(weights), ctypes.byref(h)))
        self.h = h

    def fop_encode_noalloc(self, batch: int, obs, fop_tokens, stream=None):
        """The FOP encoder without a buffer and without allocating (fixed device scratch)."""
        _check(load_library().ravel_fop_encode_noalloc(self.h, int(batch), _ptr(obs), _ptr(fop_tokens),
                                                        _stream(stream)))

    @property
    def weight_bytes(self) -> int:
        return int(load_library().ravel_model_weight_bytes(self.h))

    def close(self):
        if getattr(self, "h", None):
            load_library().ravel_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Buffer:
    """Rolling state of B environments (ravel_buffer_create); ``quantized``: tokens per scale of contexts held in 8 bits
    (ravel_buffer_create_quantized), 0: contexts in the model's dtype."""

    def __init__(self, model: Model, batch: int, seed: int = 0, quantized: int = 0):
        lib = load_library()
        self.model = model
        self.B = batch
        self.seed = seed
        h = ctypes.c_void_p()
        if quantized:
            _check(lib.ravel_buffer_create_quantized(model.h, batch, seed, int(quantized), ctypes.byref(h)))
        else:
            _check(lib.ravel_buffer_create(model.h, batch, seed, ctypes.byref(h)))
        self.h = h

    # -- options -----------------------------------------------------------
    def set_option(self, option: int, value: int):
        _check(load_library().ravel_buffer_set_option(self.h, option, int(value)))

    # -- context plane -------------------------------------------------------
    def acquire(self, env: int, stream=None) -> Tuple[int, int]:
        k, v = ctypes.c_void_p(), ctypes.c_void_p()
        _check(load_library().ravel_context_acquire(self.h, env, ctypes.byref(k), ctypes.byref(v),
                                                    _stream(stream)))
        return k.value, v.value

    def set_context(self, env: int, k, v, t_obs: int, stream=None):
        _check(load_library().ravel_set_context(self.h, env, _ptr(k), _ptr(v), int(t_obs), _stream(stream)))

    def track_context(self, on: bool = True):
        _check(load_library().ravel_context_track(self.h, int(bool(on))))

    def evict_context(self, env: int, keep: int, first: int = 0, stream=None):
        _check(load_library().ravel_context_evict(self.h, env, int(keep), int(first), _stream(stream)))

    def context_cache(self, env: int) -> "Cache":
        """env's active context as a cache of ``layers`` sequences in the buffer's memory (which must outlive it)."""
        import torch

        c = RavelCache()
        _check(load_library().ravel_context_cache(self.h, env, ctypes.byref(c)))
        lead, blocks = (c.n_seq, c.n_kv_heads), -(-c.capacity // c.block)

        def tensor(ptr, shape, kind):
            at = type("DeviceMemory", (), {"__cuda_array_interface__": {
                "shape": shape, "typestr": kind, "data": (ptr, False), "version": 2}})()
            return torch.as_tensor(at, device="cuda")

        code = lead + (c.capacity, c.head_dim)
        return Cache(tensor(c.k, code, "|u1"), tensor(c.v, code, "|u1"), tensor(c.k_scale, lead + (blocks,), "<f4"),
                     tensor(c.v_scale, lead + (blocks,), "<f4"), tensor(c.len, (c.n_seq,), "<i4"), c.block,
                     weight=tensor(c.weight, lead + (c.capacity,), "<f4"))

    # -- hot path ----------------------------------------------------------
    def step(self, fop_tokens, action_out, stream=None):
        _check(load_library().ravel_step(self.h, _ptr(fop_tokens), _ptr(action_out), _stream(stream)))

    def set_relative_dims(self, mask):
        m = None
        if mask is not None:
            m = np.ascontiguousarray(np.asarray(mask, dtype=np.int32))
            self._mask = m
        _check(load_library().ravel_set_relative_dims(self.h, None if m is None else m.ctypes.data))

    def step_state(self, fop_tokens, state, action_out, stream=None):
        _check(load_library().ravel_step_state(self.h, _ptr(fop_tokens), _ptr(state), _ptr(action_out),
                                               _stream(stream)))

    def full_denoise(self, steps: int, fop_tokens, noise, chunk_out, stream=None):
        _check(load_library().ravel_full_denoise(self.h, int(steps), _ptr(fop_tokens), _ptr(noise), _ptr(chunk_out),
                                                 _stream(stream)))

    def train_loss(self, target, noise, ages, fop_tokens, loss_out, v_out=None, stream=None):
        _check(load_library().ravel_train_loss(self.h, _ptr(target), _ptr(noise), _ptr(ages), _ptr(fop_tokens),
                                               _ptr(loss_out), _ptr(v_out), _stream(stream)))

    def fop_encode(self, obs, fop_tokens, stream=None):
        _check(load_library().ravel_fop_encode(self.h, _ptr(obs), _ptr(fop_tokens), _stream(stream)))

    def profile_step(self, fop_tokens, action_out, stream=None, capacity: int = 4096):
        recs = (KernelRecord * capacity)()
        n = ctypes.c_int32(capacity)
        _check(load_library().ravel_profile_step(self.h, _ptr(fop_tokens), _ptr(action_out), _stream(stream),
                                                 recs, ctypes.byref(n)))
        return [(recs[i].name.decode(), recs[i].bytes, recs[i].flops, recs[i].ms) for i in range(n.value)]

    # -- inspection --------------------------------------------------------
    def sync(self):
        _check(load_library().ravel_buffer_sync(self.h))

    def debug_state(self):
        s = self.model.shape
        X = np.zeros((self.B, s.horizon, s.action_dim), dtype=np.float32)
        t = ctypes.c_int64()
        t_obs = np.zeros(self.B, dtype=np.int64)
        _check(load_library().ravel_debug_state(self.h, X.ctypes.data, ctypes.addressof(t), t_obs.ctypes.data))
        return X, int(t.value), t_obs

    def publish_log(self) -> List[Tuple[int, int, int]]:
        lib = load_library()
        n = ctypes.c_int32(0)
        _check(lib.ravel_publish_log(self.h, None, ctypes.byref(n)))
        cap = max(n.value, 1)
        buf = np.zeros((cap, 3), dtype=np.int64)
        n = ctypes.c_int32(cap)
        _check(lib.ravel_publish_log(self.h, buf.ctypes.data, ctypes.byref(n)))
        return [tuple(int(x) for x in buf[i]) for i in range(n.value)]

    def query(self, key: int) -> int:
        v = ctypes.c_int64(0)
        _check(load_library().ravel_buffer_query(self.h, int(key), ctypes.byref(v)))
        return int(v.value)

    def save(self) -> bytes:
        lib = load_library()
        n = ctypes.c_size_t(0)
        _check(lib.ravel_buffer_save(self.h, None, ctypes.byref(n)))
        blob = np.zeros(n.value, dtype=np.uint8)
        _check(lib.ravel_buffer_save(self.h, blob.ctypes.data, ctypes.byref(n)))
        return blob.tobytes()

    def load(self, blob: bytes):
        a = np.frombuffer(blob, dtype=np.uint8).copy()
        _check(load_library().ravel_buffer_load(self.h, a.ctypes.data, a.size))

    def close(self):
        if getattr(self, "h", None):
            load_library().ravel_buffer_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Cache:
    """A key/value cache in 8 bits (the ravel_cache_* calls) over tensors that the caller owns.

    ``k``, ``v``: e4m3 codes ``[n_seq, n_kv_heads, capacity, head_dim]`` (float8_e4m3fn or uint8); ``k_scale``,
    ``v_scale``: float32 ``[n_seq, n_kv_heads, ceil(capacity / block)]``; ``length``: int32 ``[n_seq]``; ``weight``:
    float32 ``[n_seq, n_kv_heads, capacity]`` or None.  ``Cache.empty`` makes them.  Indices, positions and counts are
    int32 tensors on the same device.  Calls are enqueued on ``stream`` (default: torch's current one).
    """

    def __init__(self, k, v, k_scale, v_scale, length, block: int, weight=None):
        import torch

        n_seq, n_kv, cap, hd = k.shape
        blocks = (n_seq, n_kv, -(-cap // block) if block > 0 else 0)
        for name, t, shape, types in (
                ("k", k, k.shape, (torch.float8_e4m3fn, torch.uint8)), ("v", v, k.shape, (torch.float8_e4m3fn, torch.uint8)),
                ("k_scale", k_scale, blocks, (torch.float32,)), ("v_scale", v_scale, blocks, (torch.float32,)),
                ("length", length, (n_seq,), (torch.int32,)), ("weight", weight, (n_seq, n_kv, cap), (torch.float32,))):
            if t is None and name == "weight":
                continue
            if tuple(t.shape) != tuple(shape) or t.dtype not in types or t.device != k.device or not t.is_contiguous():
                raise ValueError(f"{name} must be a contiguous {types[0]} tensor {tuple(shape)} on {k.device}")
        self.k, self.v, self.k_scale, self.v_scale, self.length, self.weight = k, v, k_scale, v_scale, length, weight
        self.block, self.device, self._device_index, self._torch = block, k.device, k.get_device(), torch
        self._lib, self._workspace = load_library(), {}
        self._raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
            lambda device: torch.cuda.current_stream(device).cuda_stream)
        self._codes_shape = (n_kv, hd)
        self._c = RavelCache(n_seq, n_kv, hd, cap, block, 0, k.data_ptr(), v.data_ptr(), k_scale.data_ptr(),
                             v_scale.data_ptr(), length.data_ptr(), None if weight is None else weight.data_ptr())
        self._ref = ctypes.byref(self._c)

    @classmethod
    def empty(cls, n_seq: int, n_kv_heads: int, capacity: int, head_dim: int, block: int = 64, weight: bool = False,
              device="cuda"):
        """A cache of empty sequences: codes 0 under the smallest scale, so that positions skipped by an append are zeros
        and leave their block's scale to its tokens."""
        import torch

        codes = [torch.zeros((n_seq, n_kv_heads, capacity, head_dim), dtype=torch.uint8, device=device)
                 .view(torch.float8_e4m3fn) for _ in range(2)]
        scales = [torch.full((n_seq, n_kv_heads, -(-capacity // block)), 2.0 ** -100, device=device) for _ in range(2)]
        return cls(*codes, *scales, torch.zeros(n_seq, dtype=torch.int32, device=device), block,
                   torch.zeros((n_seq, n_kv_heads, capacity), device=device) if weight else None)

    def _on(self, stream, *tensors):
        """(guard that makes this cache's device and the call's stream current, or None; stream handle)."""
        device = self._device_index
        for t in tensors:
            if t is not None and t.get_device() != device:
                raise ValueError(f"every tensor of the call must be on {self.device}")
        if device < 0:
            raise ValueError("a cache's calls need its tensors on a GPU")
        cuda = self._torch.cuda
        if stream is None:
            if device == cuda.current_device():
                return None, self._raw_stream(device)
            return cuda.device(self.device), self._raw_stream(device)
        if isinstance(stream, int):
            stream = cuda.ExternalStream(stream, device=self.device)
        elif stream.device != self.device:
            raise ValueError(f"the stream must be one of {self.device}")
        return cuda.stream(stream), stream.cuda_stream

    def _index(self, name, t, batch):
        if t is None:
            return None
        if t.dtype is not self._torch.int32 or t.dim() != 1 or t.shape[0] != batch or not t.is_contiguous():
            raise ValueError(f"{name} must be a contiguous int32 tensor [{batch}]")
        return t.data_ptr()

    def _dtype(self, t) -> int:
        if t.dtype is self._torch.bfloat16:
            return BF16
        if t.dtype is self._torch.float32:
            return F32
        raise ValueError(f"bf16 or float32 expected, got {t.dtype}")

    def append(self, k, v, pos=None, count=None, seq=None, stream=None):
        """Store k, v ``[batch, n, n_kv_heads, head_dim]`` (bf16 or float32) from ``pos`` (default: the lengths) on."""
        shape, strides = k.shape, k.stride()
        if len(shape) != 4 or shape[2:] != self._codes_shape or v.shape != shape or v.dtype is not k.dtype:
            raise ValueError("k and v must be [batch, n, %d, %d] of one dtype" % self._codes_shape)
        if v.stride() != strides or (strides[3] != 1 and k.numel()):
            raise ValueError("k and v must have the same strides, head_dim contiguous")
        guard, s = self._on(stream, k, v, pos, count, seq)
        B = shape[0]
        args = (self._ref, B, self._index("seq", seq, B), self._index("pos", pos, B), self._index("count", count, B),
                shape[1], self._dtype(k), k.data_ptr(), v.data_ptr(), strides[0], strides[1], strides[2], s)
        if guard is None:
            _check(self._lib.ravel_cache_append(*args))
        else:
            with guard:
                _check(self._lib.ravel_cache_append(*args))

    def attention(self, q, out, self_k=None, self_v=None, seq=None, scale=None, track=False, stream=None):
        """out = attention of q ``[batch, rows, n_q_heads, head_dim]`` over the sequences' tokens and the call's own
        ``self_k``, ``self_v`` ``[batch, n_self, n_kv_heads, head_dim]``; ``track``: add to the accumulated weights."""
        shape, qs, os_, dtype = q.shape, q.stride(), out.stride(), q.dtype
        nkv, hd = self._codes_shape
        if len(shape) != 4 or shape[3] != hd or out.shape != shape or out.dtype is not dtype:
            raise ValueError(f"q and out must be [batch, rows, n_q_heads, {hd}] of one dtype")
        if (qs[3] != 1 or os_[3] != 1) and q.numel():
            raise ValueError("head_dim must be contiguous")
        B, rows, nq, _ = shape
        n_self, kp, vp, ss = 0, 0, 0, (0, 0, 0)
        if self_k is not None and self_v is not None:
            n_self, ss = self_k.shape[1], self_k.stride()
            if self_k.shape != (B, n_self, nkv, hd) or self_v.shape != self_k.shape or self_k.dtype is not dtype or \
                    self_v.dtype is not dtype:
                raise ValueError(f"self_k and self_v must be [{B}, n_self, {nkv}, {hd}] of the queries' dtype")
            if self_v.stride() != ss or (ss[3] != 1 and self_k.numel()):
                raise ValueError("self_k and self_v must have the same strides, head_dim contiguous")
            kp, vp = self_k.data_ptr(), self_v.data_ptr()
        elif self_k is not self_v:
            raise ValueError("self_k and self_v must both be given or both None")
        guard, s = self._on(stream, q, out, self_k, self_v, seq)
        sizes = (self._dtype(q), B, nq, rows, n_self, 1 if track else 0)
        fields = (hd ** -0.5 if scale is None else scale, 0, self._index("seq", seq, B) or 0, q.data_ptr(), kp, vp,
                  out.data_ptr(), *qs[:3], *ss[:3], *os_[:3])
        if guard is None:
            self._attention(sizes, fields, s)
        else:
            with guard:
                self._attention(sizes, fields, s)

    def _attention(self, sizes, fields, s):
        n = self._workspace.get(sizes)  # bytes that calls of these sizes need
        if n is None:
            need = ctypes.c_int64(0)
            _check(self._lib.ravel_cache_attention_workspace(self._ref, _pack_query(*sizes, *fields, 0, 0), ctypes.byref(need)))
            n = self._workspace[sizes] = need.value
        ws = 0
        if n:
            # of this call alone: torch keeps it from later calls on the stream until this one has run
            memory = self._torch.empty(n, dtype=self._torch.uint8, device=self.device)
            ws = memory.data_ptr()
        _check(self._lib.ravel_cache_attention(self._ref, _pack_query(*sizes, *fields, ws, n), s))

    def evict(self, keep: int, first: int = 0, seq=None, into: Optional["Cache"] = None, into_seq=None, kept=None,
              stream=None):
        """Keep the ``keep`` tokens of the largest accumulated weight per row and KV head, in place or in another cache;
        returns the index each place's token had, int32 ``[batch, n_kv_heads, keep]`` (``kept``, or a new tensor)."""
        torch, c = self._torch, self._c
        B = seq.shape[0] if seq is not None else c.n_seq
        if into is not None and into.device != self.device:
            raise ValueError(f"every tensor of the call must be on {self.device}")
        guard, s = self._on(stream, seq, into_seq, kept)
        with guard if guard is not None else contextlib.nullcontext():
            if kept is None:
                kept = torch.empty((B, c.n_kv_heads, max(keep, 0)), dtype=torch.int32, device=self.device)
            elif tuple(kept.shape) != (B, c.n_kv_heads, keep) or kept.dtype is not torch.int32 or not kept.is_contiguous():
                raise ValueError(f"kept must be a contiguous int32 tensor [{B}, {c.n_kv_heads}, {keep}]")
            lib, n = self._lib, ctypes.c_int64(0)
            _check(lib.ravel_cache_evict_workspace(self._ref, B, keep, ctypes.byref(n)))
            ws = torch.empty(n.value, dtype=torch.uint8, device=self.device)
            _check(lib.ravel_cache_evict(self._ref, B, self._index("seq", seq, B), keep, first,
                                         None if into is None else into._ref, self._index("into_seq", into_seq, B),
                                         kept.data_ptr(), ws.data_ptr(), n.value, s))
        return kept
