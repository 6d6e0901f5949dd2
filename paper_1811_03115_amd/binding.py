"""ctypes binding with the same names as include/bpd.h.  Argument marshalling only.

PyTorch is used for device memory (the workspace and result tensors) and for the stream
handle; nothing here computes anything.
"""
from __future__ import annotations

import ctypes as C
import os
import struct
from typing import Dict, Optional

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libbpd.so")

BPD_F32, BPD_BF16 = 0, 1
TREE_MAX, BLOCKS_MAX = 64, 4096          # nodes of a tree, blocks that are chosen from
PHASE_NONE, PHASE_LAYERS, PHASE_HEAD_HIDDEN, PHASE_HEAD_OUT, PHASE_VOCAB, PHASE_ACCEPT, PHASE_STEP, PHASE_EMPTY = range(8)
ERRORS = {-1: "BPD_E_ARG", -2: "BPD_E_STATE", -3: "BPD_E_CAPACITY", -4: "BPD_E_WEIGHTS", -5: "BPD_E_HIP"}


class BpdError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"{ERRORS.get(code, code)}: {msg}")
        self.code = code


class bpd_config(C.Structure):
    _fields_ = [(n, C.c_int32) for n in (
        "n_enc_layers", "n_dec_layers", "d_model", "n_heads", "d_ff", "vocab", "k_max",
        "max_batch", "max_src_len", "max_out_len", "dtype", "eos_id", "pad_id")] + [("ln_eps", C.c_float)]


class bpd_tensor(C.Structure):
    _fields_ = [("name", C.c_char_p), ("data", C.c_void_p), ("dtype", C.c_int32), ("ndim", C.c_int32),
                ("shape", C.c_int64 * 4), ("on_device", C.c_int32)]


class bpd_stats(C.Structure):
    _fields_ = [("steps", C.c_int64), ("invocations", C.c_int64), ("seq_steps", C.c_int64),
                ("accepted_total", C.c_int64), ("hist", C.c_int64 * 17), ("finished", C.c_int32)]


class bpd_cache(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p)] + [(n, C.c_int32) for n in (
        "dtype", "n_layers", "max_batch", "n_kv_heads", "head_dim", "capacity")]


class bpd_rows(C.Structure):
    _fields_ = [("data", C.c_void_p), ("dtype", C.c_int32)] + [(n, C.c_int64) for n in ("layer", "seq", "row", "head")]


class bpd_blocks(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("block", "first", "recent", "top")] + [(n, C.c_void_p) for n in ("summaries", "added", "chosen")]


EXPORTS = ["bpd_workspace_bytes", "bpd_create", "bpd_destroy", "bpd_load_weights", "bpd_encode", "bpd_step", "bpd_step_static",
           "bpd_set_acceptance", "bpd_set_top_n", "bpd_set_two_phase", "bpd_set_local_attention", "bpd_decode", "bpd_get_state", "bpd_get_output", "bpd_get_stats",
           "bpd_set_proposals", "bpd_debug_step_logits", "bpd_profile_enable", "bpd_profile_read",
           "bpd_profile_samples", "bpd_measure_hbm_read", "bpd_measure_mfma_bf16", "bpd_last_error",
           "bpd_step_tree", "bpd_set_sparse_attention", "bpd_sparse_buffer_bytes",
           "bpd_op_error", "bpd_cache_bytes", "bpd_summaries_bytes", "bpd_attention_workspace_bytes", "bpd_cache_store", "bpd_tree_attention",
           "bpd_sparse_attention", "bpd_tree_accept"]

_lib = None
_torch = None                # torch, once the library is loaded
_raw_stream = None           # its current stream's handle by device number, where torch has that call


def lib() -> C.CDLL:
    """Load libbpd.so.  There is no fallback: without the HIP library nothing runs."""
    global _lib, _torch, _raw_stream
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with `python -m paper_1811_03115_amd.build` "
                               "(there is no CPU fallback)")
        import torch  # (first: the library then uses the HIP runtime that torch brings, not a second one)
        L = C.CDLL(LIB_PATH)
        vp, i32p = C.c_void_p, C.c_void_p
        L.bpd_workspace_bytes.restype = C.c_size_t
        L.bpd_workspace_bytes.argtypes = [C.POINTER(bpd_config)]
        L.bpd_create.argtypes = [C.POINTER(bpd_config), vp, C.c_size_t, vp, C.POINTER(vp)]
        L.bpd_destroy.argtypes = [vp]
        L.bpd_load_weights.argtypes = [vp, C.POINTER(bpd_tensor), C.c_int]
        L.bpd_encode.argtypes = [vp, i32p, i32p, i32p, C.c_int, C.c_int]
        L.bpd_step.argtypes = [vp, C.c_int, i32p, i32p]
        L.bpd_step_static.argtypes = [vp, C.c_int, i32p, i32p]
        L.bpd_set_acceptance.argtypes = [vp, C.c_int, C.c_int]
        L.bpd_set_top_n.argtypes = [vp, C.c_int]
        L.bpd_set_two_phase.argtypes = [vp, C.c_int]
        L.bpd_set_local_attention.argtypes = [vp, C.c_int, C.c_int]
        L.bpd_decode.argtypes = [vp, C.c_int, i32p, C.c_int, i32p, i32p, C.POINTER(bpd_stats)]
        L.bpd_get_state.argtypes = [vp, i32p, i32p, i32p, i32p]
        L.bpd_get_output.argtypes = [vp, i32p, i32p]
        L.bpd_get_stats.argtypes = [vp, C.POINTER(bpd_stats)]
        L.bpd_set_proposals.argtypes = [vp, i32p]
        L.bpd_debug_step_logits.argtypes = [vp, C.c_int, vp]
        L.bpd_profile_enable.argtypes = [vp, C.c_int]
        L.bpd_profile_read.argtypes = [vp, C.POINTER(C.c_double), C.POINTER(C.c_int64)]
        L.bpd_profile_samples.argtypes = [vp, vp, C.c_int64, C.POINTER(C.c_double), C.POINTER(C.c_int64)]
        L.bpd_measure_hbm_read.argtypes = [vp, C.c_size_t, vp, C.c_int, C.POINTER(C.c_double)]
        L.bpd_measure_mfma_bf16.argtypes = [vp, vp, C.c_int, C.POINTER(C.c_double)]
        L.bpd_step_tree.argtypes = [vp, C.c_int, i32p, i32p]
        L.bpd_set_sparse_attention.argtypes = [vp] + [C.c_int] * 4 + [vp, C.c_size_t]
        L.bpd_sparse_buffer_bytes.restype = C.c_size_t
        L.bpd_sparse_buffer_bytes.argtypes = [vp, C.c_int]
        cp, rp, sz = vp, vp, C.c_size_t          # (bpd_cache, bpd_rows, bpd_blocks: by reference, or as packed bytes)
        L.bpd_op_error.restype = C.c_char_p
        L.bpd_op_error.argtypes = []
        for name, args in (("bpd_cache_bytes", [cp]), ("bpd_summaries_bytes", [cp, C.c_int]), ("bpd_attention_workspace_bytes", [cp] + [C.c_int] * 4)):
            getattr(L, name).restype, getattr(L, name).argtypes = sz, args
        L.bpd_cache_store.argtypes = [cp, rp, rp, vp, vp, C.c_int, C.c_int, vp]
        L.bpd_tree_attention.argtypes = [cp, rp, rp, vp, vp, C.c_int, C.c_int, C.c_int, C.c_float, vp, sz, vp]
        L.bpd_sparse_attention.argtypes = [cp, rp, rp, vp, vp, C.c_int, C.c_int, C.c_int, C.c_float, vp, vp, sz, vp]
        L.bpd_tree_accept.argtypes = [vp] * 6 + [C.c_int] * 3 + [vp] * 4 + [cp, vp]
        L.bpd_last_error.restype = C.c_char_p
        L.bpd_last_error.argtypes = [vp]
        _torch, _raw_stream = torch, getattr(torch._C, "_cuda_getCurrentRawStream", None)
        _lib = L
    return _lib


def make_config(**kw) -> bpd_config:
    c = bpd_config()
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def config_from_workload(w, max_batch: Optional[int] = None) -> bpd_config:
    """bpd_config for a workloads.Config."""
    return make_config(n_enc_layers=w.n_enc, n_dec_layers=w.n_dec, d_model=w.d_model, n_heads=w.n_heads,
                       d_ff=w.d_ff, vocab=w.vocab, k_max=w.k, max_batch=max_batch or w.batch,
                       max_src_len=w.max_src, max_out_len=w.max_out,
                       dtype=BPD_BF16 if w.dtype == "bf16" else BPD_F32, eos_id=w.eos_id, pad_id=w.pad_id,
                       ln_eps=w.ln_eps)


def _ptr(a) -> Optional[int]:
    """Raw address of a numpy array (host) or torch tensor (host or device), or None."""
    if a is None:
        return None
    if isinstance(a, np.ndarray):
        assert a.flags["C_CONTIGUOUS"]
        return a.ctypes.data
    assert a.is_contiguous()
    return a.data_ptr()


def _i32(a):
    if a is None:
        return None
    if isinstance(a, np.ndarray):
        return np.ascontiguousarray(a, dtype=np.int32)
    import torch
    assert a.dtype == torch.int32
    return a.contiguous()


# -- caches that the caller owns
def new_cache(max_batch: int, n_kv_heads: int, head_dim: int, capacity: int, dtype=None, device="cuda", n_layers: Optional[int] = None):
    """(k, v): empty cache tensors of the shapes that the cache operators take, [n_layers,] B, .. (bpd_cache in include/bpd.h).
    bf16 heads of 64 and 128 dimensions: [B, heads, capacity / 32, 32, head_dim] in operand order, the capacity rounded up to a multiple of 32;
    others: [B, capacity, heads, head_dim]."""
    import torch
    dtype = dtype or torch.bfloat16
    if dtype == torch.bfloat16 and head_dim in (64, 128):
        shape = (max_batch, n_kv_heads, (capacity + 31) // 32, 32, head_dim)
    else:
        shape = (max_batch, capacity, n_kv_heads, head_dim)
    shape = shape if n_layers is None else (n_layers,) + shape
    return torch.empty(shape, dtype=dtype, device=device), torch.empty(shape, dtype=dtype, device=device)


def new_summaries(cache, block: int):
    """Room for the summaries of one layer's blocks, zeros: the first bpd_sparse_attention that gets them has added=None, which makes all of them."""
    import torch
    (_, _, _, _, b, h, d, cap), k, _ = _cache(cache, 0)
    if block not in (32, 64, 128):
        raise _bad("block: 32, 64 or 128 rows")
    return torch.zeros((b, h, (cap // block + 63) // 64, 2, d // 8, 64, 8), dtype=k.dtype, device=k.device)


def _op_check(rc: int):
    if rc != 0:
        raise BpdError(rc, lib().bpd_op_error().decode())


def _bad(what: str):
    return BpdError(-1, what)


# (the wrappers below are most of what a call of a few microseconds costs the host: they look at each tensor once, and pack bpd_cache, bpd_rows and bpd_blocks
# as bytes, which takes a quarter of what building a ctypes structure does)
_PACK_CACHE, _PACK_ROWS, _PACK_BLOCKS = struct.Struct("PPiiiiii"), struct.Struct("Pi4xqqqq"), struct.Struct("iiiiPPP")
_DTYPES = {}                 # torch's dtypes, filled with the first call: this module imports torch late
_WORKSPACES = {}             # bytes of workspace by the sizes that they depend on


def _dtype_of(t) -> int:
    if not _DTYPES:
        import torch
        _DTYPES.update({torch.bfloat16: BPD_BF16, torch.float32: BPD_F32})
    code = _DTYPES.get(t.dtype)
    if code is None:
        raise _bad(f"tensors are bfloat16 or float32, not {t.dtype}")
    return code


def _cache(cache, layer: Optional[int] = None):
    """The tensors (k, v) as a cache; layer: that one alone.  Returns (the fields of bpd_cache, k, whether the tensors have a dimension of layers)."""
    k, v = cache
    dtype, shape = _dtype_of(k), k.shape
    d = shape[-1]
    grouped = dtype == BPD_BF16 and (d == 64 or d == 128)
    layers = len(shape) - (5 if grouped else 4)
    if layers not in (0, 1) or shape != v.shape or k.dtype != v.dtype or k.get_device() != v.get_device() or not k.is_contiguous() or not v.is_contiguous():
        raise _bad("cache: k and v are contiguous tensors of one shape, type and device, as binding.new_cache makes them")
    n = shape[0] if layers else 1
    kp, vp = k.data_ptr(), v.data_ptr()
    if grouped:
        b, h, groups, rows, _ = shape[layers:]
        if rows != 32:
            raise _bad("cache: groups of 32 keys")
        cap = 32 * groups
    else:
        b, cap, h, _ = shape[layers:]
    if layer is not None:
        if not 0 <= layer < n:
            raise _bad("cache: no such layer")
        if layer:
            at = layer * (b * h * cap * d) * (2 if dtype == BPD_BF16 else 4)
            kp, vp = kp + at, vp + at
        n = 1
    return (kp, vp, dtype, n, b, h, d, cap), k, layers


def _int(device: int, shape, name: str, t):
    """Address of an int32 array of the given shape, contiguous, on the device (None: None)."""
    if t is None:
        return None
    if t.dtype != _torch.int32 or t.shape != shape or not t.is_contiguous():
        raise _bad(f"{name}: contiguous int32 {list(shape)}")
    if t.get_device() != device:
        raise _bad(f"{name} is on {t.device}, the cache on another device")
    return t.data_ptr()


def _rows(t, layers: int = 0):
    """bpd_rows of a tensor [layers,] B, T, heads, D whose last dimension is contiguous."""
    s = t.stride()
    if s[-1] != 1 and t.shape[-1] > 1:
        raise _bad("the last dimension of rows is contiguous")
    return _PACK_ROWS.pack(t.data_ptr(), _dtype_of(t), s[0] if layers else 0, s[layers], s[layers + 1], s[layers + 2])


def _call(device: int, call, *args):
    """call(*args, stream) on the device, on torch's current stream there."""
    if device < 0:
        raise _bad("tensors are on a GPU")
    stream = _raw_stream(device) if _raw_stream else _torch.cuda.current_stream(device).cuda_stream
    if device == _torch.cuda.current_device():
        rc = call(*args, stream)
    else:
        with _torch.cuda.device(device):
            rc = call(*args, stream)
    if rc:
        _op_check(rc)


def _attention(cache, layer, q, length, parent, scale, out, workspace, block):
    """What both attentions do with their arguments: (device, the cache's fields, the call's first arguments, workspace, its address and bytes, out)."""
    lib()
    c, k, _ = _cache(cache, layer)
    device, shape = k.get_device(), q.shape
    if len(shape) != 4 or shape[3] != c[6]:
        raise _bad("q: [B, T, heads, head_dim]")
    b, t, h, d = shape
    if q.get_device() != device:
        raise _bad("q and the cache are on different devices")
    if out is None:
        out = _torch.empty_like(q) if q.is_contiguous() else _torch.empty(shape, dtype=q.dtype, device=q.device)
    elif out.shape != shape or out.get_device() != device:
        raise _bad("out: the shape and device of q")
    length_p, parent_p = _int(device, (b,), "length", length), _int(device, (b, t), "parent", parent)
    if device < 0:
        raise _bad("tensors are on a GPU")
    packed = _PACK_CACHE.pack(*c)
    if workspace is None:
        key = (device, c[2:], b, t, h, block)
        need = _WORKSPACES.get(key)
        if need is None:
            with _torch.cuda.device(device):
                need = lib().bpd_attention_workspace_bytes(packed, b, t, h, block)
            if len(_WORKSPACES) > 4096:
                _WORKSPACES.clear()
            _WORKSPACES[key] = need
        if need:
            workspace = _torch.empty(need, dtype=_torch.uint8, device=q.device)
    elif workspace.get_device() != device or not workspace.is_contiguous():
        raise _bad("workspace: contiguous, on the cache's device")
    ws, nbytes = (workspace.data_ptr(), workspace.nbytes) if workspace is not None else (None, 0)
    return device, c, (packed, _rows(q), _rows(out), length_p, parent_p, b, t, h, d ** -0.5 if scale is None else scale), workspace, ws, nbytes, out


class Context:
    """Owns the workspace tensor and the opaque bpd_ctx*.  Methods mirror the C entry points."""

    def __init__(self, cfg: bpd_config, device: str = "cuda:0", stream=None):
        import torch
        self.torch = torch
        self.L = lib()
        self.cfg = cfg
        self.device = torch.device(device)
        nbytes = self.L.bpd_workspace_bytes(C.byref(cfg))
        if nbytes == 0:
            raise BpdError(-1, "invalid configuration")
        self.workspace = torch.empty(nbytes + 256, dtype=torch.uint8, device=self.device)
        base = self.workspace.data_ptr()
        aligned = (base + 255) // 256 * 256
        self.stream = stream if stream is not None else torch.cuda.current_stream(self.device)
        handle = C.c_void_p()
        with torch.cuda.device(self.device):
            rc = self.L.bpd_create(C.byref(cfg), aligned, nbytes, self.stream.cuda_stream, C.byref(handle))
        if rc != 0:
            raise BpdError(rc, "bpd_create failed")
        self.h = handle
        self.B = 0
        self.sparse_buffers = {}                 # by rows of a block (bpd_set_sparse_attention)

    # -- helpers
    def _check(self, rc: int):
        if rc != 0:
            raise BpdError(rc, self.L.bpd_last_error(self.h).decode())

    def close(self):
        if getattr(self, "h", None):
            self.L.bpd_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # -- C ABI mirrors
    def bpd_load_weights(self, weights: Dict[str, object]):
        """weights: name -> numpy float32 array (host) or torch float32/bfloat16 tensor (host or device)."""
        torch = self.torch
        arr = (bpd_tensor * len(weights))()
        keep = []
        for i, (name, a) in enumerate(weights.items()):
            if isinstance(a, np.ndarray):
                a = np.ascontiguousarray(a, dtype=np.float32)
                dtype, on_dev, shape = BPD_F32, 0, a.shape
            else:
                a = a.contiguous()
                dtype = BPD_BF16 if a.dtype == torch.bfloat16 else BPD_F32
                assert a.dtype in (torch.bfloat16, torch.float32)
                on_dev, shape = int(a.is_cuda), tuple(a.shape)
            keep.append(a)
            t = arr[i]
            t.name = name.encode()
            t.data = _ptr(a)
            t.dtype = dtype
            t.ndim = len(shape)
            for d_, s in enumerate(shape):
                t.shape[d_] = s
            t.on_device = on_dev
        self._check(self.L.bpd_load_weights(self.h, arr, len(weights)))

    def bpd_encode(self, src_ids, src_len, max_len=None):
        src_ids, src_len, max_len = _i32(src_ids), _i32(src_len), _i32(max_len)
        B, S = src_ids.shape
        self._check(self.L.bpd_encode(self.h, _ptr(src_ids), _ptr(src_len), _ptr(max_len), B, S))
        self.B = B

    def bpd_step(self, k: int, imposed_accept=None, accepted_len=None):
        imposed_accept = _i32(imposed_accept)
        self._check(self.L.bpd_step(self.h, k, _ptr(imposed_accept), _ptr(accepted_len)))

    def bpd_step_static(self, k: int, imposed_accept=None, accepted_len=None):
        imposed_accept = _i32(imposed_accept)
        self._check(self.L.bpd_step_static(self.h, k, _ptr(imposed_accept), _ptr(accepted_len)))

    def bpd_step_tree(self, k: int, parent, accepted_len=None):
        """parent: k ints on the host (list, tuple or numpy): -1, then an earlier node for each."""
        parent = np.ascontiguousarray(parent, dtype=np.int32)
        if parent.shape != (k,):
            raise BpdError(-1, "parent: one of each node")
        self._check(self.L.bpd_step_tree(self.h, k, _ptr(parent), _ptr(accepted_len)))

    def bpd_sparse_buffer_bytes(self, block: int) -> int:
        return self.L.bpd_sparse_buffer_bytes(self.h, block)

    def bpd_set_sparse_attention(self, block: int, first: int = 1, recent: int = 2, top: int = 8):
        """block 0: all keys again.  The context keeps a buffer for each size of blocks as long as it lives: steps that have been captured under a setting have its
        address, also behind a setting of no blocks, and find the summaries that a later call of this makes."""
        torch = self.torch
        nbytes = self.bpd_sparse_buffer_bytes(block) if block else 0
        buf = self.sparse_buffers.get(block)
        if buf is None and nbytes:
            with torch.cuda.device(self.device), torch.cuda.stream(self.stream):
                buf = torch.empty(nbytes + 256, dtype=torch.uint8, device=self.device)
        self._check(self.L.bpd_set_sparse_attention(self.h, block, first, recent, top, (buf.data_ptr() + 255) // 256 * 256 if buf is not None else None, nbytes))
        if buf is not None:
            self.sparse_buffers[block] = buf

    def bpd_set_acceptance(self, distance_eps: int = 0, min_block: int = 1):
        self._check(self.L.bpd_set_acceptance(self.h, distance_eps, min_block))

    def bpd_set_top_n(self, n: int = 1):
        self._check(self.L.bpd_set_top_n(self.h, n))

    def bpd_set_two_phase(self, on: bool = True):
        self._check(self.L.bpd_set_two_phase(self.h, int(on)))

    def bpd_set_local_attention(self, query_block: int, memory_len: int):
        self._check(self.L.bpd_set_local_attention(self.h, int(query_block), int(memory_len)))

    def bpd_decode(self, k: int, schedule=None, max_steps: Optional[int] = None):
        """Returns (out_ids [B,max_out] int32 numpy, out_len [B], stats)."""
        schedule = _i32(schedule)
        if max_steps is None:
            max_steps = self.cfg.max_out_len if schedule is None else schedule.shape[0]
        out_ids = np.empty((self.B, self.cfg.max_out_len), dtype=np.int32)
        out_len = np.empty(self.B, dtype=np.int32)
        st = bpd_stats()
        self._check(self.L.bpd_decode(self.h, k, _ptr(schedule), max_steps, _ptr(out_ids), _ptr(out_len), C.byref(st)))
        return out_ids, out_len, st

    def bpd_get_state(self):
        k = self.cfg.k_max
        P = np.empty((self.B, k), dtype=np.int32)
        A = np.empty((self.B, k, k), dtype=np.int32)
        j = np.empty(self.B, dtype=np.int32)
        fin = np.empty(self.B, dtype=np.int32)
        self._check(self.L.bpd_get_state(self.h, _ptr(P), _ptr(A), _ptr(j), _ptr(fin)))
        return P, A, j, fin

    def bpd_get_output(self):
        out_ids = np.empty((self.B, self.cfg.max_out_len), dtype=np.int32)
        out_len = np.empty(self.B, dtype=np.int32)
        self._check(self.L.bpd_get_output(self.h, _ptr(out_ids), _ptr(out_len)))
        return out_ids, out_len

    def bpd_get_stats(self) -> bpd_stats:
        st = bpd_stats()
        self._check(self.L.bpd_get_stats(self.h, C.byref(st)))
        return st

    def bpd_set_proposals(self, P):
        P = _i32(P)
        assert tuple(P.shape) == (self.B, self.cfg.k_max)
        self._check(self.L.bpd_set_proposals(self.h, _ptr(P)))

    def bpd_debug_step_logits(self, k: int):
        """Returns a device float32 tensor [B, k, k, vocab]."""
        torch = self.torch
        out = torch.empty((self.B, k, k, self.cfg.vocab), dtype=torch.float32, device=self.device)
        self._check(self.L.bpd_debug_step_logits(self.h, k, out.data_ptr()))
        return out

    def bpd_profile_enable(self, phase: int):
        self._check(self.L.bpd_profile_enable(self.h, phase))

    def bpd_profile_read(self):
        ms, n = C.c_double(), C.c_int64()
        self._check(self.L.bpd_profile_read(self.h, C.byref(ms), C.byref(n)))
        return ms.value, n.value

    def bpd_profile_samples(self, capacity: int):
        """Returns (per-launch milliseconds [<= capacity] float32 numpy, total ms, launches)."""
        out = np.zeros(capacity, dtype=np.float32)
        ms, n = C.c_double(), C.c_int64()
        self._check(self.L.bpd_profile_samples(self.h, _ptr(out), capacity, C.byref(ms), C.byref(n)))
        return out[:min(capacity, n.value)], ms.value, n.value

    @staticmethod
    def bpd_measure_hbm_read(nbytes: int = 1 << 30, iters: int = 4) -> float:
        """GB/s of a streaming read over a fresh `nbytes` device buffer on torch's current stream."""
        import torch
        buf = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
        gbps = C.c_double()
        rc = lib().bpd_measure_hbm_read(buf.data_ptr(), nbytes, torch.cuda.current_stream().cuda_stream, iters, C.byref(gbps))
        if rc:
            raise BpdError(rc, "bpd_measure_hbm_read")
        return gbps.value

    @staticmethod
    def bpd_measure_mfma_bf16(iters: int = 20000) -> float:
        """TFLOP/s of back-to-back bf16 MFMAs on torch's current stream."""
        import torch
        buf = torch.zeros(64, dtype=torch.float32, device="cuda")
        tf = C.c_double()
        rc = lib().bpd_measure_mfma_bf16(buf.data_ptr(), torch.cuda.current_stream().cuda_stream, iters, C.byref(tf))
        if rc:
            raise BpdError(rc, "bpd_measure_mfma_bf16")
        return tf.value

    # -- operators on caches of the caller's (no context; torch's current stream of the tensors' device)
    @staticmethod
    def bpd_op_error() -> str:
        return lib().bpd_op_error().decode()

    @staticmethod
    def bpd_cache_bytes(cache) -> int:
        return lib().bpd_cache_bytes(_PACK_CACHE.pack(*_cache(cache)[0]))

    @staticmethod
    def bpd_summaries_bytes(cache, block: int) -> int:
        return lib().bpd_summaries_bytes(_PACK_CACHE.pack(*_cache(cache, 0)[0]), block)

    @staticmethod
    def bpd_attention_workspace_bytes(cache, B: int, T: int, n_heads: int, block: int = 0) -> int:
        c, k, _ = _cache(cache, 0)
        with lib() and _torch.cuda.device(k.device):
            return lib().bpd_attention_workspace_bytes(_PACK_CACHE.pack(*c), B, T, n_heads, block)

    @staticmethod
    def bpd_cache_store(cache, k, v, start, count=None):
        """Rows k, v [B, T, kv heads, head_dim] ([n_layers, B, ..] for a cache with layers) to rows start[b] .. of the cache; count[b] of them (None: T)."""
        L = lib()
        c, kc, layers = _cache(cache)
        device, shape = kc.get_device(), k.shape
        if len(shape) != 4 + layers or shape != v.shape or shape[-1] != c[6] or shape[-2] != c[5] or (layers and shape[0] != c[3]):
            raise _bad("k, v: [B, T, kv heads, head_dim], behind the layers if the cache has any")
        if k.get_device() != device or v.get_device() != device:
            raise _bad("k, v and the cache are on different devices")
        b, t = shape[layers], shape[layers + 1]
        _call(device, L.bpd_cache_store, _PACK_CACHE.pack(*c), _rows(k, layers), _rows(v, layers), _int(device, (b,), "start", start), _int(device, (b,), "count", count), b, t)

    @staticmethod
    def bpd_tree_attention(cache, q, length, parent=None, layer: int = 0, scale: Optional[float] = None, out=None, workspace=None):
        """q [B, T, heads, head_dim], length [B], parent [B, T] or None (a chain).  Returns out (of q's dtype, unless given; scale None: head_dim ** -0.5)."""
        device, c, args, keep, ws, n, out = _attention(cache, layer, q, length, parent, scale, out, workspace, 0)
        _call(device, _lib.bpd_tree_attention, *args, ws, n)
        return out

    @staticmethod
    def bpd_sparse_attention(cache, q, length, summaries, block: int, first: int, recent: int, top: int, parent=None, added=None, layer: int = 0,
                             scale: Optional[float] = None, out=None, chosen=None, workspace=None):
        """As bpd_tree_attention, over chosen blocks; summaries: binding.new_summaries(), one per layer; added [B]: rows committed since the call before with them, None: all
        (the first call).  Returns (out, chosen [B, kv heads, T, words] int32)."""
        if block not in (32, 64, 128):
            raise _bad("block: 32, 64 or 128 rows")
        device, c, args, keep, ws, n, out = _attention(cache, layer, q, length, parent, scale, out, workspace, block)
        _, _, dtype, _, most, kv, d, cap = c
        b, t, nb = args[5], args[6], cap // block
        if (summaries.numel() != most * kv * ((nb + 63) // 64) * 128 * d or _dtype_of(summaries) != dtype or not summaries.is_contiguous() or summaries.get_device() != device):
            raise _bad("summaries: as binding.new_summaries makes them")
        shape = (b, kv, t, (nb + 31) // 32)
        if chosen is None:
            chosen = _torch.empty(shape, dtype=_torch.int32, device=q.device)
        blocks = _PACK_BLOCKS.pack(block, first, recent, top, summaries.data_ptr(), _int(device, (b,), "added", added) or 0, _int(device, shape, "chosen", chosen))
        _call(device, _lib.bpd_sparse_attention, *args, blocks, ws, n)
        return out, chosen

    @staticmethod
    def bpd_tree_accept(parent, token, expect, best, length, cache=None, room=None, eos_id: int = -1, out=None):
        """parent, token, best [B, T], expect, length, room [B].  Returns (path [B, T], accepted [B], next [B], new_length [B]), or writes them to `out`."""
        L = lib()
        shape, device = parent.shape, parent.get_device()
        if len(shape) != 2:
            raise _bad("parent: [B, T]")
        b, t = shape
        one = (b,)
        if out is None:
            out = (_torch.empty_like(parent), _torch.empty_like(length), _torch.empty_like(length), _torch.empty_like(length))
        path, accepted, following, new_length = out
        c = None
        if cache is not None:
            c, k, _ = _cache(cache)
            if k.get_device() != device:
                raise _bad("parent and the cache are on different devices")
            c = _PACK_CACHE.pack(*c)
        _call(device, L.bpd_tree_accept, _int(device, shape, "parent", parent), _int(device, shape, "token", token), _int(device, one, "expect", expect), _int(device, shape, "best", best),
              _int(device, one, "length", length), _int(device, one, "room", room), eos_id, b, t, _int(device, shape, "path", path), _int(device, one, "accepted", accepted),
              _int(device, one, "next", following), _int(device, one, "new_length", new_length), c)
        return out
