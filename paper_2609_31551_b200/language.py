"""Binding of include/eas_language.h: the attention operators of the language model that the Encode stage feeds (argument
marshalling only; PyTorch provides device memory and streams).

Tensors keep the shapes a model has them in: queries [tokens, n_heads, head_dim], keys and values [tokens, n_kv_heads, head_dim], bf16 or
fp16, each token's heads contiguous and the tokens any multiple of 8 elements apart (views of one packed projection, for instance).
`stream` defaults to the current one of the tensors' device; what a call allocates, it allocates on that stream."""
from __future__ import annotations
import contextlib
import ctypes as C
import struct
import numpy as np
import torch

from . import binding as B

LANGUAGE_SYMBOLS = [
    "eas_prompt_attention_workspace_bytes", "eas_prompt_attention", "eas_cache_create", "eas_cache_destroy", "eas_cache_store", "eas_cache_load",
    "eas_cache_attention_workspace_bytes", "eas_cache_attention", "eas_cache_chunk_workspace_bytes", "eas_cache_chunk_attention",
    "eas_rotary_create", "eas_rotary_destroy", "eas_rotary_apply", "eas_cache_append",
]
STATUS_CACHE_RANGE = 3          # EAS_DEVICE_CACHE_RANGE
_DTYPES = {torch.bfloat16: 0, torch.float16: 1}


class PromptInputs(C.Structure):
    _fields_ = [("q", C.c_void_p), ("k", C.c_void_p), ("v", C.c_void_p), ("out", C.c_void_p),
                ("ld_q", C.c_int64), ("ld_k", C.c_int64), ("ld_v", C.c_int64), ("ld_out", C.c_int64),
                ("dtype", C.c_int32), ("n_heads", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32),
                ("scale", C.c_float), ("n_seqs", C.c_int32), ("cu_q", C.c_void_p), ("cu_k", C.c_void_p)]


class CacheDesc(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("k_scale", C.c_void_p), ("v_scale", C.c_void_p),
                ("n_blocks", C.c_int32), ("block_size", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32)]


class CacheSeqs(C.Structure):
    _fields_ = [("n_seqs", C.c_int32), ("block_table", C.c_void_p), ("max_blocks", C.c_int32), ("ld_table", C.c_int64),
                ("cu_seqlens", C.c_void_p), ("start", C.c_void_p), ("seq_lens", C.c_void_p)]


class RotaryDesc(C.Structure):
    _fields_ = [("head_dim", C.c_int32), ("rotary_dim", C.c_int32), ("pairing", C.c_int32), ("n_axes", C.c_int32), ("inv_freq", C.c_void_p),
                ("axis", C.c_void_p), ("scale", C.c_float)]


class RotaryInputs(C.Structure):
    _fields_ = [("q", C.c_void_p), ("k", C.c_void_p), ("out_q", C.c_void_p), ("out_k", C.c_void_p),
                ("ld_q", C.c_int64), ("ld_k", C.c_int64), ("ld_out_q", C.c_int64), ("ld_out_k", C.c_int64),
                ("positions", C.c_void_p), ("ld_positions", C.c_int64),
                ("n_rows", C.c_int32), ("n_heads", C.c_int32), ("n_kv_heads", C.c_int32), ("dtype", C.c_int32), ("inverse", C.c_int32)]


# The records of a call as bytes: making a ctypes structure takes 2.5 us (a prompt's) and 0.9, packing it 0.6 and 0.3
_prompt_record = struct.Struct("4P4q4ifi2P").pack
_pack_seqs = struct.Struct("iPiq3P").pack
_pack_rotary = struct.Struct("4P4qPq5i4x").pack
_declared = False


def lib():
    global _declared
    l = B.load_library()
    if not _declared:
        l.eas_prompt_attention.restype = C.c_int
        l.eas_prompt_attention.argtypes = [C.c_void_p, C.c_void_p, C.c_size_t, C.c_int32, C.c_void_p, C.c_void_p]
        l.eas_prompt_attention_workspace_bytes.restype = C.c_size_t
        l.eas_prompt_attention_workspace_bytes.argtypes = [C.c_void_p]
        l.eas_cache_create.restype = C.c_int
        l.eas_cache_create.argtypes = [C.POINTER(CacheDesc), C.POINTER(C.c_void_p)]
        l.eas_cache_destroy.restype = None
        l.eas_cache_destroy.argtypes = [C.c_void_p]
        rows = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p, C.c_int64, C.c_int32, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p]
        l.eas_cache_store.restype = C.c_int
        l.eas_cache_store.argtypes = rows
        l.eas_cache_load.restype = C.c_int
        l.eas_cache_load.argtypes = rows
        l.eas_cache_attention_workspace_bytes.restype = C.c_size_t
        l.eas_cache_attention_workspace_bytes.argtypes = [C.c_void_p, C.c_int32, C.c_int32]
        l.eas_cache_attention.restype = C.c_int
        l.eas_cache_attention.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p, C.c_int64, C.c_int32, C.c_int32,
                                          C.c_float, C.c_void_p, C.c_size_t, C.c_int32, C.c_void_p, C.c_void_p]
        l.eas_cache_chunk_workspace_bytes.restype = C.c_size_t
        l.eas_cache_chunk_workspace_bytes.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.c_int32]
        l.eas_cache_chunk_attention.restype = C.c_int
        l.eas_cache_chunk_attention.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p, C.c_int64, C.c_int32, C.c_int32, C.c_int32,
                                                C.c_int32, C.c_float, C.c_void_p, C.c_size_t, C.c_int32, C.c_void_p, C.c_void_p]
        l.eas_rotary_create.restype = C.c_int
        l.eas_rotary_create.argtypes = [C.POINTER(RotaryDesc), C.POINTER(C.c_void_p)]
        l.eas_rotary_destroy.restype = None
        l.eas_rotary_destroy.argtypes = [C.c_void_p]
        l.eas_rotary_apply.restype = C.c_int
        l.eas_rotary_apply.argtypes = [C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p]
        l.eas_cache_append.restype = C.c_int
        l.eas_cache_append.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int64, C.c_int32, C.c_void_p, C.c_void_p]
        _declared = True
    return l


def _pack_prompt(*fields):
    try:
        return _prompt_record(*fields)
    except (struct.error, OverflowError) as e:
        raise B.EasError(1, f"prompt_attention: {e}") from None


def _need(ok, text):
    if not ok:
        raise B.EasError(1, text)


# (Texts are put together only where a check fails: these run before every launch.)
def _rows(t, name, heads, head_dim, dtype, index):
    """Checks a [tokens, heads, head_dim] tensor whose tokens' heads are contiguous; returns the distance of two tokens."""
    shape, stride = t.shape, t.stride()
    if len(shape) != 3 or shape[1] != heads or shape[2] != head_dim:
        raise B.EasError(1, f"{name} has shape {tuple(shape)}, expected [tokens, {heads}, {head_dim}]")
    if t.dtype != dtype or t.get_device() != index:
        raise B.EasError(1, f"{name} is {t.dtype} on {t.device}, expected {dtype} on GPU {index}")
    if stride[2] != 1 or (stride[1] != head_dim and heads != 1):
        raise B.EasError(1, f"{name}: the heads of a token must be contiguous")
    return stride[0] if shape[0] > 1 else heads * head_dim


def _ints(t, name, n, index):
    if t.dtype != torch.int32 or t.get_device() != index or t.shape != (n,) or not t.is_contiguous():
        raise B.EasError(1, f"{name} must be a contiguous int32 tensor [{n}] on GPU {index}, not {t.dtype} {tuple(t.shape)} on {t.device}")
    return t.data_ptr()


def _elsewhere(index, stream):
    """True if a call has to run inside _on: another device is current than the tensors', or a stream is asked for."""
    return stream is not None or torch._C._cuda_getDevice() != index


@contextlib.contextmanager
def _on(index, stream):
    """The tensors' device is current inside, and so is the call's stream: allocations belong to it."""
    if stream is not None and stream.device.index != index:
        raise B.EasError(1, f"the stream is on {stream.device}, the tensors on GPU {index}")
    with torch.cuda.device(index), torch.cuda.stream(stream):
        yield


def _whole(x, name):
    if x.dtype.kind != "f" or not (np.isfinite(x) & (x == np.floor(x)) & (np.abs(x) < 2 ** 53)).all():
        raise B.EasError(1, f"{name} must be whole numbers of 32 bits")
    return x.astype(np.int64)


def _host_ints(x, name):
    if type(x) is not np.ndarray or x.dtype != np.int32 or not x.flags.c_contiguous:
        try:
            given = np.asarray(x)
        except (TypeError, ValueError, RuntimeError) as e:
            raise B.EasError(1, f"{name}: {e}") from None
        if given.dtype.kind not in "biu":
            given = _whole(given, name)
        x = np.ascontiguousarray(given, dtype=np.int32)
        if np.count_nonzero(x != given):
            raise B.EasError(1, f"{name} must be whole numbers of 32 bits")          # (the conversion cut them off)
    if x.ndim != 1 or x.size < 1:
        raise B.EasError(1, f"{name} must be a list of at least one offset")
    return x, x.__array_interface__["data"][0]


def prompt_attention(q, k, v, cu_seqlens_host, cu_seqlens_k_host=None, scale=None, out=None, sm_budget=0, stream=None, status=None, workspace=None):
    """eas_prompt_attention: causal attention of packed prompts.  q [T, n_heads, head_dim], k and v [T_k, n_kv_heads, head_dim];
    cu_seqlens_host (int32 [n + 1]) gives the queries of each sequence, cu_seqlens_k_host its keys (default: the same; a sequence's
    queries are the last tokens among its keys).  scale: 1 / sqrt(head_dim).  Returns (out, device status word); `out`, `status` (device
    int32, zeroed by the caller) and `workspace` (uint8, on a 256-byte boundary; few calls need one, and calls that may run at the same
    time one each) can be passed in so that a call allocates nothing."""
    dtype, index = q.dtype, q.get_device()
    if index < 0 or dtype not in _DTYPES or q.dim() != 3 or k.dim() != 3:
        raise B.EasError(1, f"q and k must be bf16 or fp16 tensors [tokens, heads, head_dim] on a GPU, q is {dtype} {tuple(q.shape)} on {q.device}")
    if _elsewhere(index, stream):
        with _on(index, stream):
            return prompt_attention(q, k, v, cu_seqlens_host, cu_seqlens_k_host, scale, out, sm_budget, None, status, workspace)
    T, H, hd = q.shape
    Tk, G, _ = k.shape
    ld_q, ld_k, ld_v = _rows(q, "q", H, hd, dtype, index), _rows(k, "k", G, hd, dtype, index), _rows(v, "v", G, hd, dtype, index)
    cu_q, at_q = _host_ints(cu_seqlens_host, "cu_seqlens")
    cu_k, at_k = (cu_q, at_q) if cu_seqlens_k_host is None else _host_ints(cu_seqlens_k_host, "cu_seqlens_k")
    if cu_k.size != cu_q.size or cu_q[-1] > T or cu_k[-1] > Tk or Tk != v.shape[0]:
        raise B.EasError(1, "cu_seqlens are two lists of the same length that end within the rows of q, and of k and v")
    if out is None:
        out = torch.empty_like(q, memory_format=torch.contiguous_format)
        ld_out = H * hd
    else:
        ld_out = _rows(out, "out", H, hd, dtype, index)
        if out.shape[0] < cu_q[-1]:
            raise B.EasError(1, "out has fewer rows than cu_seqlens name")
    if status is None:
        status = torch.zeros(4, dtype=torch.int32, device=q.device)
    elif status.dtype != torch.int32 or status.get_device() != index or status.numel() < 1:
        raise B.EasError(1, "status must be an int32 tensor on the GPU of q")
    pin = _pack_prompt(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), ld_q, ld_k, ld_v, ld_out, _DTYPES[dtype], H, G, hd,
                       hd ** -0.5 if scale is None else scale, cu_q.size - 1, at_q, at_k)
    l = lib()
    if workspace is None:
        need = l.eas_prompt_attention_workspace_bytes(pin)
        at, size = None, 0
        if need:
            workspace = q.new_empty(need, dtype=torch.uint8)
    elif workspace.get_device() != index or not workspace.is_contiguous():
        raise B.EasError(1, "workspace must be a contiguous tensor on the GPU of q")
    if workspace is not None:
        at, size = workspace.data_ptr(), workspace.nbytes
    rc = l.eas_prompt_attention(pin, at, size, sm_budget, torch._C._cuda_getCurrentRawStream(index), status.data_ptr())
    if rc:
        B._check(rc)
    return out, status


def prompt_attention_workspace_bytes(n_heads, n_kv_heads, head_dim, cu_seqlens_host, cu_seqlens_k_host=None):
    """eas_prompt_attention_workspace_bytes: scratch of a prompt_attention call of these shapes on the current device (0 for most)."""
    cu_q, at_q = _host_ints(cu_seqlens_host, "cu_seqlens")
    cu_k, at_k = (cu_q, at_q) if cu_seqlens_k_host is None else _host_ints(cu_seqlens_k_host, "cu_seqlens_k")
    if cu_k.size != cu_q.size:
        raise B.EasError(1, "cu_seqlens are two lists of the same length")
    pin = _pack_prompt(0, 0, 0, 0, 0, 0, 0, 0, 0, n_heads, n_kv_heads, head_dim, 1.0, cu_q.size - 1, at_q, at_k)
    return lib().eas_prompt_attention_workspace_bytes(pin)


class Rotary:
    """Rotary positions with one or several axes (eas_rotary_*).

    The first rotary_dim dimensions of a head (default: all; a multiple of 16) are pairs, dimension i and i + rotary_dim / 2, or 2 i and 2 i + 1 with
    neighbours=True.  Pair i turns by position * inv_freq[i], inv_freq being base ** (-2 i / rotary_dim) unless given (fp64, for scaled frequencies); scale
    multiplies cosines and sines.  sections: how many of the pairs, one section behind the other, turn with the first axis (time), the second
    (height), the third (width), ...; or axes: the axis of each pair.  Default: one axis.  A Rotary belongs to no device."""

    def __init__(self, head_dim, rotary_dim=None, base=10000.0, sections=None, axes=None, inv_freq=None, neighbours=False, scale=1.0):
        self.handle = None
        self.lib = lib()
        self.head_dim, self.rotary_dim = head_dim, head_dim if rotary_dim is None else rotary_dim
        pairs = max(self.rotary_dim // 2, 0)
        try:
            if inv_freq is None:
                inv_freq = float(base) ** (-np.arange(pairs, dtype=np.float64) / max(pairs, 1))
            freq = np.ascontiguousarray(inv_freq, dtype=np.float64)
            if sections is not None:
                _need(axes is None, "sections or axes, not both")
                counts = [int(n) for n in sections]
                _need(counts and min(counts) >= 0 and sum(counts) == pairs, f"sections {counts} must name {pairs} pairs")
                axes = np.repeat(np.arange(len(counts)), counts)
                self.n_axes = len(counts)
            else:
                self.n_axes = 1 if axes is None else int(max(axes)) + 1
            axis = np.zeros(pairs, dtype=np.int32) if axes is None else np.ascontiguousarray(axes, dtype=np.int32)
            desc = RotaryDesc(head_dim, self.rotary_dim, 1 if neighbours else 0, self.n_axes, freq.ctypes.data, axis.ctypes.data, scale)
        except (TypeError, ValueError, OverflowError, ZeroDivisionError) as e:
            raise B.EasError(1, f"rotary positions: {e}") from None
        _need(freq.shape == (pairs,) and axis.shape == (pairs,), f"inv_freq and axes must be lists of {pairs}")
        h = C.c_void_p()
        B._check(self.lib.eas_rotary_create(C.byref(desc), C.byref(h)))
        self.handle = h

    def close(self):
        if getattr(self, "handle", None):
            self.lib.eas_rotary_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _positions(self, positions, rows, index):
        """-> address, distance of two axes."""
        shape = positions.shape
        if (positions.dtype != torch.int32 or positions.get_device() != index or shape[-1:] != (rows,) or positions.stride(-1) != 1 and rows > 1
                or (shape[:-1] != (self.n_axes,) and not (self.n_axes == 1 and len(shape) == 1))):
            raise B.EasError(1, f"positions must be int32 [{self.n_axes}, {rows}] on GPU {index}, not {positions.dtype} {tuple(shape)} on {positions.device}")
        return positions.data_ptr(), positions.stride(0) if self.n_axes > 1 else rows

    def apply(self, q, k, positions, out=None, inverse=False, sm_budget=0, stream=None):
        """eas_rotary_apply: q [T, n_heads, head_dim] and k [T, n_kv_heads, head_dim] (one of them may be None) at positions (int32 [n_axes, T], which may be one
        row expanded, or [T] with one axis, on the device) -> rotated (q, k).  out: a pair of tensors for them, (q, k) themselves to rotate in place.  inverse takes a
        rotation back; a gradient goes through apply by inverse=True."""
        x = k if q is None else q
        if x is None:
            raise B.EasError(1, "queries, keys or both")
        dtype, index = x.dtype, x.get_device()
        if self.handle is None:
            raise B.EasError(1, "the rotary positions are closed")
        if index < 0 or dtype not in _DTYPES or x.dim() != 3 or (k is not None and k.dim() != 3):
            raise B.EasError(1, f"q and k must be bf16 or fp16 tensors [tokens, heads, head_dim] on a GPU, not {dtype} {tuple(x.shape)} on {x.device}")
        if _elsewhere(index, stream):
            with _on(index, stream):
                return self.apply(q, k, positions, out, inverse, sm_budget)
        T, hd = x.shape[0], self.head_dim
        H, ld_q, at_q, at_out_q, ld_out_q, out_q = 0, 0, 0, 0, 0, None
        G, ld_k, at_k, at_out_k, ld_out_k, out_k = 0, 0, 0, 0, 0, None
        if out is not None:
            if len(out) != 2 or (q is not None and out[0] is None) or (k is not None and out[1] is None):
                raise B.EasError(1, "out must be a pair of tensors, for q and for k")
            out_q, out_k = out
        if q is not None:
            H = q.shape[1]
            ld_q = _rows(q, "q", H, hd, dtype, index)
            if out is None:
                out_q = torch.empty_like(q, memory_format=torch.contiguous_format)
                ld_out_q = H * hd
            else:
                ld_out_q = _rows(out_q, "out of q", H, hd, dtype, index)
            at_q, at_out_q = q.data_ptr(), out_q.data_ptr()
            if out_q.shape[0] != T:
                raise B.EasError(1, "the output of q must have as many tokens as q")
        if k is not None:
            G = k.shape[1]
            ld_k = _rows(k, "k", G, hd, dtype, index)
            if out is None:
                out_k = torch.empty_like(k, memory_format=torch.contiguous_format)
                ld_out_k = G * hd
            else:
                ld_out_k = _rows(out_k, "out of k", G, hd, dtype, index)
            at_k, at_out_k = k.data_ptr(), out_k.data_ptr()
            if k.shape[0] != T or out_k.shape[0] != T:
                raise B.EasError(1, "k and its output must have as many tokens as q")
        at, ld_pos = self._positions(positions, T, index)
        rec = _pack_rotary(at_q, at_k, at_out_q, at_out_k, ld_q, ld_k, ld_out_q, ld_out_k, at, ld_pos, T, H, G, _DTYPES[dtype], 1 if inverse else 0)
        rc = self.lib.eas_rotary_apply(self.handle, rec, sm_budget, torch._C._cuda_getCurrentRawStream(index))
        if rc:
            B._check(rc)
        return out_q, out_k


class KvCache:
    """An 8-bit paged key/value cache (eas_cache_*): n_blocks blocks of block_size tokens.

    k, v: int8 [n_blocks, n_kv_heads, block_size, head_dim]; k_scale, v_scale: fp32 [n_blocks, n_kv_heads]; value = number * scale.
    They are allocated here (scales and numbers 0) unless given as `tensors`.  Sequences are rows of a block table (int32
    [n_seqs, max_blocks], on the device): token t of sequence s lies in block table[s, t // block_size].  Tables, lengths and starts are read
    on the device when a call's work runs, so captured calls can be replayed with other values in them."""

    def __init__(self, n_blocks, block_size, n_kv_heads, head_dim, device="cuda", tensors=None):
        self.handle = None
        self.lib = lib()
        shape = (n_blocks, n_kv_heads, block_size, head_dim)
        if tensors is None:
            _need(min(shape) > 0, f"bad cache shape {shape}")
            tensors = (torch.zeros(shape, dtype=torch.int8, device=device), torch.zeros(shape, dtype=torch.int8, device=device),
                       torch.zeros(shape[:2], device=device), torch.zeros(shape[:2], device=device))
        self.k, self.v, self.k_scale, self.v_scale = tensors
        self.device = self.k.device
        self._index = self.k.get_device()
        for t, name, dt, s in ((self.k, "k", torch.int8, shape), (self.v, "v", torch.int8, shape), (self.k_scale, "k_scale", torch.float32, shape[:2]),
                               (self.v_scale, "v_scale", torch.float32, shape[:2])):
            _need(t.is_cuda and t.device == self.device and t.dtype == dt and tuple(t.shape) == s and t.is_contiguous(),
                  f"{name} must be a contiguous {dt} tensor of shape {s} on one GPU")
        self.n_blocks, self.block_size, self.n_kv_heads, self.head_dim = n_blocks, block_size, n_kv_heads, head_dim
        with torch.cuda.device(self.device):
            self._status = torch.zeros(4, dtype=torch.int32, device=self.device)
            self._status_at = self._status.data_ptr()
            desc = CacheDesc(self.k.data_ptr(), self.v.data_ptr(), self.k_scale.data_ptr(), self.v_scale.data_ptr(), n_blocks, block_size, n_kv_heads, head_dim)
            h = C.c_void_p()
            B._check(self.lib.eas_cache_create(C.byref(desc), C.byref(h)))
            torch.cuda.current_stream().synchronize()        # the zeros above, whatever stream the first call is on
        self.handle = h

    def close(self):
        if getattr(self, "handle", None):
            self.lib.eas_cache_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _seqs(self, block_table, n, cu_seqlens, start, seq_lens):
        shape = block_table.shape
        if self.handle is None:
            raise B.EasError(1, "the cache is closed")
        if (len(shape) != 2 or shape[0] != n or block_table.dtype != torch.int32 or block_table.get_device() != self._index
                or (shape[1] > 1 and block_table.stride(1) != 1)):
            raise B.EasError(1, f"block_table must be an int32 tensor [{n}, max_blocks] on {self.device}")
        return _pack_seqs(n, block_table.data_ptr(), shape[1], block_table.stride(0) if n > 1 else shape[1], cu_seqlens, start, seq_lens)

    def _move(self, call, k, v, rows, cu_seqlens, start, block_table, sm_budget, new=False):
        """new: k and v are the call's own, made for it."""
        if len(start.shape) != 1:
            raise B.EasError(1, "start must be a list of one place a sequence")
        n, index, dtype = start.shape[0], self._index, k.dtype
        seqs = self._seqs(block_table, n, _ints(cu_seqlens, "cu_seqlens", n + 1, index), _ints(start, "start", n, index), 0)
        if dtype not in _DTYPES:
            raise B.EasError(1, f"k and v must be bf16 or fp16, not {dtype}")
        if new:
            ld_k = ld_v = self.n_kv_heads * self.head_dim
        else:
            if k.shape[0] != v.shape[0] or k.shape[0] < rows:
                raise B.EasError(1, "k and v must have as many rows, and at least the rows of the call")
            ld_k, ld_v = _rows(k, "k", self.n_kv_heads, self.head_dim, dtype, index), _rows(v, "v", self.n_kv_heads, self.head_dim, dtype, index)
        rc = call(self.handle, seqs, k.data_ptr(), ld_k, v.data_ptr(), ld_v, rows, _DTYPES[dtype], sm_budget,
                  torch._C._cuda_getCurrentRawStream(index), self._status_at)
        if rc:
            B._check(rc)

    def store(self, k, v, cu_seqlens, start, block_table, sm_budget=0, stream=None):
        """eas_cache_store: rows cu_seqlens[s] .. cu_seqlens[s + 1] - 1 of k and v ([rows, n_kv_heads, head_dim]) go to places start[s], ... of
        sequence s.  cu_seqlens (int32 [n + 1]), start (int32 [n]) and block_table are on the device.  A prompt starts at 0; a
        decoding step writes one row per sequence, cu_seqlens = 0, 1, 2, ..., start = the lengths so far."""
        if _elsewhere(self._index, stream):
            with _on(self._index, stream):
                return self.store(k, v, cu_seqlens, start, block_table, sm_budget)
        self._move(self.lib.eas_cache_store, k, v, k.shape[0], cu_seqlens, start, block_table, sm_budget)

    def append(self, q, k, v, cu_seqlens, start, block_table, rotary, positions=None, out=None, sm_budget=0, stream=None):
        """eas_cache_append: store() of the keys rotated by `rotary` and the values, and the queries rotated: one launch.  q [rows, n_heads, head_dim] or None, k and v
        [rows, n_kv_heads, head_dim]; cu_seqlens, start and block_table as for store().  positions: int32 [n_axes, rows] (or [rows] with one axis);
        default: a token's place in its sequence.  Returns the rotated queries: in `out` if given (q itself to rotate it in place), where rows that
        cu_seqlens does not name stay as they were."""
        index, dtype = self._index, k.dtype
        if _elsewhere(index, stream):
            with _on(index, stream):
                return self.append(q, k, v, cu_seqlens, start, block_table, rotary, positions, out, sm_budget)
        if rotary.handle is None:
            raise B.EasError(1, "the rotary positions are closed")
        if dtype not in _DTYPES or len(start.shape) != 1:
            raise B.EasError(1, f"k and v must be bf16 or fp16, not {dtype}; start a list of one place a sequence")
        n, rows, G, hd = start.shape[0], k.shape[0], self.n_kv_heads, self.head_dim
        seqs = self._seqs(block_table, n, _ints(cu_seqlens, "cu_seqlens", n + 1, index), _ints(start, "start", n, index), 0)
        ld_k, ld_v = _rows(k, "k", G, hd, dtype, index), _rows(v, "v", G, hd, dtype, index)
        H, at_q, at_out, ld_q, ld_out = 0, 0, 0, 0, 0
        if q is not None:
            if q.dim() != 3:
                raise B.EasError(1, f"q must be [rows, n_heads, head_dim], not {tuple(q.shape)}")
            H = q.shape[1]
            ld_q = _rows(q, "q", H, hd, dtype, index)
            if out is None:
                out = torch.empty_like(q, memory_format=torch.contiguous_format)
                ld_out = H * hd
            else:
                ld_out = _rows(out, "out", H, hd, dtype, index)
            at_q, at_out = q.data_ptr(), out.data_ptr()
            if q.shape[0] != rows or out.shape[0] != rows:
                raise B.EasError(1, "q and its output must have as many rows as k")
        if v.shape[0] != rows:
            raise B.EasError(1, "k and v must have as many rows")
        at_pos, ld_pos = (0, 0) if positions is None else rotary._positions(positions, rows, index)
        rec = _pack_rotary(at_q, k.data_ptr(), at_out, 0, ld_q, ld_k, ld_out, 0, at_pos, ld_pos, rows, H, G, _DTYPES[dtype], 0)
        rc = self.lib.eas_cache_append(self.handle, seqs, rotary.handle, rec, v.data_ptr(), ld_v, sm_budget, torch._C._cuda_getCurrentRawStream(index),
                                       self._status_at)
        if rc:
            B._check(rc)
        return out

    def load(self, cu_seqlens, start, block_table, n_rows, dtype=torch.bfloat16, out=None, sm_budget=0, stream=None):
        """eas_cache_load: the values of the same places -> (k, v), [n_rows, n_kv_heads, head_dim].  Rows that cu_seqlens does not name are
        left as they were (`out`, a pair of tensors of at least n_rows rows, whose type counts) or are not set."""
        if _elsewhere(self._index, stream):
            with _on(self._index, stream):
                return self.load(cu_seqlens, start, block_table, n_rows, dtype, out, sm_budget)
        new = out is None
        if n_rows < 0:
            raise B.EasError(1, f"n_rows {n_rows}")
        if new:
            shape = (n_rows, self.n_kv_heads, self.head_dim)
            out = self.k.new_empty(shape, dtype=dtype), self.k.new_empty(shape, dtype=dtype)
        self._move(self.lib.eas_cache_load, out[0], out[1], n_rows, cu_seqlens, start, block_table, sm_budget, new)
        return out

    def attention_workspace_bytes(self, n_seqs, n_heads):
        """eas_cache_attention_workspace_bytes: scratch of an attention call."""
        return self.lib.eas_cache_attention_workspace_bytes(self.handle, n_seqs, n_heads)

    def attention(self, q, seq_lens, block_table, scale=None, out=None, workspace=None, sm_budget=0, stream=None):
        """eas_cache_attention: q [n_seqs, n_heads, head_dim], one token a sequence, attends to places 0 .. seq_lens[s] - 1 (the token's own key
        and value among them, stored before).  workspace: a uint8 tensor of attention_workspace_bytes(), on a 256-byte boundary;
        calls that may run at the same time need one each (default: allocated by the call)."""
        index, dtype = self._index, q.dtype
        if _elsewhere(index, stream):
            with _on(index, stream):
                return self.attention(q, seq_lens, block_table, scale, out, workspace, sm_budget)
        if q.dim() != 3 or dtype not in _DTYPES:
            raise B.EasError(1, f"q must be bf16 or fp16 [n_seqs, n_heads, head_dim], not {dtype} {tuple(q.shape)}")
        n, H, hd = q.shape
        ld_q = _rows(q, "q", H, self.head_dim, dtype, index)
        seqs = self._seqs(block_table, n, 0, 0, _ints(seq_lens, "seq_lens", n, index))
        if out is None:
            out = torch.empty_like(q, memory_format=torch.contiguous_format)
            ld_out = H * hd
        else:
            ld_out = _rows(out, "out", H, hd, dtype, index)
            if out.shape[0] < n:
                raise B.EasError(1, "out has fewer rows than q")
        if workspace is None:
            size = self.attention_workspace_bytes(n, H)
            workspace = q.new_empty(size, dtype=torch.uint8)
        elif workspace.get_device() != index or not workspace.is_contiguous():
            raise B.EasError(1, "workspace must be a contiguous tensor on the cache's GPU")
        else:
            size = workspace.nbytes
        rc = self.lib.eas_cache_attention(self.handle, seqs, q.data_ptr(), ld_q, out.data_ptr(), ld_out, H, _DTYPES[dtype],
                                          hd ** -0.5 if scale is None else scale, workspace.data_ptr(), size, sm_budget,
                                          torch._C._cuda_getCurrentRawStream(index), self._status_at)
        if rc:
            B._check(rc)
        return out

    def chunk_workspace_bytes(self, n_seqs, n_rows, max_new, n_heads):
        """eas_cache_chunk_workspace_bytes: scratch of a chunk_attention call."""
        return self.lib.eas_cache_chunk_workspace_bytes(self.handle, n_seqs, n_rows, max_new, n_heads)

    def chunk_attention(self, q, cu_seqlens, seq_lens, block_table, max_new=None, scale=None, out=None, workspace=None, sm_budget=0, stream=None):
        """eas_cache_chunk_attention: rows cu_seqlens[s] .. cu_seqlens[s + 1] - 1 of q [rows, n_heads, head_dim] are the last tokens among places
        0 .. seq_lens[s] - 1 of sequence s (stored before); each sees the places up to its own.  max_new: the most new tokens of a sequence, which
        chooses the kernels: the exact number is the fastest (default: any number); a captured call can be replayed for other cu_seqlens and seq_lens within it.  Rows that cu_seqlens does not name are
        left as they were (`out`, which overlaps no input) or are not set.  A sequence's last bits may depend on max_new, on the table's width and on the other sequences.
        workspace: a uint8 tensor of chunk_workspace_bytes(), on a 256-byte boundary; calls that may run at the same time need one each (default: allocated by the call)."""
        index, dtype = self._index, q.dtype
        if _elsewhere(index, stream):
            with _on(index, stream):
                return self.chunk_attention(q, cu_seqlens, seq_lens, block_table, max_new, scale, out, workspace, sm_budget)
        if q.dim() != 3 or dtype not in _DTYPES or len(seq_lens.shape) != 1:
            raise B.EasError(1, f"q must be bf16 or fp16 [rows, n_heads, head_dim], not {dtype} {tuple(q.shape)}; seq_lens a list of one length a sequence")
        rows, H, hd = q.shape
        n = seq_lens.shape[0]
        ld_q = _rows(q, "q", H, self.head_dim, dtype, index)
        seqs = self._seqs(block_table, n, _ints(cu_seqlens, "cu_seqlens", n + 1, index), 0, _ints(seq_lens, "seq_lens", n, index))
        if max_new is None:
            max_new = rows
        if out is None:
            out = torch.empty_like(q, memory_format=torch.contiguous_format)
            ld_out = H * hd
        else:
            ld_out = _rows(out, "out", H, hd, dtype, index)
            if out.shape[0] < rows:
                raise B.EasError(1, "out has fewer rows than q")
        if workspace is None:
            size = self.chunk_workspace_bytes(n, rows, max_new, H)
            workspace = q.new_empty(size, dtype=torch.uint8)
        elif workspace.get_device() != index or not workspace.is_contiguous():
            raise B.EasError(1, "workspace must be a contiguous tensor on the cache's GPU")
        else:
            size = workspace.nbytes
        rc = self.lib.eas_cache_chunk_attention(self.handle, seqs, q.data_ptr(), ld_q, out.data_ptr(), ld_out, rows, max_new, H, _DTYPES[dtype],
                                                hd ** -0.5 if scale is None else scale, workspace.data_ptr(), size, sm_budget,
                                                torch._C._cuda_getCurrentRawStream(index), self._status_at)
        if rc:
            B._check(rc)
        return out

    def check(self, stream=None):
        """Waits for the stream, then reads and clears the status word of this cache's calls; raises if one of them found a block or place
        outside the cache (EAS_ERR_DEVICE_CHECK) or gave up waiting (EAS_ERR_DEVICE_TIMEOUT)."""
        with torch.cuda.device(self.device):
            st = torch.cuda.current_stream() if stream is None else stream
            st.synchronize()
            with torch.cuda.stream(st):
                word = int(self._status[0])
                if word:
                    self._status.zero_()
                    st.synchronize()
        if word == STATUS_CACHE_RANGE:
            raise B.EasError(7, "a block number, start or length points outside the cache")
        if word:
            raise B.EasError(5, "a device-side wait expired")
