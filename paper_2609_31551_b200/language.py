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
    "eas_cache_attention_workspace_bytes", "eas_cache_attention",
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


# The records of a call as bytes: making a ctypes structure takes 2.5 us (a prompt's) and 0.9, packing it 0.6 and 0.3
_prompt_record = struct.Struct("4P4q4ifi2P").pack
_pack_seqs = struct.Struct("iPiq3P").pack
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
