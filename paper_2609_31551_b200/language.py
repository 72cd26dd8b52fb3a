"""Binding of include/eas_language.h: the attention operators of the language model that the Encode stage feeds (argument
marshalling only; PyTorch provides device memory and streams).

Tensors keep the shapes a model has them in: queries [tokens, n_heads, head_dim], keys and values [tokens, n_kv_heads, head_dim], bf16 or
fp16, each token's heads contiguous and the tokens any multiple of 8 elements apart (views of one packed projection, for instance).
`stream` defaults to the current one of the tensors' device; what a call allocates, it allocates on that stream."""
from __future__ import annotations
import contextlib
import ctypes as C
import numpy as np
import torch

from . import binding as B

LANGUAGE_SYMBOLS = [
    "eas_prompt_attention", "eas_cache_create", "eas_cache_destroy", "eas_cache_store", "eas_cache_load",
    "eas_cache_attention_workspace_bytes", "eas_cache_attention",
]
STATUS_CACHE_RANGE = 3          # EAS_DEVICE_CACHE_RANGE
_DTYPES = {torch.bfloat16: 0, torch.float16: 1}
_I32P = C.POINTER(C.c_int32)


class PromptInputs(C.Structure):
    _fields_ = [("q", C.c_void_p), ("k", C.c_void_p), ("v", C.c_void_p), ("out", C.c_void_p),
                ("ld_q", C.c_int64), ("ld_k", C.c_int64), ("ld_v", C.c_int64), ("ld_out", C.c_int64),
                ("dtype", C.c_int32), ("n_heads", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32),
                ("scale", C.c_float), ("n_seqs", C.c_int32), ("cu_q", _I32P), ("cu_k", _I32P)]


class CacheDesc(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("k_scale", C.c_void_p), ("v_scale", C.c_void_p),
                ("n_blocks", C.c_int32), ("block_size", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32)]


class CacheSeqs(C.Structure):
    _fields_ = [("n_seqs", C.c_int32), ("block_table", C.c_void_p), ("max_blocks", C.c_int32), ("ld_table", C.c_int64),
                ("cu_seqlens", C.c_void_p), ("start", C.c_void_p), ("seq_lens", C.c_void_p)]


_declared = False


def lib():
    global _declared
    l = B.load_library()
    if not _declared:
        l.eas_prompt_attention.restype = C.c_int
        l.eas_prompt_attention.argtypes = [C.POINTER(PromptInputs), C.c_int32, C.c_void_p, C.c_void_p]
        l.eas_cache_create.restype = C.c_int
        l.eas_cache_create.argtypes = [C.POINTER(CacheDesc), C.POINTER(C.c_void_p)]
        l.eas_cache_destroy.restype = None
        l.eas_cache_destroy.argtypes = [C.c_void_p]
        rows = [C.c_void_p, C.POINTER(CacheSeqs), C.c_void_p, C.c_int64, C.c_void_p, C.c_int64, C.c_int32, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p]
        l.eas_cache_store.restype = C.c_int
        l.eas_cache_store.argtypes = rows
        l.eas_cache_load.restype = C.c_int
        l.eas_cache_load.argtypes = rows
        l.eas_cache_attention_workspace_bytes.restype = C.c_size_t
        l.eas_cache_attention_workspace_bytes.argtypes = [C.c_void_p, C.c_int32, C.c_int32]
        l.eas_cache_attention.restype = C.c_int
        l.eas_cache_attention.argtypes = [C.c_void_p, C.POINTER(CacheSeqs), C.c_void_p, C.c_int64, C.c_void_p, C.c_int64, C.c_int32, C.c_int32,
                                          C.c_float, C.c_void_p, C.c_size_t, C.c_int32, C.c_void_p, C.c_void_p]
        _declared = True
    return l


def _need(ok, text):
    if not ok:
        raise B.EasError(1, text)


def _rows(t, name, heads=None, head_dim=None, dtype=None, device=None):
    """Checks a [tokens, heads, head_dim] tensor whose tokens' heads are contiguous; returns the distance of two tokens."""
    _need(t.dim() == 3, f"{name} must be [tokens, heads, head_dim]")
    _need(dtype is None or t.dtype == dtype, f"{name} is {t.dtype}, expected {dtype}")
    _need(device is None or t.device == device, f"{name} is on {t.device}, expected {device}")
    _need((heads is None or t.shape[1] == heads) and (head_dim is None or t.shape[2] == head_dim), f"{name} has shape {tuple(t.shape)}")
    _need(t.stride(2) == 1 and (t.shape[1] == 1 or t.stride(1) == t.shape[2]), f"{name}: the heads of a token must be contiguous")
    return t.stride(0) if t.shape[0] > 1 else t.shape[1] * t.shape[2]


def _ints(t, name, shape, device):
    _need(t.dtype == torch.int32 and t.device == device and t.is_contiguous() and tuple(t.shape) == shape,
          f"{name} must be a contiguous int32 tensor of shape {shape} on {device}")
    return t.data_ptr()


@contextlib.contextmanager
def _on(device, stream):
    """The tensors' device is current inside, and allocations belong to the call's stream."""
    with torch.cuda.device(device):
        if stream is None or stream == torch.cuda.current_stream(device):
            yield torch.cuda.current_stream(device).cuda_stream
        else:
            with torch.cuda.stream(stream):
                yield stream.cuda_stream


def prompt_attention(q, k, v, cu_seqlens_host, cu_seqlens_k_host=None, scale=None, out=None, sm_budget=0, stream=None, status=None):
    """eas_prompt_attention: causal attention of packed prompts.  q [T, n_heads, head_dim], k and v [T_k, n_kv_heads, head_dim];
    cu_seqlens_host (int32 [n + 1]) gives the queries of each sequence, cu_seqlens_k_host its keys (default: the same; a sequence's
    queries are the last tokens among its keys).  scale: 1 / sqrt(head_dim).  Returns (out, device status word); `out` and
    `status` (device int32, zeroed by the caller) can be passed in so that a call allocates nothing."""
    _need(q.is_cuda and q.dtype in _DTYPES, f"q must be a bf16 or fp16 tensor on a GPU, not {q.dtype} on {q.device}")
    H, hd = q.shape[-2], q.shape[-1]
    ld_q = _rows(q, "q")
    ld_k = _rows(k, "k", head_dim=hd, dtype=q.dtype, device=q.device)
    ld_v = _rows(v, "v", heads=k.shape[1], head_dim=hd, dtype=q.dtype, device=q.device)
    cu_q = np.ascontiguousarray(cu_seqlens_host, dtype=np.int32)
    cu_k = cu_q if cu_seqlens_k_host is None else np.ascontiguousarray(cu_seqlens_k_host, dtype=np.int32)
    _need(cu_q.ndim == 1 and cu_q.size >= 1 and cu_k.shape == cu_q.shape, "cu_seqlens must be two lists of the same length")
    _need(cu_q[-1] <= q.shape[0] and cu_k[-1] <= k.shape[0] and k.shape[0] == v.shape[0], "cu_seqlens reach past the rows of q, k or v")
    with _on(q.device, stream) as s:
        if out is None:
            out = torch.empty((q.shape[0], H, hd), dtype=q.dtype, device=q.device)
        ld_out = _rows(out, "out", heads=H, head_dim=hd, dtype=q.dtype, device=q.device)
        _need(out.shape[0] >= cu_q[-1], "out has fewer rows than q")
        if status is None:
            status = torch.zeros(4, dtype=torch.int32, device=q.device)
        pin = PromptInputs(q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), ld_q, ld_k, ld_v, ld_out, _DTYPES[q.dtype], H, k.shape[1], hd,
                           hd ** -0.5 if scale is None else scale, cu_q.size - 1, cu_q.ctypes.data_as(_I32P), cu_k.ctypes.data_as(_I32P))
        B._check(lib().eas_prompt_attention(C.byref(pin), sm_budget, s, status.data_ptr()))
    return out, status


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
        for t, name, dt, s in ((self.k, "k", torch.int8, shape), (self.v, "v", torch.int8, shape), (self.k_scale, "k_scale", torch.float32, shape[:2]),
                               (self.v_scale, "v_scale", torch.float32, shape[:2])):
            _need(t.is_cuda and t.device == self.device and t.dtype == dt and tuple(t.shape) == s and t.is_contiguous(),
                  f"{name} must be a contiguous {dt} tensor of shape {s} on one GPU")
        self.n_blocks, self.block_size, self.n_kv_heads, self.head_dim = n_blocks, block_size, n_kv_heads, head_dim
        with torch.cuda.device(self.device):
            self._status = torch.zeros(4, dtype=torch.int32, device=self.device)
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

    def _seqs(self, block_table, n):
        _need(self.handle is not None, "the cache is closed")
        _need(block_table.dim() == 2 and block_table.dtype == torch.int32 and block_table.device == self.device and block_table.shape[0] == n
              and (block_table.stride(1) == 1 or block_table.shape[1] <= 1), f"block_table must be an int32 tensor [{n}, max_blocks] on {self.device}")
        return CacheSeqs(n, block_table.data_ptr(), block_table.shape[1], block_table.stride(0) if n > 1 else block_table.shape[1], None, None, None)

    def _move(self, call, k, v, cu_seqlens, start, block_table, sm_budget, s):
        n = start.shape[0]
        seqs = self._seqs(block_table, n)
        seqs.cu_seqlens = _ints(cu_seqlens, "cu_seqlens", (n + 1,), self.device)
        seqs.start = _ints(start, "start", (n,), self.device)
        ld_k = _rows(k, "k", self.n_kv_heads, self.head_dim, device=self.device)
        ld_v = _rows(v, "v", self.n_kv_heads, self.head_dim, dtype=k.dtype, device=self.device)
        _need(k.dtype in _DTYPES and k.shape[0] == v.shape[0], "k and v must be bf16 or fp16, with as many rows")
        B._check(call(self.handle, C.byref(seqs), k.data_ptr(), ld_k, v.data_ptr(), ld_v, k.shape[0], _DTYPES[k.dtype], sm_budget, s,
                      self._status.data_ptr()))

    def store(self, k, v, cu_seqlens, start, block_table, sm_budget=0, stream=None):
        """eas_cache_store: rows cu_seqlens[s] .. cu_seqlens[s + 1] - 1 of k and v ([rows, n_kv_heads, head_dim]) go to places start[s], ... of
        sequence s.  cu_seqlens (int32 [n + 1]), start (int32 [n]) and block_table are on the device.  A prompt starts at 0; a
        decoding step writes one row per sequence, cu_seqlens = 0, 1, 2, ..., start = the lengths so far."""
        with _on(self.device, stream) as s:
            self._move(self.lib.eas_cache_store, k, v, cu_seqlens, start, block_table, sm_budget, s)

    def load(self, cu_seqlens, start, block_table, n_rows, dtype=torch.bfloat16, out=None, sm_budget=0, stream=None):
        """eas_cache_load: the values of the same places -> (k, v), [n_rows, n_kv_heads, head_dim].  Rows that cu_seqlens does not name are
        left as they were (`out`, a pair of tensors) or are not set."""
        with _on(self.device, stream) as s:
            if out is None:
                out = tuple(torch.empty((n_rows, self.n_kv_heads, self.head_dim), dtype=dtype, device=self.device) for _ in range(2))
            self._move(self.lib.eas_cache_load, out[0], out[1], cu_seqlens, start, block_table, sm_budget, s)
        return out

    def attention_workspace_bytes(self, n_seqs, n_heads):
        return self.lib.eas_cache_attention_workspace_bytes(self.handle, n_seqs, n_heads)

    def attention(self, q, seq_lens, block_table, scale=None, out=None, workspace=None, sm_budget=0, stream=None):
        """eas_cache_attention: q [n_seqs, n_heads, head_dim], one token a sequence, attends to places 0 .. seq_lens[s] - 1 (the token's own key
        and value among them, stored before).  workspace: a uint8 tensor of attention_workspace_bytes(), on a 256-byte boundary;
        calls that may run at the same time need one each (default: allocated by the call)."""
        n = q.shape[0]
        _need(q.dtype in _DTYPES, f"q is {q.dtype}")
        ld_q = _rows(q, "q", head_dim=self.head_dim, device=self.device)
        seqs = self._seqs(block_table, n)
        seqs.seq_lens = _ints(seq_lens, "seq_lens", (n,), self.device)
        H = q.shape[1]
        with _on(self.device, stream) as s:
            if out is None:
                out = torch.empty((n, H, self.head_dim), dtype=q.dtype, device=self.device)
            ld_out = _rows(out, "out", H, self.head_dim, dtype=q.dtype, device=self.device)
            _need(out.shape[0] >= n, "out has fewer rows than q")
            if workspace is None:
                need = self.attention_workspace_bytes(n, H)
                workspace = torch.empty(need, dtype=torch.uint8, device=self.device)
            _need(workspace.is_cuda and workspace.device == self.device and workspace.is_contiguous(), "workspace must be a tensor on the cache's GPU")
            B._check(self.lib.eas_cache_attention(self.handle, C.byref(seqs), q.data_ptr(), ld_q, out.data_ptr(), ld_out, H, _DTYPES[q.dtype],
                                                  self.head_dim ** -0.5 if scale is None else scale, workspace.data_ptr(),
                                                  workspace.numel() * workspace.element_size(), sm_budget, s, self._status.data_ptr()))
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
