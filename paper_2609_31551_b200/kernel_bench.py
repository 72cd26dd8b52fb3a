"""Micro-benchmarks of the single-kernel entry points (CUDA events on the launching stream).

    python -m paper_2609_31551_b200.kernel_bench gemm --M 18464 --N 4096 --K 1024 --act 1
    python -m paper_2609_31551_b200.kernel_bench norm --rows 18464 --d 1024 --kind 0
    python -m paper_2609_31551_b200.kernel_bench attention --lens 577x32 --heads 16 --head-dim 64
    python -m paper_2609_31551_b200.kernel_bench prompt --lens 2048x8 --heads 32 --kv-heads 8 --head-dim 128 --before 0
    python -m paper_2609_31551_b200.kernel_bench token --lens 4096x64 --heads 32 --kv-heads 8 --head-dim 128 --block 64
    python -m paper_2609_31551_b200.kernel_bench store --lens 2048x8 --kv-heads 8 --head-dim 128 --block 64      (or load)
    python -m paper_2609_31551_b200.kernel_bench chunk --lens 4096x64 --new 4 --heads 32 --kv-heads 8 --head-dim 128 --block 64
    python -m paper_2609_31551_b200.kernel_bench append --lens 2048x8 --before 0 --heads 32 --kv-heads 8 --head-dim 128 --block 64      (or rotate)

Prints one JSON line per run: milliseconds per launch and TFLOP/s (GEMM, attention, prompt, chunk) or GB/s (norm, token, chunk, store, load, append, rotate)."""
from __future__ import annotations
import argparse
import json
import numpy as np
import torch

from . import binding as B
from . import language as L


def _time(fn, iters, warmup):
    for _ in range(warmup):
        fn()
    torch.cuda.synchronize()
    e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    e0.record()
    for _ in range(iters):
        fn()
    e1.record()
    torch.cuda.synchronize()
    return e0.elapsed_time(e1) / iters


def bench_gemm(a):
    g = torch.Generator(device="cuda").manual_seed(1)
    A = torch.randn(a.M, a.K, device="cuda", generator=g).bfloat16()
    W = (torch.randn(a.N, a.K, device="cuda", generator=g) * 0.05).bfloat16()
    b = torch.randn(a.N, device="cuda", generator=g).bfloat16()
    out = torch.empty((a.M, a.N // 2 if a.act == 2 else a.N), dtype=torch.float32 if a.fp32 else torch.bfloat16, device="cuda")
    if a.fp32:
        out.zero_()
    resid = out if a.fp32 else None
    ms = _time(lambda: B.kernel_gemm(A, W, b, act=a.act, out_fp32=a.fp32, resid=resid, sm_budget=a.sm_budget, out=out),
               a.iters, a.warmup)
    return {"kernel": "gemm", "M": a.M, "N": a.N, "K": a.K, "act": a.act, "fp32_resid": a.fp32, "sm_budget": a.sm_budget,
            "ms": ms, "tflops": 2.0 * a.M * a.N * a.K / ms / 1e9}


def bench_norm(a):
    x = torch.randn(a.rows, a.d, device="cuda")
    g = torch.ones(a.d, device="cuda").bfloat16()
    b = torch.zeros(a.d, device="cuda").bfloat16()
    ms = _time(lambda: B.kernel_norm(x, g, b, a.kind, 1e-5, sm_budget=a.sm_budget), a.iters, a.warmup)
    return {"kernel": "norm", "rows": a.rows, "d": a.d, "kind": a.kind, "sm_budget": a.sm_budget, "ms": ms,
            "gbs": a.rows * a.d * 6 / ms / 1e6}


def _lens(text):
    lens = []
    for part in text.split(","):
        if "x" in part:
            s, n = part.split("x")
            lens += [int(s)] * int(n)
        else:
            lens.append(int(part))
    return lens


def bench_prompt(a):
    lens = _lens(a.lens)
    cu_q = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    cu_k = np.concatenate([[0], np.cumsum([n + a.before for n in lens])]).astype(np.int32)
    dtype = torch.float16 if a.fp16 else torch.bfloat16
    q = torch.randn(int(cu_q[-1]), a.heads, a.head_dim, device="cuda").to(dtype)
    k, v = (torch.randn(int(cu_k[-1]), a.kv_heads, a.head_dim, device="cuda").to(dtype) for _ in range(2))
    out, status = torch.empty_like(q), torch.zeros(4, dtype=torch.int32, device="cuda")
    ms = _time(lambda: L.prompt_attention(q, k, v, cu_q, cu_k, out=out, status=status, sm_budget=a.sm_budget), a.iters, a.warmup)
    seen = sum(n * a.before + n * (n + 1) // 2 for n in lens)
    return {"kernel": "prompt", "lens": a.lens, "before": a.before, "heads": a.heads, "kv_heads": a.kv_heads, "head_dim": a.head_dim,
            "sm_budget": a.sm_budget, "ms": ms, "tflops": 4.0 * a.heads * a.head_dim * seen / ms / 1e9}


def _bench_cache(a):
    lens = _lens(a.lens)
    need = [(n + a.block - 1) // a.block for n in lens]
    cache = L.KvCache(sum(need), a.block, a.kv_heads, a.head_dim)
    for t in (cache.k, cache.v):
        t.random_(-127, 128)
    for t in (cache.k_scale, cache.v_scale):
        t.fill_(0.03)
    table, perm, at = torch.zeros(len(lens), max(need), dtype=torch.int32), torch.randperm(sum(need)).to(torch.int32), 0
    for i, n in enumerate(need):
        table[i, :n] = perm[at:at + n]
        at += n
    return lens, cache, table.cuda(), torch.float16 if a.fp16 else torch.bfloat16


def bench_token(a):
    lens, cache, table, dtype = _bench_cache(a)
    q = torch.randn(len(lens), a.heads, a.head_dim, device="cuda").to(dtype)
    held, out = torch.tensor(lens, dtype=torch.int32, device="cuda"), torch.empty_like(q)
    ws = torch.empty(cache.attention_workspace_bytes(len(lens), a.heads), dtype=torch.uint8, device="cuda")
    ms = _time(lambda: cache.attention(q, held, table, out=out, workspace=ws, sm_budget=a.sm_budget), a.iters, a.warmup)
    cache.check()
    return {"kernel": "token", "lens": a.lens, "heads": a.heads, "kv_heads": a.kv_heads, "head_dim": a.head_dim, "block": a.block,
            "sm_budget": a.sm_budget, "ms": ms, "gbs": 2.0 * a.kv_heads * a.head_dim * sum(lens) / ms / 1e6}


def bench_rows(a):
    lens, cache, table, dtype = _bench_cache(a)
    T = sum(lens)
    k, v = (torch.randn(T, a.kv_heads, a.head_dim, device="cuda").to(dtype) for _ in range(2))
    cu = torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32, device="cuda")
    start = torch.zeros(len(lens), dtype=torch.int32, device="cuda")
    if a.which == "store":
        ms = _time(lambda: cache.store(k, v, cu, start, table, sm_budget=a.sm_budget), a.iters, a.warmup)
    else:
        ms = _time(lambda: cache.load(cu, start, table, T, dtype=dtype, out=(k, v), sm_budget=a.sm_budget), a.iters, a.warmup)
    cache.check()
    return {"kernel": a.which, "lens": a.lens, "kv_heads": a.kv_heads, "head_dim": a.head_dim, "block": a.block, "sm_budget": a.sm_budget, "ms": ms,
            "gbs": 6.0 * a.kv_heads * a.head_dim * T / ms / 1e6}


def bench_chunk(a):
    """--lens: cached tokens of each sequence, the new ones among them; --new: new tokens of each."""
    lens, cache, table, dtype = _bench_cache(a)
    new = [min(a.new, n) for n in lens]
    q = torch.randn(sum(new), a.heads, a.head_dim, device="cuda").to(dtype)
    held, out = torch.tensor(lens, dtype=torch.int32, device="cuda"), torch.empty_like(q)
    cu = torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32, device="cuda")
    ws = torch.empty(cache.chunk_workspace_bytes(len(lens), sum(new), max(new), a.heads), dtype=torch.uint8, device="cuda")
    ms = _time(lambda: cache.chunk_attention(q, cu, held, table, max_new=max(new), out=out, workspace=ws, sm_budget=a.sm_budget), a.iters, a.warmup)
    cache.check()
    seen = sum(n * (h - n) + n * (n + 1) // 2 for n, h in zip(new, lens))
    return {"kernel": "chunk", "lens": a.lens, "new": a.new, "heads": a.heads, "kv_heads": a.kv_heads, "head_dim": a.head_dim, "block": a.block,
            "sm_budget": a.sm_budget, "ms": ms, "gbs": 2.0 * a.kv_heads * a.head_dim * sum(lens) / ms / 1e6, "tflops": 4.0 * a.heads * a.head_dim * seen / ms / 1e9}


def bench_rotary(a):
    """rotate: --lens tokens of queries and keys; append: the same into the cache behind --before tokens of each sequence."""
    new = _lens(a.lens)
    a.lens = ",".join(str(n + a.before) for n in new)
    held, cache, table, dtype = _bench_cache(a)
    T = sum(new)
    qkv = torch.randn(T, a.heads + 2 * a.kv_heads, a.head_dim, device="cuda").to(dtype)
    q, k, v = qkv[:, :a.heads], qkv[:, a.heads:a.heads + a.kv_heads], qkv[:, a.heads + a.kv_heads:]
    quarter = a.head_dim // 8
    rotary = L.Rotary(a.head_dim, base=1e6, sections=(2 * quarter, quarter, quarter))
    positions = torch.randint(0, 30000, (3, T), dtype=torch.int32, device="cuda")
    out = torch.empty_like(q, memory_format=torch.contiguous_format), torch.empty_like(k, memory_format=torch.contiguous_format)
    if a.which == "rotate":
        ms = _time(lambda: rotary.apply(q, k, positions, out=out, sm_budget=a.sm_budget), a.iters, a.warmup)
    else:
        cu = torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32, device="cuda")
        start = torch.full((len(new),), a.before, dtype=torch.int32, device="cuda")
        ms = _time(lambda: cache.append(q, k, v, cu, start, table, rotary, positions, out=out[0], sm_budget=a.sm_budget), a.iters, a.warmup)
        cache.check()
    width = 4.0 * (a.heads + a.kv_heads) if a.which == "rotate" else 4.0 * a.heads + 6.0 * a.kv_heads
    return {"kernel": a.which, "tokens": T, "before": a.before, "heads": a.heads, "kv_heads": a.kv_heads, "head_dim": a.head_dim, "block": a.block,
            "sm_budget": a.sm_budget, "ms": ms, "gbs": width * a.head_dim * T / ms / 1e6}


def bench_attention(a):
    lens = _lens(a.lens)
    T, d = sum(lens), a.heads * a.head_dim
    qkv = torch.randn(T, 3 * d, device="cuda").bfloat16()
    cu = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    ms = _time(lambda: B.kernel_attention(qkv, cu, a.heads, a.head_dim, sm_budget=a.sm_budget, impl=a.impl), a.iters, a.warmup)
    return {"kernel": "attention", "lens": a.lens, "heads": a.heads, "head_dim": a.head_dim, "impl": a.impl,
            "sm_budget": a.sm_budget, "ms": ms, "tflops": 4.0 * d * sum(s * s for s in lens) / ms / 1e9}


def main():
    ap = argparse.ArgumentParser()
    sub = ap.add_subparsers(dest="which", required=True)
    for name in ("gemm", "norm", "attention", "prompt", "token", "store", "load", "chunk", "rotate", "append"):
        sp = sub.add_parser(name)
        sp.add_argument("--iters", type=int, default=20)
        sp.add_argument("--warmup", type=int, default=3)
        sp.add_argument("--sm-budget", type=int, default=0)
        if name == "gemm":
            sp.add_argument("--M", type=int, default=18464); sp.add_argument("--N", type=int, default=4096)
            sp.add_argument("--K", type=int, default=1024); sp.add_argument("--act", type=int, default=0)
            sp.add_argument("--fp32", action="store_true")
        elif name == "norm":
            sp.add_argument("--rows", type=int, default=18464); sp.add_argument("--d", type=int, default=1024)
            sp.add_argument("--kind", type=int, default=0)
        elif name != "attention":
            sp.add_argument("--lens", default="4096x64" if name in ("token", "chunk") else "2048x8"); sp.add_argument("--heads", type=int, default=32)
            sp.add_argument("--kv-heads", type=int, default=8); sp.add_argument("--head-dim", type=int, default=128)
            sp.add_argument("--block", type=int, default=64); sp.add_argument("--before", type=int, default=0); sp.add_argument("--fp16", action="store_true")
            sp.add_argument("--new", type=int, default=4)
        else:
            sp.add_argument("--lens", default="577x32"); sp.add_argument("--heads", type=int, default=16)
            sp.add_argument("--head-dim", type=int, default=64); sp.add_argument("--impl", type=int, default=0)
    a = ap.parse_args()
    res = {"gemm": bench_gemm, "norm": bench_norm, "attention": bench_attention, "prompt": bench_prompt, "token": bench_token, "store": bench_rows,
           "load": bench_rows, "chunk": bench_chunk, "rotate": bench_rotary, "append": bench_rotary}[a.which](a)
    print(json.dumps(res))


if __name__ == "__main__":
    main()
