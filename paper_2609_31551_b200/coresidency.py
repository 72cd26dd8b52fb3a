"""Co-residency of the Encode stage with a "local prefill" neighbour on one GPU (Section 3.4).

The paper gives the encoder a share of the SMs and the co-located prefill worker the rest, and picks the share from a
table so that encoding is slowed by at most 20 %.  Here the share is the `sm_budget` argument of every call: the
encoder's persistent kernels launch `sm_budget` CTAs (each fills an SM: its shared-memory request excludes a second
one), and a neighbour that launches `sm_total - sm_budget` CTAs of the same kind fits beside it, so the two never
queue behind one another for SMs.  What they still share is L2 and HBM.  This module measures that remaining
interference: encode latency at budget N alone, then with a stream of large GEMMs (the synthetic prefill: a
compute-bound bf16 matrix product, like the projections of a language-model prefill step) running on the other
SMs, and the neighbour's own slow-down.

    python -m paper_2609_31551_b200.coresidency --config c1 --micro-batch 8

`--neighbour` chooses what else a language model's workers would run there: `prompt`, the causal attention of a prefill batch (compute-bound
like the matrix products, with bursts of K and V from L2), `token`, the attention of a decoding step over 8-bit caches (bound by HBM, which no
partition of the SMs divides), or `chunk`, the attention of a worker that does both: chunks of prompts and drafts of a few tokens over the same caches.

The neighbour's kernels never wait for the encoder's or the reverse: they are independent launches on two streams."""
from __future__ import annotations
import argparse
import json
import os
import sys

import numpy as np
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import eas_synth as S  # noqa: E402
from . import binding as B  # noqa: E402


def _check_word(status):
    word = int(status[0])
    if word:
        raise RuntimeError(f"the neighbour's kernels raised status {word}")


class PrefillNeighbour:
    """A stream of out = A W^T products (M x N x K, bf16) on `sm_budget` SMs of its own stream."""

    def __init__(self, m: int = 4096, n: int = 8192, k: int = 8192):
        g = torch.Generator(device="cuda").manual_seed(7)
        self.a = (torch.randn(m, k, device="cuda", generator=g) * 0.05).bfloat16()
        self.w = (torch.randn(n, k, device="cuda", generator=g) * 0.05).bfloat16()
        self.bias = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
        self.out = torch.empty(m, n, dtype=torch.bfloat16, device="cuda")
        self.status = torch.zeros(4, dtype=torch.int32, device="cuda")
        self.flops = 2.0 * m * n * k
        self.stream = torch.cuda.Stream()

    def enqueue(self, count: int, sm_budget: int):
        for _ in range(count):
            B.kernel_gemm(self.a, self.w, self.bias, sm_budget=sm_budget, stream=self.stream, out=self.out, status=self.status)

    def check(self):
        _check_word(self.status)


class PromptNeighbour:
    """Prefill attention: a batch of prompts (32 query heads, 8 key/value heads of 128), causal, packed."""

    def __init__(self, lens=(4096, 2048, 1024, 1024)):
        from . import language as L
        self._call = L.prompt_attention
        g = torch.Generator(device="cuda").manual_seed(7)
        self.cu = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
        qkv = torch.randn(int(self.cu[-1]), 48, 128, device="cuda", generator=g).bfloat16()
        self.q, self.k, self.v = qkv[:, :32], qkv[:, 32:40], qkv[:, 40:]
        self.out = torch.empty_like(self.q, memory_format=torch.contiguous_format)
        self.status = torch.zeros(4, dtype=torch.int32, device="cuda")
        self.flops = sum(2.0 * n * (n + 1) for n in lens) * 32 * 128
        self.stream = torch.cuda.Stream()

    def enqueue(self, count: int, sm_budget: int):
        for _ in range(count):
            self._call(self.q, self.k, self.v, self.cu, out=self.out, status=self.status, sm_budget=sm_budget, stream=self.stream)

    def check(self):
        _check_word(self.status)


class TokenNeighbour:
    """Decode attention: one token of each of `n` sequences (32 query heads, 8 key/value heads of 128) over its 8-bit cache."""

    def __init__(self, n: int = 64, tokens: int = 4096, block: int = 64):
        self._fill(n, tokens, block)
        self.q = torch.randn(n, 32, 128, device="cuda").bfloat16()
        self.out = torch.empty_like(self.q)
        self.workspace = torch.empty(self.cache.attention_workspace_bytes(n, 32), dtype=torch.uint8, device="cuda")
        self.flops = 4.0 * 32 * 128 * n * tokens
        torch.cuda.synchronize()

    def _fill(self, n, tokens, block):
        from . import language as L
        blocks = tokens // block
        self.cache = L.KvCache(n * blocks, block, 8, 128)
        self.cache.k.random_(-127, 128)
        self.cache.v.random_(-127, 128)
        self.cache.k_scale.fill_(0.03)
        self.cache.v_scale.fill_(0.03)
        self.lens = torch.full((n,), tokens, dtype=torch.int32, device="cuda")
        self.table = torch.randperm(n * blocks, device="cuda").to(torch.int32).view(n, blocks)
        self.stream = torch.cuda.Stream()

    def enqueue(self, count: int, sm_budget: int):
        for _ in range(count):
            self.cache.attention(self.q, self.lens, self.table, out=self.out, workspace=self.workspace, sm_budget=sm_budget, stream=self.stream)

    def check(self):
        self.cache.check()


class ChunkNeighbour(TokenNeighbour):
    """Chunk attention: `chunk` new tokens of the first sequence and four of each other one, over the same caches."""

    def __init__(self, n: int = 32, tokens: int = 4096, block: int = 64, chunk: int = 1024):
        self._fill(n, tokens, block)
        new = [chunk] + [4] * (n - 1)
        self.cu = torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32, device="cuda")
        self.max_new = chunk
        self.q = torch.randn(sum(new), 32, 128, device="cuda").bfloat16()
        self.out = torch.empty_like(self.q)
        self.workspace = torch.empty(self.cache.chunk_workspace_bytes(n, sum(new), chunk, 32), dtype=torch.uint8, device="cuda")
        self.flops = 4.0 * 32 * 128 * sum(m * (tokens - m) + m * (m + 1) / 2 for m in new)
        torch.cuda.synchronize()

    def enqueue(self, count: int, sm_budget: int):
        for _ in range(count):
            self.cache.chunk_attention(self.q, self.cu, self.lens, self.table, max_new=self.max_new, out=self.out, workspace=self.workspace, sm_budget=sm_budget,
                                       stream=self.stream)


NEIGHBOURS = {"gemm": PrefillNeighbour, "prompt": PromptNeighbour, "token": TokenNeighbour, "chunk": ChunkNeighbour}


def _encode_ms(enc, batch, sm_budget, reps, stream):
    data, shapes, offsets, cu, cu_dev, out, ws = batch
    e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    e0.record(stream)
    for _ in range(reps):
        enc.encode_microbatch(data, shapes, offsets, cu, cu_seqlens_dev=cu_dev, sm_budget=sm_budget, out=out, workspace=ws,
                              stream=stream)
    e1.record(stream)
    return e0, e1


def measure(config: str, micro_batch: int, levels=(0.3, 0.5, 0.7), reps: int = 5, neighbour_shape=(4096, 8192, 8192),
            partition: str = "grid", neighbour: str = "gemm"):
    """-> list of dicts, one per SM level: encode latency alone / beside the neighbour, and the neighbour's rate.

    partition = "grid": both sides bound their SM use by their grid sizes (`sm_budget`) on ordinary streams.
    partition = "green": eas_sm_partition splits the SMs into two driver-enforced sets (green contexts) and each side
    runs on its set's stream; the level is rounded up to the driver's granularity.
    neighbour: one of NEIGHBOURS; neighbour_shape is the matrix product's."""
    cfg = S.get_config(config)
    enc = B.Encoder(cfg, B.weights_to_device(S.make_weights(cfg)))
    shapes = S.draw_item_shapes(cfg, micro_batch, 3000 + micro_batch)
    items = S.make_items(cfg, shapes, 2000 + micro_batch)
    data, offsets = B.pack_items(items)
    cu = np.concatenate([[0], np.cumsum([S.tokens_per_item(cfg, s) for s in shapes])]).astype(np.int32)
    cu_dev = torch.from_numpy(cu).cuda()
    out = torch.empty((enc.out_rows(cu), cfg["d_out"]), dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(enc.workspace_bytes(int(cu[-1]), len(shapes)) + 1024, dtype=torch.uint8, device="cuda")
    batch = (data, shapes, offsets, cu, cu_dev, out, ws)
    sm_total = torch.cuda.get_device_properties(0).multi_processor_count
    nb = PrefillNeighbour(*neighbour_shape) if neighbour == "gemm" else NEIGHBOURS[neighbour]()
    enc_stream = torch.cuda.Stream()
    torch.cuda.synchronize()

    def encode_alone(budget, stream=None):
        stream = stream or enc_stream
        best = float("inf")
        for _ in range(3):              # the first passes also bring the clocks up after an idle stretch: keep the best
            e0, e1 = _encode_ms(enc, batch, budget, reps, stream)
            torch.cuda.synchronize()
            best = min(best, e0.elapsed_time(e1) / reps)
        return best

    def neighbour_alone(budget, count):
        nb.enqueue(2, budget)
        e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        e0.record(nb.stream)
        nb.enqueue(count, budget)
        e1.record(nb.stream)
        torch.cuda.synchronize()
        return e0.elapsed_time(e1) / count

    rows = []
    exclusive = encode_alone(0)
    plain_streams = (enc_stream, nb.stream)
    for f in levels:
        n_enc = max(2, int(sm_total * f) // 2 * 2)
        n_nb = sm_total - n_enc
        part = None
        if partition == "green":
            part = B.SmPartition(n_enc)
            n_enc, n_nb = part.sm_count(0), part.sm_count(1)
            enc_stream, nb.stream = part.stream(0), part.stream(1)
        alone = encode_alone(n_enc, enc_stream)
        nb_ms = neighbour_alone(n_nb, 4)
        # enough neighbour launches to cover the encoder's timed region with margin on both sides
        count = int(np.ceil((reps + 2) * alone / nb_ms)) + 4
        n0, n1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        n0.record(nb.stream)
        nb.enqueue(count, n_nb)
        n1.record(nb.stream)
        enc_stream.wait_event(n0)                                            # start beside the neighbour's first product
        _encode_ms(enc, batch, n_enc, 1, enc_stream)
        e0, e1 = _encode_ms(enc, batch, n_enc, reps, enc_stream)
        torch.cuda.synchronize()
        enc.status(enc_stream)
        nb.check()
        beside = e0.elapsed_time(e1) / reps
        nb_beside = n0.elapsed_time(n1) / count
        if part is not None:
            enc_stream, nb.stream = plain_streams
            part.close()
        rows.append({"partition": partition, "neighbour": neighbour, "sm_encode": n_enc, "sm_neighbour": n_nb, "encode_ms_exclusive": exclusive, "encode_ms_alone": alone,
                     "encode_ms_beside_neighbour": beside, "inflation": beside / alone,
                     "vs_exclusive": beside / exclusive,
                     "neighbour_tflops_alone": nb.flops / (nb_ms * 1e-3) / 1e12,
                     "neighbour_tflops_beside_encoder": nb.flops / (nb_beside * 1e-3) / 1e12})
    return rows


def main():
    ap = argparse.ArgumentParser()
    ap.add_argument("--config", default="c1")
    ap.add_argument("--micro-batch", type=int, default=8)
    ap.add_argument("--levels", default="0.3,0.5,0.7")
    ap.add_argument("--partition", default="grid", choices=("grid", "green"))
    ap.add_argument("--neighbour", default="gemm", choices=tuple(NEIGHBOURS))
    a = ap.parse_args()
    for r in measure(a.config, a.micro_batch, tuple(float(x) for x in a.levels.split(",")), partition=a.partition, neighbour=a.neighbour):
        print(json.dumps(r))


if __name__ == "__main__":
    main()
