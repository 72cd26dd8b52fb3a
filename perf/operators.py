"""What the language-model operators are timed on: the attention of a prompt, the 8-bit key/value cache (written, read back) and
the attention of single tokens over it, each through its public entry point.

A case is one call of one operator.  Fields:

  op            "prompt": causal attention of packed prompts; "store", "load": keys and values into the cache and back out of it;
                "token": one new token per sequence attends to its cache
  heads, kv_heads, head_dim     query heads, key/value heads, width of a head
  dtype         "bf16" or "fp16": queries, keys, values and outputs
  lens          new tokens per sequence (prompt, store, load), or how many sequences draw theirs from low..high
  before        tokens that came before them: further keys in front of the prompt's own, or tokens that the cache holds already
  block         tokens of a cache block
  size_seed     seed of the drawn lengths

Rows of queries, keys and values lie in one packed [tokens, (heads + 2 kv_heads) * head_dim] matrix, as a projection leaves them."""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


def _case(name, op, lens, heads, kv_heads, head_dim, *, dtype="bf16", before=0, block=0, size_seed=0, low=0, high=0):
    c = {"op": op, "heads": heads, "kv_heads": kv_heads, "head_dim": head_dim, "dtype": dtype, "lens": lens, "low": low, "high": high,
         "before": before, "block": block, "size_seed": size_seed}
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # a spoken command's transcript, nothing else on the GPU: the smallest prompt
        _case("prompt-1-short", "prompt", "39", 16, 4, 64),
        # a prefill batch: questions around images (576 or 196 embeddings each), a speech clip (1500), text alone, one token
        _case("prompt-8-media", "prompt", "617,213,1563,1,1193,88,640,305", 32, 8, 128),
        # the embeddings of a 64-frame clip twice over and the question about them: the largest call
        _case("prompt-1-long", "prompt", "16411", 32, 8, 128),
        # a chunk of a long prompt whose first part is in the cache already; heads in groups of five
        _case("prompt-1-chunk", "prompt", "512", 40, 8, 128, dtype="fp16", before=11801),
        # the keys and values of a prefill batch on their way into the cache
        _case("store-6-prompts", "store", "617,2213,1563,1,1193,640", 32, 8, 128, block=64),
        # one decoding step of 64 answers: each writes one token into a block that has others already
        _case("store-64-tokens", "store", 64, 32, 8, 128, block=16, low=1, high=1, before=900, size_seed=64),
        # two long prefixes read back for the next chunk of their prompts
        _case("load-2-prefixes", "load", "11801,8192", 32, 8, 128, block=64),
        # short prefixes of many requests, small blocks
        _case("load-16-short", "load", 16, 16, 16, 64, dtype="fp16", block=16, low=5, high=700, size_seed=16),
        # one answer being written, nothing else on the GPU: the smallest decoding step
        _case("token-1", "token", "713", 32, 8, 128, block=16),
        # an ordinary decoding step: 48 answers of all ages
        _case("token-48-ragged", "token", 48, 32, 8, 128, block=64, low=1, high=8192, size_seed=48),
        # answers about long clips: eight caches of tens of thousands of tokens
        _case("token-8-long", "token", 8, 64, 8, 128, block=128, low=24000, high=65536, size_seed=8),
        # a small model with a head of its own for every query head
        _case("token-128-small", "token", 128, 16, 16, 64, dtype="fp16", block=32, low=500, high=3500, size_seed=128),
    ]


def _log_uniform(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    most = 0.9 * max(_cost(c) for c in listed())
    op = rng.choice(["prompt", "prompt", "store", "load", "token", "token"])
    while True:
        kv, group = rng.choice([1, 2, 4, 8, 8, 16]), rng.choice([1, 2, 3, 4, 4, 5, 7, 8, 12])
        hd, dtype = rng.choice([64, 128, 128]), rng.choice(["bf16", "bf16", "fp16"])
        block, seed = rng.choice([16, 32, 64, 128]), rng.randrange(1 << 20)
        if kv * group > 64:
            continue
        if op == "prompt":
            n = _log_uniform(rng, 1, 24)
            high = _log_uniform(rng, 1, 12000)
            before = _log_uniform(rng, 1, 16000) if rng.random() < 0.3 else 0
            c = _case("", op, n, kv * group, kv, hd, dtype=dtype, low=max(1, high // 20), high=high, before=before, size_seed=seed)
        elif op == "token":
            high = _log_uniform(rng, 1, 65536)
            c = _case("", op, _log_uniform(rng, 1, 192), kv * group, kv, hd, dtype=dtype, block=block, low=max(1, high // 20), high=high, size_seed=seed)
        else:
            single = op == "store" and rng.random() < 0.4
            high = 1 if single else _log_uniform(rng, 1, 12000)
            c = _case("", op, _log_uniform(rng, 1, 256 if single else 24), kv * group, kv, hd, dtype=dtype, block=block, low=max(1, high // 20), high=high,
                      before=_log_uniform(rng, 1, 3000) if single or rng.random() < 0.3 else 0, size_seed=seed)
        w = work(c)
        if _cost(c) <= most and w["bytes"] <= 2e9:
            return c


def _cost(case):
    w = work(case)
    return max(w["bytes"] / 6.5e12, w["flops"] / 1.6e15)


def _lens(case):
    """-> new tokens and earlier tokens of each sequence.  Where `before` belongs to several drawn sequences it is their most."""
    if isinstance(case["lens"], str):
        lens = [int(x) for x in case["lens"].split(",")]
        return lens, [case["before"]] * len(lens)
    rng = random.Random(case["size_seed"])
    lens = [_log_uniform(rng, case["low"], case["high"]) for _ in range(case["lens"])]
    return lens, [rng.randint(0, case["before"]) for _ in lens]


def _offsets(lens):
    o = [0]
    for n in lens:
        o.append(o[-1] + n)
    return o


def _rows(tokens, case, gen):
    """Queries, keys and values of `tokens` tokens, views of one packed matrix.  Heads differ in how sharply they attend, and some
    channels of the keys stand out, as they do in trained models."""
    H, G, D = case["heads"], case["kv_heads"], case["head_dim"]
    x = torch.empty((tokens, (H + 2 * G) * D), dtype=torch.float32, device="cuda").normal_(generator=gen)
    x[:, :H * D].view(tokens, H, D).mul_(torch.empty((H, 1), device="cuda").uniform_(0.5, 3.0, generator=gen))
    loud = torch.empty((G, D), device="cuda").uniform_(generator=gen)
    x[:, H * D:(H + G) * D].view(tokens, G, D).add_(torch.where(loud > 0.95, 4.0, 0.0))
    x = x.to(DTYPES[case["dtype"]])
    return (x[:, :H * D].view(tokens, H, D), x[:, H * D:(H + G) * D].view(tokens, G, D), x[:, (H + G) * D:].view(tokens, G, D))


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    lens, before = _lens(case)
    H, G, D = case["heads"], case["kv_heads"], case["head_dim"]
    st = {"op": case["op"], "lens": lens, "before": before, "dtype": DTYPES[case["dtype"]], "block": case["block"], "scale": D ** -0.5}
    if case["op"] == "prompt":
        total = [a + b for a, b in zip(lens, before)]
        st["cu_q"], st["cu_k"] = _offsets(lens), _offsets(total)
        if any(before):
            q, k, v = _rows(st["cu_q"][-1], case, gen)[0], *_rows(st["cu_k"][-1], case, gen)[1:]
        else:
            q, k, v = _rows(st["cu_q"][-1], case, gen)
        st.update(q=q, k=k, v=v)
        if own:
            import numpy as np
            st["cu_q_host"] = np.asarray(st["cu_q"], dtype=np.int32)
            st["cu_k_host"] = np.asarray(st["cu_k"], dtype=np.int32)
            st["status"] = torch.zeros(4, dtype=torch.int32, device="cuda")
        return st
    # the cache: every sequence's blocks lie anywhere in it, and as many again belong to others
    bs = case["block"]
    held = [a + b for a, b in zip(lens, before)]
    need = [(n + bs - 1) // bs for n in held]
    n_blocks = sum(need) + sum(need) // 4 + 4
    perm = torch.randperm(n_blocks, device="cuda", generator=gen).to(torch.int32)
    table = torch.zeros((len(lens), max(need)), dtype=torch.int32)
    at = 0
    host = perm.cpu()
    for i, n in enumerate(need):
        table[i, :n] = host[at:at + n]
        at += n
    shape = (n_blocks, G, bs, D)
    cache = {}
    for name in ("k", "v"):
        x = torch.empty(shape, dtype=torch.int8, device="cuda")
        step = max(1, (1 << 26) // (G * bs * D))
        for a in range(0, n_blocks, step):
            x[a:a + step] = torch.empty(x[a:a + step].shape, device="cuda").normal_(0.0, 36.0, generator=gen).clamp_(-127, 127).round_()
        cache[name] = x
        cache[name + "_scale"] = torch.empty((n_blocks, G), device="cuda").uniform_(0.02, 0.04, generator=gen)
    st.update(cache=cache, table=table.cuda(), held=held, cu=torch.tensor(_offsets(lens), dtype=torch.int32, device="cuda"),
              start=torch.tensor(before, dtype=torch.int32, device="cuda"), cu_held=torch.tensor(_offsets(held), dtype=torch.int32, device="cuda"),
              zero=torch.zeros(len(lens), dtype=torch.int32, device="cuda"), seq_lens=torch.tensor(held, dtype=torch.int32, device="cuda"))
    if case["op"] == "store":
        _, st["k"], st["v"] = _rows(sum(lens), case, gen)
    if case["op"] == "token":
        st["q"] = _rows(len(lens), case, gen)[0]
    if own:
        import paper_2609_31551_b200 as P
        st["handle"] = P.KvCache(n_blocks, bs, G, D, tensors=(cache["k"], cache["v"], cache["k_scale"], cache["v_scale"]))
    return st


# ------------------------------------------------------------------------------------------------ one pass
def run(st):
    if st["op"] == "prompt":
        if own:
            import paper_2609_31551_b200 as P
            return P.prompt_attention(st["q"], st["k"], st["v"], st["cu_q_host"], st["cu_k_host"], status=st["status"])[0]
        return _plain_prompt(st)
    if own:
        c = st["handle"]
        if st["op"] == "store":
            # a decoding step or a prefill batch writes; all that the sequences hold then is read back, so that the values can be seen
            c.store(st["k"], st["v"], st["cu"], st["start"], st["table"])
            k, v = c.load(st["cu_held"], st["zero"], st["table"], sum(st["held"]), dtype=st["dtype"])
            return [k, v, c.k_scale, c.v_scale]
        if st["op"] == "load":
            return list(c.load(st["cu"], st["start"], st["table"], sum(st["lens"]), dtype=st["dtype"]))
        return c.attention(st["q"], st["seq_lens"], st["table"])
    c = st["cache"]
    if st["op"] == "store":
        for i in range(len(st["lens"])):
            for name in ("k", "v"):
                _plain_store(st, i, c[name], c[name + "_scale"], st[name])
        zeros = [0] * len(st["held"])
        return [_plain_load(st, c["k"], c["k_scale"], st["held"], zeros), _plain_load(st, c["v"], c["v_scale"], st["held"], zeros), c["k_scale"], c["v_scale"]]
    if st["op"] == "load":
        return [_plain_load(st, c["k"], c["k_scale"], st["lens"], st["before"]), _plain_load(st, c["v"], c["v_scale"], st["lens"], st["before"])]
    return _plain_token(st)


def _plain_prompt(st):
    """softmax(scale q k^T) v over the keys up to the query's own place, the queries being the last of their sequence."""
    q, k, v = st["q"], st["k"], st["v"]
    G, group = k.shape[1], q.shape[1] // k.shape[1]
    out = torch.empty((q.shape[0], q.shape[1], q.shape[2]), dtype=q.dtype, device=q.device)
    for s, n in enumerate(st["lens"]):
        a, b0, b1 = st["cu_q"][s], st["cu_k"][s], st["cu_k"][s + 1]
        ahead = (b1 - b0) - n
        rows = max(1, min(n, (1 << 27) // (group * (b1 - b0))))
        for h in range(G):
            kh, vh = k[b0:b1, h].float(), v[b0:b1, h].float()
            for r in range(0, n, rows):
                m = min(rows, n - r)
                qh = q[a + r:a + r + m, h * group:(h + 1) * group].float()                       # [m, group, D]
                x = (qh.reshape(m * group, -1) @ kh.T).mul_(st["scale"]).view(m, group, -1)
                last = torch.arange(r, r + m, device=q.device) + ahead
                x.masked_fill_(torch.arange(b1 - b0, device=q.device)[None, None, :] > last[:, None, None], -math.inf)
                x = (x - x.amax(-1, keepdim=True)).exp_()
                x /= x.sum(-1, keepdim=True)
                out[a + r:a + r + m, h * group:(h + 1) * group] = (x.view(m * group, -1) @ vh).view(m, group, -1).to(q.dtype)
    return out


def _plain_store(st, i, cache, scales, x):
    """Rounds sequence i's new rows to 8 bits, one scale for each block and head: the largest magnitude of the block over 127, never less
    than the scale that the tokens already in the block had; those are rounded again where it grew."""
    bs, n, before = st["block"], st["lens"][i], st["before"][i]
    a = sum(st["lens"][:i])
    new = x[a:a + n].double()                                                                    # [n, G, D]
    first, last, inside = before // bs, (before + n - 1) // bs, before % bs
    ids = st["table"][i, first:last + 1].long()
    G, D = new.shape[1], new.shape[2]
    pad = torch.zeros(((last - first + 1) * bs, G, D), dtype=torch.float64, device=x.device)
    pad[inside:inside + n] = new
    pad = pad.view(-1, bs, G, D).permute(0, 2, 1, 3)                                             # [blocks, G, bs, D]
    s = (pad.abs().amax((2, 3)) / 127.0).float().clamp_min(2.0 ** -100)
    if inside:
        was = scales[ids[0]].clone()
        s[0] = torch.maximum(s[0], was)
        kept = cache[ids[0], :, :inside].double() * was.double()[:, None, None] / s[0].double()[:, None, None]
        cache[ids[0], :, :inside] = kept.round().clamp_(-127, 127).to(torch.int8)
    val = (pad / s.double()[:, :, None, None]).round().clamp_(-127, 127).to(torch.int8)
    place = torch.arange(before, before + n, device=x.device)
    cache[st["table"][i].long()[place // bs], :, place % bs] = val.permute(0, 2, 1, 3).reshape(-1, G, D)[inside:inside + n]
    scales[ids] = s


def _plain_load(st, cache, scales, lens, starts):
    parts = []
    for i, (n, b) in enumerate(zip(lens, starts)):
        place = torch.arange(b, b + n, device=cache.device)
        ids = st["table"][i].long()[place // st["block"]]
        parts.append((cache[ids, :, place % st["block"]].float() * scales[ids][:, :, None]).to(st["dtype"]))
    return torch.cat(parts)


def _plain_token(st):
    q, c, bs = st["q"], st["cache"], st["block"]
    G = c["k"].shape[1]
    group = q.shape[1] // G
    out = torch.empty((q.shape[0], q.shape[1], q.shape[2]), dtype=q.dtype, device=q.device)
    for i, n in enumerate(st["held"]):
        ids = st["table"][i, :(n + bs - 1) // bs].long()

        def rows(name):                                                                          # [G, n, D]
            x = c[name][ids].float() * c[name + "_scale"][ids][:, :, None, None]
            return x.permute(1, 0, 2, 3).reshape(G, -1, q.shape[2])[:, :n]
        x = torch.matmul(q[i].view(G, group, -1).float(), rows("k").transpose(1, 2)) * st["scale"]
        x = (x - x.amax(-1, keepdim=True)).exp_()
        x /= x.sum(-1, keepdim=True)
        out[i] = torch.matmul(x, rows("v")).reshape(q.shape[1], -1).to(q.dtype)
    return out


# ------------------------------------------------------------------------------------------------ what a pass cannot do without
def work(case):
    lens, before = _lens(case)
    H, G, D = case["heads"], case["kv_heads"], case["head_dim"]
    if case["op"] == "prompt":
        # query i of n, with b keys in front of the prompt, sees b + i + 1 keys: 2 D for its scores and 2 D for the values, each
        seen = sum(n * b + n * (n + 1) // 2 for n, b in zip(lens, before))
        return {"bytes": 2 * D * (2 * H * sum(lens) + 2 * G * (sum(lens) + sum(before))), "flops": 4 * H * D * seen}
    bs = case["block"]
    held = [a + b for a, b in zip(lens, before)]

    def blocks(ls, starts):
        return sum((b + n - 1) // bs - b // bs + 1 for n, b in zip(ls, starts))
    if case["op"] == "token":
        return {"bytes": 2 * H * D * 2 * len(lens) + 2 * G * (D * sum(held) + 4 * blocks(held, [0] * len(held))), "flops": 4 * H * D * sum(held)}
    back = 2 * G * (3 * D * sum(held) + 4 * blocks(held, [0] * len(held)))     # 1 byte read, 2 written
    if case["op"] == "load":
        back = 2 * G * (3 * D * sum(lens) + 4 * blocks(lens, before))
        return {"bytes": back, "flops": 2 * G * D * sum(lens)}
    kept = sum(b % bs for b in before)                                          # tokens in front of the new ones in their block: read, written
    return {"bytes": back + 2 * G * (3 * D * sum(lens) + 2 * D * kept + 4 * blocks(lens, before)), "flops": 4 * G * D * (sum(lens) + sum(held))}


# ------------------------------------------------------------------------------------------------ the definitions in 64 bits
def exact(case, seed):
    global own
    was, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = was
    dbl = torch.float64
    if case["op"] == "prompt":
        H, G = case["heads"], case["kv_heads"]
        out = torch.zeros(st["q"].shape, dtype=dbl, device="cuda")
        for s, n in enumerate(st["lens"]):
            n_k = n + st["before"][s]
            q0, k0 = st["cu_q"][s], st["cu_k"][s]
            for h in range(H):
                kk, vv = st["k"][k0:k0 + n_k, h * G // H].to(dbl), st["v"][k0:k0 + n_k, h * G // H].to(dbl)
                step = max(1, (1 << 27) // n_k)
                for r in range(0, n, step):
                    e = min(n, r + step)
                    seen = e + n_k - n                                          # the last of these rows sees this many keys
                    z = st["q"][q0 + r:q0 + e, h].to(dbl) @ kk[:seen].T / math.sqrt(case["head_dim"])
                    z = torch.where(torch.ones_like(z, dtype=torch.bool).tril(seen - (e - r)), z, -math.inf)
                    out[q0 + r:q0 + e, h] = torch.softmax(z, dim=1) @ vv[:seen]
        return out
    c, bs, G = st["cache"], st["block"], case["kv_heads"]
    values = {name: c[name].to(dbl) * c[name + "_scale"].to(dbl)[:, :, None, None] for name in ("k", "v")} if case["op"] != "store" else None

    def gather(x, i, n):                                                        # [n, G, D]
        return torch.cat([x[int(b)].transpose(0, 1) for b in st["table"][i, :(n + bs - 1) // bs].tolist()])[:n]
    if case["op"] == "load":
        return [torch.cat([gather(values[name], i, b + n)[b:] for i, (n, b) in enumerate(zip(st["lens"], st["before"]))]) for name in ("k", "v")]
    if case["op"] == "token":
        out = []
        for i, n in enumerate(st["held"]):
            kk, vv = (gather(values[name], i, n).repeat_interleave(case["heads"] // G, dim=1) for name in ("k", "v"))
            p = torch.softmax(torch.einsum("hd,nhd->hn", st["q"][i].to(dbl), kk) / math.sqrt(case["head_dim"]), dim=1)
            out.append(torch.einsum("hn,nhd->hd", p, vv))
        return torch.stack(out)
    res = []
    for name in ("k", "v"):
        scales = c[name + "_scale"].clone()
        parts, a = [], 0
        for i, (n, b) in enumerate(zip(st["lens"], st["before"])):
            row = st["table"][i].tolist()
            x = st[name][a:a + n].to(dbl)
            a += n
            done = 0
            for j in range((b + n + bs - 1) // bs):
                lo, hi = j * bs, min((j + 1) * bs, b + n)
                old = c[name][row[j], :, :max(0, min(hi, b) - lo)].to(dbl)      # [G, tokens, D] as 8-bit numbers
                s_old = scales[row[j]].to(dbl)
                if hi <= b:
                    parts.append((old * s_old[:, None, None]).transpose(0, 1))
                    continue
                fresh = x[done:done + hi - max(lo, b)].transpose(0, 1)
                done += hi - max(lo, b)
                s = (fresh.abs().amax((1, 2)) / 127).clamp(min=2.0 ** -100).to(torch.float32)
                if old.shape[1]:
                    s = torch.maximum(s, scales[row[j]])
                scales[row[j]] = s
                s = s.to(dbl)[:, None, None]
                ints = torch.cat([torch.round(old * s_old[:, None, None] / s), torch.round(fresh / s)], dim=1)
                parts.append((ints.clamp(-127, 127) * s).transpose(0, 1))
        res.append((torch.cat(parts), scales.to(dbl)))
    return [res[0][0], res[1][0], res[0][1], res[1][1]]
