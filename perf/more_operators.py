"""What the operators between a language model's projections and its cache are timed on: rotary positions, keys and values appended to the
8-bit cache with the rotation on the way, and the attention of several new tokens a sequence over that cache, each through its public entry point.

A case is one call of one operator.  Fields:

  op            "rotate": queries and keys of packed tokens; "append": queries rotated, keys rotated and stored, values stored;
                "chunk": the new tokens of each sequence attend to its cache, themselves included
  heads, kv_heads, head_dim     query heads, key/value heads, width of a head
  dtype         "bf16" or "fp16": queries, keys, values and outputs
  lens          new tokens per sequence, or how many sequences draw theirs from low..high
  before        tokens that came before them (drawn lengths: at most)
  block         tokens of a cache block
  rotary_dim    dimensions of a head that are rotated
  sections      pairs of dimensions that turn with time, height and width ("" : one axis)
  neighbours    pairs are neighbouring dimensions (else the halves of rotary_dim)
  base          of the frequencies
  far           positions begin there
  inverse       the rotation is taken back
  size_seed     seed of the drawn lengths

Rows of queries, keys and values lie in one packed [tokens, (heads + 2 kv_heads) * head_dim] matrix, as a projection leaves them."""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


def _case(name, op, lens, heads, kv_heads, head_dim, *, dtype="bf16", before=0, block=0, rotary_dim=0, sections="", neighbours=False, base=10000.0, far=0,
          inverse=False, size_seed=0, low=0, high=0):
    c = {"op": op, "heads": heads, "kv_heads": kv_heads, "head_dim": head_dim, "dtype": dtype, "lens": lens, "low": low, "high": high, "before": before,
         "block": block, "rotary_dim": rotary_dim, "sections": sections, "neighbours": neighbours, "base": base, "far": far, "inverse": inverse, "size_seed": size_seed}
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # a prefill batch of questions around images and clips, on its way to the prompts' attention
        _case("rotate-6-media", "rotate", "617,2213,1563,1,1193,640", 32, 8, 128, rotary_dim=128, sections="16,24,24", base=1e6),
        # one decoding step of a small model, a quarter of a head rotated, neighbouring dimensions: latency
        _case("rotate-40-tokens", "rotate", 40, 16, 16, 64, dtype="fp16", rotary_dim=16, neighbours=True, low=1, high=1, before=3000, size_seed=40),
        # the embeddings of a 64-frame clip twice over, at positions far behind a long history, turned back: the largest call
        _case("rotate-1-far", "rotate", "16411", 32, 8, 128, rotary_dim=128, sections="24,20,20", base=5e6, far=700000, inverse=True),
        # the same prefill batch on its way into the cache
        _case("append-6-media", "append", "617,2213,1563,1,1193,640", 32, 8, 128, block=64, rotary_dim=128, sections="16,24,24", base=1e6),
        # one decoding step of 64 answers: each writes one token into a block that has others already
        _case("append-64-tokens", "append", 64, 32, 8, 128, block=16, rotary_dim=128, low=1, high=1, before=900, size_seed=64),
        # drafts of 1 to 6 tokens for 24 answers, heads of 64 of which half is rotated
        _case("append-24-drafts", "append", 24, 16, 4, 64, dtype="fp16", block=32, rotary_dim=32, neighbours=True, low=1, high=6, before=5000, size_seed=24),
        # a draft of four tokens of one answer, nothing else on the GPU: the smallest attention
        _case("chunk-1-draft", "chunk", "4", 16, 4, 128, before=713, block=16),
        # drafts to be verified: 48 answers of all ages
        _case("chunk-48-drafts", "chunk", 48, 32, 8, 128, before=8192, block=64, low=1, high=8, size_seed=48),
        # a chunk of a long prompt whose first part is in the cache already; heads in groups of five
        _case("chunk-1-prefix", "chunk", "512", 40, 8, 128, dtype="fp16", before=11801, block=64),
        # one prompt's chunk together with a decoding step of other sequences
        _case("chunk-24-mixed", "chunk", "1187,1,1,1,3,1,1,1,1,2,1,1,1,1,1,1,1,4,1,1,1,1,1,1", 32, 8, 128, before=6000, block=32, size_seed=3),
        # chunks of two conversations about long videos: the largest call
        _case("chunk-2-long", "chunk", "2048,2048", 32, 8, 128, before=32768, block=128, size_seed=2),
        # whole prompts of a small model straight from the cache, a head of its own for every query head
        _case("chunk-12-small", "chunk", 12, 16, 16, 64, dtype="fp16", before=0, block=32, low=40, high=1500, size_seed=12),
    ]


def _log_uniform(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    most = {op: 0.9 * max(_cost(c) for c in listed() if c["op"] == op) for op in ("rotate", "append", "chunk")}
    op = rng.choice(["rotate", "append", "append", "chunk", "chunk", "chunk"])
    while True:
        kv, group = rng.choice([1, 2, 4, 8, 8, 16]), rng.choice([1, 2, 3, 4, 4, 5, 7, 8, 12])
        hd, dtype = rng.choice([64, 128, 128]), rng.choice(["bf16", "bf16", "fp16"])
        block, seed = rng.choice([16, 32, 64, 128]), rng.randrange(1 << 20)
        if kv * group > 64:
            continue
        single = rng.random() < 0.3
        n = _log_uniform(rng, 1, 192 if single else 24)
        high = _log_uniform(rng, 1, 8 if single else 8000)
        before = _log_uniform(rng, 1, 40000) if single or rng.random() < 0.7 else 0
        rotary = {}
        if op != "chunk":
            width = rng.choice([hd, hd, hd // 2, 16, 48])
            a, b = rng.randint(1, width // 4), rng.randint(1, width // 8)
            rotary = {"rotary_dim": width, "sections": rng.choice(["", "%d,%d,%d" % (width // 2 - a - b, a, b)]), "neighbours": rng.random() < 0.3,
                      "base": rng.choice([1e4, 5e5, 1e6, 1e7]), "far": rng.choice([0, 0, 0, 1000000]), "inverse": op == "rotate" and rng.random() < 0.3}
        c = _case("", op, n, kv * group, kv, hd, dtype=dtype, before=before, block=0 if op == "rotate" else block, low=max(1, high // 20), high=high, size_seed=seed,
                  **rotary)
        if _cost(c) <= most[op] and work(c)["bytes"] <= 2e9 and sum(_lens(c)[1]) <= 2500000:
            return c


def _cost(case):
    w = work(case)
    return max(w["bytes"] / 6.5e12, w["flops"] / 1.6e15)


def _lens(case):
    """-> new tokens and earlier tokens of each sequence.  `before` is the most that a sequence has, unless there is one sequence of a given length."""
    rng = random.Random(case["size_seed"])
    if isinstance(case["lens"], str):
        lens = [int(x) for x in case["lens"].split(",")]
        if len(lens) == 1:
            return lens, [case["before"]]
    else:
        lens = [_log_uniform(rng, case["low"], case["high"]) for _ in range(case["lens"])]
    return lens, [rng.randint(case["before"] // 8, case["before"]) for _ in lens]


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


def _media_positions(lens, before, seed, far):
    """Time, height and width of packed tokens: runs of text (all three the same) and grids of image or clip embeddings between them."""
    rng = random.Random(seed)
    cols = [[], [], []]
    for n, b in zip(lens, before):
        at, left = b + far, n
        while left > 0:
            text = min(left, rng.randint(5, 200))
            for c in cols:
                c.extend(range(at, at + text))
            at, left = at + text, left - text
            t, h, w = rng.choice([1, 1, 4]), rng.randint(6, 24), rng.randint(6, 24)
            if left >= t * h * w:
                for i in range(t * h * w):
                    cols[0].append(at + i // (h * w))
                    cols[1].append(at + i // w % h)
                    cols[2].append(at + i % w)
                at, left = at + max(t, h, w), left - t * h * w
    return torch.tensor(cols, dtype=torch.int32).cuda()


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    lens, before = _lens(case)
    H, G, D = case["heads"], case["kv_heads"], case["head_dim"]
    T, cu = sum(lens), _offsets(lens)
    st = {"op": case["op"], "lens": lens, "before": before, "dtype": DTYPES[case["dtype"]], "scale": D ** -0.5, "inverse": case["inverse"],
          "pairs": case["rotary_dim"] // 2, "neighbours": case["neighbours"]}
    st["q"], st["k"], st["v"] = _rows(T, case, gen)
    st["cu"] = torch.tensor(cu, dtype=torch.int32, device="cuda")
    st["start"] = torch.tensor(before, dtype=torch.int32, device="cuda")
    if case["op"] != "chunk":
        if case["sections"]:
            counts = [int(x) for x in case["sections"].split(",")]
            st["axis"] = torch.repeat_interleave(torch.arange(3), torch.tensor(counts)).cuda()
            st["positions"] = _media_positions(lens, before, seed, case["far"])
        else:
            st["axis"] = torch.zeros(case["rotary_dim"] // 2, dtype=torch.int64, device="cuda")
            seq = torch.repeat_interleave(torch.arange(len(lens)), torch.tensor(lens))
            place = torch.arange(T) - torch.tensor(cu)[seq] + torch.tensor(before)[seq] + case["far"]
            st["positions"] = place.to(torch.int32).cuda().view(1, T)
        st["inv_freq"] = case["base"] ** (-torch.arange(0, case["rotary_dim"], 2, dtype=torch.float64, device="cuda") / case["rotary_dim"])
        if own:
            import paper_2609_31551_b200 as P
            st["rotary"] = P.Rotary(D, rotary_dim=case["rotary_dim"], base=case["base"], neighbours=case["neighbours"],
                                    sections=[int(x) for x in case["sections"].split(",")] if case["sections"] else None)
    if case["op"] == "rotate":
        return st
    # the cache: every sequence's blocks lie anywhere in it, and some belong to others
    bs = st["block"] = case["block"]
    held = [a + b for a, b in zip(lens, before)]
    need = [(n + bs - 1) // bs for n in held]
    n_blocks = sum(need) + sum(need) // 8 + 4
    perm = torch.randperm(n_blocks, device="cuda", generator=gen).to(torch.int32)
    table = torch.zeros((len(lens), max(need)), dtype=torch.int32)
    at = 0
    host = perm.cpu()
    for i, n in enumerate(need):
        table[i, :n] = host[at:at + n]
        at += n
    cache = {}
    for name in ("k", "v"):
        x = torch.empty((n_blocks, G, bs, D), dtype=torch.int8, device="cuda")
        step = max(1, (1 << 26) // (G * bs * D))
        for a in range(0, n_blocks, step):
            x[a:a + step] = torch.empty(x[a:a + step].shape, device="cuda").normal_(0.0, 36.0, generator=gen).clamp_(-127, 127).round_()
        cache[name] = x
        cache[name + "_scale"] = torch.empty((n_blocks, G), device="cuda").uniform_(0.02, 0.04, generator=gen)
    st.update(cache=cache, table=table.cuda(), held=held, seq_lens=torch.tensor(held, dtype=torch.int32, device="cuda"))
    # the blocks that an append touches, from their first tokens on
    back = [a + b % bs for a, b in zip(lens, before)]
    st.update(back=back, cu_back=torch.tensor(_offsets(back), dtype=torch.int32, device="cuda"),
              start_back=torch.tensor([b - b % bs for b in before], dtype=torch.int32, device="cuda"))
    if own:
        import paper_2609_31551_b200 as P
        st["handle"] = P.KvCache(n_blocks, bs, G, D, tensors=(cache["k"], cache["v"], cache["k_scale"], cache["v_scale"]))
    return st


# ------------------------------------------------------------------------------------------------ one pass
def run(st):
    if st["op"] == "rotate":
        if own:
            return list(st["rotary"].apply(st["q"], st["k"], st["positions"], inverse=st["inverse"]))
        return [_plain_rotate(st, st["q"]).to(st["dtype"]), _plain_rotate(st, st["k"]).to(st["dtype"])]
    if st["op"] == "append":
        if own:
            # what the touched blocks hold then is read back, so that the values can be seen
            c = st["handle"]
            q = c.append(st["q"], st["k"], st["v"], st["cu"], st["start"], st["table"], st["rotary"], st["positions"])
            k, v = c.load(st["cu_back"], st["start_back"], st["table"], sum(st["back"]), dtype=st["dtype"])
            return [q, k, v, c.k_scale, c.v_scale]
        return _plain_append(st)
    if own:
        return st["handle"].chunk_attention(st["q"], st["cu"], st["seq_lens"], st["table"], max_new=max(st["lens"]))
    return _plain_chunk(st)


def _plain_rotate(st, x):
    """Each pair of dimensions (a, b) of a head turned by its angle; fp32, not rounded."""
    angle = st["positions"].double()[st["axis"]].T * st["inv_freq"] * (-1.0 if st["inverse"] else 1.0)      # [T, pairs]
    angle = angle[:, None, :]
    cos, sin = angle.cos().float(), angle.sin().float()
    n = st["pairs"]
    y = x.float()
    if st["neighbours"]:
        a, b = y[..., 0:2 * n:2], y[..., 1:2 * n:2]
        return torch.cat([torch.stack([a * cos - b * sin, b * cos + a * sin], dim=-1).flatten(-2), y[..., 2 * n:]], dim=-1)
    a, b = y[..., :n], y[..., n:2 * n]
    return torch.cat([a * cos - b * sin, b * cos + a * sin, y[..., 2 * n:]], dim=-1)


def _row_places(st, lens, cu, start):
    """Of each packed row: its block in the cache, and its place in that block."""
    seq = torch.repeat_interleave(torch.arange(len(lens), device="cuda"), (cu[1:] - cu[:-1]).long(), output_size=sum(lens))
    place = torch.arange(sum(lens), device="cuda") - cu[seq] + start[seq]
    return st["table"][seq, place // st["block"]].long(), place % st["block"]


def _plain_append(st):
    """Rounds the rotated keys and the values to 8 bits, one scale for each block and head: the largest magnitude of the block's new tokens over
    127, never less than the scale that the tokens already in the block had; those are rounded again where it grew."""
    c, bs = st["cache"], st["block"]
    ids, place = _row_places(st, st["lens"], st["cu"], st["start"])
    inside = (st["start"] % bs).long()                                                             # tokens that a sequence's first block holds
    first = st["table"].gather(1, (st["start"] // bs).long()[:, None])[:, 0].long()
    out = []
    for name, x in (("k", _plain_rotate(st, st["k"])), ("v", st["v"].float())):
        numbers, scales = c[name], c[name + "_scale"]
        largest = torch.zeros(scales.shape, device="cuda").scatter_reduce_(0, ids[:, None].expand(-1, scales.shape[1]), x.abs().amax(-1), "amax")
        touched = torch.zeros(scales.shape[0], dtype=torch.bool, device="cuda").index_fill_(0, ids, True)
        s = (largest.double() / 127.0).float().clamp_min(2.0 ** -100)
        was = scales[first]
        s[first] = torch.where((inside > 0)[:, None], torch.maximum(s[first], was), s[first])
        again = (numbers[first].double() * (was.double() / s[first].double())[:, :, None, None]).round().clamp(-127, 127).to(torch.int8)
        kept = torch.arange(bs, device="cuda")[None, :] < inside[:, None]                          # [sequences, bs]
        numbers[first] = torch.where(kept[:, None, :, None], again, numbers[first])
        numbers[ids, :, place] = (x.double() / s[ids].double()[:, :, None]).round().clamp(-127, 127).to(torch.int8)
        scales.copy_(torch.where(touched[:, None], s, scales))
        ids_back, place_back = _row_places(st, st["back"], st["cu_back"], st["start_back"])
        out.append((numbers[ids_back, :, place_back].float() * scales[ids_back][:, :, None]).to(st["dtype"]))
    return [_plain_rotate(st, st["q"]).to(st["dtype"]), out[0], out[1], c["k_scale"], c["v_scale"]]


def _plain_chunk(st):
    """softmax(scale q k^T) v over the places up to the token's own, the new tokens being the last of their sequence."""
    q, c, bs = st["q"], st["cache"], st["block"]
    G, D = c["k"].shape[1], q.shape[2]
    group = q.shape[1] // G
    out = torch.empty((q.shape[0], q.shape[1], D), dtype=q.dtype, device=q.device)
    a = 0
    for i, n in enumerate(st["lens"]):
        held, ahead = st["held"][i], st["before"][i]
        ids = st["table"][i, :(held + bs - 1) // bs].long()
        k, v = ((c[name][ids].float() * c[name + "_scale"][ids][:, :, None, None]).permute(1, 0, 2, 3).reshape(G, -1, D)[:, :held] for name in ("k", "v"))
        rows = max(1, min(n, (1 << 29) // (q.shape[1] * held)))
        for r in range(0, n, rows):
            m = min(rows, n - r)
            qr = q[a + r:a + r + m].float().view(m, G, group, D).permute(1, 0, 2, 3).reshape(G, m * group, D)
            x = torch.matmul(qr, k.transpose(1, 2)).mul_(st["scale"]).view(G, m, group, held)
            last = torch.arange(r + ahead, r + ahead + m, device=q.device)
            x.masked_fill_(torch.arange(held, device=q.device) > last[None, :, None, None], -math.inf)
            x = (x - x.amax(-1, keepdim=True)).exp_()
            x /= x.sum(-1, keepdim=True)
            y = torch.matmul(x.view(G, m * group, held), v).view(G, m, group, D)
            out[a + r:a + r + m] = y.permute(1, 0, 2, 3).reshape(m, -1, D).to(q.dtype)
        a += n
    return out


# ------------------------------------------------------------------------------------------------ what a pass cannot do without
def work(case):
    lens, before = _lens(case)
    H, G, D, T = case["heads"], case["kv_heads"], case["head_dim"], sum(lens)
    axes = 3 if case["sections"] else 1
    if case["op"] == "rotate":
        return {"bytes": 4 * (H + G) * D * T + 4 * axes * T, "flops": 3 * (H + G) * case["rotary_dim"] * T}
    bs = case["block"]
    if case["op"] == "chunk":
        held = [a + b for a, b in zip(lens, before)]
        # new token i of n, with b tokens in front of them, sees b + i + 1: 2 D for its scores and 2 D for the values, each
        seen = sum(n * b + n * (n + 1) // 2 for n, b in zip(lens, before))
        blocks = sum((n + bs - 1) // bs for n in held)
        return {"bytes": 4 * H * D * T + 2 * G * (D * sum(held) + 4 * blocks), "flops": 4 * H * D * seen}
    kept = sum(b % bs for b in before)                                          # tokens in front of the new ones in their block: read, written
    blocks = sum((b + n - 1) // bs - b // bs + 1 for n, b in zip(lens, before))
    back = 2 * G * (3 * D * (T + kept) + 4 * blocks)                            # 1 byte read, 2 written
    return {"bytes": back + 4 * H * D * T + 2 * G * (3 * D * T + 2 * D * kept + 4 * blocks) + 4 * axes * T,
            "flops": 3 * (H + G) * case["rotary_dim"] * T + 4 * G * D * (2 * T + kept)}


# ------------------------------------------------------------------------------------------------ the definitions in 64 bits
def exact(case, seed):
    global own
    was, own = own, False
    try:
        st = prepare(case, seed)
    finally:
        own = was
    dbl = torch.float64

    def turned(x):                                                              # as complex numbers
        x = x.to(dbl)
        w = case["rotary_dim"]
        i = torch.arange(w // 2, device="cuda")
        lo, hi = (2 * i, 2 * i + 1) if case["neighbours"] else (i, i + w // 2)
        pos = st["positions"].to(dbl)[st["axis"]]                               # [pairs, T]
        rate = torch.tensor([case["base"] ** (-2.0 * j / w) for j in range(w // 2)], dtype=dbl, device="cuda")
        turn = torch.polar(torch.ones_like(pos), pos * rate[:, None]).T[:, None]
        z = torch.complex(x[..., lo], x[..., hi]) * (turn.conj() if case["inverse"] else turn)
        y = x.clone()
        y[..., lo], y[..., hi] = z.real, z.imag
        return y
    if case["op"] == "rotate":
        return [turned(st["q"]), turned(st["k"])]
    c, bs, G = st["cache"], st["block"], case["kv_heads"]
    if case["op"] == "append":
        res = []
        for name, x in (("k", turned(st["k"])), ("v", st["v"].to(dbl))):
            scales, parts, a = c[name + "_scale"].clone(), [], 0
            table = st["table"].tolist()
            for row, n, b in zip(table, st["lens"], st["before"]):
                fresh, a = x[a:a + n], a + n
                for j in range(b // bs, (b + n - 1) // bs + 1):
                    lo, hi = max(j * bs, b), min((j + 1) * bs, b + n)
                    new = fresh[lo - b:hi - b].transpose(0, 1)
                    old = c[name][row[j], :, :lo - j * bs].to(dbl)
                    s = (new.abs().amax((1, 2)) / 127).clamp(min=2.0 ** -100).to(torch.float32)
                    s_old = scales[row[j]].clone()
                    if old.shape[1]:
                        s = torch.maximum(s, s_old)
                    scales[row[j]] = s
                    s = s.to(dbl)[:, None, None]
                    ints = torch.cat([torch.round(old * s_old.to(dbl)[:, None, None] / s), torch.round(new / s)], dim=1)
                    parts.append((ints.clamp(-127, 127) * s).transpose(0, 1))
            res.append((torch.cat(parts), scales.to(dbl)))
        return [turned(st["q"]), res[0][0], res[1][0], res[0][1], res[1][1]]
    if work(case)["flops"] > 4e12:
        return None
    H, a = case["heads"], 0
    out = torch.zeros(st["q"].shape, dtype=dbl, device="cuda")
    for i, n in enumerate(st["lens"]):
        held = st["held"][i]
        blocks = st["table"][i, :(held + bs - 1) // bs].tolist()
        for g in range(G):
            kk, vv = (torch.cat([c[name][b, g].to(dbl) * c[name + "_scale"][b, g].to(dbl) for b in blocks])[:held] for name in ("k", "v"))
            for h in range(g * H // G, (g + 1) * H // G):
                step = max(1, (1 << 27) // held)
                for r in range(0, n, step):
                    e = min(n, r + step)
                    seen = e + held - n                                         # the last of these rows sees this many places
                    z = st["q"][a + r:a + e, h].to(dbl) @ kk[:seen].T / math.sqrt(case["head_dim"])
                    z = torch.where(torch.ones_like(z, dtype=torch.bool).tril(seen - (e - r)), z, -math.inf)
                    out[a + r:a + e, h] = torch.softmax(z, dim=1) @ vv[:seen]
        a += n
    return out
