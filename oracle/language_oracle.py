"""Plain CPU fp64 definitions of the language-model operators (include/eas_language.h).

Test infrastructure only.  One function per operator, loops over sequences and heads, numbers as the definition has them: softmax over the
visible keys, one scale per cache block and head, round to nearest even.  Nothing is read that a sequence does not own."""
import numpy as np
import torch

F64 = torch.float64


def attend(q, k, v, scale):
    """q [hd], k and v [n, hd] -> (softmax(scale q k^T) v, the same of |v|, largest sum |q_i k_i| scale).  n = 0: zeros."""
    if k.shape[0] == 0:
        return torch.zeros_like(q), torch.zeros_like(q), 0.0
    p = torch.softmax((k @ q) * scale, dim=0)
    return p @ v, p @ v.abs(), float((k.abs() @ q.abs()).max() * scale)


def prompt_attention(q, k, v, cu_q, cu_k, scale):
    """Causal, the queries being the last of their sequence's keys.  q [T, H, hd], k, v [Tk, G, hd] (any dtype).
    Returns out, the attention over |v| and the largest absolute score sum per row and head, for error bounds; rows of no sequence are NaN."""
    H, G = q.shape[1], k.shape[1]
    q, k, v = q.to(F64), k.to(F64), v.to(F64)
    out, mag = torch.full_like(q, float("nan")), torch.full_like(q, float("nan"))
    smax = torch.zeros(q.shape[:2], dtype=F64)
    for s in range(len(cu_q) - 1):
        a, b, c, d = (int(x) for x in (cu_q[s], cu_q[s + 1], cu_k[s], cu_k[s + 1]))
        for i in range(b - a):
            seen = max(i + 1 + (d - c) - (b - a), 0)
            for h in range(H):
                g = h * G // H
                out[a + i, h], mag[a + i, h], smax[a + i, h] = attend(q[a + i, h], k[c:c + seen, g], v[c:c + seen, g], scale)
    return out, mag, smax


MIN_SCALE = 2.0 ** -100


def cache_store(numbers, scales, x, cu, start, table):
    """numbers int8 [blocks, G, bs, hd] and scales float32 [blocks, G] are changed in place; x [rows, G, hd]."""
    bs = numbers.shape[2]
    x = x.to(F64).numpy()
    for s in range(len(start)):
        rows, at = x[int(cu[s]):int(cu[s + 1])], int(start[s])
        for b in range(at // bs, (at + len(rows) + bs - 1) // bs if len(rows) else 0):
            lo, hi = max(at, b * bs), min(at + len(rows), (b + 1) * bs)
            blk = int(table[s, b])
            for g in range(numbers.shape[1]):
                new = rows[lo - at:hi - at, g]
                scale = np.float32(max(np.abs(new).max() / 127.0, MIN_SCALE))
                kept = lo - b * bs
                if kept:
                    was = np.float32(scales[blk, g])
                    if scale > was:
                        again = np.rint(numbers[blk, g, :kept].numpy().astype(np.float64) * np.float64(was) / np.float64(scale))
                        numbers[blk, g, :kept] = torch.from_numpy(again.astype(np.int8))
                    scale = max(scale, was)
                numbers[blk, g, kept:kept + hi - lo] = torch.from_numpy(np.rint(new / np.float64(scale)).astype(np.int8))
                scales[blk, g] = float(scale)


def cache_values(numbers, scales, table_row, n):
    """The first n tokens of a sequence as values: [n, G, hd] fp64."""
    bs = numbers.shape[2]
    ids = [int(b) for b in table_row[:(n + bs - 1) // bs]]
    if not ids:
        return torch.zeros((0, numbers.shape[1], numbers.shape[3]), dtype=F64)
    vals = numbers[ids].to(F64) * scales[ids].to(F64)[:, :, None, None]
    return vals.permute(0, 2, 1, 3).reshape(-1, numbers.shape[1], numbers.shape[3])[:n]


def cache_attention(q, k_numbers, v_numbers, k_scales, v_scales, seq_lens, table, scale):
    """q [n, H, hd] -> out, attention over |v|, largest absolute score sum."""
    H, G = q.shape[1], k_numbers.shape[1]
    q = q.to(F64)
    out, mag, smax = torch.zeros_like(q), torch.zeros_like(q), torch.zeros(q.shape[:2], dtype=F64)
    for s in range(q.shape[0]):
        n = max(int(seq_lens[s]), 0)
        k, v = cache_values(k_numbers, k_scales, table[s], n), cache_values(v_numbers, v_scales, table[s], n)
        for h in range(H):
            out[s, h], mag[s, h], smax[s, h] = attend(q[s, h], k[:, h * G // H], v[:, h * G // H], scale)
    return out, mag, smax


def chunk_attention(q, k_numbers, v_numbers, k_scales, v_scales, cu, seq_lens, table, scale):
    """q [rows, H, hd]: rows cu[s] .. cu[s + 1] - 1 are the last tokens among the first seq_lens[s] of sequence s.  -> out, attention over |v| and the
    largest absolute score sum, as prompt_attention; rows of no sequence are NaN."""
    H, G = q.shape[1], k_numbers.shape[1]
    q = q.to(F64)
    out, mag = torch.full_like(q, float("nan")), torch.full_like(q, float("nan"))
    smax = torch.zeros(q.shape[:2], dtype=F64)
    for s in range(len(cu) - 1):
        a, b, n = int(cu[s]), int(cu[s + 1]), max(int(seq_lens[s]), 0)
        k, v = cache_values(k_numbers, k_scales, table[s], n), cache_values(v_numbers, v_scales, table[s], n)
        seen = torch.arange(b - a) + 1 + n - (b - a)
        hidden = torch.arange(n)[None] >= seen[:, None]
        for h in range(H):
            g = h * G // H
            x = (q[a:b, h] @ k[:, g].T * scale).masked_fill(hidden, -float("inf"))
            p = torch.where((seen > 0)[:, None], torch.softmax(x, dim=1), 0.0) if n else x
            out[a:b, h], mag[a:b, h] = p @ v[:, g], p @ v[:, g].abs()
            if n and b > a:
                smax[a:b, h] = (q[a:b, h].abs() @ k[:, g].abs().T).amax(1) * scale
    return out, mag, smax


def rotate(x, positions, axis, inv_freq, neighbours=False, scale=1.0, inverse=False):
    """x [rows, heads, hd], positions [n_axes][rows], axis and inv_freq [pairs] -> fp64.  Angles in extended precision: a position of 2^31 times a
    frequency has bits that fp64 drops."""
    y = x.to(F64).numpy().copy()
    n = len(inv_freq)
    for i in range(n):
        a, b = (2 * i, 2 * i + 1) if neighbours else (i, i + n)
        angle = np.asarray(positions[axis[i]]).astype(np.longdouble) * np.longdouble(inv_freq[i]) * (-1 if inverse else 1)
        c, s = (scale * f(angle).astype(np.float64)[:, None] for f in (np.cos, np.sin))
        u, w = x[:, :, a].to(F64).numpy(), x[:, :, b].to(F64).numpy()
        y[:, :, a], y[:, :, b] = u * c - w * s, w * c + u * s
    return torch.from_numpy(y)
