"""Rotary positions, appending to the cache and chunk attention on a GPU against the fp64 oracle.

Bounds.  u = eps / 2 of the data type is the largest relative error of one rounding to it (bf16 2^-8, fp16 2^-11).
Rotation, y = s (a cos - b sin):
  - the angle: cut to 2^-32 turns and rounded to fp32 (2^-25 of a half turn), so below pi (2^-25 + 2^-31) + 2^-33 < 2^-23.3; its cosine or sine: cut off below
    2^-25, 2^-25 for the last rounding (of a value up to 1) and less for those before it, 2^-23.  Together below 2^-22 for a cosine or sine, twice that with its
    product by s, the two products and the difference (2^-24 of a term each):
                                                                                                 2^-21 s (|a| + |b|)
  - the output is rounded once: u |y|, and half of 2^-24 where fp16 has no more bits.
Numbers of the cache: half a step of the scale, and the rotation's error; the scale: that error and 2^-23 of itself.  Kept numbers, rounded again: half a step of the new one.
Chunk attention, with A the attention over |v| (as for single tokens over the cache):
  - probabilities rounded to fp16:  2^-11 A;  the output:  u A
  - a score, a sum of head_dim products in fp32 (2^-23 an addition), twice:                       2 (head_dim + 8) 2^-23 smax A
  - exponentials, logarithms, products and rescalings, fp32 sums cut into steps:                  2^-17 A
  - fp16 probabilities below 2^-14 are multiples of 2^-24; sum p >= 1:                            n 2^-25 max |v|
"""
import numpy as np
import pytest
import torch

from oracle import language_oracle as LO

pytestmark = pytest.mark.gpu
U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
DTYPES = [torch.bfloat16, torch.float16]
BF, FP = DTYPES


def _rand(shape, dtype, seed, scale=1.0):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * scale).to(dtype)


def _cu(lens):
    return np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)


def _dev(x):
    return torch.as_tensor(np.asarray(x), dtype=torch.int32).cuda()


def _table(seed, lens, bs, spare=3):
    need = [(max(n, 0) + bs - 1) // bs for n in lens]
    perm = torch.randperm(sum(need) + spare, generator=torch.Generator().manual_seed(seed)).to(torch.int32)
    table, at = torch.full((len(lens), max(need + [1])), -7, dtype=torch.int32), 0
    for i, n in enumerate(need):
        table[i, :n] = perm[at:at + n]
        at += n
    return table, sum(need) + spare


def _filled(n_blocks, G, bs, hd, seed):
    gen = torch.Generator().manual_seed(seed)
    return ([torch.randint(-127, 128, (n_blocks, G, bs, hd), generator=gen, dtype=torch.int8) for _ in range(2)],
            [torch.rand(n_blocks, G, generator=gen) * 0.03 + 0.005 for _ in range(2)])


def _cache(numbers, scales):
    import paper_2609_31551_b200 as P
    n, G, bs, hd = numbers[0].shape
    return P.KvCache(n, bs, G, hd, tensors=(numbers[0].cuda(), numbers[1].cuda(), scales[0].cuda(), scales[1].cuda()))


# ------------------------------------------------------------------------------------------------ rotary positions
def _pair_sum(x, pairs, neighbours):
    """|a| + |b| of the pair that an element belongs to; 0 where it is not rotated."""
    y, z = x.double().abs(), torch.zeros(x.shape, dtype=torch.float64)
    i = torch.arange(pairs)
    a, b = (2 * i, 2 * i + 1) if neighbours else (i, i + pairs)
    z[..., a] = z[..., b] = y[..., a] + y[..., b]
    return z


def _rotation_tol(x, ref, rot, scale=1.0):
    return 2.0 ** -21 * scale * _pair_sum(x, rot["pairs"], rot["neighbours"])


def _check_rotated(x, got, rot, positions, scale=1.0, inverse=False):
    ref = LO.rotate(x, positions, rot["axis"], rot["inv_freq"], rot["neighbours"], scale, inverse)
    u = U[x.dtype]
    tol = _rotation_tol(x, ref, rot, scale) * (1 + u) + u * 1.001 * ref.abs() + (2.0 ** -25 if x.dtype == FP else 0.0)
    err = (got.double().cpu() - ref).abs()
    assert (err <= tol).all(), float((err / tol.clamp_min(1e-300)).max())
    tail = 2 * rot["pairs"]
    assert torch.equal(got[..., tail:].cpu(), x[..., tail:])


def _rotary(hd, width, sections=None, neighbours=False, base=1e4, **kw):
    import paper_2609_31551_b200 as P
    pairs = width // 2
    rot = {"pairs": pairs, "neighbours": neighbours, "inv_freq": base ** (-np.arange(pairs, dtype=np.float64) / pairs),
           "axis": np.repeat(np.arange(len(sections)), sections) if sections else np.zeros(pairs, dtype=np.int64)}
    return P.Rotary(hd, rotary_dim=width, base=base, sections=sections, neighbours=neighbours, **kw), rot


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("hd,width,sections", [(128, 128, (16, 24, 24)), (128, 128, None), (64, 64, (8, 12, 12)), (64, 16, None), (128, 48, (10, 6, 8)), (128, 96, (20, 0, 28)), (64, 48, (24,))])
@pytest.mark.parametrize("neighbours", [False, True])
@pytest.mark.parametrize("T,H,G", [(1, 1, 1), (5, 4, 2), (67, 33, 3), (300, 8, 8)])
def test_rotation(dtype, hd, width, sections, neighbours, T, H, G):
    r, rot = _rotary(hd, width, sections, neighbours)
    q, k = _rand((T, H, hd), dtype, 1, 3.0), _rand((T, G, hd), dtype, 2)
    pos = torch.randint(-50, 5000, (r.n_axes, T), generator=torch.Generator().manual_seed(3), dtype=torch.int32)
    out_q, out_k = r.apply(q.cuda(), k.cuda(), pos.cuda())
    _check_rotated(q, out_q, rot, pos.numpy())
    _check_rotated(k, out_k, rot, pos.numpy())
    for budget in (1, 50):
        again = r.apply(q.cuda(), k.cuda(), pos.cuda(), sm_budget=budget)
        assert torch.equal(again[0], out_q) and torch.equal(again[1], out_k)
    back = r.apply(out_q, out_k, pos.cuda(), inverse=True)
    _check_rotated(out_q.cpu(), back[0], rot, pos.numpy(), inverse=True)
    _check_rotated(out_k.cpu(), back[1], rot, pos.numpy(), inverse=True)


def test_rotation_of_far_positions():
    """Every 32-bit position, the frequency 1 among them, where fp32 would not know the angle at all."""
    r, rot = _rotary(128, 128, None, base=5e6)
    pos = np.array([2 ** 31 - 1, -2 ** 31, 2 ** 30 + 1, 700001, 16777217, -1, 0, 1 << 24], dtype=np.int32)
    q = _rand((8, 2, 128), FP, 5)
    out, none = r.apply(q.cuda(), None, _dev(pos))
    assert none is None
    _check_rotated(q, out, rot, pos[None])


def test_rotation_with_given_frequencies_and_axes():
    import paper_2609_31551_b200 as P
    gen = np.random.Generator(np.random.PCG64(4))
    freq = np.concatenate([gen.uniform(-9.0, 9.0, 30), [0.0, 2 * np.pi]])      # more than a turn a position, backwards, none
    axes = gen.integers(0, 4, 32)
    axes[0] = 3
    r = P.Rotary(64, inv_freq=freq, axes=axes, scale=0.75)
    assert r.n_axes == 4
    rot = {"pairs": 32, "neighbours": False, "inv_freq": freq, "axis": axes}
    q, pos = _rand((40, 3, 64), BF, 6), gen.integers(-3000, 3000, (4, 40)).astype(np.int32)
    _check_rotated(q, r.apply(q.cuda(), None, _dev(pos))[0], rot, pos, scale=0.75)


@pytest.mark.parametrize("width,neighbours", [(128, False), (32, True), (32, False)])
def test_rotation_in_place_of_views_leaves_the_rest(width, neighbours):
    """Queries and keys inside one packed projection, turned where they lie."""
    H, G, hd, T = 6, 2, 128, 37
    r, rot = _rotary(hd, width, (width // 4, width // 8, width // 8), neighbours)
    x = _rand((T, (H + 2 * G) * hd + 24), BF, 7)
    xd = x.cuda()

    def parts(t):
        return t[:, 8:8 + H * hd].view(T, H, hd), t[:, 8 + H * hd:8 + (H + G) * hd].view(T, G, hd)
    pos = torch.randint(0, 900, (3, T), generator=torch.Generator().manual_seed(8), dtype=torch.int32)
    wide = torch.full((3, T + 9), -1, dtype=torch.int32)
    wide[:, :T] = pos
    q, k = parts(xd)
    out_q, out_k = r.apply(q, k, wide.cuda()[:, :T], out=(q, k))
    assert out_q is q and out_k is k
    for a, b in zip(parts(x), (q, k)):
        _check_rotated(a, b, rot, pos.numpy())
    rest, was = xd.cpu(), x.clone()
    for t in (rest, was):
        for p in parts(t):
            p.zero_()
    assert torch.equal(rest, was)


def test_rotation_keeps_what_is_not_finite_in_its_pairs():
    r, rot = _rotary(64, 32, None)
    q = _rand((3, 2, 64), BF, 9)
    q[1, 0, 3], q[2, 1, 40] = float("inf"), float("nan")
    out = r.apply(q.cuda(), None, _dev([5, 6, 7]))[0].cpu()
    bad = ~torch.isfinite(out)
    want = torch.zeros_like(bad)
    want[1, 0, 3] = want[1, 0, 19] = want[2, 1, 40] = True
    assert torch.equal(bad, want)


def test_gradient_of_the_rotation_is_its_inverse():
    """<g, R x> = <R^T g, x> by apply(inverse=True), and R x against differences of the oracle's fp64 map."""
    r, rot = _rotary(128, 64, (16, 8, 8), scale=1.25)
    pos = torch.randint(0, 4000, (3, 9), generator=torch.Generator().manual_seed(10), dtype=torch.int32)
    x, g = _rand((9, 4, 128), FP, 11), _rand((9, 4, 128), FP, 12)
    grad = r.apply(g.cuda(), None, pos.cuda(), inverse=True)[0]
    _check_rotated(g, grad, rot, pos.numpy(), scale=1.25, inverse=True)
    f = lambda y: float((LO.rotate(y, pos.numpy(), rot["axis"], rot["inv_freq"], False, 1.25) * g.double()).sum())      # noqa: E731
    # the map is linear: a difference over any step is the derivative; the gradient is rounded to fp16 once, 2^-11 of it
    for at in ((0, 0, 0), (3, 1, 40), (8, 3, 63), (5, 2, 100)):
        y = x.double().clone()
        y[at] += 1.0
        want = f(y) - f(x.double())
        assert abs(float(grad[at]) - want) <= 2.0 ** -11 * abs(want) + 2.0 ** -20 * 1.25 * 8, at


# ------------------------------------------------------------------------------------------------ append
def _check_append(c, before, numbers, scales, rot, q, k, v, cu, start, table, positions, out, scale=1.0):
    """before: numbers and scales as they were; the cache against exact quotients with the scale that it chose, the scale against the exact one."""
    bs, hd = c.block_size, c.head_dim
    turned = LO.rotate(k, positions, rot["axis"], rot["inv_freq"], rot["neighbours"], scale)
    slack = _rotation_tol(k, turned, rot, scale)
    for x, tol, now, now_s, old, old_s in ((turned, slack, c.k.cpu(), c.k_scale.cpu(), before[0][0], before[1][0]),
                                           (v.double(), torch.zeros(v.shape, dtype=torch.float64), c.v.cpu(), c.v_scale.cpu(), before[0][1], before[1][1])):
        untouched = torch.ones(now.shape[0], dtype=torch.bool)
        for s in range(len(start)):
            a, b, at = int(cu[s]), int(cu[s + 1]), int(start[s])
            for blk in range(at // bs, (at + b - a + bs - 1) // bs if b > a else 0):
                lo, hi, i = max(at, blk * bs), min(at + b - a, (blk + 1) * bs), int(table[s, blk])
                untouched[i] = False
                new, new_tol = x[a + lo - at:a + hi - at].transpose(0, 1), tol[a + lo - at:a + hi - at].transpose(0, 1)      # [G, n, hd]
                kept = lo - blk * bs
                want = (new.abs().amax((1, 2)) / 127).clamp_min(LO.MIN_SCALE)
                far = new_tol.amax((1, 2)) / 127 + want * 2.0 ** -23
                if kept:
                    want = torch.maximum(want, old_s[i].double())
                assert ((now_s[i].double() - want).abs() <= far).all()
                step = now_s[i].double()[:, None, None]
                got = now[i, :, kept:kept + hi - lo].double() * step
                assert ((got - new).abs() <= 0.5 * step * (1 + 2.0 ** -20) + new_tol).all()
                again = old[i, :, :kept].double() * old_s[i].double()[:, None, None]
                same = now_s[i] == old_s[i]
                assert torch.equal(now[i, same, :kept], old[i, same, :kept]) or not kept
                assert ((now[i, :, :kept].double() * step - again).abs() <= 0.5 * step * (1 + 2.0 ** -20)).all()
                assert torch.equal(now[i, :, kept + hi - lo:], old[i, :, kept + hi - lo:])
        assert torch.equal(now[untouched], old[untouched]) and torch.equal(now_s[untouched], old_s[untouched])
    if q is not None:
        _check_rotated(q, out, rot, positions, scale)


def _places(cu, start):
    return np.concatenate([np.arange(int(b) - int(a)) + int(s) for a, b, s in zip(cu[:-1], cu[1:], start)] + [np.zeros(0)]).astype(np.int32)[None]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("hd,width,neighbours", [(128, 128, False), (64, 64, False), (128, 32, True), (64, 48, False)])
@pytest.mark.parametrize("bs", [16, 32, 64, 128])
@pytest.mark.parametrize("lens,before", [([1], [0]), ([1, 1, 1], [5, 0, 31]), ([40, 0, 129], [0, 7, 3]), ([300, 2], [17, 127]), ([16, 128], [16, 0])])
def test_append(dtype, hd, width, neighbours, bs, lens, before):
    G, H = 3, 6
    r, rot = _rotary(hd, width, (width // 4, width // 8, width // 2 - width // 4 - width // 8), neighbours)
    table, n_blocks = _table(bs + hd, [a + b for a, b in zip(lens, before)], bs)
    was = _filled(n_blocks, G, bs, hd, 40)
    cu = _cu(lens)
    T = int(cu[-1])
    q = _rand((T, H, hd), dtype, 39, 2.0)
    k, v = (_rand((T, G, hd), dtype, s) * torch.rand(T, G, 1, generator=torch.Generator().manual_seed(s)).mul(4).exp().to(dtype) for s in (41, 42))
    k[::3] *= 0.0625                                                    # tokens that leave the scale alone, and ones that raise it
    pos = np.random.Generator(np.random.PCG64(bs)).integers(0, 90000, (3, T)).astype(np.int32)
    results = []
    for budget in (0, 1, 37):
        c = _cache(*was)
        out = c.append(q.cuda(), k.cuda(), v.cuda(), _dev(cu), _dev(before), table.cuda(), r, _dev(pos), sm_budget=budget)
        c.check()
        results.append((c.k.cpu(), c.v.cpu(), c.k_scale.cpu(), c.v_scale.cpu(), out.cpu()))
        if budget == 0:
            _check_append(c, was, *was, rot, q, k, v, cu, before, table, pos, out)
    for other in results[1:]:
        assert all(torch.equal(a, b) for a, b in zip(results[0], other))


@pytest.mark.parametrize("G,H", [(1, 1), (8, 32), (16, 16), (5, 0)])
@pytest.mark.parametrize("lens,before", [([1] * 70, "random"), ([1, 6, 3, 0, 2] * 5, "random"), ([700, 1, 33], [0, 900, 64])])
def test_append_at_the_tokens_own_places(G, H, lens, before):
    """Positions that are not given are the places; steps of many sequences, and no queries."""
    hd, bs = 128, 16
    r, rot = _rotary(hd, hd)
    if before == "random":
        before = np.random.Generator(np.random.PCG64(G)).integers(0, 300, len(lens))
    table, n_blocks = _table(G, [a + int(b) for a, b in zip(lens, before)], bs)
    was = _filled(n_blocks, G, bs, hd, 43)
    cu = _cu(lens)
    T = int(cu[-1])
    q = _rand((T, H, hd), BF, 44) if H else None
    k, v = _rand((T, G, hd), BF, 45), _rand((T, G, hd), BF, 46, 4.0)
    c = _cache(*was)
    out = c.append(q.cuda() if H else None, k.cuda(), v.cuda(), _dev(cu), _dev(before), table.cuda(), r)
    c.check()
    assert H or out is None
    _check_append(c, was, *was, rot, q, k, v, cu, before, table, _places(cu, before), out)
    # the positions spelt out give the same bytes
    d = _cache(*was)
    again = d.append(q.cuda() if H else None, k.cuda(), v.cuda(), _dev(cu), _dev(before), table.cuda(), r, _dev(_places(cu, before)))
    assert torch.equal(c.k, d.k) and torch.equal(c.k_scale, d.k_scale) and (not H or torch.equal(out, again))


def test_append_without_rotation_is_store():
    """Frequencies of 0: what the cache holds then is what store() writes, bit for bit."""
    import paper_2609_31551_b200 as P
    hd, bs, G = 64, 32, 4
    lens, before = [70, 1, 9], [5, 31, 64]
    table, n_blocks = _table(1, [a + b for a, b in zip(lens, before)], bs)
    was = _filled(n_blocks, G, bs, hd, 47)
    cu = _cu(lens)
    k, v = _rand((80, G, hd), FP, 48, 3.0), _rand((80, G, hd), FP, 49)
    a, b = _cache(*was), _cache(*was)
    a.store(k.cuda(), v.cuda(), _dev(cu), _dev(before), table.cuda())
    q = b.append(k.cuda(), k.cuda(), v.cuda(), _dev(cu), _dev(before), table.cuda(), P.Rotary(hd, inv_freq=[0.0] * 32))
    for x, y in ((a.k, b.k), (a.v, b.v), (a.k_scale, b.k_scale), (a.v_scale, b.v_scale), (q.cpu(), k)):
        assert torch.equal(x, y)


def test_append_skips_and_reports_what_lies_outside_and_leaves_unnamed_rows():
    import paper_2609_31551_b200 as P
    hd, bs, G = 64, 16, 2
    r, rot = _rotary(hd, hd)
    was = _filled(6, G, bs, hd, 50)
    x = _rand((12, G, hd), BF, 51)
    q = _rand((12, 4, hd), BF, 52)

    def call(cu, start, table):
        c = _cache(*was)
        out = torch.full((12, 4, hd), 5.0, dtype=BF, device="cuda")
        c.append(q.cuda(), x.cuda(), x.cuda(), _dev(cu), _dev(start), _dev(table), r, out=out)
        return c, out.cpu()
    for start, table in (([0, 16], [[9, 0], [1, 2]]), ([0, 40], [[0, 3], [1, 2]]), ([-1, 16], [[0, 3], [1, 2]]), ([0, 16], [[-1, 0], [1, 2]])):
        c, out = call([2, 5, 9], start, table)
        with pytest.raises(P.EasError) as e:
            c.check()
        assert e.value.status == 7
        assert (out[:2] == 5).all() and (out[9:] == 5).all() and not (out[2:9] == 5).all(dim=-1).any()
        c.check()                                                           # the word is cleared
    c, out = call([2, 5, 9], [0, 16], [[0, 3], [1, 2]])
    c.check()
    full = [torch.cat([torch.zeros((2, *t.shape[1:]), dtype=t.dtype), t[2:]]) for t in (x, x)]
    _check_append(c, was, *was, rot, None, full[0], full[1], [2, 5, 9], [0, 16], torch.tensor([[0, 3], [1, 2]]), np.concatenate([[0, 0], [0, 1, 2], [16, 17, 18, 19], [0, 0, 0]])[None], None)
    # rows past the tensor: cu_seqlens is cut to them
    c, out = call([0, 8, 99], [0, 0], [[0, 3], [1, 2]])
    c.check()
    assert not (out == 5).all(dim=-1).any()


def test_append_non_finite_keys_stay_in_their_block_and_head():
    hd, bs, G = 64, 16, 2
    r, rot = _rotary(hd, hd)
    was = _filled(4, G, bs, hd, 53)
    k = _rand((20, G, hd), BF, 54)
    k[17, 1, 4] = float("inf")
    c = _cache(*was)
    c.append(None, k.cuda(), k.cuda(), _dev([0, 20]), _dev([0]), _dev([[2, 0]]), r)
    c.check()
    bad = torch.isnan(c.k_scale).cpu()
    assert bad.sum() == 1 and bad[0, 1] and torch.isnan(c.v_scale[0, 1])
    kk, _ = c.load(_dev([0, 20]), _dev([0]), _dev([[2, 0]]), 20)
    assert torch.isnan(kk[16:, 1]).all() and torch.isfinite(kk[:16]).all() and torch.isfinite(kk[:, 0]).all()


# ------------------------------------------------------------------------------------------------ chunk attention
def _check_chunk(c, numbers, scales, q, cu, lens, table, scale=None, max_new=None, **kw):
    hd = q.shape[2]
    out = c.chunk_attention(q.cuda(), _dev(cu), _dev(lens), table.cuda(), max_new=max_new, scale=scale, **kw)
    c.check()
    ref, mag, smax = LO.chunk_attention(q, numbers[0], numbers[1], scales[0], scales[1], cu, lens, table, hd ** -0.5 if scale is None else scale)
    got, named = out.double().cpu(), ~torch.isnan(ref[:, 0, 0])
    assert torch.isfinite(got[named]).all()
    vmax = float((numbers[1].float().abs().amax((2, 3)) * scales[1]).max())
    u = U[q.dtype]
    tol = mag * (2.0 ** -11 + u * 1.01 + 2 * (hd + 8) * 2.0 ** -23 * smax[..., None] + 2.0 ** -17) + max(list(lens) + [0]) * 2.0 ** -25 * vmax + (2.0 ** -24 if q.dtype == FP else 0.0)
    err = (got - ref).abs()
    assert (err[named] <= tol[named]).all(), float((err / tol)[named].max())
    for s in range(len(lens)):
        blind = max(min(int(cu[s + 1]) - int(cu[s]) - max(int(lens[s]), 0), int(cu[s + 1]) - int(cu[s])), 0)
        assert not got[int(cu[s]):int(cu[s]) + blind].any()
    return out


CHUNKS = [([1], [0]), ([3], [0]), ([4], [713]), ([1, 1, 1], [15, 16, 32]), ([2, 0, 5, 1], [40, 0, 0, 300]), ([80, 81, 1], [0, 79, 1000]), ([129, 3], [500, 0]), ([17], [2000]),
          ([0, 7, 0], [5, 5, 5]), ([333], [64])]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("H,G", [(1, 1), (8, 2), (5, 1), (16, 2), (17, 1)])
@pytest.mark.parametrize("bs", [16, 64])
@pytest.mark.parametrize("lens,before", CHUNKS)
def test_chunk_attention(dtype, hd, H, G, bs, lens, before):
    held = [a + b for a, b in zip(lens, before)]
    table, n_blocks = _table(H + bs, held, bs)
    numbers, scales = _filled(n_blocks, G, bs, hd, 60)
    cu = _cu(lens)
    q = _rand((int(cu[-1]), H, hd), dtype, 61, 2.0)
    c = _cache(numbers, scales)
    for max_new in {max(lens), None}:
        out = _check_chunk(c, numbers, scales, q, cu, held, table, max_new=max_new)
        for budget in (1, 37):
            assert torch.equal(out, c.chunk_attention(q.cuda(), _dev(cu), _dev(held), table.cuda(), max_new=max_new, sm_budget=budget))


@pytest.mark.parametrize("hd,H,G,bs,lens,before", [
    (128, 8, 1, 16, [9], [30011]), (64, 4, 4, 64, [40, 1, 3], [9000, 5000, 77]), (128, 32, 8, 128, [5] * 3, [4097] * 3), (64, 12, 1, 32, [200, 7], [12000, 40]),
    (128, 40, 8, 32, [150], [6000]), (64, 16, 16, 16, [70, 300], [100, 0]), (128, 128, 1, 64, [3, 2], [900, 10]), (64, 65, 1, 16, [4], [333]),
    (128, 4, 4, 64, [300, 1, 1, 1, 260], [3000, 2500, 1, 0, 700])])
@pytest.mark.parametrize("dtype", DTYPES)
def test_chunk_attention_over_long_caches(hd, H, G, bs, lens, before, dtype):
    held = [a + b for a, b in zip(lens, before)]
    table, n_blocks = _table(hd + H, held, bs)
    numbers, scales = _filled(n_blocks, G, bs, hd, 62)
    cu = _cu(lens)
    q = _rand((int(cu[-1]), H, hd), dtype, 63, 1.5)
    c = _cache(numbers, scales)
    out = _check_chunk(c, numbers, scales, q, cu, held, table, max_new=max(lens))
    assert torch.equal(out, c.chunk_attention(q.cuda(), _dev(cu), _dev(held), table.cuda(), max_new=max(lens), sm_budget=74))
    assert torch.equal(out, c.chunk_attention(q.cuda(), _dev(cu), _dev(held), table.cuda(), max_new=max(lens)))


@pytest.mark.parametrize("max_new", [2, 40, None])
def test_chunk_attention_of_more_sequences_than_a_launch_holds(max_new):
    n, hd, bs = 2300, 64, 16
    rng = np.random.Generator(np.random.PCG64(6))
    lens = rng.integers(0, 3, n)
    before = rng.integers(0, 40, n)
    if max_new == 40:
        lens[[0, 1030, 2299]] = 40
    held = lens + before
    table, n_blocks = _table(3, held, bs)
    numbers, scales = _filled(n_blocks, 2, bs, hd, 64)
    cu = _cu(lens)
    q = _rand((int(cu[-1]), 4, hd), BF, 65)
    _check_chunk(_cache(numbers, scales), numbers, scales, q, cu, held, table, max_new=max_new)


@pytest.mark.parametrize("max_new", [3, 30])
@pytest.mark.parametrize("hd", [64, 128])
def test_chunk_attention_rows_that_see_nothing(hd, max_new):
    """Sequences shorter than their chunk, of length 0 and below."""
    lens, held = [3, 3, 3, 2, 1], [1, 0, -5, 2, 700]
    if max_new == 30:
        lens, held = [30, 20, 30, 30, 1], [11, 0, -5, 30, 700]
    table, n_blocks = _table(2, held, 16)
    numbers, scales = _filled(n_blocks, 2, 16, hd, 66)
    cu = _cu(lens)
    q = _rand((int(cu[-1]), 8, hd), BF, 67)
    _check_chunk(_cache(numbers, scales), numbers, scales, q, cu, held, table, max_new=max_new)


@pytest.mark.parametrize("max_new", [4, 60])
@pytest.mark.parametrize("hd", [64, 128])
def test_chunk_attention_scales_of_all_sizes(hd, max_new):
    """Value scales from 2^-99 to 2^100 and key scales that leave one block to decide: the weights fit whatever they are."""
    lens, before, bs, G = [max_new, 1], [200, 90], 16, 2
    held = [a + b for a, b in zip(lens, before)]
    table, n_blocks = _table(8, held, bs)
    numbers, scales = _filled(n_blocks, G, bs, hd, 68)
    cu = _cu(lens)
    q = _rand((int(cu[-1]), 4, hd), FP, 69)
    for factor in (2.0 ** -95, 2.0 ** 100):
        sc = [scales[0], scales[1] * factor]
        c = _cache(numbers, sc)
        out = c.chunk_attention(q.cuda(), _dev(cu), _dev(held), table.cuda(), max_new=max_new)
        c.check()
        if factor > 1:
            assert not torch.isnan(out).any() and torch.isinf(out).any()          # (the values pass fp16)
    mixed = scales[1] * (2.0 ** (torch.arange(n_blocks) % 13 - 6).float())[:, None]
    for sc in ([scales[0], mixed], [scales[0] * 20, mixed], [torch.where(torch.arange(n_blocks)[:, None] % 3 == 0, 0.0, scales[0]), scales[1]]):
        _check_chunk(_cache(numbers, sc), numbers, sc, q, cu, held, table, max_new=max_new)


@pytest.mark.parametrize("max_new", [4, 60])
@pytest.mark.parametrize("hd", [64, 128])
def test_chunk_attention_non_finite_blocks_and_queries(hd, max_new):
    """A block whose scale is NaN reaches the rows that see it and no others; a query with Inf or NaN in it is NaN alone."""
    lens, before, bs, G, H = [max_new, 2], [100, 70], 16, 2, 4
    held = [a + b for a, b in zip(lens, before)]
    table, n_blocks = _table(9, held, bs)
    for which in (0, 1):
        for first_bad in (40, 96, (held[0] - 1) // bs * bs):                    # a block in front of the chunk, one that it begins in, its last
            numbers, scales = _filled(n_blocks, G, bs, hd, 70)
            scales[which][int(table[0, first_bad // bs]), 1] = float("nan")
            cu = _cu(lens)
            q = _rand((int(cu[-1]), H, hd), BF, 71)
            c = _cache(numbers, scales)
            out = c.chunk_attention(q.cuda(), _dev(cu), _dev(held), table.cuda(), max_new=max_new).cpu()
            c.check()
            sees = torch.arange(int(cu[-1])) + before[0] >= first_bad // bs * bs
            sees[lens[0]:] = False
            want = torch.zeros(out.shape, dtype=torch.bool)
            want[sees, 2:] = True
            assert torch.equal(torch.isnan(out), want)
    numbers, scales = _filled(n_blocks, G, bs, hd, 72)
    q[1, 3, 5], q[2, 0, 0] = float("inf"), float("nan")
    out = _cache(numbers, scales).chunk_attention(q.cuda(), _dev(cu), _dev(held), table.cuda(), max_new=max_new).cpu()
    want = torch.zeros(out.shape, dtype=torch.bool)
    want[1, 3] = want[2, 0] = True
    assert torch.equal(torch.isnan(out), want)


@pytest.mark.parametrize("max_new", [4, 50])
@pytest.mark.parametrize("hd", [64, 128])
def test_chunk_attention_skips_and_reports_what_lies_outside(hd, max_new):
    import paper_2609_31551_b200 as P
    lens, held, bs = [max_new, 2, 3], [60, 40, 33], 16
    table, n_blocks = _table(10, held, bs)
    numbers, scales = _filled(n_blocks, 1, bs, hd, 73)
    cu = _cu(lens)
    q = _rand((int(cu[-1]), 3, hd), BF, 74)
    c = _cache(numbers, scales)
    good = _check_chunk(c, numbers, scales, q, cu, held, table, max_new=max_new).cpu()
    others = torch.ones(int(cu[-1]), dtype=torch.bool)
    others[cu[1]:cu[2]] = False

    def call(tab, lens_now=held, most=max_new, cu_now=cu):
        out = torch.full(q.shape, 5.0, dtype=BF, device="cuda")
        c.chunk_attention(q.cuda(), _dev(cu_now), _dev(lens_now), tab.cuda(), max_new=most, out=out)
        with pytest.raises(P.EasError) as e:
            c.check()
        assert e.value.status == 7
        return out.cpu()
    for bad in (n_blocks, -1, 2 ** 30):
        t = table.clone()
        t[1, 1] = bad
        out = call(t)
        assert torch.equal(out[others], good[others]) and torch.isfinite(out).all()
        # tokens of the missing block do not count: as if the other blocks were all there is
        keep = list(range(16)) + list(range(32, 40))
        num = [torch.zeros(2, 1, bs, hd, dtype=torch.int8) for _ in range(2)]
        kv = [LO.cache_values(numbers[i], scales[i], table[1], 40)[keep] for i in range(2)]
        ref = torch.stack([LO.attend(q[cu[1] + 1, h].double(), kv[0][:, 0], kv[1][:, 0], hd ** -0.5)[0] for h in range(3)])
        assert torch.allclose(out[cu[1] + 1].double(), ref, rtol=2.0 ** -7, atol=2.0 ** -7)
    # a length behind the table's end is cut to it
    out = call(table, [60, 16 * table.shape[1] + 1, 33])
    assert torch.equal(out[others], good[others])
    # more new tokens than max_new: that sequence is left alone
    out = call(table, most=max_new - 1)
    assert (out[:cu[1]] == 5).all() and torch.equal(out[cu[1]:], good[cu[1]:])


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("lens", [[3, 2], [70, 9]])
def test_chunk_attention_reads_views_and_leaves_other_rows_alone(hd, lens):
    H, G, bs, before = 4, 2, 32, [100, 260]
    held = [a + b for a, b in zip(lens, before)]
    table, n_blocks = _table(11, held, bs)
    numbers, scales = _filled(n_blocks, G, bs, hd, 75)
    for s in range(2):                                                          # what lies behind a sequence's end in its last block does not count
        used = held[s] % bs
        for x in numbers:
            x[int(table[s, held[s] // bs]), :, used:] = 127 if s else -128
    cu = _cu(lens) + 6
    T = int(cu[-1]) + 8
    x = _rand((T, (H + 2) * hd + 24), BF, 76)
    x[:6], x[int(cu[-1]):] = float("nan"), float("nan")                        # rows of no sequence
    q = x[:, 8:8 + H * hd].view(T, H, hd)
    buf = torch.full((T, H * hd + 40), 5.0, dtype=BF, device="cuda")
    xd = x.cuda()
    c = _cache(numbers, scales)
    out = c.chunk_attention(xd[:, 8:8 + H * hd].view(T, H, hd), _dev(cu), _dev(held), table.cuda(), max_new=max(lens), out=buf[:, 8:8 + H * hd].view(T, H, hd), scale=0.2)
    c.check()
    plain = _check_chunk(c, numbers, scales, q[6:int(cu[-1])].contiguous(), cu - 6, held, table, max_new=max(lens), scale=0.2)
    assert torch.equal(out[6:int(cu[-1])], plain)
    buf[6:int(cu[-1]), 8:8 + H * hd] = 5.0
    assert (buf == 5.0).all()


def test_chunk_of_one_token_is_the_attention_of_single_tokens():
    """The same formula: both against each other within both bounds' rounding of the output and the weights."""
    lens = [700, 1, 64, 0, 333]
    table, n_blocks = _table(12, lens, 32)
    numbers, scales = _filled(n_blocks, 2, 32, 128, 77)
    q = _rand((5, 8, 128), FP, 78)
    c = _cache(numbers, scales)
    _check_chunk(c, numbers, scales, q, np.arange(6), lens, table, max_new=1)
    a = c.attention(q.cuda(), _dev(lens), table.cuda())
    b = c.chunk_attention(q.cuda(), _dev(range(6)), _dev(lens), table.cuda(), max_new=1)
    assert torch.allclose(a.float(), b.float(), rtol=2.0 ** -9, atol=2.0 ** -9 * 4)


@pytest.mark.parametrize("max_new", [4, 90])
def test_chunk_attention_replays_for_other_lengths(max_new):
    """A captured call, replayed with other chunks and lengths in its tensors, on its own stream and workspace; beside it an eager one."""
    hd, bs, G, H, n = 128, 32, 2, 8, 6
    rng = np.random.Generator(np.random.PCG64(13))
    most = [max_new + 900] * n
    table, n_blocks = _table(13, most, bs)
    numbers, scales = _filled(n_blocks, G, bs, hd, 79)
    rows = max_new * n
    q = _rand((rows, H, hd), BF, 80)
    c = _cache(numbers, scales)
    qd, cu_d, len_d, td = q.cuda(), _dev([0] * (n + 1)), _dev([0] * n), table.cuda()
    out = torch.full(q.shape, 5.0, dtype=BF, device="cuda")
    ws = torch.empty(c.chunk_workspace_bytes(n, rows, max_new, H), dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    c.chunk_attention(qd, cu_d, len_d, td, max_new=max_new, out=out, workspace=ws)
    torch.cuda.synchronize()
    assert (out == 5).all()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        c.chunk_attention(qd, cu_d, len_d, td, max_new=max_new, out=out, workspace=ws, stream=None)
    for trial in range(3):
        lens = rng.integers(0, max_new + 1, n)
        held = [int(a + rng.integers(0, 900)) for a in lens]
        cu = _cu(lens)
        cu_d.copy_(_dev(cu))
        len_d.copy_(_dev(held))
        out.fill_(5.0)
        graph.replay()
        eager = _check_chunk(c, numbers, scales, q, cu, held, table, max_new=max_new)
        assert torch.equal(out[:cu[-1]], eager[:cu[-1]]) and (out[cu[-1]:] == 5).all()


def test_offsets_past_32_bits():
    """A cache of more than 4 GB a side, and blocks at its end."""
    import paper_2609_31551_b200 as P
    hd, bs, G, n_blocks = 128, 128, 8, 33000
    c = P.KvCache(n_blocks, bs, G, hd)
    held, n = [300, 200], 3
    table = torch.tensor([[n_blocks - 1, n_blocks - 3, 32767], [n_blocks - 2, 16384, 0]], dtype=torch.int32)
    r, rot = _rotary(hd, hd)
    k, v = _rand((500, G, hd), BF, 81), _rand((500, G, hd), BF, 82)
    c.append(None, k.cuda(), v.cuda(), _dev([0, 300, 500]), _dev([0, 0]), table.cuda(), r)
    small = P.KvCache(6, bs, G, hd)
    small.append(None, k.cuda(), v.cuda(), _dev([0, 300, 500]), _dev([0, 0]), _dev([[0, 1, 2], [3, 4, 5]]), r)
    for most in (n, 40):
        q = _rand((2 * most, 8, hd), BF, 83)
        a = c.chunk_attention(q.cuda(), _dev([0, most, 2 * most]), _dev(held), table.cuda(), max_new=most)
        b = small.chunk_attention(q.cuda(), _dev([0, most, 2 * most]), _dev(held), _dev([[0, 1, 2], [3, 4, 5]]), max_new=most)
        assert torch.equal(a, b) and torch.isfinite(a).all()
    c.check()
    small.check()


def test_refusals_on_the_device():
    import paper_2609_31551_b200 as P
    c = P.KvCache(8, 16, 2, 64)
    r = P.Rotary(64)
    x, q = torch.zeros(4, 2, 64, dtype=BF, device="cuda"), torch.zeros(4, 8, 64, dtype=BF, device="cuda")
    cu, start, table, pos = _dev([0, 4]), _dev([0]), _dev([[0, 1]]), _dev([0, 1, 2, 3])

    def refused(call):
        with pytest.raises(P.EasError):
            call()
    for bad in (q.float(), q.cpu(), q[:, :, :32], q.transpose(0, 1), torch.zeros(4, 8 * 64 + 4, dtype=BF, device="cuda")[:, 4:].view(4, 8, 64)):
        refused(lambda: r.apply(bad, x, pos))
        refused(lambda: c.append(bad, x, x, cu, start, table, r))
        refused(lambda: c.chunk_attention(bad, cu, start, table))
    for bad in (pos[:3], pos.long(), pos.cpu(), pos.view(2, 2), _dev([0] * 8)[::2]):
        refused(lambda: r.apply(q, x, bad))
        refused(lambda: c.append(q, x, x, cu, start, table, r, bad))
    refused(lambda: r.apply(q, x[:3], pos))
    refused(lambda: r.apply(q, x, pos, out=(q[:3], x)))
    refused(lambda: r.apply(q, x.half(), pos))
    refused(lambda: r.apply(q, x, pos, sm_budget=4096))
    refused(lambda: r.apply(q, x, pos, sm_budget=-1))
    refused(lambda: P.Rotary(64, sections=(16, 8, 8)).apply(q, x, pos))
    refused(lambda: c.append(q, x, x[:3], cu, start, table, r))
    refused(lambda: c.append(q[:3], x, x, cu, start, table, r))
    refused(lambda: c.append(q, q, q, cu, start, table, r))
    refused(lambda: c.append(q, x, x, cu, start, table, P.Rotary(128)))
    refused(lambda: c.append(q, x, x, cu[:1], start, table, r))
    refused(lambda: c.append(q, x, x, cu, start, table.long(), r))
    refused(lambda: c.chunk_attention(q, cu[:1], start, table))
    refused(lambda: c.chunk_attention(q, cu, start, table, max_new=-1))
    refused(lambda: c.chunk_attention(q, cu, start, table, scale=0.0))
    refused(lambda: c.chunk_attention(q, cu, start, table, scale=float("nan")))
    refused(lambda: c.chunk_attention(q[:, :7], cu, start, table))
    refused(lambda: c.chunk_attention(q, cu, start, table, out=torch.zeros(3, 8, 64, dtype=BF, device="cuda")))
    refused(lambda: c.chunk_attention(q, cu, start, table, workspace=torch.zeros(16, dtype=torch.uint8, device="cuda")))
    refused(lambda: c.chunk_attention(q, cu, start, table, workspace=torch.zeros(1 << 26, dtype=torch.uint8, device="cuda")[8:]))
    refused(lambda: c.chunk_attention(q, cu, start, table, sm_budget=4096))
    r.close()
    refused(lambda: r.apply(q, x, pos))
    refused(lambda: c.append(q, x, x, cu, start, table, r))
    c.close()
    refused(lambda: c.chunk_attention(q, cu, start, table))
    # nothing to do is no error
    c = P.KvCache(8, 16, 2, 64)
    r = P.Rotary(64)
    a, b = r.apply(q[:0], x[:0], pos[:0])
    assert a.shape == (0, 8, 64) and b.shape == (0, 2, 64)
    assert c.append(q[:0], x[:0], x[:0], _dev([0]), start[:0], table[:0], r).shape == (0, 8, 64)
    assert c.chunk_attention(q[:0], _dev([0]), start[:0], table[:0]).shape == (0, 8, 64)
    assert c.chunk_attention(q[:0], _dev([0, 0]), start, table).shape == (0, 8, 64)
    c.check()


# ------------------------------------------------------------------------------------------------ together
@pytest.mark.parametrize("hd,dtype,bs", [(128, BF, 16), (64, FP, 64)])
def test_a_conversation_from_projections_to_answers(hd, dtype, bs):
    """Prompts appended and attended from the cache in two chunks, then drafts of a few tokens and single ones, on a side stream: every output against the oracle on what
    the cache holds."""
    import paper_2609_31551_b200 as P
    H, G, n = 8, 2, 3
    r, rot = _rotary(hd, hd, (hd // 8, hd // 8 + hd // 16, hd // 8 + hd // 16))
    most = 400
    table, n_blocks = _table(14, [most] * n, bs)
    c = P.KvCache(n_blocks, bs, G, hd)
    td = table.cuda()
    held = [0] * n
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for step, lens in enumerate(([90, 1, 200], [60, 130, 0], [4, 1, 3], [1, 1, 1], [2, 4, 4], [1, 1, 1])):
        cu, T = _cu(lens), sum(lens)
        qkv = _rand((T, H + 2 * G, hd), dtype, 100 + step, 1.5)
        x = qkv.cuda()
        pos = torch.randint(0, 500, (3, T), generator=torch.Generator().manual_seed(step), dtype=torch.int32)
        after = [a + b for a, b in zip(held, lens)]
        args = _dev(cu), _dev(held), _dev(after), pos.cuda()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            q = c.append(x[:, :H], x[:, H:H + G], x[:, H + G:], args[0], args[1], td, r, args[3])
            out = c.chunk_attention(q, args[0], args[2], td, max_new=max(lens))
        c.check(side)
        _check_rotated(qkv[:, :H], q, rot, pos.numpy())
        held = after
        numbers, scales = [c.k.cpu(), c.v.cpu()], [c.k_scale.cpu(), c.v_scale.cpu()]
        again = _check_chunk(c, numbers, scales, q.cpu(), cu, held, table, max_new=max(lens))
        assert torch.equal(out, again)
        if max(lens) == 1:
            single = c.attention(q, args[2], td)
            assert torch.allclose(single.float(), out.float(), rtol=4 * U[dtype], atol=4 * U[dtype])
