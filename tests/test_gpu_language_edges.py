"""The language-model operators where sums, references and infinities go wrong, against the fp64 oracle.

Bounds.  u_p, u are the largest relative errors of one rounding to the type of the probabilities and of the output (2^-8 bf16, 2^-11 fp16), A the
attention over |v|, smax the largest sum |q k| scale of a row.  An output element is off by at most
  u_p A + u |out| + 2 (head_dim + 8) 2^-23 smax A + 2^-17 A
(probabilities, output, scores, exponentials and sums).  fp16 weights are kept 2^7 above the reference, so that the row's largest is at least 2^7;
below 2^-14 they are rounded to multiples of 2^-24, each off by at most 2^-25.  Prompts: the sum of the weights is at least 2^7, so together that is
  n 2^-25 / 2^7 max |v| = n 2^-32 max |v|.
Tokens: a weight is 2^(score + log2 scale of the value's block), the numbers are at most 127, and the sum of weight / value scale is at least 2^7 / (value scale
v* of the token whose weight is the largest): n 2^-32 127 v*.  fp16 outputs below 2^-14 are off by at most 2^-25."""
import numpy as np
import pytest
import torch

from oracle import language_oracle as LO

pytestmark = pytest.mark.gpu
U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
DTYPES = [torch.bfloat16, torch.float16]
INF, NAN = float("inf"), float("nan")


def _rand(shape, dtype, seed, scale=1.0):
    gen = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=gen) * scale).to(dtype)


def _dev(x):
    return torch.as_tensor(np.asarray(x), dtype=torch.int32).cuda()


def _prompt(q, k, v, cu_q, cu_k, **kw):
    import paper_2609_31551_b200 as P
    out, status = P.prompt_attention(q.cuda(), k.cuda(), v.cuda(), cu_q, cu_k, **kw)
    assert int(status[0]) == 0
    return out.cpu()


def _is_cut(q, k, cu_q, cu_k):
    import paper_2609_31551_b200 as P
    return P.prompt_attention_workspace_bytes(q.shape[1], k.shape[1], q.shape[2], cu_q, cu_k) > 0


def _prompt_tol(q, mag, smax, n, vmax):
    hd, u = q.shape[2], U[q.dtype]
    tol = mag * (u + u * 1.01 + 2 * (hd + 8) * 2.0 ** -23 * smax[..., None] + 2.0 ** -17)
    return tol + (1.1 * n * 2.0 ** -32 * vmax + 2.0 ** -25 if q.dtype == torch.float16 else 0.0)


def _same_where_not_finite(got, ref):
    assert torch.equal(torch.isnan(got), torch.isnan(ref))
    assert torch.equal(got == INF, ref == INF) and torch.equal(got == -INF, ref == -INF)


def _check(got, q, k, v, cu_q, cu_k):
    """All of a call's rows: the same infinities and NaN as the definition, the rest within the bound (of the finite values)."""
    hd = q.shape[2]
    ref, _, smax = LO.prompt_attention(q, k, v, cu_q, cu_k, hd ** -0.5)
    tame = torch.nan_to_num(v.double(), nan=0.0, posinf=0.0, neginf=0.0)
    mag = LO.prompt_attention(q, k, tame, cu_q, cu_k, hd ** -0.5)[1]
    got = got.double()
    _same_where_not_finite(got, ref)
    fin = torch.isfinite(ref)
    tol = _prompt_tol(q, mag, torch.nan_to_num(smax, nan=0.0, posinf=0.0), int(max(np.diff(cu_k))), float(tame.abs().max()))
    err = (got - ref).abs()
    assert (err[fin] <= tol[fin]).all(), float((err / tol)[fin].max())


CHUNK = [(0, False), (9000, True)]       # keys in front of the chunk; with many the key steps are cut


# ------------------------------------------------------------------------------------------------ prompts: seen and hidden values
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("ahead,cut", CHUNK)
def test_prompt_seen_infinities_beside_hidden_values(hd, dtype, ahead, cut):
    """In one tile: a row sees an infinity of its own while later rows' values hold NaN or the opposite infinity in the same column."""
    cu_q, cu_k = [0, 200], [0, ahead + 200]
    q, k, v = _rand((200, 4, hd), dtype, 1, 2.0), _rand((ahead + 200, 2, hd), dtype, 2), _rand((ahead + 200, 2, hd), dtype, 3)
    t = v[ahead:]
    t[120, 0, 3], t[140, 0, 3] = INF, NAN
    t[110, 0, 5], t[150, 0, 5] = INF, -INF
    t[100, 0, 7], t[130, 0, 7] = -INF, INF
    t[125, 0, 9], t[131, 1, hd - 1], t[132, 1, hd - 1] = NAN, -INF, NAN
    assert _is_cut(q, k, cu_q, cu_k) == cut
    got = _prompt(q, k, v, cu_q, cu_k)
    _check(got, q, k, v, cu_q, cu_k)
    assert torch.equal(got.isnan(), _prompt(q, k, v, cu_q, cu_k, sm_budget=3).isnan())


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("ahead,cut", CHUNK)
def test_prompt_infinite_value_of_a_key_that_hardly_counts(hd, dtype, ahead, cut):
    """A weight below the smallest fp32 number times Inf is Inf; the weight of a key that scores -Inf is 0, and 0 x Inf NaN."""
    cu_q, cu_k = [0, 150], [0, ahead + 150]
    q = torch.full((150, 4, hd), 4.0).to(dtype)
    k, v = _rand((ahead + 150, 2, hd), dtype, 4, 0.25), _rand((ahead + 150, 2, hd), dtype, 5)
    at = ahead + 90
    k[at, 0], v[at, 0, 2] = -0.8 * hd ** 0.5, INF                     # score about -3.2 hd = -205 or -410
    k[at + 3, 1, 0], v[at + 3, 1, 4] = -INF, INF
    assert _is_cut(q, k, cu_q, cu_k) == cut
    _check(_prompt(q, k, v, cu_q, cu_k), q, k, v, cu_q, cu_k)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("ahead,cut", CHUNK)
def test_prompt_values_near_the_largest_number(hd, ahead, cut):
    """The weighted sum of the values passes the fp32 range although their mean does not."""
    cu_q, cu_k = [0, 150], [0, ahead + 150]
    q, k = _rand((150, 4, hd), torch.bfloat16, 6, 0.5), _rand((ahead + 150, 2, hd), torch.bfloat16, 7)
    v = (_rand((ahead + 150, 2, hd), torch.float32, 8).sign() * 0.2 + 0.7).mul(3.3e38).bfloat16()
    v[:, 1] = 3.0e38
    assert _is_cut(q, k, cu_q, cu_k) == cut
    got = _prompt(q, k, v, cu_q, cu_k)
    assert torch.isfinite(got).all()
    _check(got, q, k, v, cu_q, cu_k)


@pytest.mark.parametrize("hd,dtype", [(64, torch.bfloat16), (128, torch.float16)])
@pytest.mark.parametrize("lens", [[300, 40, 513, 1, 130], [90, 5, 260, 33, 1, 130, 77, 128, 129, 200, 64, 3]])
def test_prompt_second_looks_in_many_units(hd, dtype, lens):
    """Hidden NaN and infinities in every sequence and head; a CTA has one unit or many, dealt in order or by a list."""
    cu = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    q, k, v = _rand((cu[-1], 6, hd), dtype, 20, 2.0), _rand((cu[-1], 2, hd), dtype, 21), _rand((cu[-1], 2, hd), dtype, 22)
    for i, n in enumerate(lens):
        for g in range(2):
            v[cu[i] + n - 1, g, (3 * i + g) % hd] = (NAN, INF, -INF)[i % 3]
            v[cu[i] + n // 2, g, (5 * i + 7 * g) % hd] = (INF, NAN)[(i + g) % 2]
            k[cu[i] + n - 1, g, 1] = (1.0, NAN, INF)[i % 3]
    got = _prompt(q, k, v, cu, cu)
    _check(got, q, k, v, cu, cu)
    for budget in (1, 5, 60):
        again = _prompt(q, k, v, cu, cu, sm_budget=budget)
        assert torch.equal(got.isnan(), again.isnan()) and torch.equal(got[~got.isnan()], again[~got.isnan()])


def test_prompt_second_looks_that_take_longer_than_a_wait():
    """The rows of the last tile hide a NaN from one another, and each has 600000 keys: a warp's second looks take longer than a wait
    of the pipeline may, and its CTA has other units to do."""
    T, hd = 600_000, 64
    q, k, v = (_rand((T, 1, hd), torch.bfloat16, 23 + i) for i in range(3))
    v[T - 1, 0, 5], v[T - 40, 0, 6] = NAN, INF
    got = _prompt(q, k, v, [0, T], [0, T])
    assert torch.isnan(got[T - 1, 0, 5]) and (got[T - 40:, 0, 6] == INF).all()
    got[T - 1, 0, 5] = got[T - 40:, 0, 6] = 0.0
    assert torch.isfinite(got).all()
    for i in (T - 2, T - 41, T - 100, T - 200_000, T // 3):
        ref, mag, smax = LO.prompt_attention(q[i:i + 1], k[:i + 1], v[:i + 1], [0, 1], [0, i + 1], hd ** -0.5)
        err, tol = (got[i:i + 1].double() - ref).abs(), _prompt_tol(q, mag, smax, i + 1, 0.0)
        fin = torch.isfinite(ref)
        assert (err[fin] <= tol[fin]).all()


# ------------------------------------------------------------------------------------------------ prompts: references
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("later", [-200.0, -40.0, 3.0])
@pytest.mark.parametrize("lead,n,ahead,cut", [(1, 200, 0, False), (80, 200, 0, False), (165, 240, 0, False), (8960, 100, 8960, True)])
def test_prompt_first_keys_score_minus_infinity(hd, dtype, later, lead, n, ahead, cut):
    """Keys that score -Inf do not count, however many of them come first and however small the later scores are."""
    cu_q, cu_k = [0, n], [0, ahead + n]
    q = torch.ones(n, 4, hd).to(dtype)
    k = (_rand((ahead + n, 2, hd), torch.float32, 9, 0.2) + later / hd ** 0.5).to(dtype)
    k[:lead, :, 1] = -INF
    v = _rand((ahead + n, 2, hd), dtype, 10)
    assert _is_cut(q, k, cu_q, cu_k) == cut
    _check(_prompt(q, k, v, cu_q, cu_k), q, k, v, cu_q, cu_k)


@pytest.mark.parametrize("w24", [75.5, 6.5])
@pytest.mark.parametrize("hd,H,G,T,rows,cut", [(128, 8, 2, 20011, 20011, False), (64, 48, 6, 16009, 16009, False), (128, 4, 1, 24000, 3, True)])
def test_prompt_one_key_in_front_of_many_equal_ones_fp16(w24, hd, H, G, T, rows, cut):
    """The first key holds most of the weight and next to no value; what comes out is what thousands of keys with weights of w24 2^-24 have."""
    q = torch.ones(rows, H, hd).half()
    k, v = torch.zeros(T, G, hd).half(), (_rand((T, G, hd), torch.float32, 11).abs() * 0.2 + 0.8).half()
    k[0] = float(np.log(2.0 ** 24 / w24) / hd ** 0.5)
    v[0] = 2.0 ** -14
    cu_q, cu_k = [0, rows], [0, T]
    assert _is_cut(q, k, cu_q, cu_k) == cut
    got = _prompt(q, k, v, cu_q, cu_k).double()
    for i in (0, 1, 77, T // 2, T - 2, T - 1):
        if i < T - rows:
            continue
        r = i - (T - rows)
        ref, mag, smax = LO.prompt_attention(q[r:r + 1], k[:i + 1], v[:i + 1], [0, 1], [0, i + 1], hd ** -0.5)
        err, tol = (got[r:r + 1] - ref).abs(), _prompt_tol(q, mag, smax, i + 1, 2.0)
        assert (err <= tol).all(), (i, float((err / tol).max()))


# ------------------------------------------------------------------------------------------------ single tokens
def _cache(numbers, scales):
    import paper_2609_31551_b200 as P
    n, G, bs, hd = numbers[0].shape
    return P.KvCache(n, bs, G, hd, tensors=(numbers[0].cuda(), numbers[1].cuda(), scales[0].cuda(), scales[1].cuda()))


def _filled(n_blocks, G, bs, hd, seed):
    gen = torch.Generator().manual_seed(seed)
    numbers = [torch.randint(-127, 128, (n_blocks, G, bs, hd), generator=gen, dtype=torch.int8) for _ in range(2)]
    scales = [torch.rand(n_blocks, G, generator=gen) * 0.03 + 0.005 for _ in range(2)]
    return numbers, scales


def _token_bound(numbers, scales, q, lens, table):
    """The definition and each row's own bound: n, value scale and magnitude of what this row reads."""
    H, G, hd, bs = q.shape[1], numbers[0].shape[1], q.shape[2], numbers[0].shape[2]
    scale = hd ** -0.5
    ref, mag, smax = LO.cache_attention(q, numbers[0], numbers[1], scales[0], scales[1], lens, table, scale)
    top = torch.zeros(q.shape[:2], dtype=torch.float64)              # value scale of the token of the largest weight
    for s, n in enumerate(lens):
        if n <= 0:
            continue
        k = LO.cache_values(numbers[0], scales[0], table[s], n)
        vs = scales[1][table[s, torch.arange(n) // bs].long()].double().clamp_min(2.0 ** -100)       # [n, G]
        for h in range(H):
            g = h * G // H
            t = (k[:, g] @ q[s, h].double()) * scale * 1.4426950408889634 + vs[:, g].log2()
            top[s, h] = vs[t.argmax(), g]
    u = U[q.dtype]
    n_tok = torch.tensor([max(n, 0) for n in lens], dtype=torch.float64)
    tol = mag * (2.0 ** -11 + u * 1.01 + 2 * (hd + 8) * 2.0 ** -23 * smax[..., None] + 2.0 ** -17)
    return ref, tol + (1.1 * 2.0 ** -32 * 127 * n_tok[:, None] * top)[..., None] + (2.0 ** -25 if q.dtype == torch.float16 else 0.0)


def _check_tokens(numbers, scales, q, lens, table, c=None):
    c = c or _cache(numbers, scales)
    out = c.attention(q.cuda(), _dev(lens), table.cuda())
    c.check()
    ref, tol = _token_bound(numbers, scales, q, lens, table)
    err = (out.double().cpu() - ref).abs()
    assert (err <= tol).all(), float((err / tol.clamp_min(1e-300)).max())
    return out


@pytest.mark.parametrize("hd,group", [(64, 1), (128, 4), (128, 12)])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("w24", [40.5, 3.5])
@pytest.mark.parametrize("unequal", [False, True])
def test_token_one_place_in_front_of_many_equal_ones(hd, group, dtype, w24, unequal):
    """One place holds most of the weight and next to no value, 20000 others a weight of w24 2^-24 of it each; value scales equal, or of several sizes.
    More rows than the device has warps (every sequence reads the same blocks), so that most are one warp's from end to end."""
    bs, n, n_seqs, G = 128, 20000, 128, 16
    H, blocks = G * group, (n + bs - 1) // bs
    gen = torch.Generator().manual_seed(12)
    numbers = [torch.zeros(blocks, G, bs, hd, dtype=torch.int8), torch.randint(90, 128, (blocks, G, bs, hd), generator=gen, dtype=torch.int8)]
    scales = [torch.full((blocks, G), 0.01), torch.full((blocks, G), 0.01)]
    if unequal:
        scales[1][5::3] = 0.16
    numbers[0][0, :, 0], numbers[1][0, :, 0] = 127, 1
    scales[0][0] = float(np.log(2.0 ** 24 / w24) / (127 * hd ** 0.5))
    table = torch.arange(blocks, dtype=torch.int32).repeat(n_seqs, 1)
    c = _cache(numbers, scales)
    got = c.attention(torch.ones(n_seqs, H, hd).to(dtype).cuda(), _dev([n] * n_seqs), table.cuda()).double().cpu()
    c.check()
    ref, tol = _token_bound(numbers, scales, torch.ones(1, H, hd).to(dtype)[:, ::group], [n], table)
    err = (got - ref.repeat_interleave(group, 1)).abs()
    assert (err <= tol.repeat_interleave(group, 1)).all(), float((err / tol.repeat_interleave(group, 1)).max())


@pytest.mark.parametrize("dtype", DTYPES)
def test_token_value_scales_of_all_sizes_row_by_row(dtype):
    """Blocks whose value scales lie many powers of ten apart: each row within what its own blocks allow."""
    bs, hd, G, H = 16, 128, 2, 6
    numbers, scales = _filled(16, G, bs, hd, 13)
    exps = torch.tensor([-12.0, 0.0, -3.0, -30.0, 1.0, -6.0, -1.0, -20.0, 0.0, -2.0, -9.0, -4.0, 0.5, -0.5, -8.0, -5.0])
    if dtype == torch.float16:
        exps = exps.clamp_min(-6.0)
    scales[1] = (10.0 ** exps)[:, None].float().repeat(1, G)
    table = torch.tensor([[3, 14, 0, 7, 9, 1, 11, 5, 2, 10], [4, 6, 8, 12, 13, 15, 0, 0, 0, 0]], dtype=torch.int32)
    q = _rand((2, H, hd), dtype, 14)
    q[0, 0] *= 1e-3
    q[0, 1] *= 60.0
    q[1, 2] = 0.0
    _check_tokens(numbers, scales, q, [160, 83], table)


@pytest.mark.parametrize("hd,H,G", [(64, 4, 4), (128, 8, 1), (128, 12, 1)])
@pytest.mark.parametrize("scale", [2.6e36, 2.0 ** -100])
def test_token_value_scales_at_the_ends_of_their_range(hd, H, G, scale):
    """Values of up to 3.3e38, and the smallest scale that a store leaves."""
    bs, lens = 32, [5000, 17, 0, 9000]
    need = [(n + bs - 1) // bs for n in lens]
    numbers, scales = _filled(sum(need), G, bs, hd, 34)
    scales[1].fill_(scale)
    table = torch.zeros(len(lens), max(need), dtype=torch.int32)
    for i, n in enumerate(need):
        table[i, :n] = torch.arange(sum(need[:i]), sum(need[:i + 1]))
    out = _check_tokens(numbers, scales, _rand((len(lens), H, hd), torch.bfloat16, 35, 2.0), lens, table)
    assert float(out.abs().max()) > scale


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("H,G", [(2, 1), (12, 1)])
@pytest.mark.parametrize("dtype", DTYPES)
def test_token_queries_that_are_not_finite(hd, H, G, dtype):
    """Every score of such a row is Inf, -Inf or NaN, and so its softmax NaN; rows beside it and sequences without tokens do not notice."""
    bs, lens = 16, [600, 0, 30, 2100]
    need = [(n + bs - 1) // bs for n in lens]
    numbers, scales = _filled(sum(need), G, bs, hd, 15)
    numbers[0][..., 3] = numbers[0][..., 3].abs().clamp_min(1)            # a dimension in which all keys are positive
    table = torch.zeros(len(lens), max(need), dtype=torch.int32)
    for i, n in enumerate(need):
        table[i, :n] = torch.arange(sum(need[:i]), sum(need[:i + 1]))
    q = _rand((4, H, hd), dtype, 16, 2.0)
    c = _cache(numbers, scales)
    want = _check_tokens(numbers, scales, q, lens, table, c)
    for at, bad in ((0, INF), (0, NAN), (3, -INF), (3, INF)):
        for s in range(4):
            p = q.clone()
            p[s, 1, at] = bad
            out = c.attention(p.cuda(), _dev(lens), table.cuda())
            c.check()
            ref = want.clone()
            if lens[s]:
                ref[s, 1] = NAN
            assert torch.equal(out.isnan(), ref.isnan()) and torch.equal(out[~out.isnan()], ref[~out.isnan()])


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("H,G", [(32, 1), (64, 1), (71, 1), (66, 2), (16, 1)])
def test_token_many_heads_a_group(hd, dtype, H, G):
    bs, lens = 32, [700, 1, 0, 4100]
    need = [(n + bs - 1) // bs for n in lens]
    numbers, scales = _filled(sum(need) + 1, G, bs, hd, 17)
    perm = torch.randperm(sum(need) + 1, generator=torch.Generator().manual_seed(18)).to(torch.int32)
    table = torch.full((len(lens), max(need)), 10 ** 6, dtype=torch.int32)
    for i, n in enumerate(need):
        table[i, :n] = perm[sum(need[:i]):sum(need[:i + 1])]
    q = _rand((len(lens), H, hd), dtype, 19, 2.0)
    c = _cache(numbers, scales)
    out = _check_tokens(numbers, scales, q, lens, table, c)
    assert torch.equal(out, c.attention(q.cuda(), _dev(lens), table.cuda(), sm_budget=41))


def test_row_counts_and_starts_that_make_no_sense_are_refused():
    import paper_2609_31551_b200 as P
    c = P.KvCache(4, 16, 2, 64)
    x, t, cu, one = torch.zeros(3, 2, 64, dtype=torch.bfloat16, device="cuda"), _dev([[0, 1]]), _dev([0, 3]), _dev([5])
    for call in (lambda: c.load(cu, one, t, -1), lambda: c.load(cu, one, t, -1, out=(x, x.clone())), lambda: c.load(cu, _dev(5), t, 3), lambda: c.store(x, x, cu, _dev(5), t),
                 lambda: P.prompt_attention(x, x, x, [0, 2.5]), lambda: P.prompt_attention(x, x, x, np.array([0, 2 ** 32 + 3]))):
        with pytest.raises(P.EasError) as e:
            call()
        assert e.value.status == 1
    c.check()


def test_token_and_store_calls_follow_one_another_without_a_pause():
    """Each store grows the scale of a block that the attention behind it reads, and nothing waits between them on the host."""
    import paper_2609_31551_b200 as P
    G, H, hd, bs, n, steps = 16, 32, 128, 16, 40, 64
    blocks = (steps + bs - 1) // bs
    table = torch.arange(n * blocks, dtype=torch.int32).view(n, blocks).cuda()
    rows = [(_rand((n, G, hd), torch.bfloat16, 500 + t, 1.0 + t).cuda(), _rand((n, G, hd), torch.bfloat16, 700 + t, 1.0 + t).cuda()) for t in range(steps)]
    q, cu = _rand((n, H, hd), torch.bfloat16, 24).cuda(), _dev(np.arange(n + 1))
    at, lens = [_dev([t] * n) for t in range(steps)], [_dev([t + 1] * n) for t in range(steps)]
    seen = []
    for paused in (True, False):
        c = P.KvCache(n * blocks, bs, G, hd)
        outs = []
        for t in range(steps):
            c.store(rows[t][0], rows[t][1], cu, at[t], table)
            if paused:
                torch.cuda.synchronize()
            outs.append(c.attention(q, lens[t], table))
            if paused:
                torch.cuda.synchronize()
        c.check()
        seen.append(torch.stack(outs))
    assert torch.equal(seen[0], seen[1])


# ------------------------------------------------------------------------------------------------ calls at the end of what is allowed
@pytest.mark.parametrize("hd", [64, 128])
def test_prompt_without_any_key_gives_zeros(hd):
    import paper_2609_31551_b200 as P
    q = _rand((40, 4, hd), torch.bfloat16, 25)
    k = torch.zeros(0, 2, hd, dtype=torch.bfloat16)
    out = torch.full((40, 4, hd), 7.0, dtype=torch.bfloat16, device="cuda")
    got, status = P.prompt_attention(q.cuda(), k.cuda(), k.cuda(), [1, 30, 39], [0, 0, 0], out=out)
    assert int(status[0]) == 0 and not got[1:39].any() and (got[0] == 7).all() and (got[39] == 7).all()


@pytest.mark.parametrize("hd", [64, 128])
def test_prompt_of_two_launches_that_are_both_cut(hd):
    """More sequences than a launch holds: both launches leave their parts in one workspace."""
    import paper_2609_31551_b200 as P
    lens, keys = [1 + i % 3 for i in range(140)], [3500 - 7 * i for i in range(140)]
    keys[77] = 40000
    cu_q, cu_k = (np.concatenate([[0], np.cumsum(x)]).astype(np.int32) for x in (lens, keys))
    q = _rand((cu_q[-1], 2, hd), torch.float16, 26, 2.0)
    k, v = _rand((cu_k[-1], 1, hd), torch.float16, 27), _rand((cu_k[-1], 1, hd), torch.float16, 28)
    order = sorted(range(140), key=lambda i: -keys[i])
    for part in (order[:128], order[128:]):
        assert P.prompt_attention_workspace_bytes(2, 1, hd, *(np.concatenate([[0], np.cumsum([x[i] for i in part])]) for x in (lens, keys))) > 0
    _check(_prompt(q, k, v, cu_q, cu_k), q, k, v, cu_q, cu_k)


def test_cache_calls_about_nothing():
    import paper_2609_31551_b200 as P
    numbers, scales = _filled(3, 2, 16, 64, 29)
    c = _cache(numbers, scales)
    x, q = torch.zeros(0, 2, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(0, 4, 64, dtype=torch.bfloat16, device="cuda")
    none, table = torch.zeros(0, dtype=torch.int32, device="cuda"), torch.zeros(0, 5, dtype=torch.int32, device="cuda")
    c.store(x, x, _dev([0]), none, table)
    assert c.load(_dev([0]), none, table, 0)[0].shape == (0, 2, 64) and c.attention(q, none, table).shape == (0, 4, 64)
    no_blocks = torch.zeros(2, 0, dtype=torch.int32, device="cuda")
    q = _rand((2, 4, 64), torch.bfloat16, 30).cuda()
    assert not c.attention(q, _dev([0, 0]), no_blocks).any()
    c.store(x, x, _dev([0, 0, 0]), _dev([0, 5]), no_blocks)
    c.check()
    assert not c.attention(q, _dev([0, 3]), no_blocks).any()
    with pytest.raises(P.EasError) as e:
        c.check()
    assert e.value.status == 7
    assert torch.equal(c.k.cpu(), numbers[0]) and torch.equal(c.v_scale.cpu(), scales[1])


def test_cut_prompt_captured_and_replayed():
    import paper_2609_31551_b200 as P
    cu_q, cu_k = [0, 60, 61], [0, 4000, 4100]
    q, k, v = _rand((61, 16, 128), torch.bfloat16, 31).cuda(), _rand((4100, 4, 128), torch.bfloat16, 32).cuda(), _rand((4100, 4, 128), torch.bfloat16, 33).cuda()
    ws = torch.empty(P.prompt_attention_workspace_bytes(16, 4, 128, cu_q, cu_k), dtype=torch.uint8, device="cuda")
    P.prompt_attention(q, k, v, cu_q, cu_k)
    torch.cuda.synchronize()
    graphs = []
    for space in (ws, ws, None):                                        # two on one workspace, one with its own
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out, status = P.prompt_attention(q, k, v, cu_q, cu_k, workspace=space)
        graphs.append((g, out, status))
    for i in range(3):
        q.copy_(q.flip(1))
        v.copy_(v.flip(0))
        want = P.prompt_attention(q, k, v, cu_q, cu_k)[0]
        ws.fill_(0xFF)
        for g, out, status in graphs:
            g.replay()
        torch.cuda.synchronize()
        for g, out, status in graphs:
            assert torch.equal(out, want) and int(status[0]) == 0


def test_decoding_steps_captured_once_and_replayed():
    """A step of a server in one graph: rows stored at the lengths, the lengths raised, attention over them, and the rows read back."""
    import paper_2609_31551_b200 as P
    G, H, hd, bs, n, steps = 4, 16, 64, 16, 5, 40
    blocks = (steps + 30 + bs - 1) // bs
    table = torch.randperm(n * blocks, generator=torch.Generator().manual_seed(36)).to(torch.int32).view(n, blocks).cuda()
    first = _dev([0, 3, 16, 29, 30])
    cu, cu_all = _dev(np.arange(n + 1)), _dev([0, 20, 20, 20, 20, 20])
    rows = [[_rand((n, h, hd), torch.float16, 800 + 3 * t + i, 1.0 + 0.1 * t).cuda() for i, h in enumerate((H, G, G))] for t in range(steps)]
    caches = [P.KvCache(n * blocks, bs, G, hd) for _ in range(2)]

    def step(c, q, k, v, lens):
        c.store(k, v, cu, lens, table)
        lens.add_(1)
        out = c.attention(q, lens, table)
        return out, *c.load(cu_all, first.new_zeros(n), table, 20, dtype=torch.float16)
    lens, want = first.clone(), []
    for t in range(steps):
        want.append([x.clone() for x in step(caches[0], *rows[t], lens)])
    caches[0].check()
    held, live = [x.clone() for x in rows[0]], first.clone()
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        outs = step(caches[1], *held, live)
    live.copy_(first)
    for t in range(steps):
        for x, y in zip(held, rows[t]):
            x.copy_(y)
        g.replay()
        for x, y in zip(outs, want[t]):
            assert torch.equal(x, y)
    caches[1].check()
    assert torch.equal(caches[0].k, caches[1].k) and torch.equal(caches[0].v_scale, caches[1].v_scale) and torch.equal(live, lens)
