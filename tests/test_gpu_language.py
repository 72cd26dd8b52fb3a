"""The language-model operators on a GPU against the fp64 oracle.

Bounds.  u = eps / 2 of the data type is the largest relative error of one rounding to it (bf16 2^-8, fp16 2^-11).  An output element is
sum p v / sum p.  With A the attention over |v|:
  - the probabilities are rounded once (prompts: to the data type, cache: to fp16), sums are not:   u_p A
  - the output is rounded once:                                                                  u |out| <= u A
  - a score is a sum of head_dim products in fp32, 2^-23 an addition (the matrix unit may truncate), of magnitude smax = max sum |q k| scale; it
    moves a probability by as much, relatively, twice (numerator and sum):                             2 (head_dim + 8) 2^-23 smax A
  - exponentials, logarithms, reciprocal, the products and rescalings around them, the fp32 sums over n keys
    (a running sum of n positive terms, cut into steps of 80 or tiles of 16 and lanes):                  2^-17 A
  - fp16 probabilities below 2^-14 are rounded to multiples of 2^-24; the reference is at most the row's maximum, so sum p >= 1:   n 2^-25 max |v|
"""
import numpy as np
import pytest
import torch

from oracle import language_oracle as LO

pytestmark = pytest.mark.gpu
U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
DTYPES = [torch.bfloat16, torch.float16]


def _bound(mag, smax, hd, u_p, u_out, n, vmax, half_p):
    rel = u_p + u_out * 1.01 + 2 * (hd + 8) * 2.0 ** -23 * smax[..., None] + 2.0 ** -17
    return mag * rel + (n * 2.0 ** -25 * vmax if half_p else 0.0) + 2.0 ** -24 * (u_out == 2.0 ** -11)   # (fp16 outputs below 2^-14: half of 2^-24, and margin)


def _rand(shape, dtype, seed, scale=1.0):
    gen = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=gen) * scale).to(dtype)


def _cu(lens):
    return np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)


# ------------------------------------------------------------------------------------------------ prompts
def _check_prompt(q, k, v, cu_q, cu_k, out, scale, rows=None):
    ref, mag, smax = LO.prompt_attention(q, k, v, cu_q, cu_k, scale)
    named = ~torch.isnan(ref[:, 0, 0])
    got = out.double().cpu()
    assert torch.isfinite(got[named]).all()
    n = int(max(np.diff(cu_k)))
    tol = _bound(mag, smax, q.shape[2], U[q.dtype], U[q.dtype], n, float(v.float().abs().max()) if len(v) else 0.0, q.dtype == torch.float16)
    err = (got - ref).abs()
    assert (err[named] <= tol[named]).all(), float((err / tol)[named].max())


PROMPTS = [
    ([1], None), ([39], None), ([80, 81, 1], None), ([129, 0, 127, 128], None), ([0, 3, 0, 0], None), ([333], None), ([1, 1, 1, 1, 1], None),
    ([17], [400]), ([1, 16, 130], [1, 257, 130]), ([9, 5], [4, 0]), ([200], [71]), ([64, 3], [64 + 80, 3 + 159]),
]


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("H,G", [(2, 2), (8, 2), (5, 1), (16, 2)])
@pytest.mark.parametrize("lens,keys", PROMPTS)
def test_prompt_attention(hd, dtype, H, G, lens, keys):
    import paper_2609_31551_b200 as P
    cu_q, cu_k = _cu(lens), _cu(keys or lens)
    q = _rand((cu_q[-1], H, hd), dtype, 1, 2.0)
    k, v = _rand((cu_k[-1], G, hd), dtype, 2), _rand((cu_k[-1], G, hd), dtype, 3)
    args = (q.cuda(), k.cuda(), v.cuda(), cu_q, cu_k)
    out, status = P.prompt_attention(*args)
    torch.cuda.synchronize()
    assert int(status[0]) == 0
    _check_prompt(q, k, v, cu_q, cu_k, out, hd ** -0.5)
    for budget in (1, 3, 74):
        again, status = P.prompt_attention(*args, sm_budget=budget)
        assert int(status[0]) == 0 and torch.equal(out, again)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("H,G", [(3, 1), (7, 1), (12, 1), (33, 1), (128, 1), (65, 1)])
def test_prompt_attention_odd_groups(hd, H, G):
    import paper_2609_31551_b200 as P
    lens = [45, 7, 1]
    cu = _cu(lens)
    q, k, v = _rand((cu[-1], H, hd), torch.bfloat16, 4, 2.0), _rand((cu[-1], G, hd), torch.bfloat16, 5), _rand((cu[-1], G, hd), torch.bfloat16, 6)
    out, status = P.prompt_attention(q.cuda(), k.cuda(), v.cuda(), cu)
    assert int(status[0]) == 0
    _check_prompt(q, k, v, cu, cu, out, hd ** -0.5)


@pytest.mark.parametrize("hd", [64, 128])
def test_prompt_attention_reads_views_and_leaves_other_rows_alone(hd):
    import paper_2609_31551_b200 as P
    H, G, lens = 4, 2, [50, 30]
    T, cu = 100, _cu(lens) + 10
    x = _rand((T, (H + 2 * G) * hd + 24), torch.bfloat16, 7)
    x[:10], x[90:] = float("nan"), float("nan")                      # rows of no sequence, in front and behind
    xd = x.cuda()

    def thirds(t):
        return (t[:, 8:8 + H * hd].view(T, H, hd), t[:, 8 + H * hd:8 + (H + G) * hd].view(T, G, hd), t[:, 8 + (H + G) * hd:8 + (H + 2 * G) * hd].view(T, G, hd))
    buf = torch.full((T, H * hd + 16), 5.0, dtype=torch.bfloat16, device="cuda")
    out = buf[:, :H * hd].view(T, H, hd)
    got, status = P.prompt_attention(*thirds(xd), cu, out=out, scale=0.2)
    assert int(status[0]) == 0 and got is out
    _check_prompt(*thirds(x), cu, cu, out, 0.2)
    rest = buf.clone()
    rest[10:90, :H * hd] = 5.0
    assert (rest == 5.0).all()


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("offset,gap", [(8, 0), (0, 8), (8, 8), (24, 40), (16, 16)])
@pytest.mark.parametrize("lens,keys", [([150, 3], None), ([40], [9000])])
def test_prompt_attention_output_rows_on_any_16_byte_boundary(hd, offset, gap, lens, keys):
    import paper_2609_31551_b200 as P
    H, G = 10, 2
    cu_q, cu_k = _cu(lens), _cu(keys or lens)
    T = int(cu_q[-1])
    q, k, v = _rand((T, H, hd), torch.float16, 70, 2.0), _rand((cu_k[-1], G, hd), torch.float16, 71), _rand((cu_k[-1], G, hd), torch.float16, 72)
    want = P.prompt_attention(q.cuda(), k.cuda(), v.cuda(), cu_q, cu_k)[0]
    flat = torch.full((offset + T * (H * hd + gap),), 5.0, dtype=torch.float16, device="cuda")
    buf = flat[offset:].view(T, H * hd + gap)
    out, status = P.prompt_attention(q.cuda(), k.cuda(), v.cuda(), cu_q, cu_k, out=buf[:, :H * hd].view(T, H, hd))
    assert int(status[0]) == 0 and torch.equal(out, want)
    assert (flat[:offset] == 5.0).all() and (buf[:, H * hd:] == 5.0).all()


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("H,G", [(2, 2), (8, 1)])
@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
@pytest.mark.parametrize("where", ["behind in the sequence", "first key of the next sequence"])
def test_prompt_attention_non_finite_values_reach_only_rows_that_see_them(hd, H, G, bad, where):
    import paper_2609_31551_b200 as P
    lens = [200, 40]
    cu = _cu(lens)
    q, k, v = _rand((240, H, hd), torch.bfloat16, 8, 2.0), _rand((240, G, hd), torch.bfloat16, 9), _rand((240, G, hd), torch.bfloat16, 10)
    clean = P.prompt_attention(q.cuda(), k.cuda(), v.cuda(), cu)[0].cpu()
    at = 100 if where == "behind in the sequence" else 200
    k[at, 0, 3], v[at, 0, 5], v[at, 0, hd - 1] = bad, bad, bad
    out, status = P.prompt_attention(q.cuda(), k.cuda(), v.cuda(), cu)
    out = out.cpu()
    assert int(status[0]) == 0
    end = 200 if at == 100 else 240
    blind = torch.ones(240, H, dtype=torch.bool)
    blind[at:end, :H // G] = False
    ref, mag, smax = LO.prompt_attention(q, k, v, cu, cu, hd ** -0.5)
    tol = _bound(mag, smax, hd, U[q.dtype], U[q.dtype], 200, 5.0, False)
    assert torch.isfinite(out[blind]).all()
    assert ((out.double() - ref).abs()[blind] <= tol[blind]).all()
    far = blind.clone()
    far[max(0, at - 128):at] = False                                   # rows of other tiles keep their bits
    assert torch.equal(out[far], clean[far])
    if bad != bad:
        assert torch.isnan(out[at:end, :H // G]).any(-1).all()


@pytest.mark.parametrize("hd,dtype", [(64, torch.float16), (128, torch.bfloat16)])
def test_prompt_attention_value_infinity_alone(hd, dtype):
    """Only v holds Inf: rows that see it get Inf in that element and the others' values elsewhere; rows that do not, nothing of it."""
    import paper_2609_31551_b200 as P
    cu = _cu([150])
    q, k, v = _rand((150, 4, hd), dtype, 11), _rand((150, 1, hd), dtype, 12), _rand((150, 1, hd), dtype, 13)
    v[120, 0, 7] = float("inf")
    out = P.prompt_attention(q.cuda(), k.cuda(), v.cuda(), cu)[0].double().cpu()
    ref, mag, smax = LO.prompt_attention(q, k, v, cu, cu, hd ** -0.5)
    assert (out[120:, :, 7] == float("inf")).all()
    fin = torch.isfinite(ref)
    assert torch.isfinite(out[fin]).all()
    tol = _bound(mag, smax, hd, U[dtype], U[dtype], 150, 5.0, dtype == torch.float16)
    assert ((out - ref).abs()[fin] <= tol[fin]).all()


@pytest.mark.parametrize("hd", [64, 128])
def test_prompt_attention_large_and_growing_scores(hd):
    """Row maxima that rise by far more than 2^8 in the exponent from step to step, and rows dominated by one key."""
    import paper_2609_31551_b200 as P
    T = 500
    q = torch.ones(T, 2, hd, dtype=torch.bfloat16)
    k = (torch.arange(T)[:, None, None] * torch.ones(1, 1, hd) * (40.0 / T)).bfloat16()
    v = _rand((T, 1, hd), torch.bfloat16, 14)
    cu = _cu([T])
    for sign in (1, -1):
        kk = k * sign
        out, status = P.prompt_attention(q.cuda(), kk.cuda(), v.cuda(), cu)
        assert int(status[0]) == 0
        _check_prompt(q, kk, v, cu, cu, out, hd ** -0.5)


@pytest.mark.parametrize("hd", [64, 128])
def test_prompt_attention_does_not_depend_on_the_packing(hd):
    import paper_2609_31551_b200 as P
    lens = [300, 40, 513, 1]
    cu = _cu(lens)
    q, k, v = (_rand((cu[-1], h, hd), torch.bfloat16, 15 + h).cuda() for h in (6, 2, 2))
    out = P.prompt_attention(q, k, v, cu)[0]
    for i in range(len(lens)):
        a, b = cu[i], cu[i + 1]
        assert torch.equal(out[a:b], P.prompt_attention(q[a:b], k[a:b], v[a:b], [0, b - a])[0])
    # a prompt in two chunks, the second behind the keys of the first
    a, m, b = cu[2], cu[2] + 200, cu[3]
    two = P.prompt_attention(q[m:b], k[a:b], v[a:b], [0, b - m], [0, b - a])[0]
    assert torch.equal(out[m:b], two)


def test_prompt_attention_of_many_short_sequences():
    import paper_2609_31551_b200 as P
    lens = [(7 * i) % 23 for i in range(300)]                           # more than one launch's worth, empty ones among them
    cu = _cu(lens)
    q, k, v = _rand((cu[-1], 4, 64), torch.float16, 20), _rand((cu[-1], 2, 64), torch.float16, 21), _rand((cu[-1], 2, 64), torch.float16, 22)
    out, status = P.prompt_attention(q.cuda(), k.cuda(), v.cuda(), cu)
    assert int(status[0]) == 0
    _check_prompt(q, k, v, cu, cu, out, 0.125)


@pytest.mark.parametrize("lens,G", [([2500] + [1] * 110, 16), ([700, 30, 1, 250, 90] * 5, 8), ([129] * 60 + [1000], 5)])
def test_prompt_attention_units_of_unequal_cost(lens, G):
    """Lists with empty entries, and (the first) more rounds than a list holds."""
    import paper_2609_31551_b200 as P
    rng = np.random.Generator(np.random.PCG64(12))
    lens = [lens[i] for i in rng.permutation(len(lens))]
    cu = _cu(lens)
    q, k, v = (_rand((cu[-1], G, 64), torch.float16, 90 + i, 1.5) for i in range(3))
    args = (q.cuda(), k.cuda(), v.cuda(), cu)
    out, status = P.prompt_attention(*args)
    assert int(status[0]) == 0
    _check_prompt(q, k, v, cu, cu, out, 0.125)
    for budget in (5, 100):
        again, status = P.prompt_attention(*args, sm_budget=budget)
        assert int(status[0]) == 0 and torch.equal(out, again)


def test_prompt_attention_long_sequence_tail_rows():
    """20 011 keys (some 250 steps a tile): the last rows and some others against the oracle."""
    import paper_2609_31551_b200 as P
    T, hd = 20011, 128
    q, k, v = _rand((T, 8, hd), torch.bfloat16, 23, 1.5), _rand((T, 2, hd), torch.bfloat16, 24), _rand((T, 2, hd), torch.bfloat16, 25)
    out, status = P.prompt_attention(q.cuda(), k.cuda(), v.cuda(), [0, T])
    assert int(status[0]) == 0
    for i in (0, 1, 79, 80, 4095, 12345, T - 2, T - 1):
        ref, mag, smax = LO.prompt_attention(q[i:i + 1], k[:i + 1], v[:i + 1], [0, 1], [0, i + 1], hd ** -0.5)
        tol = _bound(mag, smax, hd, U[q.dtype], U[q.dtype], T, 0.0, False)
        assert ((out[i:i + 1].double().cpu() - ref).abs() <= tol).all()


@pytest.mark.parametrize("hd,dtype", [(64, torch.float16), (128, torch.bfloat16), (128, torch.float16)])
@pytest.mark.parametrize("H,G,lens,keys", [(10, 2, [40], [9000]), (8, 8, [5, 0, 33], [4001, 77, 6000]), (4, 1, [1], [12345]), (3, 1, [131], [2400]), (8, 2, [60, 20], [2500, 3])])
def test_prompt_attention_few_queries_many_keys(hd, dtype, H, G, lens, keys):
    """Too few tiles for the device: the key steps are cut and joined (workspace), rows that see few or no keys among them."""
    import paper_2609_31551_b200 as P
    cu_q, cu_k = _cu(lens), _cu(keys)
    need = P.prompt_attention_workspace_bytes(H, G, hd, cu_q, cu_k)
    assert need > 0
    q = _rand((cu_q[-1], H, hd), dtype, 1, 2.0)
    k, v = _rand((cu_k[-1], G, hd), dtype, 2), _rand((cu_k[-1], G, hd), dtype, 3)
    args = (q.cuda(), k.cuda(), v.cuda(), cu_q, cu_k)
    out, status = P.prompt_attention(*args)
    assert int(status[0]) == 0
    _check_prompt(q, k, v, cu_q, cu_k, out, hd ** -0.5)
    ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")     # whatever the workspace holds
    for budget in (1, 50):
        again, status = P.prompt_attention(*args, sm_budget=budget, workspace=ws)
        assert int(status[0]) == 0 and torch.equal(out, again)
    with pytest.raises(P.EasError) as e:
        P.prompt_attention(*args, workspace=ws[:need - 256])
    assert e.value.status == 3


@pytest.mark.parametrize("hd,H,G,seed", [(64, 8, 2, 1), (128, 8, 2, 2), (128, 5, 5, 3), (64, 24, 3, 4), (128, 4, 1, 5)])
def test_prompt_attention_cut_lines_of_many_units(hd, H, G, seed):
    """Units of very different lengths, some without keys, so that a piece of the line holds ends, whole units and beginnings."""
    import paper_2609_31551_b200 as P
    rng = np.random.Generator(np.random.PCG64(seed))
    n = int(rng.integers(3, 30))
    lens = [int(x) for x in rng.choice([0, 1, 2, 7, 40, 130], n)]
    keys = [int(x) for x in rng.integers(1, 600, n)]
    keys[1], keys[2], lens[1], lens[2] = 9000, 0, 33, 5
    cu_q, cu_k = _cu(lens), _cu(keys)
    assert P.prompt_attention_workspace_bytes(H, G, hd, cu_q, cu_k) > 0
    q = _rand((cu_q[-1], H, hd), torch.bfloat16, 75, 2.0)
    k, v = _rand((cu_k[-1], G, hd), torch.bfloat16, 76), _rand((cu_k[-1], G, hd), torch.bfloat16, 77)
    args = (q.cuda(), k.cuda(), v.cuda(), cu_q, cu_k)
    out, status = P.prompt_attention(*args)
    assert int(status[0]) == 0
    _check_prompt(q, k, v, cu_q, cu_k, out, hd ** -0.5)
    for budget in (1, 20, 147):
        again, status = P.prompt_attention(*args, sm_budget=budget)
        assert int(status[0]) == 0 and torch.equal(out, again)


@pytest.mark.parametrize("hd", [64, 128])
def test_prompt_attention_split_and_non_finite_values(hd):
    import paper_2609_31551_b200 as P
    cu_q, cu_k = _cu([50]), _cu([5000])
    q, k, v = _rand((50, 4, hd), torch.bfloat16, 4, 2.0), _rand((5000, 2, hd), torch.bfloat16, 5), _rand((5000, 2, hd), torch.bfloat16, 6)
    v[4980, 0, 3], k[4990, 1, 5], v[100, 1, 9] = float("inf"), float("nan"), float("-inf")
    assert P.prompt_attention_workspace_bytes(4, 2, hd, cu_q, cu_k) > 0
    out, status = P.prompt_attention(q.cuda(), k.cuda(), v.cuda(), cu_q, cu_k)
    assert int(status[0]) == 0
    out = out.double().cpu()
    ref, mag, smax = LO.prompt_attention(q, k, v, cu_q, cu_k, hd ** -0.5)
    assert (out[30:, :2, 3] == float("inf")).all() and (out[:40, 2:, 9] == float("-inf")).all() and torch.isnan(out[40:, 2:]).any(-1).all()
    fin = torch.isfinite(ref)
    tol = _bound(mag, smax, hd, U[q.dtype], U[q.dtype], 5000, 5.0, False)
    assert torch.isfinite(out[fin]).all() and ((out - ref).abs()[fin] <= tol[fin]).all()


def test_prompt_attention_other_stream_and_graph():
    import paper_2609_31551_b200 as P
    cu = _cu([100, 33])
    q, k, v = (_rand((133, h, 128), torch.bfloat16, 30 + h).cuda() for h in (4, 2, 2))
    want = P.prompt_attention(q, k, v, cu)[0]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got, _ = P.prompt_attention(q, k, v, cu, stream=side)
    side.synchronize()
    assert torch.equal(got, want)
    status = torch.zeros(4, dtype=torch.int32, device="cuda")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out, _ = P.prompt_attention(q, k, v, cu, status=status)
    q.copy_(q.flip(0))
    want = P.prompt_attention(q, k, v, cu)[0]
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want) and int(status[0]) == 0


def test_prompt_attention_refusals():
    import paper_2609_31551_b200 as P
    x = torch.zeros(8, 2, 64, dtype=torch.bfloat16, device="cuda")
    for call in (lambda: P.prompt_attention(x.float(), x, x, [0, 8]), lambda: P.prompt_attention(x, x.half(), x, [0, 8]),
                 lambda: P.prompt_attention(x, x, x, [0, 9]), lambda: P.prompt_attention(x, x[:, :1], x, [0, 8]),
                 lambda: P.prompt_attention(x, x, x, [0, 8], [0, 4, 8]), lambda: P.prompt_attention(x, x, x, [0, 8], scale=0.0),
                 lambda: P.prompt_attention(x, x, x, [0, 8], sm_budget=1000), lambda: P.prompt_attention(x, x, x, [0, 8], out=x[:4]),
                 lambda: P.prompt_attention(x.transpose(1, 2), x, x, [0, 8]), lambda: P.prompt_attention(x, x, x, [0, 5, 4])):
        with pytest.raises(P.EasError) as e:
            call()
        assert e.value.status == 1
    y = torch.zeros(8, 2, 80, dtype=torch.bfloat16, device="cuda")
    with pytest.raises(P.EasError) as e:
        P.prompt_attention(y, y, y, [0, 8])
    assert e.value.status == 2
    for status in (torch.zeros(4, dtype=torch.int32), torch.zeros(4, device="cuda"), torch.zeros(0, dtype=torch.int32, device="cuda")):
        with pytest.raises(P.EasError) as e:
            P.prompt_attention(x, x, x, [0, 8], status=status)
        assert e.value.status == 1
    out, _ = P.prompt_attention(x[:0], x[:0], x[:0], [0])               # no sequence, no row: nothing to do
    assert out.shape == (0, 2, 64)


# ------------------------------------------------------------------------------------------------ the cache
def _table(rng, lens, bs, n_blocks):
    need = [(n + bs - 1) // bs for n in lens]
    perm = rng.permutation(n_blocks)
    table = np.full((len(lens), max(need + [1])), 10 ** 6, dtype=np.int32)       # unused entries point outside: never read
    at = 0
    for i, n in enumerate(need):
        table[i, :n] = perm[at:at + n]
        at += n
    assert at <= n_blocks
    return torch.from_numpy(table)


def _dev(x):
    return torch.as_tensor(np.asarray(x), dtype=torch.int32).cuda()


def _filled(n_blocks, G, bs, hd, seed):
    gen = torch.Generator().manual_seed(seed)
    numbers = [torch.randint(-127, 128, (n_blocks, G, bs, hd), generator=gen, dtype=torch.int8) for _ in range(2)]
    scales = [torch.rand(n_blocks, G, generator=gen) * 0.03 + 0.005 for _ in range(2)]
    return numbers, scales


def _cache(numbers, scales):
    import paper_2609_31551_b200 as P
    n, G, bs, hd = numbers[0].shape
    return P.KvCache(n, bs, G, hd, tensors=(numbers[0].cuda(), numbers[1].cuda(), scales[0].cuda(), scales[1].cuda()))


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("bs", [16, 32, 64, 128])
@pytest.mark.parametrize("lens,before", [([1], [0]), ([1, 1, 1], [5, 0, 31]), ([40, 0, 129], [0, 7, 3]), ([300, 2], [17, 127]), ([16, 128], [16, 0])])
def test_cache_store_and_load_are_exact(hd, dtype, bs, lens, before):
    """The numbers and scales are the oracle's, bit for bit; what the call does not name stays as it was."""
    G = 3
    rng = np.random.Generator(np.random.PCG64(bs + hd + sum(lens)))
    held = [a + b for a, b in zip(lens, before)]
    n_blocks = sum((n + bs - 1) // bs for n in held) + 3
    table = _table(rng, held, bs, n_blocks)
    numbers, scales = _filled(n_blocks, G, bs, hd, 40)
    c = _cache(numbers, scales)
    cu = _cu(lens)
    k, v = (_rand((cu[-1], G, hd), dtype, s) * torch.rand(cu[-1], G, 1, generator=torch.Generator().manual_seed(s)).mul(4).exp().to(dtype) for s in (41, 42))
    k[::3] *= 0.0625                                                    # tokens that leave the scale alone, and ones that raise it
    c.store(k.cuda(), v.cuda(), _dev(cu), _dev(before), table.cuda())
    c.check()
    for x, num, sc in ((k, numbers[0], scales[0]), (v, numbers[1], scales[1])):
        LO.cache_store(num, sc, x, cu, before, table)
    assert torch.equal(c.k_scale.cpu(), scales[0]) and torch.equal(c.v_scale.cpu(), scales[1])
    assert torch.equal(c.k.cpu(), numbers[0]) and torch.equal(c.v.cpu(), numbers[1])
    # and back: all tokens, then a part
    for starts, parts in (([0] * len(lens), held), (before, lens)):
        cu_h = _cu(parts)
        kk, vv = c.load(_dev(cu_h), _dev(starts), table.cuda(), int(cu_h[-1]), dtype=dtype)
        for got, num, sc in ((kk, numbers[0], scales[0]), (vv, numbers[1], scales[1])):
            for i in range(len(lens)):
                want = LO.cache_values(num, sc, table[i], starts[i] + parts[i])[starts[i]:]
                assert torch.equal(got[cu_h[i]:cu_h[i + 1]].cpu(), want.float().to(dtype))      # number * scale in fp32, one more rounding
    c.check()
    for budget in (1, 5):
        d = _cache(*_filled(n_blocks, G, bs, hd, 40))
        d.store(k.cuda(), v.cuda(), _dev(cu), _dev(before), table.cuda(), sm_budget=budget)
        assert torch.equal(d.k, c.k) and torch.equal(d.v_scale, c.v_scale)


@pytest.mark.parametrize("dtype", DTYPES)
def test_cache_store_ties_zeros_and_extremes(dtype):
    """Halves of the largest value are ties of 63.5 steps up to the scale's own rounding; blocks of zeros; the type's largest and smallest numbers."""
    bs, hd, G = 16, 64, 1
    info = torch.finfo(dtype)
    x = torch.zeros(6 * bs, G, hd, dtype=dtype)
    for b, top in enumerate([1.0, 1.2734375, 0.0, info.max, info.tiny, info.smallest_normal / 128 if dtype == torch.bfloat16 else 2.0 ** -24]):
        blk = x[b * bs:(b + 1) * bs]
        blk.copy_((torch.linspace(-1, 1, bs * hd).view(bs, 1, hd) * top).to(dtype))
        blk[0, 0, 0], blk[0, 0, 1], blk[0, 0, 2] = top, top / 2, -top / 2
    numbers, scales = _filled(8, G, bs, hd, 44)
    table = torch.tensor([[7, 2, 3, 0, 6, 1]], dtype=torch.int32)
    c = _cache(numbers, scales)
    c.store(x.cuda(), x.cuda(), _dev([0, 6 * bs]), _dev([0]), table.cuda())
    c.check()
    LO.cache_store(numbers[0], scales[0], x, [0, 6 * bs], [0], table)
    assert torch.equal(c.k_scale.cpu(), scales[0])
    assert torch.equal(c.k.cpu(), numbers[0])


def test_cache_store_non_finite_values_stay_in_their_block_and_head():
    bs, hd, G = 16, 64, 2
    c = _cache(*_filled(4, G, bs, hd, 45))
    x = _rand((48, G, hd), torch.bfloat16, 46)
    x[20, 1, 3], x[40, 0, 0] = float("inf"), float("nan")
    c.store(x.cuda(), x.cuda(), _dev([0, 48]), _dev([0]), _dev([[0, 1, 2]]))
    c.check()
    k, _ = c.load(_dev([0, 48]), _dev([0]), _dev([[0, 1, 2]]), 48)
    fine = torch.ones(48, G, dtype=torch.bool)
    fine[16:32, 1], fine[32:48, 0] = False, False
    k = k.cpu()
    assert torch.isfinite(k[fine]).all() and torch.isnan(k[~fine]).all()


def test_cache_calls_skip_and_report_what_lies_outside():
    import paper_2609_31551_b200 as P
    bs, hd, G = 16, 64, 2
    x = _rand((40, G, hd), torch.bfloat16, 47).cuda()
    for table, start in (([[0, 4, 1]], [0]), ([[0, -1, 1]], [0]), ([[0, 1]], [0]), ([[0, 1, 2]], [-3]), ([[0, 1, 2]], [2 ** 31 - 20])):
        c = _cache(*_filled(4, G, bs, hd, 48))
        before = [t.clone() for t in (c.k, c.v, c.k_scale, c.v_scale)]
        c.store(x, x, _dev([0, 40]), _dev(start), _dev(table))
        with pytest.raises(P.EasError) as e:
            c.check()
        assert e.value.status == 7
        c.check()                                                       # reading clears it
        assert torch.equal(c.k[3], before[0][3])
        if start[0] != 0:
            assert torch.equal(c.k, before[0]) and torch.equal(c.v_scale, before[3])
        out = tuple(torch.full((40, G, hd), 9.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        c.load(_dev([0, 40]), _dev(start), _dev(table), 40, out=out)
        with pytest.raises(P.EasError):
            c.check()
        assert (out[0][16:32] == 9.0).all() or len(table[0]) == 2 or start[0] != 0
        q = _rand((1, 2, hd), torch.bfloat16, 49).cuda()
        if start[0] == 0:
            got = c.attention(q, _dev([40]), _dev(table))
            with pytest.raises(P.EasError):
                c.check()
            assert torch.isfinite(got).all()


def test_cache_store_ignores_rows_past_the_tensor():
    c = _cache(*_filled(4, 1, 16, 64, 50))
    want = c.k.clone()
    x = _rand((5, 1, 64), torch.bfloat16, 51).cuda()
    c.store(x, x, _dev([0, 40]), _dev([0]), _dev([[3, 2, 1]]))          # 40 rows announced, 5 exist
    assert torch.equal(c.k[:3], want[:3]) and torch.equal(c.k[3, 0, 5:], want[3, 0, 5:])


def test_cache_load_writes_no_row_behind_n_rows():
    numbers, scales = _filled(3, 2, 16, 64, 52)
    c = _cache(numbers, scales)
    k, v = (torch.full((12, 2, 64), 5.0, dtype=torch.float16, device="cuda") for _ in range(2))
    cu, start, table = _dev([0, 40]), _dev([0]), _dev([[2, 0, 1]])      # 40 rows announced, 9 asked for, 12 there
    got = c.load(cu, start, table, 9, out=(k, v))
    c.check()
    assert got[0] is k and (k[9:] == 5.0).all() and (v[9:] == 5.0).all()
    want = c.load(cu, start, table, 40, dtype=torch.float16)
    assert torch.equal(k[:9], want[0][:9]) and torch.equal(v[:9], want[1][:9])
    import paper_2609_31551_b200 as P
    with pytest.raises(P.EasError) as e:
        c.load(cu, start, table, 13, out=(k, v))
    assert e.value.status == 1


# ------------------------------------------------------------------------------------------------ single tokens
def _check_tokens(c, numbers, scales, q, lens, table, scale=None, **kw):
    hd, bs = q.shape[2], numbers[0].shape[2]
    out = c.attention(q.cuda(), _dev(lens), table.cuda(), scale=scale, **kw)
    c.check()
    ref, mag, smax = LO.cache_attention(q, numbers[0], numbers[1], scales[0], scales[1], lens, table, hd ** -0.5 if scale is None else scale)
    got = out.double().cpu()
    assert torch.isfinite(got).all()
    vmax = float((numbers[1].float().abs().amax((2, 3)) * scales[1]).max())
    tol = _bound(mag, smax, hd, 2.0 ** -11, U[q.dtype], max(list(lens) + [0]), vmax, True)
    assert ((got - ref).abs() <= tol).all(), float(((got - ref).abs() / tol).max())
    assert not got[torch.tensor([n <= 0 for n in lens])].any()
    return out


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("H,G", [(1, 1), (8, 2), (10, 2), (16, 1), (17, 1), (24, 2)])
@pytest.mark.parametrize("bs,lens", [(16, [1]), (16, [15, 16, 17, 0, 33]), (32, [700, 1, 64]), (64, [63, 65, 1000]), (128, [129, 0, 2050])])
def test_cache_attention(hd, dtype, H, G, bs, lens):
    rng = np.random.Generator(np.random.PCG64(H + bs + hd))
    n_blocks = sum((n + bs - 1) // bs for n in lens) + 2
    table = _table(rng, lens, bs, n_blocks)
    numbers, scales = _filled(n_blocks, G, bs, hd, 60)
    q = _rand((len(lens), H, hd), dtype, 61, 2.0)
    c = _cache(numbers, scales)
    out = _check_tokens(c, numbers, scales, q, lens, table)
    for budget in (1, 37):
        assert torch.equal(out, c.attention(q.cuda(), _dev(lens), table.cuda(), sm_budget=budget))


@pytest.mark.parametrize("hd,H,G,bs,lens", [(128, 8, 1, 16, [30011]), (64, 4, 4, 64, [9000, 1, 5000, 0, 77]), (128, 32, 8, 128, [4097] * 3), (64, 12, 1, 32, [12000, 40])])
def test_cache_attention_split_over_many_pieces(hd, H, G, bs, lens):
    rng = np.random.Generator(np.random.PCG64(hd + H))
    n_blocks = sum((n + bs - 1) // bs for n in lens)
    table = _table(rng, lens, bs, n_blocks)
    numbers, scales = _filled(n_blocks, G, bs, hd, 62)
    q = _rand((len(lens), H, hd), torch.bfloat16, 63, 2.0)
    c = _cache(numbers, scales)
    out = _check_tokens(c, numbers, scales, q, lens, table)
    assert torch.equal(out, c.attention(q.cuda(), _dev(lens), table.cuda(), sm_budget=50))


def test_cache_attention_many_sequences_in_two_launches():
    rng = np.random.Generator(np.random.PCG64(5))
    lens = [int(x) for x in rng.integers(0, 60, 1300)]
    n_blocks = sum((n + 15) // 16 for n in lens)
    table = _table(rng, lens, 16, n_blocks)
    numbers, scales = _filled(n_blocks, 2, 16, 64, 64)
    _check_tokens(_cache(numbers, scales), numbers, scales, _rand((1300, 2, 64), torch.bfloat16, 65, 2.0), lens, table)


def test_cache_attention_scales_of_all_sizes():
    """Blocks whose scales lie many powers of ten apart, zero scales, queries of very different size, and a strided table, q and out."""
    bs, hd, G, H = 16, 128, 1, 3
    lens = [160, 33]
    rng = np.random.Generator(np.random.PCG64(6))
    numbers, scales = _filled(16, G, bs, hd, 66)
    table = _table(rng, lens, bs, 16)
    exps = torch.tensor([-12.0, 0.0, -3.0, -30.0, 1.0, -6.0, -1.0, -20.0, 0.0, -2.0, -9.0, -4.0, 0.5, -0.5, -8.0, -5.0])
    scales[1] = (10.0 ** exps)[:, None].float()
    scales[1][int(table[0, 4])] = 0.0
    scales[0][int(table[0, 2])] = 0.0
    q = _rand((2, H, hd), torch.bfloat16, 67)
    q[0, 0] *= 1e-20
    q[0, 1] *= 60.0
    q[1, 2] = 0.0
    wide = torch.zeros(2, H * hd + 8, dtype=torch.bfloat16)
    wide[:, :H * hd] = q.reshape(2, -1)
    c = _cache(numbers, scales)
    out = _check_tokens(c, numbers, scales, q, lens, table)
    buf = torch.full((3, H * hd + 16), 2.0, dtype=torch.bfloat16, device="cuda")
    big = torch.full((2, 40), -1, dtype=torch.int32)
    big[:, :table.shape[1]] = table
    got = c.attention(wide.cuda()[:, :H * hd].view(2, H, hd), _dev(lens), big.cuda()[:, :table.shape[1]], out=buf[:2, :H * hd].view(2, H, hd))
    assert torch.equal(got, out)
    assert (buf[2] == 2.0).all() and (buf[:, H * hd:] == 2.0).all()


def test_cache_attention_reads_nothing_behind_the_lengths():
    bs, hd = 32, 128
    numbers, scales = _filled(6, 2, bs, hd, 68)
    table = torch.tensor([[0, 1, 2], [3, 4, 5]], dtype=torch.int32)
    q = _rand((2, 4, hd), torch.bfloat16, 69, 2.0)
    c = _cache(numbers, scales)
    out = c.attention(q.cuda(), _dev([40, 64]), table.cuda())
    c.k_scale[2], c.v_scale[2], c.k_scale[5], c.v_scale[5] = (float("nan"),) * 4
    c.k[1, :, 8:], c.v[1, :, 8:] = -128, -128
    assert torch.equal(out, c.attention(q.cuda(), _dev([40, 64]), table.cuda()))
    c.v_scale[0, 1] = float("nan")                                      # one block and head that sequence 0 does read
    got = c.attention(q.cuda(), _dev([40, 64]), table.cuda())
    assert torch.isnan(got[0, 2:]).all() and torch.equal(got[0, :2], out[0, :2]) and torch.equal(got[1], out[1])


def test_cache_attention_replays_for_other_lengths_and_shared_workspace():
    bs, hd, G, H = 16, 128, 2, 8
    rng = np.random.Generator(np.random.PCG64(7))
    numbers, scales = _filled(300, G, bs, hd, 70)
    c = _cache(numbers, scales)
    table = _table(rng, [1000, 1000, 1000], bs, 300)
    td, q, lens = table.cuda(), _rand((3, H, hd), torch.bfloat16, 71, 2.0).cuda(), _dev([3, 0, 900])
    ws = torch.empty(c.attention_workspace_bytes(3, H), dtype=torch.uint8, device="cuda")
    graphs, outs = [], []
    for _ in range(2):                                                  # two captures on one workspace, replayed one behind the other
        g = torch.cuda.CUDAGraph()
        c.attention(q, lens, td, workspace=ws)
        torch.cuda.synchronize()
        with torch.cuda.graph(g):
            outs.append(c.attention(q, lens, td, workspace=ws))
        graphs.append(g)
    for now in ([3, 0, 900], [1000, 17, 1], [0, 0, 0], [512, 513, 514]):
        lens.copy_(_dev(now))
        want = c.attention(q, _dev(now), td)
        for g, o in zip(graphs, outs):
            ws.fill_(0xFF)
            g.replay()
            assert torch.equal(o, want)
    c.check()
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = c.attention(q, lens, td, stream=side)
    side.synchronize()
    assert torch.equal(got, want)


def test_cache_refusals():
    import paper_2609_31551_b200 as P
    c = _cache(*_filled(4, 2, 16, 64, 72))
    x, q = torch.zeros(3, 2, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(1, 4, 64, dtype=torch.bfloat16, device="cuda")
    t, one, cu = _dev([[0, 1]]), _dev([5]), _dev([0, 3])
    bad = [
        lambda: c.store(x.float(), x.float(), cu, one, t), lambda: c.store(x, x[:2], cu, one, t), lambda: c.store(x, x.half(), cu, one, t),
        lambda: c.store(x[:, :1], x[:, :1], cu, one, t), lambda: c.store(x, x, cu.long(), one, t), lambda: c.store(x, x, one, one, t),
        lambda: c.store(x, x, cu, one, t.cpu()), lambda: c.store(x, x, cu, one, t[0]), lambda: c.store(x, x, cu, one, t, sm_budget=-1),
        lambda: c.attention(q[:, :3], one, t), lambda: c.attention(q.float(), one, t), lambda: c.attention(q, one, t, scale=float("nan")),
        lambda: c.attention(q, cu, t), lambda: c.attention(q, one, t, out=q.half()), lambda: c.attention(q, one, t, workspace=torch.zeros(1 << 20, dtype=torch.uint8)),
        lambda: c.load(cu, one, t, 3, dtype=torch.float32), lambda: P.KvCache(4, 16, 2, 64, tensors=(c.k, c.v, c.k_scale, c.v_scale.half())),
    ]
    for call in bad:
        with pytest.raises(P.EasError) as e:
            call()
        assert e.value.status in (1, 2)
    with pytest.raises(P.EasError) as e:
        c.attention(q, one, t, workspace=torch.zeros(256, dtype=torch.uint8, device="cuda"))
    assert e.value.status == 3
    for shape in ((4, 24, 2, 64), (4, 16, 2, 96)):
        with pytest.raises(P.EasError) as e:
            P.KvCache(*shape)
        assert e.value.status == 2
    c.close()
    with pytest.raises(P.EasError):
        c.store(x, x, cu, one, t)


# ------------------------------------------------------------------------------------------------ a run of them together
@pytest.mark.parametrize("hd,dtype,bs", [(128, torch.bfloat16, 16), (64, torch.float16, 64)])
def test_prompts_then_tokens(hd, dtype, bs):
    """A batch is answered as a server would: the prompts attend to themselves and go into the cache, a second chunk of one of them attends to
    the prefix read back, then every sequence writes and attends one token at a time."""
    import paper_2609_31551_b200 as P
    H, G, steps = 8, 2, 20
    lens = [70, 5, 200]
    total = [n + steps for n in lens]
    rng = np.random.Generator(np.random.PCG64(8))
    n_blocks = sum((n + bs - 1) // bs for n in total)
    table = _table(rng, total, bs, n_blocks)
    td = table.cuda()
    cache = P.KvCache(n_blocks, bs, G, hd)
    nums, scs = [torch.zeros(n_blocks, G, bs, hd, dtype=torch.int8) for _ in range(2)], [torch.zeros(n_blocks, G) for _ in range(2)]
    cu = _cu(lens)
    q, k, v = _rand((cu[-1], H, hd), dtype, 80, 2.0), _rand((cu[-1], G, hd), dtype, 81), _rand((cu[-1], G, hd), dtype, 82)
    out, status = P.prompt_attention(q.cuda(), k.cuda(), v.cuda(), cu)
    cache.store(k.cuda(), v.cuda(), _dev(cu), _dev([0, 0, 0]), td)
    assert int(status[0]) == 0
    _check_prompt(q, k, v, cu, cu, out, hd ** -0.5)
    for x, i in ((k, 0), (v, 1)):
        LO.cache_store(nums[i], scs[i], x, cu, [0, 0, 0], table)
    # the last 30 tokens of the longest prompt once more, behind the prefix as the cache holds it
    kk, vv = cache.load(_dev([0, 200]), _dev([0]), td[2:], 200, dtype=dtype)
    kc, vc = torch.cat([kk[:170].cpu(), k[cu[2] + 170:]]), torch.cat([vv[:170].cpu(), v[cu[2] + 170:]])
    chunk = P.prompt_attention(q[cu[3] - 30:].cuda(), kc.cuda(), vc.cuda(), [0, 30], [0, 200])[0]
    _check_prompt(q[cu[3] - 30:], kc, vc, _cu([30]), _cu([200]), chunk, hd ** -0.5)
    now = list(lens)
    for t in range(steps):
        q, k, v = _rand((3, H, hd), dtype, 90 + t, 2.0), _rand((3, G, hd), dtype, 190 + t, 0.5 + 0.2 * t), _rand((3, G, hd), dtype, 290 + t)
        cache.store(k.cuda(), v.cuda(), _dev([0, 1, 2, 3]), _dev(now), td)
        for x, i in ((k, 0), (v, 1)):
            LO.cache_store(nums[i], scs[i], x, [0, 1, 2, 3], now, table)
        now = [n + 1 for n in now]
        _check_tokens(cache, nums, scs, q, now, table)
    assert torch.equal(cache.k.cpu(), nums[0]) and torch.equal(cache.v_scale.cpu(), scs[1])


def test_offsets_past_32_bits():
    """Blocks whose bytes lie past 2^32, and token rows past 2^31 elements: the same bits as the same data near the start."""
    import paper_2609_31551_b200 as P
    H, G, hd, bs, n = 8, 8, 128, 128, 400
    far = 2 ** 32 // (G * bs * hd) + 1                                  # the first block behind 2^32 bytes
    cu, zero = _dev([0, n]), _dev([0])
    k, v, q = _rand((n, G, hd), torch.bfloat16, 400).cuda(), _rand((n, G, hd), torch.bfloat16, 401).cuda(), _rand((n, H, hd), torch.bfloat16, 402, 2.0).cuda()
    near, big = P.KvCache(4, bs, G, hd), P.KvCache(far + 4, bs, G, hd)
    wide = torch.empty(n * 2 ** 23, dtype=torch.bfloat16, device="cuda")     # rows 2^23 elements apart: row 256 begins at 2^31

    def spread(x, at):
        y = wide[at:].as_strided(x.shape, (2 ** 23, x.shape[2], 1))
        y.copy_(x)
        return y
    kw, vw, qw = spread(k, 0), spread(v, 4096), spread(q, 8192)
    ow = wide[16384:].as_strided(q.shape, (2 ** 23, hd, 1))
    want, got = P.prompt_attention(q, k, v, [0, n]), P.prompt_attention(qw, kw, vw, [0, n], out=ow)
    assert int(want[1][0]) == 0 and int(got[1][0]) == 0 and torch.equal(want[0], got[0])
    table = _dev([[1, 3, 0, 2]])
    near.store(k, v, cu, zero, table)
    big.store(kw, vw, cu, zero, table + far)
    want, got = near.load(cu, zero, table, n), big.load(cu, zero, table + far, n, out=(kw, vw))
    assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1]) and float(want[0].abs().max()) > 1
    lens, tables = _dev([n - i for i in range(n)]), table.expand(n, 4).contiguous()
    a, b = near.attention(q, lens, tables), big.attention(qw, lens, tables + far, out=ow)
    near.check(), big.check()
    assert torch.equal(a, b) and float(a.abs().max()) > 0.01


def test_calls_on_two_streams_at_once():
    """Calls that share the cache and its status word but no workspace, on shares of the SMs and on all of them."""
    import paper_2609_31551_b200 as P
    H, G, hd, bs, lens = 16, 4, 128, 32, [3000, 50, 900]
    rng = np.random.Generator(np.random.PCG64(41))
    n_blocks = sum((n + bs - 1) // bs for n in lens)
    table = _table(rng, lens, bs, n_blocks).cuda()
    numbers, scales = _filled(n_blocks, G, bs, hd, 410)
    c = _cache(numbers, scales)
    q1, lens_d = _rand((3, H, hd), torch.bfloat16, 411).cuda(), _dev(lens)
    cu_q, cu_k = [0, 60, 61], [0, 4000, 4100]
    q = _rand((61, H, hd), torch.bfloat16, 412).cuda()
    k, v = _rand((4100, G, hd), torch.bfloat16, 413).cuda(), _rand((4100, G, hd), torch.bfloat16, 414).cuda()
    assert P.prompt_attention_workspace_bytes(H, G, hd, cu_q, cu_k) > 0
    tok, (pro, status) = c.attention(q1, lens_d, table), P.prompt_attention(q, k, v, cu_q, cu_k)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    seen = []
    for i in range(40):
        st, budget = streams[i % 2], (0, 60)[i // 20]
        seen.append((tok, c.attention(q1, lens_d, table, stream=st, sm_budget=budget)))
        out, s = P.prompt_attention(q, k, v, cu_q, cu_k, stream=streams[1 - i % 2], sm_budget=budget)
        seen.append((pro, out))
        seen.append((status, s))
    torch.cuda.synchronize()
    c.check()
    assert int(status[0]) == 0 and all(torch.equal(a, b) for a, b in seen)


# ------------------------------------------------------------------------------------------------ the commands that call them
@pytest.mark.parametrize("neighbour", ["prompt", "token"])
def test_coresidency_with_a_language_model_neighbour(neighbour):
    from paper_2609_31551_b200 import coresidency
    rows = coresidency.measure("c0", 2, levels=(0.5,), reps=2, neighbour=neighbour)
    assert len(rows) == 1 and rows[0]["neighbour"] == neighbour
    assert rows[0]["encode_ms_beside_neighbour"] > 0 and rows[0]["neighbour_tflops_beside_encoder"] > 0


@pytest.mark.parametrize("argv", [["prompt", "--lens", "300x2,17", "--before", "40"], ["token", "--lens", "500x3,1", "--block", "16", "--sm-budget", "20"],
                                  ["store", "--lens", "300x2,17", "--fp16"], ["load", "--lens", "300x2,17", "--head-dim", "64"]])
def test_kernel_bench_runs(argv, monkeypatch, capsys):
    import json
    from paper_2609_31551_b200 import kernel_bench
    monkeypatch.setattr("sys.argv", ["kernel_bench"] + argv + ["--iters", "2", "--warmup", "1"])
    kernel_bench.main()
    line = json.loads(capsys.readouterr().out)
    assert line["kernel"] == argv[0] and line["ms"] > 0 and line.get("tflops", line.get("gbs")) > 0
