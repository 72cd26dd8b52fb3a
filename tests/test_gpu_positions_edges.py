"""Calls of rotary positions, appending and chunk attention that lie off the beaten track: axes that share memory, keys alone, bounds that are not met, tables as wide as
they may be, quiet keys under loud scales, queries and scales at the ends of their ranges.  The bounds are those of test_gpu_positions.py."""
import pytest
import torch

from tests.test_gpu_positions import _cache, _check_append, _check_chunk, _check_rotated, _cu, _dev, _filled, _rand, _rotary, _table

pytestmark = pytest.mark.gpu
BF, FP = torch.bfloat16, torch.float16


# ------------------------------------------------------------------------------------------------ positions
@pytest.mark.parametrize("T", [1, 2, 37])
def test_axes_may_share_their_positions(T):
    """Text tokens on three axes: one row of positions, seen three times."""
    import paper_2609_31551_b200 as P
    hd, G, bs = 64, 2, 16
    r, rot = _rotary(hd, hd, (16, 8, 8))
    q, k = _rand((T, 4, hd), BF, 1), _rand((T, G, hd), BF, 2)
    pos = torch.randint(0, 5000, (T,), generator=torch.Generator().manual_seed(3), dtype=torch.int32).cuda()
    shared, apart = pos.expand(3, -1), pos.repeat(3, 1)
    assert shared.stride(0) == 0
    out = r.apply(q.cuda(), k.cuda(), shared)
    _check_rotated(q, out[0], rot, apart.cpu().numpy())
    _check_rotated(k, out[1], rot, apart.cpu().numpy())
    table, n_blocks = _table(1, [T + 5], bs)
    was = _filled(n_blocks, G, bs, hd, 4)
    c = _cache(*was)
    turned = c.append(q.cuda(), k.cuda(), k.cuda(), _dev([0, T]), _dev([5]), table.cuda(), r, shared)
    c.check()
    _check_append(c, was, *was, rot, q, k, k, [0, T], [5], table, apart.cpu().numpy(), turned)
    if T > 2:                                                              # axes that overlap otherwise are a mistake
        for call in (lambda p: r.apply(q.cuda(), k.cuda(), p), lambda p: c.append(q.cuda(), k.cuda(), k.cuda(), _dev([0, T]), _dev([5]), table.cuda(), r, p)):
            with pytest.raises(P.EasError):
                call(torch.zeros(3 * T, dtype=torch.int32, device="cuda").as_strided((3, T), (1, 1)))


def test_rotation_of_keys_alone():
    import paper_2609_31551_b200 as P
    r, rot = _rotary(128, 64, (16, 8, 8))
    k = _rand((21, 3, 128), FP, 5)
    pos = torch.randint(0, 900, (3, 21), generator=torch.Generator().manual_seed(6), dtype=torch.int32)
    kd = k.cuda()
    none, out = r.apply(None, kd, pos.cuda())
    assert none is None
    _check_rotated(k, out, rot, pos.numpy())
    assert torch.equal(r.apply(kd, None, pos.cuda())[0], out)
    buf = torch.empty_like(kd)
    assert r.apply(None, kd, pos.cuda(), out=(None, buf))[1] is buf and torch.equal(buf, out)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    again = r.apply(None, kd, pos.cuda(), stream=side)[1]
    side.synchronize()
    assert torch.equal(again, out)
    for call in (lambda: r.apply(None, None, pos.cuda()), lambda: r.apply(kd, kd, pos.cuda(), out=(buf, None)), lambda: r.apply(kd, kd, pos.cuda(), out=(None, buf)),
                 lambda: r.apply(kd, kd, pos.cuda(), out=buf[:2]), lambda: r.apply(kd, None, pos.cuda(), out=(buf,)), lambda: r.apply(None, kd.float(), pos.cuda())):
        with pytest.raises(P.EasError):
            call()


# ------------------------------------------------------------------------------------------------ which kernel
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("lens", [[4] * 12, [3, 4, 8, 1, 5], [4, 2, 1], [1] * 9])
def test_drafts_without_a_bound_go_to_the_kernels_for_few_rows(hd, lens):
    """max_new left out says nothing of how the rows are spread: single tokens, and drafts of 9 to 32 rows a key/value head, are computed by the same kernels as with their bound, to the same bits."""
    H, G, bs = 8, 2, 16
    held = [n + b for n, b in zip(lens, range(300, 1500, 100))]
    table, n_blocks = _table(hd, held, bs)
    numbers, scales = _filled(n_blocks, G, bs, hd, 11)
    q = _rand((sum(lens), H, hd), BF, 12, 2.0)
    c = _cache(numbers, scales)
    exact = _check_chunk(c, numbers, scales, q, _cu(lens), held, table, max_new=max(lens))
    for loose in (None, sum(lens) + 7):
        assert torch.equal(_check_chunk(c, numbers, scales, q, _cu(lens), held, table, max_new=loose), exact)


@pytest.mark.parametrize("hd,H,G", [(128, 8, 8), (64, 16, 8)])
@pytest.mark.parametrize("lens", [[1] * 8, [2, 1, 4, 1, 1, 0, 3, 1], [40, 1, 1, 1, 1, 1, 1, 1], [33, 40, 38, 1, 2, 40, 12, 39]])
def test_tables_as_wide_as_they_may_be(hd, H, G, lens):
    """2^30 places a sequence, of which a few hundred are used."""
    bs, width = 128, 1 << 23
    held = [n + b for n, b in zip(lens, (700, 0, 90, 33, 5, 260, 128, 127))]
    narrow, n_blocks = _table(13, held, bs)
    numbers, scales = _filled(n_blocks, G, bs, hd, 14)
    table = torch.full((len(lens), width), -7, dtype=torch.int32)
    table[:, :narrow.shape[1]] = narrow
    q = _rand((sum(lens), H, hd), BF, 15, 2.0)
    c = _cache(numbers, scales)
    for max_new in (max(lens), None):
        workspace = torch.empty(c.chunk_workspace_bytes(len(lens), sum(lens), sum(lens) if max_new is None else max_new, H), dtype=torch.uint8, device="cuda")
        _check_chunk(c, numbers, scales, q, _cu(lens), held, table, max_new=max_new, workspace=workspace)


# ------------------------------------------------------------------------------------------------ ranges
@pytest.mark.parametrize("dtype", [BF, FP])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("max_new", [3, 60])
def test_quiet_keys_under_a_loud_scale(dtype, hd, max_new):
    """Numbers of -1, 0 and 1, most of them 0, in blocks whose scale another token has set, and queries of one sign: the sum over |q| times 127 steps of the scale is some
    thousand times a score, and must not stand in its error.  Scores are within a few units of each other, so every key counts."""
    bs, G, H = 16, 2, 8
    lens, before = [max_new, 1], [5, 40]
    held = [a + b for a, b in zip(lens, before)]
    table, n_blocks = _table(17, held, bs)
    gen = torch.Generator().manual_seed(18)
    numbers, scales = _filled(n_blocks, G, bs, hd, 19)
    keys = (torch.rand(numbers[0].shape, generator=gen) < 4.0 / hd).to(torch.int8) * (torch.randint(0, 2, numbers[0].shape, generator=gen, dtype=torch.int8) * 2 - 1)
    q = ((torch.rand((sum(lens), H, hd), generator=gen) * 0.5 + 0.5) * 8.0).to(dtype)
    numbers, scales = [keys, numbers[1]], [torch.full_like(scales[0], 6.0), scales[1]]
    _check_chunk(_cache(numbers, scales), numbers, scales, q, _cu(lens), held, table, max_new=max_new)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("max_new", [3, 60])
@pytest.mark.parametrize("power", [100, 117, 120, 125])
def test_queries_at_the_upper_end_of_bf16(hd, max_new, power):
    """Queries of up to 2^127 over keys whose scale takes it back: the scores are those of ordinary ones."""
    bs, G, H = 16, 2, 4
    lens, before = [max_new, 1], [50, 40]
    held = [a + b for a, b in zip(lens, before)]
    table, n_blocks = _table(20, held, bs)
    numbers, scales = _filled(n_blocks, G, bs, hd, 21)
    q = (_rand((sum(lens), H, hd), BF, 22).float().clamp(-3.9, 3.9) * 2.0 ** power).to(BF)
    assert torch.isfinite(q).all()
    for split in (0, 30):                                                  # the scale of the scores may take part of it
        sc = [scales[0] * 2.0 ** (split - power), scales[1]]
        _check_chunk(_cache(numbers, sc), numbers, sc, q, _cu(lens), held, table, scale=hd ** -0.5 * 2.0 ** -split, max_new=max_new)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("max_new", [4, 60])
@pytest.mark.parametrize("power", [-92, -60, 100])
def test_value_scales_at_both_ends(hd, max_new, power):
    """Values of 2^-97 and 2^107 and their sums in bf16, against the oracle."""
    lens, before, bs, G = [max_new, 1], [200, 90], 16, 2
    held = [a + b for a, b in zip(lens, before)]
    table, n_blocks = _table(23, held, bs)
    numbers, scales = _filled(n_blocks, G, bs, hd, 24)
    q = _rand((sum(lens), 4, hd), BF, 25)
    sc = [scales[0], scales[1] * 2.0 ** power]
    assert float(sc[1].min()) >= 2.0 ** -100
    out = _check_chunk(_cache(numbers, sc), numbers, sc, q, _cu(lens), held, table, max_new=max_new)
    assert (out != 0).any(dim=-1).all()
