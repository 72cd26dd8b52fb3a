"""How rotary positions, appending and chunk attention are called: streams, captured graphs, workspaces, shapes as they come, the commands that use them.

Results are compared bit for bit: what a call computes depends on its inputs and the device, not on its stream, its share of the SMs or what runs beside it.  The one
comparison with the oracle has the bounds of test_gpu_positions.py."""
import numpy as np
import pytest
import torch

from tests.test_gpu_positions import _cache, _check_chunk, _cu, _dev, _filled, _places, _rand, _table

pytestmark = pytest.mark.gpu
BF, FP = torch.bfloat16, torch.float16


class Job:
    """One step of a worker: append the new tokens, attend."""

    def __init__(self, seed, lens, before, H=8, G=2, hd=128, bs=32, dtype=BF):
        import paper_2609_31551_b200 as P
        held = [a + b for a, b in zip(lens, before)]
        table, n_blocks = _table(seed, held, bs)
        self.was = _filled(n_blocks, G, bs, hd, seed)
        self.cache = _cache(*self.was)
        self.rotary = P.Rotary(hd, sections=(hd // 4, hd // 8, hd // 8))
        T = sum(lens)
        self.q, self.k, self.v = (_rand((T, h, hd), dtype, seed + i).cuda() for i, h in enumerate((H, G, G)))
        self.cu, self.before, self.held, self.table = _dev(_cu(lens)), _dev(before), _dev(held), table.cuda()
        self.positions = _dev(np.repeat(_places(_cu(lens), before), 3, axis=0))
        self.max_new = max(lens)

    def reset(self):
        for now, was in zip((self.cache.k, self.cache.v, self.cache.k_scale, self.cache.v_scale), (*self.was[0], *self.was[1])):
            now.copy_(was)

    def run(self, **kw):
        q = self.cache.append(self.q, self.k, self.v, self.cu, self.before, self.table, self.rotary, self.positions, **kw)
        return self.cache.chunk_attention(q, self.cu, self.held, self.table, max_new=self.max_new, **kw)

    def result(self, out):
        return [x.clone() for x in (out, self.cache.k, self.cache.v, self.cache.k_scale, self.cache.v_scale)]


STEPS = [([300, 1, 2], [700, 90, 0]), ([2, 4, 1], [1000, 31, 16]), ([40, 1, 1, 1, 1, 1, 1], [100, 3, 900, 2000, 64, 65, 31])]


def test_steps_on_two_streams_at_once():
    """Two caches, two streams, the same Rotary: no call waits for another, and none sees another's scratch."""
    jobs = [Job(10 + i, *STEPS[i % 3]) for i in range(2)] + [Job(20, *STEPS[2], H=5, G=1, hd=64, dtype=FP)]
    for j in jobs[1:2]:
        j.rotary = jobs[0].rotary
    alone = []
    for j in jobs:
        alone.append(j.result(j.run()))
        j.reset()
    streams = [torch.cuda.Stream() for _ in jobs]
    torch.cuda.synchronize()
    for i in range(12):
        outs = []
        for j, st in zip(jobs, streams):
            outs.append(j.run(stream=st, sm_budget=(0, 60)[i % 2]))
        torch.cuda.synchronize()
        for j, out, ref in zip(jobs, outs, alone):
            j.cache.check()
            assert all(torch.equal(a, b) for a, b in zip(j.result(out), ref))
            j.reset()
        torch.cuda.synchronize()


@pytest.mark.parametrize("lens,before", STEPS)
def test_a_step_again_and_on_any_share_is_the_same(lens, before):
    j = Job(31, lens, before)
    ref = j.result(j.run())
    for budget in (0, 1, 2, 73, 0):
        j.reset()
        assert all(torch.equal(a, b) for a, b in zip(j.result(j.run(sm_budget=budget)), ref))


def test_two_captured_graphs_share_a_workspace_and_follow_one_another():
    jobs = [Job(41, *STEPS[0]), Job(42, *STEPS[2])]
    size = max(j.cache.chunk_workspace_bytes(j.held.numel(), j.q.shape[0], j.max_new, 8) for j in jobs)
    workspace = torch.empty(size, dtype=torch.uint8, device="cuda")
    refs = []
    for j in jobs:
        refs.append(j.result(j.run(sm_budget=0)))
        j.reset()
    outs, graphs = [torch.empty_like(j.q) for j in jobs], []
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for j, out in zip(jobs, outs):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=side):
            q = j.cache.append(j.q, j.k, j.v, j.cu, j.before, j.table, j.rotary, j.positions)
            j.cache.chunk_attention(q, j.cu, j.held, j.table, max_new=j.max_new, out=out, workspace=workspace)
    for _ in range(3):
        for j, g, out in zip(jobs, graphs, outs):
            j.reset()
            out.fill_(7)
        workspace.fill_(0xFF)
        for g in graphs + graphs:            # (what is appended again is the same)
            g.replay()
        torch.cuda.synchronize()
        for j, out, ref in zip(jobs, outs, refs):
            j.cache.check()
            assert torch.equal(out, ref[0])


def test_a_capture_replays_for_other_places_and_tokens():
    """One capture of append and attention, replayed for other rows, places, blocks and positions written into its inputs."""
    a, b = Job(51, [6, 1, 3], [50, 200, 0]), Job(51, [2, 5, 3], [64, 7, 190])
    wide = max(a.table.shape[1], b.table.shape[1])
    for j in (a, b):
        j.table = torch.nn.functional.pad(j.table, (0, wide - j.table.shape[1]), value=-7).contiguous()
        j.max_new = 6
    n = min(a.cache.n_blocks, b.cache.n_blocks)
    assert max(int(j.table.max()) for j in (a, b)) < a.cache.n_blocks and n > 0
    b.cache.close()
    b.cache, b.was = a.cache, a.was
    refs = []
    for j in (a, b):
        j.reset()
        refs.append(j.result(j.run()))
    a.reset()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        out = a.run()
    keep = {n: getattr(a, n).clone() for n in ("q", "k", "v", "cu", "before", "held", "table", "positions")}
    for j, src, ref in ((b, vars(b), refs[1]), (a, keep, refs[0]), (b, vars(b), refs[1])):
        for name in keep:
            getattr(a, name).copy_(src[name])
        a.reset()
        graph.replay()
        torch.cuda.synchronize()
        a.cache.check()
        assert all(torch.equal(x, y) for x, y in zip(a.result(out), ref))


def test_sequences_may_share_blocks_that_are_read():
    """A prefix that two sequences have in common lies in the cache once."""
    H, G, hd, bs = 8, 2, 128, 16
    numbers, scales = _filled(9, G, bs, hd, 61)
    table = torch.tensor([[3, 1, 4, 0, 5], [3, 1, 4, 8, 2]], dtype=torch.int32)
    c = _cache(numbers, scales)
    for lens, held in (([5, 2], [70, 64]), ([60, 33], [80, 51])):
        q = _rand((sum(lens), H, hd), BF, 62, 2.0)
        _check_chunk(c, numbers, scales, q, _cu(lens), held, table, max_new=max(lens))


def test_shapes_as_they_come():
    rng = np.random.Generator(np.random.PCG64(71))
    for i in range(24):
        G, group, hd = int(rng.choice([1, 2, 3, 8])), int(rng.choice([1, 2, 3, 4, 5, 7, 8, 12, 33])), int(rng.choice([64, 128]))
        bs, n = int(rng.choice([16, 32, 64, 128])), int(rng.integers(1, 12))
        high = int(rng.choice([2, 9, 60, 400]))
        lens = rng.integers(0, high + 1, n).tolist()
        lens[int(rng.integers(n))] = high
        held = [a + int(b) for a, b in zip(lens, rng.integers(0, int(rng.choice([2, 100, 1500])), n))]
        table, n_blocks = _table(i, held, bs)
        numbers, scales = _filled(n_blocks, G, bs, hd, 700 + i)
        q = _rand((sum(lens), G * group, hd), (BF, FP)[i % 2], 800 + i, 2.0)
        _check_chunk(_cache(numbers, scales), numbers, scales, q, _cu(lens), held, table, max_new=(high, None, high + 5)[i % 3])


@pytest.mark.parametrize("hd,dtype", [(128, BF), (128, FP), (64, BF)])
@pytest.mark.parametrize("lens", [[5] * 6, [8, 8, 7, 8, 0, 8], [6, 1, 5, 5, 8, 5]])
def test_drafts_behind_a_table_of_any_width(hd, dtype, lens):
    """The width of the table, of which most is not used, may choose other kernels; a workspace of the stated size does for all."""
    H, G, bs = 8, 2, 16
    held = [n + b for n, b in zip(lens, (700, 0, 90, 33, 5, 1500))]
    narrow, n_blocks = _table(91, held, bs)
    numbers, scales = _filled(n_blocks, G, bs, hd, 92)
    q = _rand((sum(lens), H, hd), dtype, 93, 2.0)
    c = _cache(numbers, scales)
    workspace = torch.empty(c.chunk_workspace_bytes(len(lens), sum(lens), max(lens), H), dtype=torch.uint8, device="cuda")
    for width in (narrow.shape[1], 4096, 40000):
        table = torch.full((len(lens), width), -7, dtype=torch.int32)
        table[:, :narrow.shape[1]] = narrow
        _check_chunk(c, numbers, scales, q, _cu(lens), held, table, max_new=max(lens), workspace=workspace)


@pytest.mark.parametrize("H,G", [(8, 2), (16, 2), (9, 1), (2, 2)])
@pytest.mark.parametrize("lens", [[70, 1, 1, 1, 1], [70, 1, 1, 0, 1, 1], [70, 3, 0, 0, 1], [70, 2, 1, 1, 1], [70]])
def test_a_chunk_beside_single_tokens_and_drafts(H, G, lens):
    before = [300, 900, 0, 31, 64, 1000][:len(lens)]
    held = [a + b for a, b in zip(lens, before)]
    table, n_blocks = _table(121, held, 16)
    numbers, scales = _filled(n_blocks, G, 16, 128, 122)
    q = _rand((sum(lens), H, 128), BF, 123, 2.0)
    c = _cache(numbers, scales)
    _check_chunk(c, numbers, scales, q, _cu(lens), held, table, max_new=70)
    _check_chunk(c, numbers, scales, q, _cu(lens), held, table)


@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("H,G,lens,before", [(128, 1, [3, 1, 9], [40, 700, 0]), (100, 1, [2, 5], [333, 80]), (130, 2, [70], [100]), (64, 64, [1, 129, 2], [500, 31, 0]),
                                             (24, 24, [33, 300], [0, 1000])])
def test_groups_of_all_sizes(hd, H, G, lens, before):
    held = [a + b for a, b in zip(lens, before)]
    table, n_blocks = _table(101, held, 32)
    numbers, scales = _filled(n_blocks, G, 32, hd, 102)
    q = _rand((sum(lens), H, hd), BF, 103, 2.0)
    c = _cache(numbers, scales)
    _check_chunk(c, numbers, scales, q, _cu(lens), held, table, max_new=max(lens))
    _check_chunk(c, numbers, scales, q, _cu(lens), held, table)


@pytest.mark.parametrize("lens,before", [([4], [700]), ([40, 3], [900, 0])])
def test_a_step_with_queries_turned_in_place(lens, before):
    j = Job(111, lens, before)
    ref = j.result(j.run())
    j.reset()
    q = j.q.clone()
    assert j.cache.append(q, j.k, j.v, j.cu, j.before, j.table, j.rotary, j.positions, out=q) is q
    out = j.cache.chunk_attention(q, j.cu, j.held, j.table, max_new=j.max_new)
    assert all(torch.equal(a, b) for a, b in zip(j.result(out), ref))


def test_coresidency_with_chunks_beside_the_encoder():
    from paper_2609_31551_b200 import coresidency
    rows = coresidency.measure("c0", 2, levels=(0.5,), reps=2, neighbour="chunk")
    assert len(rows) == 1 and rows[0]["neighbour"] == "chunk"
    assert rows[0]["encode_ms_beside_neighbour"] > 0 and rows[0]["neighbour_tflops_beside_encoder"] > 0


@pytest.mark.parametrize("argv", [["chunk", "--lens", "500x3,90", "--new", "4", "--block", "16"], ["chunk", "--lens", "900,700", "--new", "70", "--sm-budget", "20", "--fp16"],
                                  ["rotate", "--lens", "300x2,17"], ["append", "--lens", "300x2,17", "--before", "40", "--head-dim", "64"]])
def test_kernel_bench_runs(argv, monkeypatch, capsys):
    import json
    from paper_2609_31551_b200 import kernel_bench
    monkeypatch.setattr("sys.argv", ["kernel_bench"] + argv + ["--iters", "2", "--warmup", "1"])
    kernel_bench.main()
    line = json.loads(capsys.readouterr().out)
    assert line["kernel"] == argv[0] and line["ms"] > 0 and line.get("tflops", line.get("gbs")) > 0
