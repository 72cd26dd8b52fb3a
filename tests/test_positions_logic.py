"""CPU-only checks of rotary positions, appending and chunk attention: the oracle against independent formulas, and the refusals that the host gives before it
touches a GPU."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import language_oracle as LO


@pytest.fixture(scope="module")
def lang():
    from paper_2609_31551_b200.build import build_library
    build_library()
    from paper_2609_31551_b200 import language
    language.lib()
    return language


def test_oracle_rotation_is_complex_multiplication():
    x = torch.randn(5, 2, 12, generator=torch.Generator().manual_seed(1), dtype=torch.float64)
    pos = np.array([[0, 1, -7, 400, 5], [9, 2, 3, 4, 100]])
    freq, axis = np.array([1.0, 0.3, 0.02, 0.5]), np.array([0, 1, 1, 0])
    angle = torch.from_numpy(pos[axis].T * freq)[:, None]
    for neighbours in (False, True):
        y = LO.rotate(x, pos, axis, freq, neighbours, 1.5)
        a, b = (x[..., 0:8:2], x[..., 1:8:2]) if neighbours else (x[..., :4], x[..., 4:8])
        z = torch.complex(a, b) * torch.polar(torch.full_like(angle, 1.5), angle)
        want = x.clone()
        if neighbours:
            want[..., 0:8:2], want[..., 1:8:2] = z.real, z.imag
        else:
            want[..., :4], want[..., 4:8] = z.real, z.imag
        assert torch.allclose(y, want, atol=1e-12)
        assert torch.allclose(LO.rotate(y, pos, axis, freq, neighbours, 1 / 1.5, inverse=True), x, atol=1e-12)


def test_rotated_scores_depend_on_the_distance_alone():
    q, k = torch.randn(1, 1, 8, dtype=torch.float64), torch.randn(1, 1, 8, dtype=torch.float64)
    freq, axis = 100.0 ** (-np.arange(4) / 4), np.zeros(4, dtype=int)
    dots = [float((LO.rotate(q, np.array([[a + 3]]), axis, freq) * LO.rotate(k, np.array([[a]]), axis, freq)).sum()) for a in (0, 5, 1000, 10 ** 6)]
    assert np.allclose(dots, dots[0], atol=1e-9)


def test_oracle_chunk_is_prompt_attention_over_the_values():
    gen = torch.Generator().manual_seed(2)
    numbers = [torch.randint(-127, 128, (5, 2, 16, 8), generator=gen, dtype=torch.int8) for _ in range(2)]
    scales = [torch.rand(5, 2, generator=gen) * 0.05 for _ in range(2)]
    table, q = torch.tensor([[3, 1], [0, 2], [4, 4]]), torch.randn(9, 4, 8, generator=gen, dtype=torch.float64)
    cu, lens = [1, 5, 7, 7], [30, 1, 0]
    out, _, _ = LO.chunk_attention(q, numbers[0], numbers[1], scales[0], scales[1], cu, lens, table, 0.4)
    k, v = (torch.cat([LO.cache_values(numbers[i], scales[i], table[s], lens[s]) for s in range(3)]) for i in range(2))
    ref, _, _ = LO.prompt_attention(q, k, v, cu, [0, 30, 31, 31], 0.4)
    assert torch.allclose(out[1:7], ref[1:7]) and not out[5].any() and out[6].any() and torch.isnan(out[[0, 7, 8]]).all()


@pytest.mark.parametrize("change,status", [
    ({"head_dim": 96}, 2), ({"rotary_dim": 24}, 2), ({"rotary_dim": 144}, 2), ({"rotary_dim": 0}, 2), ({"rotary_dim": -16}, 2), ({"pairing": 2}, 1), ({"n_axes": 0}, 2),
    ({"n_axes": 5}, 2), ({"scale": 0.0}, 1), ({"scale": float("inf")}, 1), ({"scale": float("nan")}, 1), ({"inv_freq": None}, 1)])
def test_rotary_create_refuses(lang, change, status):
    freq = np.ones(64)
    fields = {"head_dim": 128, "rotary_dim": 128, "pairing": 0, "n_axes": 1, "inv_freq": freq.ctypes.data, "axis": None, "scale": 1.0}
    desc, h = lang.RotaryDesc(**{**fields, **change}), C.c_void_p(5)
    assert lang.lib().eas_rotary_create(C.byref(desc), C.byref(h)) == status
    assert h.value is None
    assert lang.lib().eas_rotary_create(None, C.byref(h)) == 1
    assert lang.lib().eas_rotary_create(C.byref(desc), None) == 1


def test_rotary_refuses_bad_lists(lang):
    import paper_2609_31551_b200 as P
    bad = [{"sections": (16, 8)}, {"sections": (-1, 33)}, {"sections": ()}, {"axes": [4] * 32}, {"axes": [-1] + [0] * 31}, {"axes": [0] * 31}, {"axes": [0] * 32, "sections": (32,)},
           {"inv_freq": [1.0]}, {"inv_freq": [float("nan")] * 32}, {"inv_freq": "abc"}, {"base": "x"}, {"sections": 7}, {"rotary_dim": 128}, {"scale": "x"}, {"base": 0.0}]
    for kw in bad:
        with pytest.raises(P.EasError):
            P.Rotary(64, **kw)
    for kw in ({}, {"sections": (32,)}, {"sections": (8, 12, 12)}, {"axes": [0, 3] * 16}, {"rotary_dim": 16, "neighbours": True}, {"inv_freq": np.zeros(32)}):
        r = P.Rotary(64, **kw)
        r.close()
        r.close()


def test_calls_refuse_null_and_bad_arguments_before_the_device(lang):
    import paper_2609_31551_b200 as P
    l = lang.lib()
    rec = lang._pack_rotary(*[0] * 15)
    r = P.Rotary(64)
    assert l.eas_rotary_apply(None, rec, 0, None) == 1
    assert l.eas_rotary_apply(r.handle, None, 0, None) == 1
    fields = ("q", "k", "out_q", "out_k", "ld_q", "ld_k", "ld_out_q", "ld_out_k", "positions", "ld_positions", "n_rows", "n_heads", "n_kv_heads", "dtype", "inverse")
    good = dict(zip(fields, (4096, 8192, 4096, 8192, 256, 128, 256, 128, 4096, 3, 3, 4, 2, 0, 0)))
    for change in ({"q": 0}, {"k": 0}, {"out_q": 0}, {"out_k": 0}, {"q": 4104}, {"out_k": 8200}, {"ld_q": 255}, {"ld_q": 248}, {"ld_k": 120}, {"ld_out_q": 260}, {"positions": 0},
                   {"ld_positions": 2}, {"n_rows": -1}, {"n_heads": -4}, {"n_kv_heads": -1}, {"dtype": 2}, {"inverse": 2}):
        got = l.eas_rotary_apply(r.handle, lang._pack_rotary(*[{**good, **change}[f] for f in fields]), 0, None)
        assert got == (2 if "dtype" in change else 1), change
    seqs = lang._pack_seqs(0, 0, 0, 0, 0, 0, 0)
    assert l.eas_cache_append(None, seqs, r.handle, rec, None, 0, 0, None, None) == 1
    assert l.eas_cache_append(None, seqs, None, rec, None, 0, 0, None, None) == 1
    assert l.eas_cache_chunk_attention(None, seqs, None, 0, None, 0, 0, 0, 1, 0, 1.0, None, 0, 0, None, None) == 1
    assert l.eas_cache_chunk_workspace_bytes(None, 1, 1, 1, 1) == 0
