"""CPU-only checks of the language-model operators: the oracle against independent formulas, the exported symbols, and the
refusals that the host gives before it touches a GPU."""
import ctypes as C
import os
import re

import numpy as np
import pytest
import torch
import torch.nn.functional as F

from oracle import language_oracle as LO

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lang():
    from paper_2609_31551_b200.build import build_library
    build_library()
    from paper_2609_31551_b200 import language
    language.lib()
    return language


def test_every_declared_symbol_is_exported(lang):
    header = open(os.path.join(ROOT, "include", "eas_language.h")).read()
    header = re.sub(r"/\*.*?\*/", "", header, flags=re.S)
    declared = set(re.findall(r"\b(eas_[a-z_0-9]+)\s*\(", header))
    assert declared == set(lang.LANGUAGE_SYMBOLS)
    for name in declared:
        assert hasattr(lang.lib(), name)


# ------------------------------------------------------------------------------------------------ the oracle
@pytest.mark.parametrize("H,G", [(4, 4), (6, 2), (5, 1)])
def test_oracle_prompt_is_masked_softmax_attention(H, G):
    gen = torch.Generator().manual_seed(H)
    lens, before = [5, 1, 7], [0, 3, 4]
    cu_q, cu_k = np.cumsum([0] + lens), np.cumsum([0] + [a + b for a, b in zip(lens, before)])
    q = torch.randn(cu_q[-1], H, 8, generator=gen, dtype=torch.float64)
    k, v = (torch.randn(cu_k[-1], G, 8, generator=gen, dtype=torch.float64) for _ in range(2))
    out, _, _ = LO.prompt_attention(q, k, v, cu_q, cu_k, 0.3)
    for s, (n, b) in enumerate(zip(lens, before)):
        qs = q[cu_q[s]:cu_q[s + 1]].transpose(0, 1)
        ks, vs = (x[cu_k[s]:cu_k[s + 1]].repeat_interleave(H // G, 1).transpose(0, 1) for x in (k, v))
        mask = torch.ones(n, n + b, dtype=torch.bool).tril(b)
        ref = F.scaled_dot_product_attention(qs, ks, vs, attn_mask=mask, scale=0.3).transpose(0, 1)
        assert torch.allclose(out[cu_q[s]:cu_q[s + 1]], ref, atol=1e-12)


def test_oracle_prompt_rows_that_see_nothing_are_zero():
    q, k = torch.ones(4, 1, 2), torch.ones(2, 1, 2)
    out, _, _ = LO.prompt_attention(q, k, k * 3, [0, 4], [0, 2], 1.0)
    assert torch.equal(out[:, 0, 0], torch.tensor([0.0, 0.0, 3.0, 3.0], dtype=torch.float64))


def test_oracle_cache_round_trip_and_growing_scale():
    numbers, scales = torch.zeros(3, 1, 16, 4, dtype=torch.int8), torch.zeros(3, 1)
    table = torch.tensor([[2, 0]])
    x = torch.tensor([[[1.27, -0.5, 0.005, 0.0]], [[0.01, 0.02, 0.03, -1.27]]], dtype=torch.float64)
    LO.cache_store(numbers, scales, x, [0, 2], [0], table)
    assert numbers[2, 0, :2].tolist() == [[127, -50, 1, 0], [1, 2, 3, -127]]          # fp32 0.01 is below 0.01, so 0.005 is just above half a step
    assert scales[2, 0] == np.float32(0.01)
    LO.cache_store(numbers, scales, torch.full((1, 1, 4), 2.54, dtype=torch.float64), [0, 1], [2], table)   # the scale doubles: 0.02
    assert numbers[2, 0, :3].tolist() == [[64, -25, 0, 0], [0, 1, 2, -64], [127] * 4]       # 63.5 and 1.5 to even, 0.5 to 0
    LO.cache_store(numbers, scales, torch.full((1, 1, 4), 0.02, dtype=torch.float64), [0, 1], [3], table)   # it never shrinks
    assert scales[2, 0] == np.float32(0.02) and numbers[2, 0, 3].tolist() == [1] * 4
    assert torch.equal(LO.cache_values(numbers, scales, table[0], 2)[:, 0], numbers[2, 0, :2].double() * float(np.float32(0.02)))


def test_oracle_cache_attention_is_prompt_attention_of_the_last_token():
    gen = torch.Generator().manual_seed(3)
    numbers = [torch.randint(-127, 128, (4, 2, 16, 8), generator=gen, dtype=torch.int8) for _ in range(2)]
    scales = [torch.rand(4, 2, generator=gen) * 0.05 for _ in range(2)]
    table, q = torch.tensor([[3, 1], [0, 2]]), torch.randn(2, 4, 8, generator=gen, dtype=torch.float64)
    out, _, _ = LO.cache_attention(q, numbers[0], numbers[1], scales[0], scales[1], [20, 0], table, 0.4)
    k, v = (LO.cache_values(numbers[i], scales[i], table[0], 20) for i in range(2))
    ref, _, _ = LO.prompt_attention(q[:1], k, v, [0, 1], [0, 20], 0.4)
    assert torch.allclose(out[:1], ref) and not out[1].any()


# ------------------------------------------------------------------------------------------------ refusals of the host
def _inputs(lang, **over):
    cu = (C.c_int32 * 3)(0, 4, 9)
    a = dict(q=1 << 20, k=1 << 21, v=1 << 22, out=1 << 23, ld_q=512, ld_k=128, ld_v=128, ld_out=512, dtype=0, n_heads=4, n_kv_heads=1,
             head_dim=128, scale=0.1, n_seqs=2, cu_q=cu, cu_k=cu)
    a.update(over)
    at = {f: C.addressof(a[f]) if a[f] is not None else None for f in ("cu_q", "cu_k")}
    pin = lang.PromptInputs(*[at.get(f, a[f]) for f, _ in lang.PromptInputs._fields_])
    pin.keep = a
    return pin


@pytest.mark.parametrize("over,status", [
    (dict(q=None), 1), (dict(k=None), 1), (dict(out=None), 1), (dict(cu_q=None), 1), (dict(cu_k=None), 1),
    (dict(dtype=2), 2), (dict(head_dim=80), 2), (dict(head_dim=96), 2), (dict(n_heads=3, n_kv_heads=2), 1), (dict(n_heads=0), 1), (dict(n_kv_heads=0), 1),
    (dict(n_heads=129, ld_q=129 * 128, ld_out=129 * 128), 2), (dict(scale=0.0), 1), (dict(scale=-1.0), 1), (dict(scale=float("nan")), 1),
    (dict(scale=float("inf")), 1), (dict(n_seqs=-1), 1), (dict(q=(1 << 20) + 8), 1), (dict(v=(1 << 22) + 2), 1), (dict(ld_q=504), 1),
    (dict(ld_k=132), 1), (dict(ld_v=120), 1), (dict(ld_out=516), 1), (dict(cu_q=(C.c_int32 * 3)(0, 5, 4)), 1), (dict(cu_k=(C.c_int32 * 3)(-1, 4, 9)), 1),
])
def test_prompt_refusals(lang, over, status):
    pin = _inputs(lang, **over)
    assert lang.lib().eas_prompt_attention(C.byref(pin), None, 0, 0, None, 1 << 24) == status
    assert lang.lib().eas_last_error()


def test_null_arguments_are_refused(lang):
    l = lang.lib()
    pin = _inputs(lang)
    assert l.eas_prompt_attention(C.byref(pin), None, 0, 0, None, None) == 1
    assert l.eas_prompt_attention(None, None, 0, 0, None, 1 << 24) == 1
    seqs, h = lang.CacheSeqs(), C.c_void_p()
    assert l.eas_cache_create(None, C.byref(h)) == 1 and not h
    assert l.eas_cache_create(C.byref(lang.CacheDesc(16, 16, 16, 16, 1, 16, 1, 64)), None) == 1
    for call in (l.eas_cache_store, l.eas_cache_load):
        assert call(None, C.byref(seqs), 16, 64, 16, 64, 1, 0, 0, None, 16) == 1
    assert l.eas_cache_attention(None, C.byref(seqs), 16, 64, 16, 64, 1, 0, 1.0, 256, 1 << 20, 0, None, 16) == 1
    assert l.eas_cache_attention_workspace_bytes(None, 1, 1) == 0
    l.eas_cache_destroy(None)


@pytest.mark.parametrize("over,status", [
    (dict(k=None), 1), (dict(v_scale=None), 1), (dict(head_dim=80), 2), (dict(block_size=8), 2), (dict(block_size=48), 2), (dict(block_size=256), 2),
    (dict(n_blocks=0), 1), (dict(n_kv_heads=-1), 1), (dict(k=(1 << 20) + 8), 1), (dict(n_blocks=1 << 24, n_kv_heads=8), 2),
])
def test_cache_create_refusals(lang, over, status):
    a = dict(k=1 << 20, v=1 << 21, k_scale=1 << 22, v_scale=1 << 23, n_blocks=4, block_size=16, n_kv_heads=2, head_dim=64)
    a.update(over)
    h = C.c_void_p(5)
    assert lang.lib().eas_cache_create(C.byref(lang.CacheDesc(*[a[f] for f, _ in lang.CacheDesc._fields_])), C.byref(h)) == status
    assert not h


def test_python_refusals_before_any_gpu_work(lang):
    import paper_2609_31551_b200 as P
    x = torch.zeros(4, 2, 64)
    with pytest.raises(P.EasError) as e:
        P.prompt_attention(x, x, x, [0, 4])
    assert e.value.status == 1
    with pytest.raises(P.EasError):
        P.KvCache(0, 16, 2, 64)
