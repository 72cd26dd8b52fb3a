"""CPU-only checks of the language-model operators' host side: refusals and rules that need no GPU."""
import ctypes as C
import os
import re
import shutil
import time

import numpy as np
import pytest


@pytest.fixture(scope="module")
def lang():
    from paper_2609_31551_b200.build import build_library
    build_library()
    from paper_2609_31551_b200 import language
    language.lib()
    return language


@pytest.mark.parametrize("place", [0, 60, 129])
def test_too_many_query_rows_are_refused_before_any_launch(lang, place):
    """130 sequences take two launches, the ones with the most keys first; the one with too many rows has the fewest."""
    lens_q, lens_k = [1] * 130, [9] * 130
    lens_q[place], lens_k[place] = (1 << 25) + 2, 1
    cu_q, cu_k = (np.concatenate([[0], np.cumsum(x)]).astype(np.int32) for x in (lens_q, lens_k))
    pin = lang.PromptInputs(1 << 20, 1 << 21, 1 << 22, 1 << 23, 128 * 128, 128, 128, 128 * 128, 0, 128, 1, 128, 0.1, 130, cu_q.ctypes.data, cu_k.ctypes.data)
    assert lang.lib().eas_prompt_attention(C.byref(pin), None, 0, 0, None, 1 << 24) == 2
    assert b"too many query rows" in lang.lib().eas_last_error()


@pytest.mark.parametrize("bad", [[0, 4.7], [0, 2 ** 31], np.array([0, 2 ** 32 + 5]), np.array([0, 2 ** 32 + 5], dtype=np.uint64), [0, float("nan")], [0, 1e30], ["0", "5"], [[0], [1, 2]], [0, None], []])
def test_offsets_that_are_no_32_bit_numbers_are_refused(lang, bad):
    import paper_2609_31551_b200 as P
    for pair in ((bad, None), ([0, 5], bad)):
        with pytest.raises(P.EasError) as e:
            P.prompt_attention_workspace_bytes(4, 2, 64, *pair)
        assert e.value.status == 1


@pytest.mark.parametrize("good", [[0, 5], (0, 5), [0.0, 5.0], np.array([0, 5]), np.array([0, 9, 5], dtype=np.uint8)[::2]])
def test_offsets_of_other_types_are_taken(lang, good):
    x, at = lang._host_ints(good, "cu")
    assert x.dtype == np.int32 and x.tolist() == [0, 5] and at == x.ctypes.data


@pytest.mark.parametrize("name", ["kv_cache.cuh", "attention_cache.cuh", "attention_prompt.cuh"])
def test_kernels_read_what_earlier_kernels_write_by_ordered_loads(name):
    """A kernel may start before the one in front of it has ended; only loads that are not of the read-only path stay behind its wait."""
    import paper_2609_31551_b200 as P
    src = re.sub(r"//.*", "", open(os.path.join(os.path.dirname(P.__file__), "csrc", name)).read())
    assert not re.search(r"__ldg\b|ld\.global\.nc|__restrict__", src)


def test_objects_are_made_again_when_the_flags_change(tmp_path, monkeypatch):
    from paper_2609_31551_b200 import build
    (tmp_path / "csrc").mkdir()
    (tmp_path / "include").mkdir()
    (tmp_path / "csrc" / "one.cpp").write_text('extern "C" int answer() { return ANSWER; }\n')
    (tmp_path / "csrc" / "two.cpp").write_text('extern "C" int two() { return 2; }\n')
    monkeypatch.setattr(build, "HERE", str(tmp_path / "csrc"))
    monkeypatch.setattr(build, "CSRC", str(tmp_path / "csrc"))
    monkeypatch.setattr(build, "SOURCES", ["one.cpp", "two.cpp"])
    ran, run = [], build._run
    monkeypatch.setattr(build, "_run", lambda cmd: ran.append(cmd) or run(cmd))
    (tmp_path / "lib").mkdir()
    monkeypatch.setattr(build, "LIB_PATH", str(tmp_path / "lib" / "lib.so"))
    for i, (answer, compiled) in enumerate(((41, 2), (41, 0), (42, 2), (42, 0))):
        monkeypatch.setattr(build, "NVCC_FLAGS", ["-O1", "-std=c++17", "-Xcompiler", "-fPIC", f"-DANSWER={answer}"])
        ran.clear()
        path = build.build_library()
        assert sum("-c" in cmd for cmd in ran) == compiled
        assert C.CDLL(shutil.copy(path, tmp_path / f"copy{i}.so")).answer() == answer      # (a copy: a library that is loaded is not loaded again)
    (tmp_path / "csrc" / "two.cpp").write_text('extern "C" int two() { return 3; }\n')
    os.utime(tmp_path / "csrc" / "two.cpp", (time.time() + 5, time.time() + 5))
    ran.clear()
    build.build_library()
    assert sum("-c" in cmd for cmd in ran) == 1
