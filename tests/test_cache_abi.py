"""The cache's part of the C ABI: exports, layouts, argument checks (no GPU needed), and the reference that the GPU tests use."""
import ctypes
import os
import re

import numpy as np
import pytest
import torch

from paper_2607_09385_b200 import binding as B
from paper_2607_09385_b200 import cache as C

import cache_reference as R


def params(**kw):
    return C.CacheParams(**dict(dict(layers=2, pages=10, page_tokens=64, heads_kv=2, head_dim=128, slots=4, max_pages=8), **kw))


def test_library_exports_every_declared_symbol(repo_root):
    text = open(os.path.join(repo_root, "include", "steel_cache.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    names = set(re.findall(r"\b(steel_cache_[a-z_]+)\s*\(", text))
    assert names == set(C.EXPORTS)
    lib = C.load_library()
    assert all(getattr(lib, n) is not None for n in names)
    assert "free pages" in B.steel_status_string(C.STEEL_ERR_NO_PAGES)


def test_struct_layouts_match_header(tmp_path, repo_root):
    import subprocess
    src = tmp_path / "s.c"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "steel_cache.h"\nint main(void) { printf("%zu %zu %zu %zu %zu %zu %zu %zu\\n", '
                   "sizeof(steel_cache_params_t), sizeof(steel_cache_sizes_t), sizeof(steel_cache_memory_t), sizeof(steel_cache_tensor_t), "
                   "sizeof(steel_cache_attend_t), offsetof(steel_cache_attend_t, scale), offsetof(steel_cache_attend_t, q), "
                   "offsetof(steel_cache_attend_t, workspace_bytes)); return 0; }\n")
    exe = str(tmp_path / "s")
    subprocess.check_call(["gcc", "-std=c11", "-I", os.path.join(repo_root, "include"), "-o", exe, str(src)])
    got = [int(x) for x in subprocess.check_output([exe], text=True).split()]
    a = C.CacheAttend
    assert got == [ctypes.sizeof(x) for x in (C.CacheParams, C.CacheSizes, C.CacheMemory, C.CacheTensor, a)] + \
        [a.scale.offset, a.q.offset, a.workspace_bytes.offset]


@pytest.mark.parametrize("kw,status", [
    (dict(layers=0), 1), (dict(pages=-1), 1), (dict(slots=0), 1), (dict(max_pages=0), 1), (dict(heads_kv=0), 1), (dict(page_tokens=0), 1),
    (dict(head_dim=96), 2), (dict(page_tokens=8), 2), (dict(page_tokens=48), 2), (dict(slots=8193), 2), (dict(pages=(1 << 20) + 1), 2),
    (dict(max_pages=1 << 24), 2), (dict(heads_kv=1025), 2), (dict(layers=5000), 2),
    (dict(max_pages=1 << 20, page_tokens=128, heads_kv=1024), 2)])
def test_sizes_refuse(kw, status):
    assert C.load_library().steel_cache_sizes(ctypes.byref(params(**kw)), ctypes.byref(C.CacheSizes())) == status


def test_sizes():
    s = C.steel_cache_sizes(params())
    assert s["unit_bytes"] == 2304 and s["page_bytes"] == 2304 * 4 * 2 and s["pool_bytes"] == s["page_bytes"] * 20
    assert s["table_bytes"] == 4 * 8 * 4 and s["refs_bytes"] == 40 and s["lens_bytes"] == 16
    assert C.steel_cache_sizes(params(head_dim=64))["unit_bytes"] == 1152
    # extend: a move a slot; fork: a row and two lengths a slot; compact: half the pages' moves and a rank a page
    for kw in (dict(max_pages=1), dict(max_pages=8), dict(pages=5000)):
        p = params(**kw)
        most = max(p.slots * 16, p.slots * (p.max_pages + 2) * 4, (p.pages + 1) // 2 * 16 + p.pages * 4)
        assert most + 128 <= C.steel_cache_sizes(p)["scratch_bytes"] <= most + 256
    lib = C.load_library()
    assert lib.steel_cache_sizes(None, ctypes.byref(C.CacheSizes())) == B.STEEL_ERR_INVALID_ARG
    assert lib.steel_cache_sizes(ctypes.byref(params()), None) == B.STEEL_ERR_INVALID_ARG


def test_null_handles_and_arguments():
    lib, handle = C.load_library(), ctypes.c_void_p(7)
    t = ctypes.byref(C.CacheTensor())
    bad = B.STEEL_ERR_INVALID_ARG
    assert lib.steel_cache_create(None, None, ctypes.byref(handle)) == bad and handle.value is None
    assert lib.steel_cache_create(ctypes.byref(params()), None, ctypes.byref(handle)) == bad
    assert lib.steel_cache_create(ctypes.byref(params()), ctypes.byref(C.CacheMemory()), ctypes.byref(handle)) == bad
    assert lib.steel_cache_create(ctypes.byref(params()), ctypes.byref(C.CacheMemory()), None) == bad
    for at in range(6):  # each pointer has to be there, and aligned
        for wrong in (None, 4096 + (2 if 0 < at < 4 else 64)):
            m = C.CacheMemory(*[4096] * 6)
            setattr(m, C.CacheMemory._fields_[at][0], wrong)
            assert lib.steel_cache_create(ctypes.byref(params()), ctypes.byref(m), ctypes.byref(handle)) == bad, (at, wrong)
    assert lib.steel_cache_destroy(None) == B.STEEL_OK
    assert lib.steel_cache_reset(None, None) == bad and lib.steel_cache_last_status(None, None) == bad
    assert lib.steel_cache_extend(None, 1, None, None, None) == bad
    assert lib.steel_cache_append(None, 0, 1, None, None, 1, t, t, None) == bad
    assert lib.steel_cache_read(None, 0, 1, None, None, 1, t, t, None) == bad
    assert lib.steel_cache_attend(None, ctypes.byref(C.CacheAttend()), None) == bad and lib.steel_cache_attend(None, None, None) == bad
    assert lib.steel_cache_attend_workspace(None, 1, 1, 1) < 0
    assert lib.steel_cache_fork(None, 1, None, None, None) == bad and lib.steel_cache_free(None, 1, None, None, None) == bad
    assert lib.steel_cache_compact(None, None, None) == bad


def test_create_without_gpu_fails_loudly():
    if torch.cuda.is_available():
        return
    handle = ctypes.c_void_p(7)
    m = C.CacheMemory(*[4096] * 6)
    assert C.load_library().steel_cache_create(ctypes.byref(params()), ctypes.byref(m), ctypes.byref(handle)) == B.STEEL_ERR_CUDA
    assert handle.value is None


@pytest.mark.parametrize("d", [64, 128])
def test_reference_units_round_trip(d):
    # the reference's two directions are written apart; a value read back is within half a step of what went in
    rng = np.random.default_rng(d)
    k, v = (rng.standard_normal((16, d)) for _ in "kv")
    qk, qv = R.quantise(k), R.quantise(v)
    unit = np.frombuffer(R.unit_of(*qk, *qv), np.uint8)
    assert unit.size == 16 * d + d // 64 * 128
    for x, (code, scale, zero), got in zip((k, v), (qk, qv), R.decode_units(unit, d)):
        assert np.array_equal(got, scale * code + zero)
        # half a step, and what rounding scale (15 steps of it) and zero to fp16 adds
        assert (np.abs(got - x) <= scale * (0.5 + 15 * 2.0 ** -11 + 2.0 ** -11) + np.abs(zero) * 2.0 ** -11).all()


def test_reference_model_shares_copies_and_compacts():
    m = R.Model(6, 16, 3, 4)
    assert m.extend([0], [20]) == "ok" and m.rows[0] == [0, 1]
    assert m.fork([0, 0], [1, 2]) == "ok" and m.refs[:2] == [3, 3]
    assert m.extend([2, 0], [1, 13]) == "ok" and m.rows[2] == [0, 2] and m.rows[0] == [0, 3, 4] and m.copies == [(1, 2, 1), (1, 3, 1)]
    assert m.extend([1], [40]) == "no pages" and m.extend([1, 1], [1, 1]) == "invalid"
    assert m.free([0], [0]) == "ok" and m.refs == [2, 1, 1, 0, 0, 0]
    assert m.free([2], [3]) == "ok" and m.rows[2] == [0] and m.free([1], [0]) == "ok"
    assert m.extend([0], [17]) == "ok" and m.rows[0] == [1, 2] and m.free([2], [0]) == "ok"
    assert m.compact() == (2, {2: 0}) and m.rows[0] == [1, 0]


def test_debug_wait_refuses_no_cache():
    assert C.load_library().steel_cache_debug_wait(None, 0) == B.STEEL_ERR_INVALID_ARG
