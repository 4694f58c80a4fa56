"""The paged cache's host side without a GPU: refusals, the binding's structures, and the launch plans under sanitizers."""
import ctypes as C
import math
import os
import re
import shutil
import subprocess

import numpy as np
import pytest
import torch

import paper_2601_01204_amd as kvx
from oracle import paged_oracle as po
from paper_2601_01204_amd import paged

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
STUB = os.path.join(ROOT, "tests", "hip_stub")


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_host_code_under_asan_and_ubsan(tmp_path):
    exe = str(tmp_path / "paged_host_check")
    csrc = os.path.join(ROOT, "paper_2601_01204_amd", "csrc")
    cmd = ["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=undefined", "-static-libasan", "-I", STUB, "-I", csrc,
           "-include", os.path.join(STUB, "paged_host_types.h"), "-x", "c++", os.path.join(csrc, "paged_api.hip"), os.path.join(STUB, "paged_host_check.cpp"),
           "-o", exe]
    b = subprocess.run(cmd, capture_output=True, text=True, timeout=300)
    assert b.returncode == 0, b.stderr[-4000:]
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, (r.stdout + r.stderr)[-4000:]
    assert "paged host checks passed" in r.stdout


def test_structures_match_the_header():
    text = open(os.path.join(ROOT, "include", "kvx.h")).read()
    for name, struct in (("kv_paged_config", paged.KvPagedConfig), ("kv_rows", paged.KvRows), ("kv_pages", paged.KvPagesStruct),
                         ("kv_paged_batch", paged.KvPagedBatchStruct)):
        body = re.search(r"typedef struct %s \{(.*?)\} %s;" % (name, name), text, re.S).group(1)
        body = re.sub(r"/\*.*?\*/", "", body, flags=re.S)
        fields = []
        for decl in body.split(";"):
            if decl.strip():
                fields += [re.sub(r"^.*[\s*]", "", part.strip()) for part in decl.split(",")]
        assert fields == [n for n, _ in struct._fields_], name
        kinds = {"int32_t": C.c_int32, "int64_t": C.c_int64, "float": C.c_float, "double": C.c_double}
        for n, t in struct._fields_:
            decl = next(d for d in body.split(";") if re.search(r"[\s*,]%s(\s*,|\s*$)" % n, d))
            assert t is (C.c_void_p if "*" in decl else kinds[decl.split()[0]]), (name, n)


def _config(**kw):
    base = dict(n_q_heads=8, n_kv_heads=2, head_dim=64, page_size=16, dtype=kvx.KV_BF16, cache_dtype=kvx.KV_BF16, max_seqs=2, max_tokens=8, max_len=100)
    base.update(kw)
    c = kvx.KvPagedConfig()
    for k, v in base.items():
        setattr(c, k, v)
    return c


@pytest.mark.parametrize("bad", [
    dict(n_q_heads=0), dict(n_q_heads=9), dict(n_q_heads=2048, n_kv_heads=256), dict(n_kv_heads=0), dict(n_kv_heads=257, n_q_heads=257),
    dict(n_q_heads=258, n_kv_heads=2), dict(head_dim=96), dict(head_dim=0), dict(page_size=4), dict(page_size=24), dict(page_size=2048), dict(page_size=0),
    dict(dtype=kvx.KV_F32), dict(dtype=kvx.KV_E4M3), dict(dtype=9), dict(cache_dtype=kvx.KV_F16), dict(cache_dtype=-1), dict(max_seqs=0),
    dict(max_seqs=65537), dict(max_tokens=0), dict(max_tokens=(1 << 22) + 1), dict(max_len=0), dict(max_len=(1 << 27) + 1), dict(max_evicted=-1),
    dict(max_evicted=101), dict(softmax_scale=-1.0), dict(softmax_scale=math.nan), dict(rotary_dim=8), dict(rotary_dim=80), dict(rotary_dim=-16),
    dict(rope_layout=2), dict(rope_scaling=4), dict(rope_scaling=-1), dict(rope_base=1.0), dict(rope_base=math.inf), dict(rope_factor=0.5),
    dict(rope_factor=math.nan), dict(rope_magnitude=-1.0), dict(rope_magnitude=math.inf), dict(rotary_dim=16, rope_scaling=3),
    dict(rotary_dim=16, rope_scaling=3, rope_original_len=100, rope_low_turns=4.0), dict(rope_low_turns=-1.0)])
def test_bad_configurations_are_refused_with_a_message(bad):
    lib = paged._library()
    h = C.c_void_p()
    assert lib.kv_paged_init(C.byref(_config(**bad)), C.byref(h)) == -1
    assert not h.value and len(lib.kv_paged_last_error(None)) > 10


def test_frequencies_that_are_not_finite_are_refused():
    freqs = (C.c_double * 8)(*([0.5] * 7 + [math.nan]))
    h = C.c_void_p()
    assert paged._library().kv_paged_init(C.byref(_config(rotary_dim=16, rope_freqs=C.cast(freqs, C.c_void_p))), C.byref(h)) == -1


def test_null_arguments():
    lib = paged._library()
    h = C.c_void_p()
    assert lib.kv_paged_init(None, C.byref(h)) == -1
    assert lib.kv_paged_init(C.byref(_config()), None) == -1
    assert lib.kv_paged_append(None, None, None, None, None, None, None, None, None) == -1
    assert lib.kv_paged_attend(None, None, None, None, None, None, 1, 0, None, None) == -1
    assert lib.kv_paged_evict(None, None, None, 1, 0, 0, None, None, None, None) == -1
    assert lib.kv_paged_status(None, None) == -1
    lib.kv_paged_destroy(None)


def _pool(**kw):
    args = dict(k_pages=torch.zeros(4, 16, 2, 64, dtype=torch.bfloat16), v_pages=torch.zeros(4, 16, 2, 64, dtype=torch.bfloat16),
                page_table=torch.zeros(3, 2, dtype=torch.int32))
    args.update(kw)
    return kvx.KvPages(**args)


@pytest.mark.parametrize("bad", [
    dict(k_pages=torch.zeros(4, 16, 64, dtype=torch.bfloat16)), dict(v_pages=torch.zeros(4, 16, 2, 64, dtype=torch.float16)),
    dict(v_pages=torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16).transpose(1, 2)), dict(page_table=torch.zeros(3, 2)),
    dict(page_table=torch.zeros(6, dtype=torch.int32)), dict(page_table=torch.zeros(2, 3, dtype=torch.int32).T), dict(weights=torch.zeros(4, 16, 2)),
    dict(ids=torch.zeros(4, 2, 16)), dict(k_scale=torch.ones(3)), dict(v_scale=torch.ones(2, dtype=torch.float64))])
def test_the_binding_refuses_pools(bad):
    _pool()
    with pytest.raises(AssertionError):
        _pool(**bad)


def test_the_binding_refuses_tables_whose_rows_overlap():
    one = torch.zeros(1, 4, dtype=torch.int32)
    with pytest.raises(AssertionError):
        _pool(page_table=one.expand(3, 4))
    with pytest.raises(AssertionError):
        _pool(page_table=torch.zeros(8, dtype=torch.int32).as_strided((3, 4), (2, 1)))
    assert _pool(page_table=one.expand(3, 4)[:1]).struct.table_stride == 4


@pytest.mark.parametrize("bad", [dict(q_start=torch.zeros(2, dtype=torch.int32)), dict(kv_lens=torch.zeros(2)), dict(q_start=torch.zeros(6, dtype=torch.int32)[::2]),
                                 dict(seen=torch.zeros(3, dtype=torch.int32)), dict(seen=torch.zeros(2, dtype=torch.int64))])
def test_the_binding_refuses_batches(bad):
    args = dict(q_start=torch.zeros(3, dtype=torch.int32), kv_lens=torch.zeros(2, dtype=torch.int32), n_tokens=4, max_new=2, max_len=9)
    kvx.KvPagedBatch(**args)
    with pytest.raises(AssertionError):
        kvx.KvPagedBatch(**{**args, **bad})


def test_unknown_fields_are_refused():
    with pytest.raises(TypeError):
        kvx.KvPaged(n_q_heads=1, n_kv_heads=1, pages=3)


# ---- the oracle against cases worked out by hand -----------------------------------------------------------------------
def test_oracle_rotation():
    x = np.zeros((2, 1, 6))
    x[:, 0] = [1, 0, 2, 0, 5, 6]
    y = po.rotate(x, [0, 1], np.array([np.pi / 2, np.pi]), interleaved=False)
    assert np.allclose(y[0], x[0]) and np.allclose(y[1, 0], [-2, 0, 1, 0, 5, 6])           # channels 0 and 2 a quarter turn, 1 and 3 half a turn
    y = po.rotate(x, [0, 1], np.array([np.pi / 2, np.pi]), interleaved=True)
    assert np.allclose(y[1, 0], [0, 1, -2, 0, 5, 6])
    assert np.allclose(po.rope_frequencies(4, base=100.0), [1.0, 0.1]) and np.allclose(po.rope_frequencies(4, "linear", 100.0, 2.0), [0.5, 0.05])
    assert np.allclose(po.rope_frequencies(4, "base", 100.0, 3.0), [1.0, 1 / 30]) and np.allclose(po.rope_frequencies(4, "parts", 100.0, 2.0, 2 * np.pi * 10, 2.0, 4.0), [1.0, 0.05])


def test_oracle_attention():
    pool = dict(k=np.zeros((3, 8, 1, 2)), v=np.zeros((3, 8, 1, 2)), table=np.array([[2, 0]]))
    for j, (k, v) in enumerate([(0.0, 1.0), (math.log(2.0), 2.0), (math.log(3.0), 4.0)] + [(0.0, 0.0)] * 6):
        p = po.place(pool, 0, j)
        assert p == ((2, j) if j < 8 else (0, j - 8))
        pool["k"][p[0], p[1], 0], pool["v"][p[0], p[1], 0] = [k, 9], [v, -v]
    out, lse, gained, _, _ = po.attend(pool, np.array([[[1.0, 0.0]], [[1.0, 0.0]]]), [0, 2], [3], 1.0)
    assert np.allclose(out[:, 0, 0], [5 / 3, 17 / 6]) and np.allclose(out[:, 0, 1], [-5 / 3, -17 / 6]) and np.allclose(lse[:, 0], [math.log(3), math.log(6)])
    assert np.allclose(gained[2, 0, :3], [1 / 3 + 1 / 6, 2 / 3 + 1 / 3, 1 / 2]) and gained.sum() == pytest.approx(2)
    out, lse, _, _, _ = po.attend(pool, np.array([[[1.0, 0.0]]]), [0, 1], [3], 1.0, window=1)
    assert np.allclose(out[0, 0], [4, -4])
    out, lse, _, _, _ = po.attend(pool, np.ones((3, 1, 2)), [0, 3], [1], 1.0)               # two rows before the sequence begins
    assert np.array_equal(out[:2], np.zeros((2, 1, 2))) and np.isneginf(lse[:2]).all() and np.isfinite(lse[2]).all()


def test_oracle_eviction():
    pool = dict(k=np.arange(16.0).reshape(2, 8, 1, 1), v=np.zeros((2, 8, 1, 1)), table=np.array([[1, 0]]), weights=np.zeros((2, 1, 8), np.float32),
                ids=np.zeros((2, 1, 8), np.int32))
    pool["weights"][1, 0] = [5, 1, 3, 3, 0, 9, 3, np.nan]
    pool["ids"][1, 0] = range(8)
    pool["weights"][0, 0, :2] = [0, 4]
    pool["ids"][0, 0, :2] = [8, 9]
    k, _, w, ids, lens, written = po.evict(pool, [10], [10], 5, 0, 1)
    # token 9 is the last one and stays; of the others 5 (9), 0 (5) and, of weight 3, slots 2 and 3; 5 moves to slot 1, 9 to slot 4
    assert ids[1, 0, :5].tolist() == [0, 5, 2, 3, 9] and w[1, 0, :5].tolist() == [5, 9, 3, 3, 4] and lens.tolist() == [5]
    assert k[1, :5, 0, 0].tolist() == [8, 13, 10, 11, 1] and written.sum() == 5
