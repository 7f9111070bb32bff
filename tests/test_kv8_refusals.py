"""What the 8-bit cache's calls refuse, on the host, before anything is enqueued.  No GPU needed."""
import ctypes

import pytest
import torch

from paper_2509_17396_amd import binding as ep
from tests import kv8_util as ku

A, B = ctypes.c_void_p(4096), ctypes.c_void_p(8192)
ODD = ctypes.c_void_p(4104)


def fixture(**kw):
    prm = ku.params(2, 8, 2, 64, 4, 100, 4, budget=50, causal=1)
    cache = ku.Cache(2, 2, 128, 64, 32, device="cpu").kv8
    for name, val in kw.items():
        setattr(prm, name, val)
    return prm, cache


def calls(prm, cache):
    lib = ep.load()
    p, c = ctypes.byref(prm), ctypes.byref(cache)
    return {"size": lib.epicache_kv8_workspace_size(p, c, ctypes.byref(ctypes.c_size_t())),
            "append": lib.epicache_kv8_append(p, c, A, B, None, None, None),
            "attention": lib.epicache_kv8_attention(p, c, A, None, 1, A, A, A, 1 << 40, None),
            "evict": lib.epicache_kv8_evict(p, c, 0, None, None, A, None, A, 1 << 40, None)}


@pytest.mark.parametrize("field,value,status", [
    ("struct_size", 4, ep.ERR_INVALID_ARG), ("n_batch", 0, ep.ERR_INVALID_ARG), ("n_kv_heads", 3, ep.ERR_INVALID_ARG),
    ("head_dim", 0, ep.ERR_INVALID_ARG), ("head_dim", 40, ep.ERR_UNSUPPORTED), ("n_cached", -1, ep.ERR_INVALID_ARG),
    ("n_block", -1, ep.ERR_INVALID_ARG), ("n_cached", 125, ep.ERR_INVALID_ARG), ("dtype", 7, ep.ERR_INVALID_ARG),
    ("reserved", 1, ep.ERR_INVALID_ARG)])
def test_bad_params_are_refused_by_every_call(field, value, status):
    prm, cache = fixture()
    setattr(prm, field, value)
    assert set(calls(prm, cache).values()) == {status}


@pytest.mark.parametrize("field,value,status", [
    ("struct_size", 4, ep.ERR_INVALID_ARG), ("block_tokens", 8, ep.ERR_INVALID_ARG), ("block_tokens", 48, ep.ERR_INVALID_ARG),
    ("block_tokens", 256, ep.ERR_INVALID_ARG), ("capacity", 0, ep.ERR_INVALID_ARG), ("capacity", 103, ep.ERR_INVALID_ARG),
    ("reserved", 1, ep.ERR_INVALID_ARG), ("stride_t", 48, ep.ERR_INVALID_ARG), ("stride_t", 72, ep.ERR_INVALID_ARG),
    ("stride_h", 4096, ep.ERR_INVALID_ARG), ("stride_b", 8192, ep.ERR_INVALID_ARG), ("stride_b", -16, ep.ERR_INVALID_ARG),
    ("scale_stride_h", 3, ep.ERR_INVALID_ARG), ("scale_stride_b", 7, ep.ERR_INVALID_ARG), ("row_stride_h", 127, ep.ERR_INVALID_ARG),
    ("row_stride_b", 255, ep.ERR_INVALID_ARG), ("stride_t", 1 << 21, ep.ERR_UNSUPPORTED)])
def test_bad_caches_are_refused_by_every_call(field, value, status):
    prm, cache = fixture()
    setattr(cache, field, value)
    assert set(calls(prm, cache).values()) == {status}


@pytest.mark.parametrize("field", ["k", "v", "k_scale", "v_scale"])
def test_arrays_have_to_be_there_and_aligned(field):
    for value in (None, 4100):
        prm, cache = fixture()
        setattr(cache, field, value)
        got = calls(prm, cache)
        assert got.pop("size") == ep.OK and set(got.values()) == {ep.ERR_INVALID_ARG}
    prm, cache = fixture()
    cache.v = cache.k
    assert calls(prm, cache)["append"] == ep.ERR_INVALID_ARG


def test_too_many_heads_or_rows():
    prm, cache = fixture()
    prm.n_batch, cache.stride_b, cache.scale_stride_b, cache.row_stride_b = 40000, 1 << 20, 1 << 10, 1 << 10
    prm.q_stride_b = prm.kv_stride_b = 1 << 20
    assert set(calls(prm, cache).values()) == {ep.ERR_UNSUPPORTED}
    prm, cache = fixture()
    cache.capacity, cache.stride_h, cache.stride_b = (1 << 24) + 16, 1 << 31, 1 << 33
    cache.scale_stride_h, cache.scale_stride_b, cache.row_stride_h, cache.row_stride_b = 1 << 24, 1 << 26, 1 << 25, 1 << 27
    assert set(calls(prm, cache).values()) == {ep.ERR_UNSUPPORTED}


def test_append_refusals():
    lib, (prm, cache) = ep.load(), fixture()
    p, c = ctypes.byref(prm), ctypes.byref(cache)
    for args in ((None, B, None, None), (A, None, None, None), (ODD, B, None, None), (A, ODD, None, None), (A, B, ODD, None),
                 (A, B, None, ODD)):
        assert lib.epicache_kv8_append(p, c, *args, None) == ep.ERR_INVALID_ARG
    for field, value in (("kv_stride_t", 68), ("kv_stride_h", -8), ("kv_stride_b", 4)):
        prm, cache = fixture()
        setattr(prm, field, value)
        assert lib.epicache_kv8_append(ctypes.byref(prm), ctypes.byref(cache), A, B, None, None, None) == ep.ERR_INVALID_ARG
    prm, cache = fixture(n_block=0, causal_patch=0)
    assert lib.epicache_kv8_append(ctypes.byref(prm), ctypes.byref(cache), None, None, None, None, None) == ep.OK


def test_attention_refusals():
    lib, (prm, cache) = ep.load(), fixture()
    p, c = ctypes.byref(prm), ctypes.byref(cache)
    need = ep.epicache_kv8_workspace_size(prm, cache)
    call = lambda q=A, n=None, acc=0, out=A, lse=A, ws=A, size=need: \
        lib.epicache_kv8_attention(p, c, q, n, acc, out, lse, ws, size, None)
    for kw in (dict(q=None), dict(q=ODD), dict(out=None), dict(out=ODD), dict(lse=None), dict(lse=ODD), dict(n=ODD), dict(acc=2),
               dict(ws=ODD), dict(acc=1, ws=None)):
        assert call(**kw) == ep.ERR_INVALID_ARG, kw
    assert call(acc=1, size=0) == ep.ERR_WORKSPACE_TOO_SMALL
    cache.weight = None
    assert call(acc=1) == ep.ERR_INVALID_ARG
    for field, value, status in (("patch_len", 0, ep.ERR_INVALID_ARG), ("patch_len", 3, ep.ERR_INVALID_ARG),
                                 ("causal_patch", 2, ep.ERR_INVALID_ARG), ("softmax_scale", -1.0, ep.ERR_INVALID_ARG),
                                 ("softmax_scale", float("nan"), ep.ERR_INVALID_ARG), ("softmax_scale", 2e6, ep.ERR_UNSUPPORTED),
                                 ("q_stride_t", 56, ep.ERR_INVALID_ARG), ("q_stride_h", 250, ep.ERR_INVALID_ARG),
                                 ("q_stride_h", 64, ep.ERR_INVALID_ARG), ("q_stride_b", 64, ep.ERR_INVALID_ARG),
                                 ("q_stride_t", 1 << 21, ep.ERR_INVALID_ARG)):
        prm, cache = fixture()
        setattr(prm, field, value)
        assert lib.epicache_kv8_attention(ctypes.byref(prm), ctypes.byref(cache), A, None, 0, A, A, A, 1 << 40, None) == status, field


def test_too_many_queries():
    for kw in (dict(patch_len=(1 << 18) + 1), dict(patch_len=1 << 18, n_batch=30000)):
        prm, cache = fixture(causal_patch=0, n_cached=0, n_block=1)
        for name, val in kw.items():
            setattr(prm, name, val)
        prm.q_stride_h, prm.q_stride_b = 1 << 25, 1 << 29
        cache.stride_b, cache.scale_stride_b, cache.row_stride_b = 1 << 20, 1 << 10, 1 << 10
        assert ep.load().epicache_kv8_attention(ctypes.byref(prm), ctypes.byref(cache), A, None, 0, A, A, A, 1 << 40, None) == ep.ERR_UNSUPPORTED


def test_evict_refusals():
    lib, (prm, cache) = ep.load(), fixture()
    p, c = ctypes.byref(prm), ctypes.byref(cache)
    need = ep.epicache_kv8_workspace_size(prm, cache)
    call = lambda recent=0, n=None, m=None, kept=A, rows=None, ws=A, size=need: \
        lib.epicache_kv8_evict(p, c, recent, n, m, kept, rows, ws, size, None)
    for kw in (dict(recent=-1), dict(recent=51), dict(kept=None), dict(kept=ODD), dict(n=ODD), dict(m=ODD), dict(rows=ODD),
               dict(ws=None), dict(ws=ODD)):
        assert call(**kw) == ep.ERR_INVALID_ARG, kw
    assert call(size=16) == ep.ERR_WORKSPACE_TOO_SMALL
    prm.budget = 0
    assert call() == ep.ERR_INVALID_ARG
    prm.budget, cache.weight = 50, None
    assert call() == ep.ERR_INVALID_ARG


def test_struct_matches_a_c_compilers(tmp_path):
    import os
    import subprocess
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    src = tmp_path / "kv8.c"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "epicache.h"\nint main(void) { printf("%zu %zu %zu %zu\\n", '
                   "sizeof(epicache_kv8), offsetof(epicache_kv8, k), offsetof(epicache_kv8, position), "
                   "offsetof(epicache_kv8, row_stride_h)); return 0; }\n")
    subprocess.run(["gcc", "-std=c99", "-I", os.path.join(root, "include"), str(src), "-o", str(tmp_path / "kv8")], check=True)
    out = subprocess.run([str(tmp_path / "kv8")], check=True, capture_output=True, text=True).stdout.split()
    assert [int(x) for x in out] == [ctypes.sizeof(ep.Kv8), ep.Kv8.k.offset, ep.Kv8.position.offset, ep.Kv8.row_stride_h.offset]


def test_make_kv8_refuses_what_does_not_belong_together():
    k, v, ks, vs, w, pos = ep.alloc_kv8(1, 2, 64, 32, 16, device="cpu")
    ep.make_kv8(k, v, ks, vs, 16, w, pos)
    ep.make_kv8(k.view(torch.uint8), v.view(torch.uint8), ks, vs, 16)
    for bad in ((k.float(), v.float(), ks, vs, 16, w, pos), (k, v[:, :, :48], ks, vs, 16, w, pos), (k, v, ks, vs, 32, w, pos),
                (k, v, ks.double(), vs.double(), 16, w, pos), (k, v, ks, vs, 16, w[:, :1], pos), (k, v, ks, vs, 16, w.double(), pos),
                (k, v, ks, vs, 16, w, pos.long()), (k, v, ks, vs, 16, w.to("meta"), pos), (k.transpose(2, 3), v.transpose(2, 3), ks, vs, 16, w, pos)):
        with pytest.raises(ValueError):
            ep.make_kv8(*bad)
