"""The cache's and the query/key step's argument checks on the host (no GPU): every call below
is refused before anything touches the device."""
import ctypes
import math

import pytest

OK, ERR_ARG, ERR_ALIGN, ERR_WORKSPACE = 0, 1, 2, 5
A16 = 0x10000  # fake, never dereferenced
A2 = 0x10002


class Cache(ctypes.Structure):
    _fields_ = [("k_codes", ctypes.c_void_p), ("v_codes", ctypes.c_void_p),
                ("k_affine", ctypes.c_void_p), ("v_affine", ctypes.c_void_p),
                ("pages", ctypes.c_int), ("heads", ctypes.c_int), ("page_size", ctypes.c_int),
                ("head_dim", ctypes.c_int)]


@pytest.fixture(scope="module")
def lib(cuda_lib_path):
    lib = ctypes.CDLL(cuda_lib_path)
    p, i, d, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_double, ctypes.c_size_t
    lib.fdllm_qk_norm_rope.argtypes = [p, p, p, p, i, i, i, i, i, p, p, d, p, i, p, p, i, i, p, p, p]
    lib.fdllm_cache_append.argtypes = [p, p, i, i, p, p, p, p, p, p, i, i, p]
    lib.fdllm_cache_read.argtypes = [p, p, i, i, p, p, p, p, i, i, p]
    lib.fdllm_cache_attention.argtypes = [p, p, i, i, i, i, p, p, i, p, p, p, p, p, i, p, i, d, p, p,
                                          p, sz, p]
    lib.fdllm_cache_attention_workspace_bytes.argtypes = [i, i, i, i, i]
    lib.fdllm_cache_attention_workspace_bytes.restype = sz
    lib.fdllm_cache_key_weights.argtypes = [p, p, i, i, i, i, p, p, i, p, p, d, p, p, i, p]
    lib.fdllm_cache_evict.argtypes = [p, p, i, i, p, p, i, i, i, i, p, i, p, p, p, p]
    return lib


def cache(**kw):
    f = dict(k_codes=A16, v_codes=A16, k_affine=A16, v_affine=A16, pages=4, heads=2, page_size=64,
             head_dim=128)
    f.update(kw)
    return Cache(**f)


def strides(*s):
    return (ctypes.c_int64 * len(s))(*s)


BAD_CACHES = [(dict(k_codes=None), ERR_ARG), (dict(v_affine=None), ERR_ARG), (dict(pages=0), ERR_ARG),
              (dict(heads=0), ERR_ARG), (dict(page_size=48), ERR_ARG), (dict(page_size=16), ERR_ARG),
              (dict(page_size=512), ERR_ARG), (dict(head_dim=96), ERR_ARG),
              (dict(v_codes=A2), ERR_ALIGN), (dict(k_affine=A16 + 8), ERR_ALIGN)]


def append(lib, c, B=1, mp=4, table=A16, k=A16, ks=(256, 256, 128), dtype=0, n=3):
    return lib.fdllm_cache_append(ctypes.byref(c) if c else None, table, B, mp, None, None, k,
                                  strides(*ks), A16, strides(256, 256, 128), dtype, n, None)


def read(lib, c, table=A16, out=A16, n=3, dtype=0, B=1):
    return lib.fdllm_cache_read(ctypes.byref(c) if c else None, table, B, 4, None, None, out, A16,
                                dtype, n, None)


def attend(lib, c, q=A16, qs=(512, 512, 128), dtype=0, B=1, Lq=2, Hq=4, table=A16, mp=4, lens=A16,
           k=None, ks=(256, 256, 128), Ln=0, causal=0, scale=1.0, out=A16, ws=A16, wsb=1 << 40):
    s = strides(*ks)
    return lib.fdllm_cache_attention(q, strides(*qs), dtype, B, Lq, Hq,
                                     ctypes.byref(c) if c else None, table, mp, lens, k, s, k, s, Ln,
                                     None, causal, scale, out, None, ws, wsb, None)


def weigh(lib, c, q=A16, dtype=0, Lq=2, Hq=4, lse=A16, scale=1.0, out=A16, max_len=64,
          qs=(512, 512, 128)):
    return lib.fdllm_cache_key_weights(q, strides(*qs), dtype, 1, Lq, Hq,
                                       ctypes.byref(c) if c else None, A16, 4, A16, lse, scale, None,
                                       out, max_len, None)


def evict(lib, c, budget=8, first=0, last=0, weights=A16, dst=A16, dmp=1, out=A16, max_len=64):
    return lib.fdllm_cache_evict(ctypes.byref(c) if c else None, A16, 1, 4, A16, weights, max_len,
                                 budget, first, last, dst, dmp, out, A16, A16, None)


@pytest.mark.parametrize("call", [append, read, attend, weigh, evict])
@pytest.mark.parametrize("fields,want", BAD_CACHES)
def test_bad_caches(lib, call, fields, want):
    assert call(lib, cache(**fields)) == want


@pytest.mark.parametrize("call", [append, read, attend, weigh, evict])
def test_no_cache(lib, call):
    assert call(lib, None) == ERR_ARG


@pytest.mark.parametrize("kw,want", [
    (dict(B=0), ERR_ARG), (dict(mp=0), ERR_ARG), (dict(mp=1 << 25), ERR_ARG), (dict(table=None), ERR_ARG),
    (dict(k=None), ERR_ARG), (dict(dtype=3), ERR_ARG), (dict(n=-1), ERR_ARG), (dict(n=1 << 30), ERR_ARG),
    (dict(k=A2), ERR_ALIGN), (dict(ks=(256, 256, 100)), ERR_ALIGN), (dict(n=0), OK),
])
def test_append(lib, kw, want):
    assert append(lib, cache(), **kw) == want


@pytest.mark.parametrize("kw,want", [
    (dict(B=0), ERR_ARG), (dict(B=65536), ERR_ARG), (dict(table=None), ERR_ARG), (dict(out=None), ERR_ARG),
    (dict(out=A2), ERR_ALIGN), (dict(dtype=-1), ERR_ARG), (dict(n=-5), ERR_ARG), (dict(n=0), OK),
])
def test_read(lib, kw, want):
    assert read(lib, cache(), **kw) == want


@pytest.mark.parametrize("kw,want", [
    (dict(q=None), ERR_ARG), (dict(dtype=1), ERR_ARG), (dict(Lq=0), ERR_ARG), (dict(Hq=3), ERR_ARG),
    (dict(B=0), ERR_ARG), (dict(table=None), ERR_ARG), (dict(lens=None), ERR_ARG), (dict(Ln=4), ERR_ARG),
    (dict(Ln=-1), ERR_ARG), (dict(causal=2), ERR_ARG), (dict(scale=math.inf), ERR_ARG),
    (dict(scale=math.nan), ERR_ARG), (dict(out=None), ERR_ARG), (dict(q=A2), ERR_ALIGN),
    (dict(qs=(512, 512, 4)), ERR_ALIGN), (dict(out=A2), ERR_ALIGN), (dict(k=A2, Ln=4), ERR_ALIGN),
    (dict(k=A16, Ln=4, ks=(8, 12, 8)), ERR_ALIGN), (dict(ws=None), ERR_WORKSPACE),
    (dict(ws=A16 + 16), ERR_WORKSPACE), (dict(wsb=0), ERR_WORKSPACE),
])
def test_attention(lib, kw, want):
    assert attend(lib, cache(), **kw) == want


def test_attention_workspace(lib):
    f = lib.fdllm_cache_attention_workspace_bytes
    assert f(1, 1, 8, 2, 128) >= 256
    for bad in ((0, 1, 8, 2, 128), (1, 0, 8, 2, 128), (1, 1, 7, 2, 128), (1, 1, 8, 0, 128),
                (1, 1, 8, 2, 96)):
        assert f(*bad) == 0


@pytest.mark.parametrize("kw,want", [
    (dict(q=None), ERR_ARG), (dict(dtype=1), ERR_ARG), (dict(Lq=0), ERR_ARG), (dict(Hq=5), ERR_ARG),
    (dict(lse=None), ERR_ARG), (dict(scale=math.nan), ERR_ARG), (dict(out=None), ERR_ARG),
    (dict(max_len=0), ERR_ARG), (dict(q=A2), ERR_ALIGN), (dict(qs=(1, 8, 8)), ERR_ALIGN),
])
def test_key_weights(lib, kw, want):
    assert weigh(lib, cache(), **kw) == want


@pytest.mark.parametrize("kw", [
    dict(budget=0), dict(first=-1), dict(last=-1), dict(first=5, last=4), dict(weights=None),
    dict(dst=None), dict(dmp=0), dict(budget=65, dmp=1), dict(out=None), dict(max_len=0),
])
def test_evict(lib, kw):
    assert evict(lib, cache(), **kw) == ERR_ARG


def qk(lib, dtype=0, T=4, Hq=2, Hk=1, D=8, eps=1e-6, axes=1, sections=None, freq=(1.0, 0.5, 0.25, 0.1),
       pairs=None, inter=0, q=A16, pos=A16, out=A16):
    f = (ctypes.c_double * len(freq))(*freq)
    sec = None if sections is None else (ctypes.c_int * len(sections))(*sections)
    return lib.fdllm_qk_norm_rope(q, strides(64, 8), A16, strides(64, 8), dtype, T, Hq, Hk, D, None, None,
                                  eps, pos, axes, sec, f, len(freq) if pairs is None else pairs, inter,
                                  out, A16, None)


@pytest.mark.parametrize("kw,want", [
    (dict(dtype=3), ERR_ARG), (dict(T=-1), ERR_ARG), (dict(Hq=0), ERR_ARG), (dict(Hk=-1), ERR_ARG),
    (dict(D=7), ERR_ARG), (dict(D=514), ERR_ARG), (dict(eps=-1.0), ERR_ARG), (dict(eps=math.inf), ERR_ARG),
    (dict(axes=0), ERR_ARG), (dict(axes=5), ERR_ARG), (dict(axes=2), ERR_ARG),
    (dict(axes=2, sections=(2, 3)), ERR_ARG), (dict(axes=2, sections=(5, -1)), ERR_ARG),
    (dict(pairs=5), ERR_ARG), (dict(pairs=-1), ERR_ARG), (dict(freq=(1.0, math.nan)), ERR_ARG),
    (dict(inter=2), ERR_ARG), (dict(q=None), ERR_ARG), (dict(pos=None), ERR_ARG), (dict(out=None), ERR_ARG),
    (dict(T=0), OK),
])
def test_qk_norm_rope(lib, kw, want):
    assert qk(lib, **kw) == want
