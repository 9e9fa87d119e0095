"""The oracle of the paged cache against what it must agree with: the one-axis rotation, direct formulas, and what the definition of the
eviction implies.  And the entry points' refusals, which need no GPU."""
import ctypes

import numpy as np
import pytest

from oracle import cache as OC
from oracle import stack as OS


def test_one_axis_is_the_plain_rotation():
    rng = np.random.default_rng(1)
    x, pos = rng.standard_normal((9, 3, 32)), rng.integers(0, 5000, 9)
    want = OS.rope(x, pos, 10000.0)
    assert np.allclose(OC.rope_axes(x, pos[:, None], [16], 10000.0, False), want, atol=1e-12)
    # with one section the axis's own ladder is the shared one
    assert np.allclose(OC.rope_axes(x, pos[:, None], [16], 10000.0, True), want, atol=1e-12)


def test_equal_positions_on_all_axes_are_one_axis():
    rng = np.random.default_rng(2)
    x, pos = rng.standard_normal((5, 2, 48)), rng.integers(0, 300, (5, 1))
    one = OC.rope_axes(x, pos, [24], 500.0, False)
    assert np.allclose(OC.rope_axes(x, np.repeat(pos, 3, 1), [7, 9, 8], 500.0, False), one, atol=1e-12)
    # scores between two rotated rows go by the differences of the positions
    q, k = rng.standard_normal((1, 1, 48)), rng.standard_normal((1, 1, 48))
    dot = lambda a, b: float((OC.rope_axes(q, [a], [7, 9, 8], 500.0, True) * OC.rope_axes(k, [b], [7, 9, 8], 500.0, True)).sum())
    assert dot([5, 9, 2], [3, 1, 7]) == pytest.approx(dot([105, 59, 22], [103, 51, 27]), abs=1e-10)


def test_pairs_behind_the_sections_stay():
    rng = np.random.default_rng(3)
    x = rng.standard_normal((4, 2, 32))
    y = OC.rope_axes(x, rng.integers(1, 99, (4, 2)), [5, 6], 10000.0, True)
    assert np.array_equal(y[:, :, 11:16], x[:, :, 11:16]) and np.array_equal(y[:, :, 27:], x[:, :, 27:])


def test_attend_gives_probabilities():
    rng = np.random.default_rng(4)
    q, k, v = rng.standard_normal((3, 4, 8)), rng.standard_normal((7, 2, 8)), rng.standard_normal((7, 2, 8))
    o, lse, got = OC.attend(q, k, v, 0.3, False)
    assert got.sum() == pytest.approx(3.0)
    x = 0.3 * k[:, 1] @ q[2, 3]
    assert lse[2, 3] == pytest.approx(np.log(np.exp(x).sum())) and np.allclose(o[2, 3], np.exp(x - lse[2, 3]) @ v[:, 1])
    oc, lc, gc = OC.attend(q, k, v, 0.3, True)
    assert np.allclose(oc[2], o[2]) and gc[6] < got[6]           # the last row sees all, the last slot has one row
    assert np.allclose(oc[0], OC.attend(q[:1], k[:5], v[:5], 0.3, False)[0][0])
    # more rows than slots: the first ones see nothing
    oe, le, ge = OC.attend(q, k[:2], v[:2], 0.3, True)
    assert not oe[0].any() and np.isneginf(le[0]).all() and ge.sum() == pytest.approx(2.0)


def test_evict_keeps_the_heaviest_and_moves_little():
    rng = np.random.default_rng(5)
    for n, keep, first, recent in [(50, 20, 0, 0), (50, 45, 3, 7), (1, 1, 0, 0), (9, 0, 2, 2), (40, 10, 6, 8), (12, 30, 1, 1)]:
        w, tok = rng.integers(0, 6, n).astype(np.float64), rng.permutation(n)
        src = OC.evict(w, tok, keep, first, recent)
        k = min(keep, n)
        assert len(set(src.tolist())) == len(src) == k
        held = (tok < first) | (tok > n - 1 - recent)
        gone = np.setdiff1d(np.arange(n), src)
        if held.sum() <= k:
            assert held[src].sum() == held.sum()
            free = src[~held[src]]
            if len(gone) and len(free):
                assert w[gone].max() <= w[free].min()
                if w[gone].max() == w[free].min():               # the lower slot of a tie stays
                    t = w[gone].max()
                    assert gone[w[gone] == t].min() > free[w[free] == t].max()
        moved = src != np.arange(k)
        assert (src[moved] >= k).all() and (np.diff(src[moved]) > 0).all()


# ---- refusals (no GPU: the addresses are never read on the host, and a refused call enqueues nothing) -----------------------------
INVALID, SMALL, UNSUPPORTED = 1, 3, 4


@pytest.fixture(scope="module")
def B():
    from paper_2511_12280_amd import binding
    return binding


def _lib(B):
    lib = ctypes.CDLL(B.LIB_PATH)
    for f in ("d3tom_rope_axes", "d3tom_cache_append", "d3tom_attend_cache", "d3tom_cache_evict"):
        getattr(lib, f).restype = ctypes.c_int
    return lib


AT = 1 << 20
P = ctypes.c_void_p(AT)
i32, i64, f32, sz = ctypes.c_int, ctypes.c_int64, ctypes.c_float, ctypes.c_size_t


def _cache(lib, **kw):
    c = lib._PagedCacheStruct(AT, AT, AT, AT, 40, 16, 20, 2, 2, 64, lib.D3TOM_BF16)
    for name, v in kw.items():
        setattr(c, name, v)
    return c


BAD_CACHES = [(dict(k_pages=0), INVALID), (dict(v_pages=AT + 8), INVALID), (dict(page_table=0), INVALID), (dict(kv_len=0), INVALID), (dict(dt=7), INVALID),
              (dict(num_pages=0), INVALID), (dict(B=0), INVALID), (dict(Hkv=0), INVALID), (dict(page_size=0), INVALID), (dict(table_stride=0), INVALID),
              (dict(page_size=8), UNSUPPORTED), (dict(page_size=48), UNSUPPORTED), (dict(page_size=8192), UNSUPPORTED), (dict(dh=12), UNSUPPORTED),
              (dict(dh=264), UNSUPPORTED), (dict(B=65536), UNSUPPORTED)]


def _axes(B, **kw):
    a = B._AxesStruct(AT, 3, (ctypes.c_int32 * 4)(10, 12, 10, 0), 0, 10000.0)
    for name, v in kw.items():
        setattr(a, name, (ctypes.c_int32 * 4)(*v) if name == "pairs" else v)
    return a


BAD_AXES = [dict(pos=0), dict(axes=0), dict(axes=5), dict(axes=-1), dict(ladder=2), dict(theta=1.0), dict(theta=float("nan")), dict(theta=float("inf")),
            dict(pairs=(10, 0, 10, 0)), dict(pairs=(10, 13, 10, 0)), dict(pairs=(2 ** 31 - 1, 2 ** 31 - 1, 3, 0)), dict(pairs=(-4, 12, 10, 0))]


def _rope(lib, axes, q=P, qs=256, k=P, ks=128, dt=1, rows=5, H=4, Hkv=2, dh=64, qo=P, ko=P):
    return lib.d3tom_rope_axes(q, i64(qs), k, i64(ks), i32(dt), i32(rows), i32(H), i32(Hkv), i32(dh), ctypes.byref(axes) if axes is not None else None, qo, ko, None)


def test_rope_axes_refuses(B):
    lib = _lib(B)
    for bad in BAD_AXES:
        assert _rope(lib, _axes(B, **bad)) == INVALID, bad
    good = _axes(B)
    odd = ctypes.c_void_p(AT + 2)
    for kw in (dict(q=None, k=None), dict(qo=None), dict(ko=None), dict(qs=255), dict(qs=260), dict(ks=127), dict(q=odd), dict(k=odd), dict(qo=odd), dict(ko=odd),
               dict(rows=0), dict(rows=-1), dict(H=0), dict(Hkv=0), dict(dt=2), dict(dh=0)):
        assert _rope(lib, good, **kw) == INVALID, kw
    assert _rope(lib, None) == INVALID
    for kw in (dict(dh=72, qs=1024, ks=1024), dict(dh=264, qs=2048, ks=2048), dict(dh=260, dt=0, qs=2048, ks=2048), dict(rows=16000001), dict(rows=2 ** 31 - 1),
               dict(H=65536, qs=1 << 22), dict(Hkv=65536, ks=1 << 22)):
        assert _rope(lib, good, **kw) == UNSUPPORTED, kw


def _append(lib, B, cache=None, axes=None, k=P, ks=128, v=P, vs=128, off=P, rows=5, most=3, q=None, qs=256, H=4, qo=None, tok=None, st=None, sw=None, stride=0):
    return lib.d3tom_cache_append(ctypes.byref(cache if cache is not None else _cache(B)), k, i64(ks), v, i64(vs), off, i32(rows), i32(most),
                                  ctypes.byref(axes) if axes is not None else None, q, i64(qs), i32(H), qo, tok, st, sw, i32(stride), None)


def test_cache_append_refuses(B):
    lib = _lib(B)
    for bad, status in BAD_CACHES:
        assert _append(lib, B, cache=_cache(B, **bad)) == status, bad
    for bad in BAD_AXES:
        assert _append(lib, B, axes=_axes(B, **bad)) == INVALID, bad
    for kw in (dict(k=None), dict(v=None), dict(ks=120), dict(vs=132), dict(off=None), dict(rows=0), dict(most=0), dict(most=6), dict(q=P, qo=P),
               dict(axes=_axes(B), q=P), dict(axes=_axes(B), q=P, qo=P, qs=100), dict(axes=_axes(B), q=P, qo=P, H=0), dict(st=P, stride=4), dict(tok=P, st=P),
               dict(sw=P), dict(sw=P, stride=-3)):
        assert _append(lib, B, **kw) == INVALID, kw
    assert lib.d3tom_cache_append(None, P, i64(128), P, i64(128), P, i32(5), i32(3), None, None, i64(0), i32(4), None, None, None, None, i32(0), None) == INVALID
    assert _append(lib, B, cache=_cache(B, dh=8), ks=16, vs=16, axes=_axes(B, pairs=(1, 1, 1, 0))) == UNSUPPORTED
    for kw in (dict(rows=16000001, most=16000001), dict(cache=_cache(B, B=65535), rows=4000, most=245), dict(axes=_axes(B), q=P, qo=P, H=65536, qs=1 << 22)):
        assert _append(lib, B, **kw) == UNSUPPORTED, kw


def _attend(lib, B, cache=None, q=P, qs=256, off=P, rows=5, most=3, max_len=320, H=4, scale=0.125, causal=0, o=P, lse=None, wi=None, wo=None, stride=0, ws=P,
            nbytes=1 << 40):
    return lib.d3tom_attend_cache(q, i64(qs), ctypes.byref(cache if cache is not None else _cache(B)), off, i32(rows), i32(most), i32(max_len), i32(H), f32(scale),
                                  i32(causal), o, lse, wi, wo, i32(stride), ws, sz(nbytes), None)


def test_attend_cache_refuses(B):
    lib = _lib(B)
    for bad, status in BAD_CACHES:
        assert _attend(lib, B, cache=_cache(B, **bad)) == status, bad
        assert B._lib.d3tom_attend_cache_workspace_bytes(_cache(B, **bad), 5, 3, 320, 4, 0) == 0
    odd = ctypes.c_void_p(AT + 2)
    for kw in (dict(q=None), dict(q=odd), dict(qs=255), dict(qs=260), dict(off=None), dict(rows=0), dict(most=0), dict(most=6), dict(max_len=0), dict(max_len=321),
               dict(H=3), dict(H=0), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(o=None), dict(o=odd), dict(wi=P),
               dict(wo=P), dict(wo=P, stride=319), dict(ws=None)):
        assert _attend(lib, B, **kw) == INVALID, kw
    need = B._lib.d3tom_attend_cache_workspace_bytes(_cache(B), 5, 3, 320, 4, 1)
    assert need >= 256
    assert _attend(lib, B, wo=P, stride=320, nbytes=need - 1) == SMALL and _attend(lib, B, ws=ctypes.c_void_p(AT + 16)) == SMALL
    for rows, most, max_len, H in [(0, 1, 1, 4), (5, 6, 1, 4), (5, 1, 321, 4), (5, 1, 0, 4), (5, 1, 1, 5)]:
        assert B._lib.d3tom_attend_cache_workspace_bytes(_cache(B), rows, most, max_len, H, 0) == 0
    assert _attend(lib, B, cache=_cache(B, B=65535), rows=1 << 30, most=1 << 30) == UNSUPPORTED
    assert _attend(lib, B, qs=(1 << 23) + 8) == UNSUPPORTED
    endless = _cache(B, page_size=4096, table_stride=1 << 19)
    for n in ((1 << 27) + 1, 2 ** 31 - 1):
        assert _attend(lib, B, cache=endless, max_len=n, wo=P, stride=n) == UNSUPPORTED
        assert B._lib.d3tom_attend_cache_workspace_bytes(endless, 5, 3, n, 4, 1) == 0


def test_attend_cache_refuses_launches_that_are_too_large(B):
    lib = _lib(B)
    far = dict(page_size=4096, table_stride=1 << 12)
    for kw in (dict(cache=_cache(B, **far), rows=1 << 22, most=1 << 22),                                                     # rows and heads
               dict(cache=_cache(B, B=65535, **far), rows=17, most=17, H=2, max_len=62 * 4096),                               # workgroups of 512 threads
               dict(cache=_cache(B, B=65535, **far), rows=1, most=1, H=2, max_len=123 * 4096),                                # of 256
               dict(cache=_cache(B, B=65535, dh=96, **far), rows=200, most=200, H=2, qs=256)):                                # of any head size
        assert _attend(lib, B, **kw) == UNSUPPORTED, kw


def test_attend_cache_workspace_serves_smaller_calls(B):
    import random
    rng = random.Random(0)
    log_int = lambda lo, hi: int(lo * (hi / lo) ** rng.random())
    for _ in range(3000):
        nB, Hkv = log_int(1, 64), rng.choice([1, 2, 4, 8, 32])
        c = _cache(B, B=nB, Hkv=Hkv, dh=rng.choice([8, 64, 96, 128]), dt=rng.choice([0, 1]), table_stride=10 ** 5)
        need = lambda rows, most, n, w: B._lib.d3tom_attend_cache_workspace_bytes(c, rows, most, n, H, w)
        H, n, most = Hkv * rng.choice([1, 2, 4, 8, 16]), log_int(1, 200000), log_int(1, 400)
        rows = rng.randint(most, most * nB)
        all_of_it = need(rows, most, n, 1)
        assert all_of_it > 0
        for _ in range(4):
            m2 = log_int(1, most + 1)
            r2 = min(rows, rng.randint(m2, m2 * nB))
            assert 0 < need(r2, min(m2, r2), log_int(1, n + 1), rng.choice([0, 1])) <= all_of_it


def _evict(lib, B, cache=None, max_len=320, keep=P, first=4, recent=8, wi=P, ti=P, wo=P, to=P, stride=320, lo=P, src=None, ws=P, nbytes=1 << 40):
    return lib.d3tom_cache_evict(ctypes.byref(cache if cache is not None else _cache(B)), i32(max_len), keep, i32(first), i32(recent), wi, ti, wo, to, i32(stride), lo,
                                 src, ws, sz(nbytes), None)


def test_cache_evict_refuses(B):
    lib = _lib(B)
    for bad, status in BAD_CACHES:
        assert _evict(lib, B, cache=_cache(B, **bad)) == status, bad
        assert B._lib.d3tom_cache_evict_workspace_bytes(_cache(B, **bad), 320) == 0
    for kw in (dict(max_len=0), dict(max_len=321), dict(keep=None), dict(first=-1), dict(recent=-1), dict(wi=None), dict(ti=None), dict(wo=None), dict(to=None),
               dict(stride=319), dict(lo=None), dict(ws=None)):
        assert _evict(lib, B, **kw) == INVALID, kw
    need = B._lib.d3tom_cache_evict_workspace_bytes(_cache(B), 320)
    assert need >= 256 and _evict(lib, B, nbytes=need - 1) == SMALL and _evict(lib, B, ws=ctypes.c_void_p(AT + 128)) == SMALL
    large = _cache(B, page_size=4096, table_stride=400)
    assert _evict(lib, B, cache=large, max_len=(1 << 20) + 1, stride=1 << 21) == UNSUPPORTED


def test_binding_refuses_a_stream_of_another_device(B, monkeypatch):
    import torch
    from types import SimpleNamespace
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0)
    assert B._on(SimpleNamespace(cuda_stream=17, device_index=0)) == (17, 0)
    with pytest.raises(ValueError, match="another device"):
        B._on(SimpleNamespace(cuda_stream=17, device_index=1))


def test_binding_refuses_what_it_cannot_pass_on(B):
    import torch
    t = torch.zeros(2, 16, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        B.PagedCache(t, t, torch.zeros(1, 2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32))       # not on the GPU
    with pytest.raises(ValueError):
        B.Axes(torch.zeros(4, 3, dtype=torch.int32), [10, 12, 10], 10000.0)
    from paper_2511_12280_amd import _native
    cache, axes, none9 = _cache(B), _axes(B), [None] * 9
    with pytest.raises(ValueError, match="another size"):
        _native.d3tom_cache_evict(axes, 0, 1, None, 0, 0, *none9)
    with pytest.raises(TypeError):
        _native.d3tom_cache_evict(4096, 0, 1, None, 0, 0, *none9)
    with pytest.raises(TypeError):
        _native.d3tom_cache_evict(cache, 0, 1)
    with pytest.raises(ValueError, match="a cache is missing"):
        _native.d3tom_cache_evict(None, 0, 1, None, 0, 0, *none9)
    with pytest.raises(ValueError, match="a tensor is missing"):
        _native.d3tom_cache_evict(cache, 0, 1, None, 0, 0, None, None, None, None, None, 17, None, None, 0)
    host = torch.zeros(4, 2, 64)
    for bad in (host, host.as_subclass(type("Sub", (torch.Tensor,), {}))):
        with pytest.raises(ValueError, match="on the GPU"):
            _native.d3tom_rope_axes(bad, None, axes, 4, 0, None, None, None, 0)
    with pytest.raises(ValueError, match="keys and values"):
        _native.d3tom_cache_append(cache, 0, None, None, None, 1, None, 0, 0, *[None] * 6, 0)
    with pytest.raises(ValueError, match="different devices"):
        _native.d3tom_attend_cache(None, cache, 0, None, 1, 1, 0.1, 0, *[None] * 6, 0)
    assert _native.d3tom_rope_axes(None, None, axes, 4, 0, None, None, None, 0) == INVALID
