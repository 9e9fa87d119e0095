"""GPU parity of the paged cache's operators against the float64 reference in oracle/cache.py, through the binding.

Tolerances, element by element, u = 2^-24 (half a step of float32), b = 2^-8 (bf16) or u (float32) for what is stored:
  rotation   cos and sin are off by u each (they are rounded once from double), two products and a sum by u each:
             4 u (|x| + |y|) of the pair, and b |result| for the store
  logits     E = scale * max_j sum_c |q_c| |k_jc| * (dh + 4) u: dh products added in float32, scale and conversion to base 2 behind that;
             differences of logits, and log-sum-exp, are off by 2 E and a few u of their size
  attention  a probability is off by the factor 1 + d, d = exp(4 E) - 1 + (n + 64) u (its exponent twice, its row's sum, the joining), and by b where it enters the
             product as bf16: (d + b') sum_j p_j |v_j| with b' = 2^-8 (bf16) or 0, and b |result| for the store
  weights    d for every probability, their sum over rows and heads in float32: (d + (rows H + 8) u) * sum, and u for the result
What moves (appended values, evicted rows) is compared bit by bit.
"""
import numpy as np
import pytest
import torch

from oracle import cache as OC
from oracle.stack import round_bf16

pytestmark = pytest.mark.gpu

U = 2.0 ** -24


@pytest.fixture(scope="module")
def B():
    from paper_2511_12280_amd import binding
    assert torch.cuda.is_available(), "GPU tests need a device"
    return binding


DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def _round(a, dtype):
    return round_bf16(a) if dtype == "bf16" else np.asarray(a, dtype=np.float32).astype(np.float64)


def _dev(a, dtype):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).cuda().to(DT[dtype])


def _i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).cuda()


def _host(t):
    return t.detach().double().cpu().numpy()


def _off(counts):
    return np.concatenate([[0], np.cumsum(counts)])


def _rows(a, dtype, apart):
    """device rows [rows, heads, dh]; apart: columns of a wider matrix, NaN beside them"""
    t = _dev(a, dtype)
    if not apart:
        return t
    wide = torch.full((t.shape[0], t.shape[1] + 3, t.shape[2]), float("nan"), dtype=t.dtype, device="cuda")
    wide[:, 1:1 + t.shape[1]] = t
    return wide[:, 1:1 + t.shape[1]]


class Cache:
    """Samples of given lengths in pages whose other rows are NaN; the rows also on the host (float64, representable)."""

    def __init__(self, B, lens, Hkv, dh, page, dtype, seed, spare=2, behind=-1, std=1.0):
        rng = np.random.default_rng(seed)
        self.lens, self.page, self.dtype = list(lens), page, dtype
        self.table, num = OC.pages(lens, page, spare, rng, behind)
        self.k = [_round(std * rng.standard_normal((n, Hkv, dh)), dtype) for n in lens]
        self.v = [_round(rng.standard_normal((n, Hkv, dh)), dtype) for n in lens]
        shape = (num, page, Hkv, dh)
        kp, vp = np.full(shape, np.nan, np.float32), np.full(shape, np.nan, np.float32)
        for b, n in enumerate(lens):
            j = np.arange(n)
            kp[self.table[b, j // page], j % page], vp[self.table[b, j // page], j % page] = self.k[b], self.v[b]
        self.k_pages, self.v_pages = _dev(kp, dtype), _dev(vp, dtype)
        self.handle = B.PagedCache(self.k_pages, self.v_pages, _i32(self.table), _i32(lens))

    def rows(self, pages, b, n=None):
        j = torch.arange(self.lens[b] if n is None else n, device="cuda")
        return pages[self.handle.page_table[b].long()[j // self.page], j % self.page]


# ---- rotary positions ------------------------------------------------------------------------------------------------------
def _check_turned(got, x, pos, pairs, theta, own, dtype):
    want = OC.rope_axes(x, pos, pairs, theta, own)
    half = x.shape[2] // 2
    pair = np.abs(x[:, :, :half]) + np.abs(x[:, :, half:])
    tol = 4 * U * np.concatenate([pair, pair], 2) + (2.0 ** -8 if dtype == "bf16" else U) * np.abs(want) + 1e-38
    assert (np.abs(_host(got) - want) <= tol).all(), np.abs(_host(got) - want).max()


@pytest.mark.parametrize("rows,H,Hkv,dh,pairs,own,dtype", [
    (1, 1, 1, 16, [8], False, "bf16"), (7, 4, 2, 64, [10, 12, 10], False, "bf16"), (7, 4, 2, 64, [10, 12, 10], True, "bf16"), (33, 32, 8, 128, [24, 20, 20], False, "bf16"),
    (5, 3, 1, 128, [1, 61, 1, 1], True, "bf16"), (6, 5, 5, 48, [7, 3], True, "bf16"), (4, 2, 2, 256, [60, 30, 20], False, "bf16"), (300, 16, 4, 128, [64], False, "bf16"),
    (1, 4, 4, 64, [16, 16], True, "f32"), (77, 6, 2, 8, [1, 3], False, "f32"), (3, 2, 1, 256, [128], False, "f32"), (130, 16, 16, 64, [8, 8, 8], True, "f32"),
    (1025, 8, 2, 64, [32], True, "f32"), (19, 33, 11, 40, [3, 2, 1, 1], False, "f32")])
def test_rope_axes(B, rows, H, Hkv, dh, pairs, own, dtype):
    rng = np.random.default_rng([rows, H, dh])
    q, k = (_round(rng.standard_normal((rows, h, dh)), dtype) for h in (H, Hkv))
    pos = rng.integers(0, 60, (rows, len(pairs)))
    pos[:, 0] = rng.integers(-5, 200000, rows)
    for apart in (False, True):
        dq, dk = _rows(q, dtype, apart), _rows(k, dtype, apart)
        qo, ko = torch.full((rows, H, dh), 7.0, dtype=DT[dtype], device="cuda"), torch.full((rows, Hkv, dh), 7.0, dtype=DT[dtype], device="cuda")
        axes = B.Axes(_i32(pos), pairs, 10000.0, int(own))
        B.d3tom_rope_axes(dq, dk, axes, qo, ko)
        _check_turned(qo, q, pos, pairs, 10000.0, own, dtype)
        _check_turned(ko, k, pos, pairs, 10000.0, own, dtype)
        alone = torch.zeros_like(ko)
        B.d3tom_rope_axes(None, dk, axes, None, alone)
        assert torch.equal(alone, ko)
        alone = torch.zeros_like(qo)
        B.d3tom_rope_axes(dq, None, axes, alone)
        assert torch.equal(alone, qo)
        if not apart:
            B.d3tom_rope_axes(dq, dk, axes, dq, dk)
            assert torch.equal(dq, qo) and torch.equal(dk, ko)


def test_rope_axes_with_one_axis_is_rope(B):
    rng = np.random.default_rng(3)
    q, k = _dev(rng.standard_normal((50, 4, 128)), "bf16"), _dev(rng.standard_normal((50, 4, 128)), "bf16")
    pos = _i32(rng.integers(0, 4000, (50, 1)))
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    B.d3tom_rope_axes(q, k, B.Axes(pos, [64], 10000.0), qo, ko)
    B.d3tom_rope(q, k, pos.view(-1), 10000.0)
    assert torch.equal(q, qo) and torch.equal(k, ko)


# ---- appending ---------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype,H,Hkv,dh,page,lens,new,pairs", [
    ("bf16", 4, 2, 64, 16, [17, 1, 40, 33], [1, 1, 0, 33], [10, 12, 10]), ("bf16", 32, 8, 128, 64, [300], [300], [24, 20, 20]), ("bf16", 8, 8, 128, 16, [129] * 9, [1] * 9, [64]),
    ("f32", 3, 3, 64, 32, [31, 32, 33], [31, 1, 2], [16, 16]), ("bf16", 2, 1, 256, 16, [50, 7], [3, 7], [100, 20]), ("bf16", 2, 1, 24, 16, [5], [2], None), ("f32", 2, 1, 4, 128, [200, 3], [190, 3], None)])
def test_cache_append(B, dtype, H, Hkv, dh, page, lens, new, pairs):
    c = Cache(B, lens, Hkv, dh, page, dtype, seed=[dh, page, len(lens)])
    rng = np.random.default_rng(5)
    rows = sum(new)
    q, k, v = (_round(rng.standard_normal((rows, h, dh)), dtype) for h in (H, Hkv, Hkv))
    pos = rng.integers(0, 9000, (rows, len(pairs) if pairs else 1))
    tokens = rng.integers(0, 1 << 30, rows).astype(np.int32)
    off = _off(new)
    W = max(lens) + 3
    kp, vp = c.k_pages.clone(), c.v_pages.clone()
    tok0, wgt0 = rng.integers(0, 99, (len(lens), W)), rng.random((len(lens), W)).astype(np.float32)
    tok, wgt = _i32(tok0), _dev(wgt0, "f32")
    qo = torch.zeros(rows, H, dh, dtype=DT[dtype], device="cuda")
    for _ in range(2):                                             # the call can be repeated
        kw = dict(axes=B.Axes(_i32(pos), pairs, 10000.0), q=_rows(q, dtype, True), q_out=qo) if pairs else {}
        B.d3tom_cache_append(c.handle, _rows(k, dtype, True), _rows(v, dtype, True), _i32(off), max(new), tokens=_i32(tokens), slot_token=tok, slot_weight=wgt, **kw)
    want_k = OC.rope_axes(k, pos, pairs, 10000.0, False) if pairs else k
    if pairs:
        _check_turned(qo, q, pos, pairs, 10000.0, False, dtype)
    for b, (n, m) in enumerate(zip(lens, new)):
        r = slice(off[b], off[b + 1])
        gk, gv = c.rows(c.k_pages, b)[n - m:], c.rows(c.v_pages, b)[n - m:]
        assert np.array_equal(_host(gv), v[r])
        if pairs:
            _check_turned(gk, k[r], pos[r], pairs, 10000.0, False, dtype)
        else:
            assert np.array_equal(_host(gk), want_k[r])
        assert np.array_equal(tok[b, n - m:n].cpu().numpy(), tokens[r]) and not wgt[b, n - m:n].any()
        tok0[b, n - m:n], wgt0[b, n - m:n] = tokens[r], 0
        # the rows themselves are as they were everywhere else
        j = torch.arange(n - m, n, device="cuda")
        page_ids = c.handle.page_table[b].long()[j // page]
        kp[page_ids, j % page], vp[page_ids, j % page] = gk, gv
    assert torch.equal(kp.view(torch.int16 if dtype == "bf16" else torch.int32), c.k_pages.view(torch.int16 if dtype == "bf16" else torch.int32))
    assert torch.equal(vp.view(torch.int16 if dtype == "bf16" else torch.int32), c.v_pages.view(torch.int16 if dtype == "bf16" else torch.int32))
    assert np.array_equal(tok.cpu().numpy(), tok0) and np.array_equal(wgt.cpu().numpy(), wgt0)


def test_cache_append_skips_what_has_no_place(B):
    # page ids that there are not, more new rows than the length says: nothing is written for those, the others arrive
    c = Cache(B, [40, 20], 2, 64, 16, "bf16", seed=1)
    c.handle.page_table[0, 1] = 10 ** 6
    c.handle.page_table[0, 2] = -7
    c.handle.kv_len[1] = 3
    before = c.k_pages.clone()
    k = torch.ones(45, 2, 64, dtype=torch.bfloat16, device="cuda")
    wgt = torch.ones(2, 60, device="cuda")
    B.d3tom_cache_append(c.handle, k, k, _i32([0, 40, 45]), 40, slot_weight=wgt)
    changed = (c.k_pages.view(torch.int16) != before.view(torch.int16)).flatten(2).any(2)
    want = torch.zeros_like(changed)
    want[c.table[0, 0]] = True                                     # slots 0 .. 15 of sample 0
    want[c.table[1, 0], :3] = True                                 # rows 2 .. 4 of sample 1's five
    assert torch.equal(changed, want)
    assert not wgt[1, :3].any() and wgt[1, 3:].all()


# ---- attention ------------------------------------------------------------------------------------------------------------------
def _attend_case(B, dtype, H, Hkv, dh, page, lens, new, causal, weighed, seed=0, apart=False, std=1.0, behind=-1, scale=None, check=True, pad=0, more_q=0, more_len=0):
    c = Cache(B, lens, Hkv, dh, page, dtype, seed=[seed, dh, page, len(lens)], behind=behind, std=std)
    rng = np.random.default_rng([seed, 9])
    rows, off = sum(new) + pad, _off(new)
    q = _round(rng.standard_normal((rows, H, dh)), dtype)
    scale = 1.0 / np.sqrt(dh) if scale is None else scale
    dq = _rows(q, dtype, apart)
    o = torch.full((rows, H, dh), 7.0, dtype=DT[dtype], device="cuda")
    lse = torch.full((rows, H), 7.0, device="cuda")
    W = max(lens) + 5
    w_in = rng.random((len(lens), W)).astype(np.float32) if weighed else None
    w_out = torch.full((len(lens), W), -3.0, device="cuda") if weighed else None
    longest, most = max(max(lens), 1) + more_len, max(new) + more_q
    W += more_len
    if weighed and more_len:
        w_in, w_out = np.pad(w_in, ((0, 0), (0, more_len))), torch.full((len(lens), W), -3.0, device="cuda")
    ws = torch.full((B.d3tom_attend_cache_workspace_bytes(c.handle, rows, most, longest, H, weighed),), 0xFF, dtype=torch.uint8, device="cuda")
    B.d3tom_attend_cache(dq, c.handle, _i32(off), most, longest, scale, causal, o, ws, lse=lse, weight_in=_dev(w_in, "f32") if weighed else None, weight_out=w_out)
    if check:
        for b, (n, m) in enumerate(zip(lens, new)):
            r = slice(off[b], off[b + 1])
            _check_attend(_host(o[r]), _host(lse[r]), _host(w_out[b]) if weighed else None, q[r], c.k[b], c.v[b], float(np.float32(scale)), causal, dtype,
                          w_in[b] if weighed else None)
    assert (o[off[-1]:] == 7).all() and (lse[off[-1]:] == 7).all()
    return c, dq, o, lse, w_out, ws


def _check_attend(o, lse, w, q, k, v, scale, causal, dtype, w_in):
    (m, H, dh), n = q.shape, len(k)
    want, want_lse, got = OC.attend(q, k, v, scale, causal)
    G = H // k.shape[1]
    b = 2.0 ** -8 if dtype == "bf16" else U
    if n and m:
        E = max(scale * (np.abs(k[:, h // G]) @ np.abs(q[:, h]).T).max() for h in range(H)) * (dh + 4) * U
        big = scale * max(np.abs(k[:, h // G] @ q[:, h].T).max() for h in range(H))
        d = np.expm1(4 * E + 8 * U * big) + (n + 64) * U
        spread = np.stack([OC.attend(q[:, h:h + 1], k[:, h // G:h // G + 1], np.abs(v[:, h // G:h // G + 1]), scale, causal)[0][:, 0] for h in range(H)], 1)
        tol = (d + (b if dtype == "bf16" else 0.0)) * spread + b * np.abs(want) * (1 + b) + 1e-37
        bad = np.abs(o - want) - tol
        assert (bad <= 0).all(), (np.abs(o - want).max(), bad.max())
        none = np.isneginf(want_lse)
        assert np.isneginf(lse[none]).all() and not o[none].any()
        assert (np.abs(lse[~none] - want_lse[~none]) <= 2 * E + d + 4 * U * (np.abs(want_lse[~none]) + big)).all()
    if w is not None:
        assert (w[n:] == -3.0).all()
        if n:
            total = w_in[:n].astype(np.float64) + got
            dw = d + (m * H + 8) * U if m else 0.0
            assert (np.abs(w[:n] - total) <= dw * got + 2 * U * total).all(), np.abs(w[:n] - total).max()


ATTEND = [
    # dtype, H, Hkv, dh, page, lens, new, causal
    ("bf16", 4, 4, 64, 16, [1], [1], False), ("bf16", 8, 2, 128, 16, [37], [1], False), ("bf16", 32, 32, 128, 16, [129, 64, 1, 200], [1, 1, 1, 1], False),
    ("bf16", 8, 1, 128, 32, [255, 256, 257, 31, 32, 33], [1] * 6, False), ("bf16", 16, 2, 128, 64, [1000, 3], [1, 1], True), ("bf16", 4, 1, 64, 128, [2500], [1], False),
    # some new rows, causal and not; more rows than a tile has, odd counts, samples without rows, without slots, rows that see nothing
    ("bf16", 4, 2, 128, 16, [100, 5, 0, 17], [5, 2, 0, 17], True), ("bf16", 4, 2, 64, 16, [100, 5, 0, 17], [5, 2, 3, 17], False), ("bf16", 4, 1, 128, 16, [3, 90], [7, 4], True),
    ("bf16", 8, 2, 128, 64, [333, 90], [32, 32], False), ("bf16", 8, 1, 64, 16, [140, 300], [33, 47], True), ("bf16", 8, 8, 128, 16, [513], [64], False),
    ("bf16", 16, 1, 128, 32, [400, 65], [20, 65], True), ("bf16", 6, 2, 64, 16, [222], [11], True), ("bf16", 5, 1, 128, 16, [77], [1], False), ("bf16", 24, 2, 128, 16, [301], [3], True),
    ("bf16", 8, 2, 128, 16, [700], [150], True), ("bf16", 2, 1, 64, 4096, [5000], [2], False),
    # other head sizes
    ("bf16", 3, 1, 8, 16, [40, 300], [1, 2], True), ("bf16", 4, 2, 80, 16, [270], [3], False), ("bf16", 2, 2, 256, 32, [100], [9], True), ("bf16", 4, 4, 96, 16, [1100], [1], False),
    ("f32", 4, 4, 64, 16, [213], [5], True), ("f32", 8, 2, 128, 16, [1], [1], False), ("f32", 8, 2, 128, 64, [600, 33, 0], [1, 1, 0], False), ("f32", 4, 1, 64, 32, [300, 90], [30, 3], True),
    ("f32", 2, 1, 4, 16, [50], [2], False), ("f32", 3, 3, 20, 16, [65], [1], True), ("f32", 2, 1, 256, 16, [290], [4], False), ("f32", 16, 2, 64, 16, [1500], [1], True),
    ("f32", 4, 2, 128, 16, [130], [64], False), ("f32", 6, 2, 64, 128, [3000], [3], False)]


@pytest.mark.parametrize("dtype,H,Hkv,dh,page,lens,new,causal", ATTEND)
@pytest.mark.parametrize("weighed", [False, True])
def test_attend_cache(B, dtype, H, Hkv, dh, page, lens, new, causal, weighed):
    _attend_case(B, dtype, H, Hkv, dh, page, lens, new, causal, weighed, apart=weighed, behind=-1 if weighed else 10 ** 8)


@pytest.mark.parametrize("dtype,H,Hkv,dh,lens,new", [
    ("bf16", 8, 2, 128, [100, 333, 50], [1, 0, 1]), ("bf16", 8, 2, 64, [100, 333, 50], [33, 0, 7]), ("bf16", 4, 2, 80, [100, 333], [0, 3]), ("f32", 8, 2, 64, [70, 300], [0, 40])])
def test_attend_cache_samples_without_rows(B, dtype, H, Hkv, dh, lens, new):
    # their slots' entries are what they were
    _attend_case(B, dtype, H, Hkv, dh, 16, lens, new, False, True)


@pytest.mark.parametrize("dtype,H,Hkv,dh,new,causal", [("bf16", 20, 10, 128, 40, False), ("bf16", 9, 9, 64, 35, True), ("f32", 17, 17, 64, 20, False), ("f32", 24, 12, 128, 11, True)])
def test_attend_cache_weighs_more_key_heads_than_waves(B, dtype, H, Hkv, dh, new, causal):
    _attend_case(B, dtype, H, Hkv, dh, 32, [270, 99], [new, 5], causal, True)


@pytest.mark.parametrize("dtype,H,Hkv,dh,new,more_q", [("bf16", 8, 2, 128, [1, 1], 0), ("bf16", 8, 2, 128, [3, 1], 3), ("bf16", 8, 2, 64, [20, 2], 12), ("bf16", 8, 2, 128, [1, 2], 10),
                                                       ("f32", 4, 4, 64, [5, 1], 4), ("bf16", 4, 2, 96, [2, 1], 6)])
@pytest.mark.parametrize("weighed", [False, True])
def test_attend_cache_padded_rows_and_generous_maxima(B, dtype, H, Hkv, dh, new, more_q, weighed):
    # rows behind the last sample's are left as they were; max_q and max_len may exceed what there is
    _attend_case(B, dtype, H, Hkv, dh, 16, [200, 131], new, True, weighed, pad=13, more_q=more_q, more_len=17)


@pytest.mark.parametrize("H,Hkv,dh,lens,new,causal", [(8, 2, 128, [37, 5], [1, 1], False), (32, 32, 128, [300, 65], [1, 1], False), (8, 2, 64, [90, 40], [4, 2], True), (16, 1, 64, [4000], [1], False),
                                                      (4, 2, 128, [2500, 333], [3, 8], True), (4, 4, 64, [30, 17], [16, 2], False)])
def test_attend_cache_few_rows_do_not_round_probabilities(B, H, Hkv, dh, lens, new, causal):
    # probabilities enter the product with v in two bf16 parts: the upper bits leave less than 2^-7 of one, of which rounding takes 2^-8 at most: 2^-15 instead of the 2^-8 of one part
    c, dq, o, lse, _, _ = _attend_case(B, "bf16", H, Hkv, dh, 16, lens, new, causal, False, seed=12)
    q, G, scale, off = _host(dq), H // Hkv, float(np.float32(1.0 / np.sqrt(dh))), _off(new)
    for b in range(len(lens)):
        r, k, v, n = slice(off[b], off[b + 1]), c.k[b], c.v[b], lens[b]
        want = OC.attend(q[r], k, v, scale, causal)[0]
        E = max(scale * (np.abs(k[:, h // G]) @ np.abs(q[r, h]).T).max() for h in range(H)) * (dh + 4) * U
        big = scale * max(np.abs(k[:, h // G] @ q[r, h].T).max() for h in range(H))
        d = np.expm1(4 * E + 8 * U * big) + (n + 64) * U
        spread = np.stack([OC.attend(q[r, h:h + 1], k[:, h // G:h // G + 1], np.abs(v[:, h // G:h // G + 1]), scale, causal)[0][:, 0] for h in range(H)], 1)
        assert (np.abs(_host(o[r]) - want) <= (d + 2.0 ** -15) * spread * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(want)).all()


@pytest.mark.parametrize("weighed", [False, True])
def test_attend_cache_maxima_far_above_what_there_is(B, weighed):
    # samples * max_q * H * runs is beyond 2^24, the workgroups are 2^17
    _attend_case(B, "bf16", 8, 2, 64, 64, [16384] + [20, 300] * 31 + [5], [1] * 63 + [3], True, weighed, pad=8192, more_q=8189)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("std,scale", [(30.0, None), (1.0, 1e-6), (1.0, 4.0)])
def test_attend_cache_logits_far_apart_and_all_alike(B, dtype, std, scale):
    # keys 30 times as long: one key has all of a row's probability; a tiny scale: all have the same
    _attend_case(B, dtype, 8, 2, 128, 16, [500, 77], [3, 1], True, False, std=std, scale=scale)
    _attend_case(B, dtype, 8, 2, 64, 16, [500, 77], [40, 1], False, True, std=std, scale=scale)


@pytest.mark.parametrize("dtype,H,Hkv,new", [("bf16", 8, 2, 1), ("bf16", 8, 2, 40), ("f32", 4, 4, 3)])
def test_attend_cache_long(B, dtype, H, Hkv, new):
    # long enough for many runs; only some rows against float64
    n, dh = 20011, 128 if dtype == "bf16" else 64
    _attend_case(B, dtype, H, Hkv, dh, 64, [n, 301], [new, 1], False, True)


def test_attend_cache_maximum_in_the_first_and_in_the_last_slot(B):
    for at in (0, -1, 700):
        c = Cache(B, [1500], 1, 128, 16, "bf16", seed=3)
        q = _round(np.random.default_rng(1).standard_normal((1, 4, 128)), "bf16")
        c.k[0][at, 0] = _round(4.0 * q[0, 1], "bf16")
        slot = at % 1500
        c.k_pages[c.table[0, slot // 16], slot % 16, 0] = _dev(c.k[0][at, 0], "bf16")
        o, lse = torch.zeros(1, 4, 128, dtype=torch.bfloat16, device="cuda"), torch.zeros(1, 4, device="cuda")
        ws = B.workspace(B.d3tom_attend_cache_workspace_bytes(c.handle, 1, 1, 1500, 4))
        B.d3tom_attend_cache(_dev(q, "bf16"), c.handle, _i32([0, 1]), 1, 1500, 0.1, False, o, ws, lse=lse)
        _check_attend(_host(o), _host(lse), None, q, c.k[0], c.v[0], float(np.float32(0.1)), False, "bf16", None)


@pytest.mark.parametrize("dtype,H,Hkv,dh,lens,new,causal", [
    ("bf16", 32, 8, 8, [2000], [2], False), ("f32", 32, 4, 4, [4000], [2], False), ("f32", 32, 8, 12, [2000], [2], True), ("f32", 16, 16, 8, [3000, 1301], [3, 2], True),
    ("bf16", 32, 32, 8, [4096], [1], False), ("f32", 64, 1, 12, [5000, 40], [1, 1], True), ("bf16", 32, 2, 16, [2000], [2], True), ("f32", 32, 8, 20, [2000], [2], False)])
@pytest.mark.parametrize("weighed", [False, True])
def test_attend_cache_joins_runs_of_small_heads(B, dtype, H, Hkv, dh, lens, new, causal, weighed):
    # more than four runs, which groups of threads share, and one to five threads to a group: up to 256 groups in a workgroup
    _attend_case(B, dtype, H, Hkv, dh, 16, lens, new, causal, weighed)


@pytest.mark.parametrize("dtype,new", [("bf16", 1), ("bf16", 30), ("f32", 2)])
def test_attend_cache_repeats_bit_by_bit_whatever_lies_behind(B, dtype, new):
    c, dq, o, lse, w, ws = _attend_case(B, dtype, 8, 2, 128, 16, [999, 130], [new, 1], True, True)
    o2, lse2, w2 = torch.zeros_like(o), torch.zeros_like(lse), w.clone()
    w_in = torch.rand(w.shape, device="cuda")
    # dead slots, and the workspace, hold other things now
    live = torch.zeros(c.k_pages.shape[:2], dtype=torch.bool, device="cuda")
    for b, n in enumerate(c.lens):
        j = torch.arange(n, device="cuda")
        live[c.handle.page_table[b].long()[j // c.page], j % c.page] = True
    outs = []
    for fill in (float("inf"), 0.5):
        c.k_pages[~live], c.v_pages[~live] = fill, fill
        ws.fill_(17)
        B.d3tom_attend_cache(dq, c.handle, _i32([0, new, new + 1]), new, 999, 1.0 / np.sqrt(128), True, o2, ws, lse=lse2, weight_in=w_in, weight_out=w2)
        outs.append((o2.clone(), lse2.clone(), w2.clone()))
    assert torch.equal(outs[0][0], o) and torch.equal(outs[0][1], lse)
    assert all(torch.equal(a, b) for a, b in zip(*outs))
    B.d3tom_attend_cache(dq, c.handle, _i32([0, new, new + 1]), new, 999, 1.0 / np.sqrt(128), True, o2, ws, weight_in=w_in, weight_out=w_in)     # in place
    assert torch.equal(w_in[0, :999], outs[0][2][0, :999]) and torch.equal(w_in[1, :130], outs[0][2][1, :130])


def test_attend_cache_equals_attend_on_the_same_rows(B):
    # all rows of a sample new and nothing masked: what d3tom_attend gives, each within its own rounding of the formula
    c, dq, o, lse, _, _ = _attend_case(B, "bf16", 8, 8, 128, 16, [300], [300], False, False)
    full = torch.empty_like(o)
    B.d3tom_attend(dq, _dev(c.k[0], "bf16"), _dev(c.v[0], "bf16"), _i32([0, 300]), 300, 1.0 / np.sqrt(128), full)
    a, b = _host(o), _host(full)
    assert (np.abs(a - b) <= 2 * 2.0 ** -8 * (np.abs(b) + np.abs(c.v[0]).max())).all()


def test_attend_cache_shared_prefix_and_pages_that_there_are_not(B):
    # two samples read the same pages; a page id that there is not reads some page instead, and the other sample is not touched by it
    c = Cache(B, [64, 70], 2, 128, 16, "bf16", seed=8)
    c.handle.page_table[1, :3] = c.handle.page_table[0, :3]
    c.k[1][:48], c.v[1][:48] = c.k[0][:48], c.v[0][:48]
    q = _round(np.random.default_rng(2).standard_normal((2, 4, 128)), "bf16")
    o, lse = torch.zeros(2, 4, 128, dtype=torch.bfloat16, device="cuda"), torch.zeros(2, 4, device="cuda")
    ws = B.workspace(B.d3tom_attend_cache_workspace_bytes(c.handle, 2, 1, 70, 4))
    call = lambda: B.d3tom_attend_cache(_dev(q, "bf16"), c.handle, _i32([0, 1, 2]), 1, 70, 0.1, False, o, ws, lse=lse)
    call()
    for b in range(2):
        _check_attend(_host(o[b:b + 1]), _host(lse[b:b + 1]), None, q[b:b + 1], c.k[b], c.v[b], float(np.float32(0.1)), False, "bf16", None)
    first = o[0].clone()
    c.k_pages.nan_to_num_(0.0)
    c.v_pages.nan_to_num_(0.0)
    c.handle.page_table[1, 2], c.handle.page_table[1, 4] = -5, 2 ** 31 - 1
    call()
    assert torch.equal(o[0], first) and torch.isfinite(o[1]).all()


def test_attend_cache_lengths_and_offsets_that_do_not_fit(B):
    # a length above max_len and offsets behind the rows are clamped: nothing outside is written
    c = Cache(B, [64, 64], 2, 64, 16, "bf16", seed=8)
    c.handle.kv_len[0] = 10 ** 9
    c.handle.kv_len[1] = -3
    q = torch.randn(3, 2, 64, device="cuda").bfloat16()
    o = torch.full((5, 2, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    w = torch.full((2, 80), 7.0, device="cuda")
    ws = B.workspace(B.d3tom_attend_cache_workspace_bytes(c.handle, 3, 2, 64, 2, True))
    B.d3tom_attend_cache(q, c.handle, _i32([0, 2, 900]), 2, 64, 0.1, False, o[:3], ws, weight_out=w)
    assert (o[3:] == 7.0).all() and not o[2].any() and (w[1] == 7.0).all() and (w[0, 64:] == 7.0).all()
    assert float(w[0, :64].sum()) == pytest.approx(2.0, rel=1e-5)


def test_attend_and_append_in_a_cache_above_four_gigabytes(B):
    # 2^33 bytes of keys, the sample's pages at the far end
    page, Hkv, dh = 64, 8, 128
    num = (1 << 33) // (page * Hkv * dh * 2) + 1
    kp = torch.empty(num, page, Hkv, dh, dtype=torch.bfloat16, device="cuda")
    vp = torch.empty_like(kp)
    rng = np.random.default_rng(0)
    n, ids = 200, [num - 1, num - 3, 1, num - 2]
    k, v = (_round(rng.standard_normal((n, Hkv, dh)), "bf16") for _ in range(2))
    cache = B.PagedCache(kp, vp, _i32([ids]), _i32([n]))
    B.d3tom_cache_append(cache, _dev(k, "bf16"), _dev(v, "bf16"), _i32([0, n]), n)
    j = torch.arange(n, device="cuda")
    assert torch.equal(kp[cache.page_table[0].long()[j // page], j % page], _dev(k, "bf16"))
    q = _round(rng.standard_normal((1, 16, dh)), "bf16")
    o, lse = torch.zeros(1, 16, dh, dtype=torch.bfloat16, device="cuda"), torch.zeros(1, 16, device="cuda")
    w = torch.full((1, n), -3.0, device="cuda")
    ws = B.workspace(B.d3tom_attend_cache_workspace_bytes(cache, 1, 1, n, 16, True))
    B.d3tom_attend_cache(_dev(q, "bf16"), cache, _i32([0, 1]), 1, n, 0.1, False, o, ws, lse=lse, weight_out=w)
    _check_attend(_host(o), _host(lse), _host(w[0]), q, k, v, float(np.float32(0.1)), False, "bf16", np.zeros(n, np.float32))
    tok, out_t, out_w = _i32([list(range(n))]), torch.zeros(1, n, dtype=torch.int32, device="cuda"), torch.zeros(1, n, device="cuda")
    left, src = _i32([0]), torch.zeros(1, n, dtype=torch.int32, device="cuda")
    B.d3tom_cache_evict(cache, n, _i32([70]), 2, 9, w, tok, out_w, out_t, left, B.workspace(B.d3tom_cache_evict_workspace_bytes(cache, n)), src=src)
    want = OC.evict(w[0].cpu().numpy(), np.arange(n), 70, 2, 9)
    assert np.array_equal(src[0, :70].cpu().numpy(), want)
    j = torch.arange(70, device="cuda")
    assert torch.equal(kp[cache.page_table[0].long()[j // page], j % page], _dev(k[want], "bf16"))


@pytest.mark.parametrize("dtype,H,Hkv,dh,new,n,weighed", [("bf16", 2, 1, 64, 1, (1 << 27) - 4101, False), ("bf16", 4, 1, 128, 5, (1 << 25) + 77, False), ("f32", 2, 2, 64, 1, 1 << 25, False),
                                                          ("bf16", 1, 1, 80, 1, (1 << 22) - 3, False), ("bf16", 2, 1, 64, 1, (1 << 23) + 9, True), ("f32", 20, 1, 64, 1, (1 << 22) + 1, True)])
def test_attend_cache_of_the_largest_lengths(B, dtype, H, Hkv, dh, new, n, weighed):
    # one sample whose pages are the same few again and again: the attention over those, each key as often as its page comes
    # Float32 sums: no lane adds up more than the 4096 slots of a run, no thread of the joining more than 2048 runs, with a few additions between lanes and threads
    page, few = 4096, 2
    rng = np.random.default_rng([n, dh])
    k, v = (_round(rng.standard_normal((few * page, Hkv, dh)), dtype) for _ in range(2))
    q = _round(rng.standard_normal((new, H, dh)), dtype)
    entries = -(-n // page)
    table = torch.arange(entries, dtype=torch.int32, device="cuda").remainder(few)[None].contiguous()
    cache = B.PagedCache(_dev(k.reshape(few, page, Hkv, dh), dtype), _dev(v.reshape(few, page, Hkv, dh), dtype), table, _i32([n]))
    o, lse = torch.zeros(new, H, dh, dtype=DT[dtype], device="cuda"), torch.zeros(new, H, device="cuda")
    w = torch.full((1, n), -3.0, device="cuda") if weighed else None
    B.d3tom_attend_cache(_dev(q, dtype), cache, _i32([0, new]), new, n, 0.3, False, o, B.workspace(B.d3tom_attend_cache_workspace_bytes(cache, new, new, n, H, weighed)), lse=lse, weight_out=w)
    slots = np.arange(few * page)
    often = (n - slots + few * page - 1) // (few * page)                          # how often each key comes
    scale, G = float(np.float32(0.3)), H // Hkv
    E = max(scale * (np.abs(k[:, h // G]) @ np.abs(q[:, h]).T).max() for h in range(H)) * (dh + 4) * U
    big = scale * max(np.abs(k[:, h // G] @ q[:, h].T).max() for h in range(H))
    d = np.expm1(4 * E + 8 * U * (big + np.log(n))) + (4096 + 2048 + 64) * U
    b, half = 2.0 ** -8 if dtype == "bf16" else U, 2.0 ** -8 if dtype == "bf16" else 0.0
    got, total = _host(o), np.zeros(few * page)
    for i in range(new):
        for h in range(H):
            x = scale * (k[:, h // G] @ q[i, h])
            p = often * np.exp(x - x.max())
            want_lse = x.max() + np.log(p.sum())
            p /= p.sum()
            want, spread = p @ v[:, h // G], p @ np.abs(v[:, h // G])
            assert (np.abs(got[i, h] - want) <= (d + half) * spread + b * np.abs(want) * (1 + b)).all(), (i, h, np.abs(got[i, h] - want).max())
            assert abs(float(lse[i, h]) - want_lse) <= 2 * E + d + 4 * U * (abs(want_lse) + big)
            total += p / often / H
    if weighed:
        want_w = torch.from_numpy(total).cuda().repeat(-(-n // (few * page)))[:n]
        assert float(((w[0].double() - want_w).abs() / want_w).max()) <= (d + (new * H + 8) * U) * 1.01


@pytest.mark.parametrize("dtype,H,Hkv,new", [("bf16", 8, 8, [16, 1]), ("bf16", 8, 2, [40, 9]), ("f32", 4, 1, [70, 3]), ("bf16", 8, 1, [33, 128])])
def test_attend_cache_rows_far_apart(B, dtype, H, Hkv, new):
    # 16 MB between the rows of q, the most there may be: offsets of up to 2^31 bytes inside a tile
    for dh in (64, 128, 96):
        c = Cache(B, [300, 140], Hkv, dh, 16, dtype, seed=[51, dh])
        rows, n = sum(new), 300
        stride = (16 << 20) // (2 if dtype == "bf16" else 4)
        wide = torch.empty(rows, stride, dtype=DT[dtype], device="cuda")
        q = torch.randn(rows, H, dh, device="cuda").to(DT[dtype])
        far = wide[:, stride - H * dh:].view(rows, H, dh)
        far.copy_(q)
        ws = B.workspace(B.d3tom_attend_cache_workspace_bytes(c.handle, rows, max(new), n, H, True))
        outs = []
        for x in (q, far):
            o, lse, w = torch.zeros_like(q), torch.zeros(rows, H, device="cuda"), torch.zeros(2, n, device="cuda")
            B.d3tom_attend_cache(x, c.handle, _i32(_off(new)), max(new), n, 0.1, True, o, ws, lse=lse, weight_out=w)
            outs.append((o, lse, w))
        assert all(torch.equal(a, b) for a, b in zip(*outs)) and torch.isfinite(outs[0][0]).all() and outs[0][2].any()


# ---- values that are not finite ----------------------------------------------------------------------------------------------------
# (kernel and runs: waves of their own, one and many; shared tiles of 64 and 128 rows, one and many; any head size, one and many)
NOT_FINITE = [("bf16", 8, 2, 128, [100, 37], [1, 2]), ("bf16", 8, 2, 64, [3000, 700], [2, 1]), ("bf16", 8, 2, 128, [90, 33], [12, 5]), ("bf16", 8, 2, 128, [1500, 260], [33, 7]),
              ("bf16", 4, 2, 96, [200, 60], [3, 2]), ("bf16", 4, 2, 80, [2500, 60], [2, 1]), ("f32", 4, 2, 64, [100, 37], [5, 2]), ("f32", 8, 2, 128, [2100, 37], [3, 1]),
              ("f32", 8, 2, 64, [300, 290], [40, 11]), ("f32", 4, 2, 40, [600, 70], [2, 1])]


def _attend_call(B, c, q, new, causal, scale=0.1):
    """outputs of one call on a cache whose pages hold c.k and c.v, and the weights that went in"""
    nB, n, dev = len(c.lens), max(c.lens), dict(device="cuda")
    for pages, rows in ((c.k_pages, c.k), (c.v_pages, c.v)):
        for b, m in enumerate(c.lens):
            j = np.arange(m)
            pages[_i32(c.table[b, j // c.page]).long(), torch.arange(m, device="cuda") % c.page] = _dev(rows[b], c.dtype)
    o, lse = torch.full(q.shape, 7.0, dtype=DT[c.dtype], **dev), torch.full(q.shape[:2], 7.0, **dev)
    w_in, w_out = np.random.default_rng(3).random((nB, n)).astype(np.float32), torch.full((nB, n), -3.0, **dev)
    ws = torch.full((B.d3tom_attend_cache_workspace_bytes(c.handle, len(q), max(new), n, q.shape[1], True),), 0xFF, dtype=torch.uint8, **dev)
    B.d3tom_attend_cache(_dev(q, c.dtype), c.handle, _i32(_off(new)), max(new), n, scale, causal, o, ws, lse=lse, weight_in=_dev(w_in, "f32"), weight_out=w_out)
    return _host(o), _host(lse), _host(w_out), w_in


@pytest.mark.parametrize("dtype,H,Hkv,dh,lens,new", NOT_FINITE)
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_attend_cache_a_row_of_nan_is_no_empty_row(B, dtype, H, Hkv, dh, lens, new, value):
    # a key of NaN (or one of infinity, which makes NaN of its own row) in one head of the first sample: its heads give NaN, everywhere, and nothing else does
    c = Cache(B, lens, Hkv, dh, 16, dtype, seed=[41, dh])
    q = np.abs(_round(np.random.default_rng(6).standard_normal((sum(new), H, dh)), dtype))
    c.k[0][lens[0] // 3, 0, 5] = value
    o, lse, w, w_in = _attend_call(B, c, q, new, False)
    m, G, s = new[0], H // Hkv, float(np.float32(0.1))
    assert np.isnan(o[:m, :G]).all() and np.isnan(lse[:m, :G]).all() and np.isnan(w[0, :lens[0]]).all()
    _check_attend(o[:m, G:], lse[:m, G:], None, q[:m, G:], c.k[0][:, 1:], c.v[0][:, 1:], s, False, dtype, None)
    _check_attend(o[m:], lse[m:], w[1], q[m:], c.k[1], c.v[1], s, False, dtype, w_in[1])


@pytest.mark.parametrize("dtype,H,Hkv,dh,lens,new", NOT_FINITE)
def test_attend_cache_logits_of_minus_infinity(B, dtype, H, Hkv, dh, lens, new):
    # keys of one head of the first sample that no query looks at: zeros, lse -infinity, no weight.  Of the second one only the first key is seen.
    c = Cache(B, lens, Hkv, dh, 16, dtype, seed=[42, dh])
    q = np.abs(_round(np.random.default_rng(7).standard_normal((sum(new), H, dh)), dtype)) + 0.5
    q = _round(q, dtype)
    c.k[0][:, 0, 5] = -np.inf
    c.k[1][1:, :, dh - 1] = -np.inf
    o, lse, w, w_in = _attend_call(B, c, q, new, False)
    m, G, s = new[0], H // Hkv, float(np.float32(0.1))
    assert not o[:m, :G].any() and np.isneginf(lse[:m, :G]).all()
    _check_attend(o[:m, G:], lse[:m, G:], None, q[:m, G:], c.k[0][:, 1:], c.v[0][:, 1:], s, False, dtype, None)
    _check_attend(o[m:], lse[m:], None, q[m:], c.k[1][:1], c.v[1][:1], s, False, dtype, None)
    got = OC.attend(q[:m, G:], c.k[0][:, 1:], c.v[0][:, 1:], s, False)[2] * (H - G) / H
    E = s * max((np.abs(c.k[0][:, h // G]) @ np.abs(q[:m, h]).T).max() for h in range(G, H)) * (dh + 4) * U
    big = s * max(np.abs(c.k[0][:, h // G] @ q[:m, h].T).max() for h in range(G, H))
    d = np.expm1(4 * E + 8 * U * big) + (lens[0] + 64) * U
    total = w_in[0, :lens[0]] + got
    assert (np.abs(w[0, :lens[0]] - total) <= (d + (m * H + 8) * U) * got + 2 * U * total).all()
    assert w[1, 0] == pytest.approx(w_in[1, 0] + new[1], rel=1e-5) and np.array_equal(w[1, 1:lens[1]].astype(np.float32), w_in[1, 1:lens[1]])


@pytest.mark.parametrize("dtype,H,Hkv,dh,lens,new", NOT_FINITE)
@pytest.mark.parametrize("value,into", [(float("nan"), "v"), (float("inf"), "v"), (float("nan"), "k"), (-float("inf"), "kv")])
def test_attend_cache_rows_in_front_do_not_see_what_is_not_finite(B, dtype, H, Hkv, dh, lens, new, value, into):
    # causal, and some of the last slots, which later rows wrote, are not finite in one head: the rows in front of them, the other heads and the other sample are what they
    # would be without them
    c = Cache(B, lens, Hkv, dh, 16, dtype, seed=[43, dh])
    q = _round(np.random.default_rng(8).standard_normal((sum(new), H, dh)), dtype)
    n, m, G, s = lens[0], new[0], H // Hkv, float(np.float32(0.1))
    first = (m + 1) // 2                                          # the first row that sees any of them
    bad = n - m + first
    if first < m:
        for rows in [dict(k=c.k, v=c.v)[t] for t in into]:
            rows[0][bad, 1], rows[0][n - 1, 1, dh - 3] = value, value
    o, lse, w, w_in = _attend_call(B, c, q, new, True)
    front, rest = slice(0, n - m + first), slice(first, m)
    _check_attend(o[:first], lse[:first], None, q[:first], c.k[0][front], c.v[0][front], s, True, dtype, None)
    _check_attend(o[m:], lse[m:], w[1], q[m:], c.k[1], c.v[1], s, True, dtype, w_in[1])
    others = [h for h in range(H) if h // G != 1]
    keys = [g for g in range(Hkv) if g != 1]
    _check_attend(o[:m, others], lse[:m, others], None, q[:m, others], c.k[0][:, keys], c.v[0][:, keys], s, True, dtype, None)
    if first < m and "v" in into:
        assert not np.isfinite(o[rest, G:2 * G]).all()
    if into == "v":
        assert np.isfinite(lse).all() and np.isfinite(w[0, :n]).all()          # the probabilities are what they were


# ---- eviction ----------------------------------------------------------------------------------------------------------------------
def _evict_case(B, dtype, Hkv, dh, page, lens, keep, first, recent, seed=0, levels=0, aliased=False, odd=0, weights=None):
    c = Cache(B, lens, Hkv, dh, page, dtype, seed=[seed, len(lens), page])
    rng = np.random.default_rng([seed, 4])
    W = max(max(lens), 1) + 3
    w = np.exp(2 * rng.standard_normal((len(lens), W)) - 4).astype(np.float32)
    if levels:
        w = rng.integers(0, levels, w.shape).astype(np.float32) * (-1.0 if odd else 1.0) * np.float32(1e-30 if odd == 2 else 1.0)
    if weights is not None:
        w[:, :weights.shape[1]] = weights
    tok = np.stack([rng.permutation(W) for _ in lens]).astype(np.int32)
    dw, dt = _dev(w, "f32"), _i32(tok)
    w_out, t_out = (dw, dt) if aliased else (torch.full(w.shape, -3.0, device="cuda"), torch.full(w.shape, -3, dtype=torch.int32, device="cuda"))
    src = torch.full(w.shape, -3, dtype=torch.int32, device="cuda")
    left = c.handle.kv_len if aliased else torch.full((len(lens),), -3, dtype=torch.int32, device="cuda")
    kp, vp = c.k_pages.clone(), c.v_pages.clone()
    longest = max(max(lens), 1)
    ws = torch.full((B.d3tom_cache_evict_workspace_bytes(c.handle, longest),), 0xFF, dtype=torch.uint8, device="cuda")
    for _ in range(1 if aliased else 2):                          # with outputs of its own the call can be repeated
        B.d3tom_cache_evict(c.handle, longest, _i32(keep), first, recent, dw, dt, w_out, t_out, left, ws, src=src)
    for b, n in enumerate(lens):
        want = OC.evict(w[b, :n], tok[b, :n], keep[b], first, recent)
        k = len(want)
        assert int(left[b]) == k
        assert np.array_equal(src[b, :k].cpu().numpy(), want), (b, n, k)
        assert (src[b, k:] == -3).all()
        assert np.array_equal(w_out[b, :k].cpu().numpy(), w[b, want]) and np.array_equal(t_out[b, :k].cpu().numpy(), tok[b, want])
        if not aliased:
            assert (w_out[b, k:] == -3).all() and (t_out[b, k:] == -3).all()
        else:
            assert np.array_equal(w_out[b, k:].cpu().numpy(), w[b, k:])
        j = torch.arange(k, device="cuda")
        for pages, old, rows in ((c.k_pages, kp, c.k), (c.v_pages, vp, c.v)):
            assert np.array_equal(_host(c.rows(pages, b, k)), rows[b][want])
            ids = c.handle.page_table[b].long()[j // page]
            old[ids, j % page] = pages[ids, j % page]
    bits = torch.int16 if dtype == "bf16" else torch.int32
    assert torch.equal(kp.view(bits), c.k_pages.view(bits)) and torch.equal(vp.view(bits), c.v_pages.view(bits))       # nothing else has changed


@pytest.mark.parametrize("dtype,Hkv,dh,page,lens,keep,first,recent", [
    ("bf16", 2, 64, 16, [1], [1], 0, 0), ("bf16", 2, 64, 16, [1], [0], 3, 3), ("bf16", 2, 64, 16, [100, 37, 0, 64], [40, 36, 5, 64], 4, 8), ("bf16", 8, 128, 64, [300, 299], [1, 298], 0, 20),
    ("f32", 1, 4, 16, [50, 51], [25, 60], 2, 2), ("f32", 3, 20, 32, [1000], [500], 0, 0), ("bf16", 1, 8, 16, [5000, 17, 1025], [3333, 9, 1024], 10, 100),
    ("bf16", 1, 8, 16, [2048, 1023, 1024, 1025], [1024, 512, 1, 1000], 4, 64), ("bf16", 1, 16, 128, [30000], [11111], 4, 3000), ("bf16", 2, 64, 16, [90, 80], [-4, 10], 50, 60),
    ("bf16", 1, 8, 4096, [70001], [35000], 4, 64), ("bf16", 1, 8, 4096, [66000, 300, 33333, 0], [65000, 299, 3, 0], 4, 64), ("bf16", 1, 8, 64, [200003], [123456], 4, 5000)])
@pytest.mark.parametrize("aliased", [False, True])
def test_cache_evict(B, dtype, Hkv, dh, page, lens, keep, first, recent, aliased):
    _evict_case(B, dtype, Hkv, dh, page, lens, keep, first, recent, aliased=aliased)


@pytest.mark.parametrize("levels,odd", [(1, 0), (2, 0), (7, 0), (300, 0), (3, 1), (5, 2)])
def test_cache_evict_ties_go_to_the_lower_slot(B, levels, odd):
    # few different weights (zeros of both signs, negative and tiny ones among them)
    _evict_case(B, "bf16", 1, 8, 16, [3000, 64, 2049], [1700, 13, 2048], 3, 5, levels=levels, odd=odd)
    # the same over several slices of 4096 slots, ties on both sides of their borders and of the new end
    _evict_case(B, "bf16", 1, 8, 16, [9000, 4097, 12288, 1, 8192, 0], [4500, 4096, 8192, 1, 100, 0], 3, 5, levels=levels, odd=odd)
    _evict_case(B, "bf16", 1, 8, 16, [9000, 8200, 4096], [8999, 4097, 4095], 0, 0, levels=levels, odd=odd, aliased=True)


@pytest.mark.parametrize("n", [4000, 5000])
@pytest.mark.parametrize("cluster,ties", [(2, 1), (63, 1), (64, 1), (65, 1), (64, 3), (66, 2), (64, 64)])
def test_cache_evict_weights_close_together(B, n, cluster, ties):
    # `cluster` weights, `ties` of each, whose bits differ in the last places only, among others far below and above: all of them share a bin of the first count
    rng = np.random.default_rng([n, cluster, ties])
    w = np.where(rng.random(n) < 0.4, 4 + 4 * rng.random(n), 0.25 * rng.random(n)).astype(np.float32)
    w[7] = 0
    at = 8 + rng.permutation(n - 8)[:cluster]
    w[at] = (np.float32(1).view(np.int32) + np.arange(cluster, dtype=np.int32) // ties).view(np.float32)
    above = int((w > 3).sum())
    for keep in {above + 1, above + 2, above + cluster // 2, above + cluster - 1, above + cluster}:
        _evict_case(B, "bf16", 1, 8, 16, [n], [keep], 0, 0, weights=w[None])


def test_cache_evict_of_the_largest_length(B):
    # 2^20 slots, 256 slices; and a neighbour that has a few
    _evict_case(B, "bf16", 1, 8, 4096, [1 << 20, 77], [(1 << 19) + 13, 50], 4, 5000)


def test_cache_evict_of_large_rows(B):
    # rows of 2 MB, 64 of a word's slots moved: their chunks do not fit 24 bits at once
    _evict_case(B, "f32", 2048, 256, 16, [130], [64], 0, 0, weights=np.arange(130, dtype=np.float32)[None])


def test_cache_evict_protects_by_number(B):
    # recent reaches beyond all numbers; numbers at the ends of int32
    _evict_case(B, "bf16", 1, 8, 16, [200], [50], 0, 2 ** 31 - 1)
    _evict_case(B, "bf16", 1, 8, 16, [200], [50], 2 ** 31 - 1, 0)
    c = Cache(B, [6], 1, 8, 16, "bf16", seed=0)
    tok = np.array([[2 ** 31 - 1, -2 ** 31, 5, 0, 2 ** 31 - 2, 7]], dtype=np.int32)
    w = np.array([[0.0, 1.0, 9.0, 2.0, 0.0, 3.0]], dtype=np.float32)
    src, left = torch.zeros(1, 6, dtype=torch.int32, device="cuda"), _i32([0])
    B.d3tom_cache_evict(c.handle, 6, _i32([4]), 1, 2, _dev(w, "f32"), _i32(tok), torch.zeros(1, 6, device="cuda"), torch.zeros_like(src), left,
                        B.workspace(B.d3tom_cache_evict_workspace_bytes(c.handle, 6)), src=src)
    assert OC.evict(w[0], tok[0], 4, 1, 2).tolist() == src[0, :4].tolist() == [0, 1, 4, 3]


def test_cache_evict_weights_of_any_bits(B):
    # NaN weights (outside the contract) still leave keep slots, every one a row of its own
    for n in (3000, 9001):
        rng = np.random.default_rng(9)
        c = Cache(B, [n], 1, 8, 16, "bf16", seed=0)
        w = torch.from_numpy(rng.integers(-2 ** 31, 2 ** 31, (1, n)).astype(np.int32)).cuda()
        w[0, ::7] = -1                                            # all bits
        w[0, 1::7] = 0x7FFFFFFF
        src, left, tok = torch.full((1, n), -3, dtype=torch.int32, device="cuda"), _i32([0]), _i32(rng.permutation(n)[None])
        for keep in (1, 200, 430, n // 2, n - 1):
            B.d3tom_cache_evict(c.handle, n, _i32([keep]), 3, 11, w.view(torch.float32), tok, torch.zeros(1, n, device="cuda"), torch.zeros_like(tok), left,
                                B.workspace(B.d3tom_cache_evict_workspace_bytes(c.handle, n)), src=src)
            got = src[0, :keep].cpu().numpy()
            assert int(left[0]) == keep and len(set(got.tolist())) == keep and got.min() >= 0 and got.max() < n
            moved = got != np.arange(keep)
            assert (got[moved] >= keep).all() and (np.diff(got[moved]) > 0).all()


# ---- together ---------------------------------------------------------------------------------------------------------------------------
class Model:
    """One layer's cache as a program uses it: append, attend with weights, evict when a sample is over its budget."""

    def __init__(self, B, nB, H, Hkv, dh, page, slots, pairs):
        self.B, self.H, self.Hkv, self.dh, self.pairs, self.slots = B, H, Hkv, dh, pairs, slots
        per = slots // page
        shape = (nB * per, page, Hkv, dh)
        table = torch.randperm(nB * per, device="cuda").to(torch.int32).view(nB, per)
        self.kv_len = torch.zeros(nB, dtype=torch.int32, device="cuda")
        self.cache = B.PagedCache(torch.full(shape, float("nan"), device="cuda").bfloat16(), torch.full(shape, float("nan"), device="cuda").bfloat16(), table, self.kv_len)
        self.token = torch.full((nB, slots), -1, dtype=torch.int32, device="cuda")
        self.weight = torch.full((nB, slots), 5.0, device="cuda")
        self.ws = B.workspace(max(B.d3tom_attend_cache_workspace_bytes(self.cache, 4096, 4096 // nB, slots, H, True), B.d3tom_cache_evict_workspace_bytes(self.cache, slots)))

    def step(self, q, k, v, off, counts, most, pos, tokens, out):
        B = self.B
        self.kv_len += counts
        B.d3tom_cache_append(self.cache, k, v, off, most, axes=B.Axes(pos, self.pairs, 10000.0, B.D3TOM_AXES_OWN), q=q, q_out=out["q"], tokens=tokens,
                             slot_token=self.token, slot_weight=self.weight)
        B.d3tom_attend_cache(out["q"], self.cache, off, most, self.slots, 0.12, True, out["o"], self.ws, weight_in=self.weight, weight_out=self.weight)

    def evict(self, keep, first, recent):
        self.B.d3tom_cache_evict(self.cache, self.slots, keep, first, recent, self.weight, self.token, self.weight, self.token, self.kv_len, self.ws)


def test_prompts_steps_and_evictions_together(B):
    nB, H, Hkv, dh, pairs = 3, 8, 2, 64, [12, 10, 10]
    M = Model(B, nB, H, Hkv, dh, 16, 160, pairs)
    rng = np.random.default_rng(0)
    k_rows, v_rows, toks, wgts, seen = [[] for _ in range(nB)], [[] for _ in range(nB)], [[] for _ in range(nB)], [[] for _ in range(nB)], [0] * nB
    for step in range(12):
        new = [40, 75, 9] if step == 0 else [1, 1, 1] if step % 3 else [4, 0, 7]
        rows, off = sum(new), _off(new)
        q, k, v = (_round(rng.standard_normal((rows, h, dh)), "bf16") for h in (H, Hkv, Hkv))
        pos = rng.integers(0, 400, (rows, 3))
        tokens = np.concatenate([np.arange(seen[b], seen[b] + new[b]) for b in range(nB)])
        out = dict(q=torch.zeros(rows, H, dh, dtype=torch.bfloat16, device="cuda"), o=torch.zeros(rows, H, dh, dtype=torch.bfloat16, device="cuda"))
        M.step(_dev(q, "bf16"), _dev(k, "bf16"), _dev(v, "bf16"), _i32(off), _i32(new), max(new), _i32(pos), _i32(tokens), out)
        _check_turned(out["q"], q, pos, pairs, 10000.0, True, "bf16")
        for b in range(nB):
            r = slice(off[b], off[b + 1])
            # the reference goes on from the stored rows: what the rotation's rounding does to a logit is the rotation's matter
            n = len(k_rows[b]) + new[b]
            j = torch.arange(n, device="cuda")
            at = M.cache.page_table[b].long()[j // 16], j % 16
            stored = _host(M.cache.k_pages[at])
            turned = OC.rope_axes(k[r], pos[r], pairs, 10000.0, True)
            assert (np.abs(stored[n - new[b]:] - turned) <= 2.0 ** -8 * np.abs(turned) + 1e-6).all()
            assert np.array_equal(stored[:n - new[b]], np.array(k_rows[b]).reshape(-1, Hkv, dh))
            k_rows[b] = list(stored)
            v_rows[b] += list(v[r])
            toks[b] += list(tokens[r])
            wgts[b] += [0.0] * new[b]
            seen[b] += new[b]
            assert np.array_equal(_host(M.cache.v_pages[at]), np.array(v_rows[b]))
            got = _host(M.weight[b, :n])
            if new[b]:
                _check_attend(_host(out["o"][r]), OC.attend(_host(out["q"][r]), k_rows[b], v_rows[b], float(np.float32(0.12)), True)[1], None, _host(out["q"][r]),
                              np.array(k_rows[b]), np.array(v_rows[b]), float(np.float32(0.12)), True, "bf16", None)
                wgts[b] = list(np.array(wgts[b]) + OC.attend(_host(out["q"][r]), k_rows[b], v_rows[b], float(np.float32(0.12)), True)[2])
            assert np.allclose(got, wgts[b], rtol=1e-4, atol=1e-6)
            wgts[b] = list(got)
        if step % 4 == 3:
            keep = [30, 64, 12]
            M.evict(_i32(keep), 2, 5)
            for b in range(nB):
                src = OC.evict(np.array(wgts[b]), np.array(toks[b]), keep[b], 2, 5)
                for rows_of in (k_rows, v_rows, toks, wgts):
                    rows_of[b] = [rows_of[b][s] for s in src]
            assert M.kv_len.tolist() == [len(t) for t in toks]
            for b in range(nB):
                assert M.token[b, :len(toks[b])].tolist() == toks[b]


def test_captured_steps_on_another_stream(B):
    # a step with lengths that grow on the device, captured, replayed with eager work between the replays: each replay is what the same step gives eagerly
    nB, H, Hkv, dh = 2, 8, 2, 128
    torch.manual_seed(0)
    q, k, v = (torch.randn(nB, h, dh, device="cuda").bfloat16() for h in (H, Hkv, Hkv))
    pos, off, ones = torch.zeros(nB, 2, dtype=torch.int32, device="cuda"), _i32([0, 1, 2]), _i32([1, 1])
    M, E = Model(B, nB, H, Hkv, dh, 16, 1024, [32, 32]), Model(B, nB, H, Hkv, dh, 16, 1024, [32, 32])
    E.cache.page_table.copy_(M.cache.page_table)
    for m in (M, E):
        pk = torch.randn(nB * 500, Hkv, dh, device="cuda", generator=torch.Generator("cuda").manual_seed(5)).bfloat16()
        m.kv_len += 500
        B.d3tom_cache_append(m.cache, pk, pk, _i32([0, 500, 1000]), 500, tokens=torch.arange(500, dtype=torch.int32, device="cuda").repeat(2), slot_token=m.token, slot_weight=m.weight)
    tokens = _i32([500, 500])
    out_m, out_e = ({n: torch.zeros(nB, H, dh, dtype=torch.bfloat16, device="cuda") for n in ("q", "o")} for _ in range(2))
    keep = _i32([499, 300])

    def turn(m, out):
        m.step(q, k, v, off, ones, 1, pos, tokens, out)
        m.evict(keep, 1, 4)
    state = [t.clone() for t in (M.cache.k_pages, M.cache.v_pages, M.token, M.weight, M.kv_len)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        turn(M, out_m)                                            # nothing is set up inside the capture
    side.synchronize()
    for t, s in zip((M.cache.k_pages, M.cache.v_pages, M.token, M.weight, M.kv_len), state):
        t.copy_(s)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        turn(M, out_m)
    for i in range(4):
        q.normal_(); k.normal_(); pos += 3; tokens += 1
        graph.replay()
        turn(E, out_e)
        torch.cuda.synchronize()
        assert torch.equal(out_m["o"], out_e["o"]) and torch.equal(out_m["q"], out_e["q"]), i
        assert M.kv_len.tolist() == E.kv_len.tolist() == [499, 300]
        for b, n in enumerate([499, 300]):
            assert torch.equal(M.weight[b, :n], E.weight[b, :n]) and torch.equal(M.token[b, :n], E.token[b, :n])
    assert torch.isfinite(out_m["o"]).all()


def test_two_graphs_share_a_workspace(B):
    # a step for few rows with its logits kept and one for many rows, captured one by one on the same workspace and replayed in turn: nothing is carried from one to the other
    nB, H, Hkv, dh, lens = 2, 8, 2, 128, [700, 300]
    c = Cache(B, lens, Hkv, dh, 16, "bf16", seed=7)
    calls = []
    for m in (1, 24):
        q = torch.randn(nB * m, H, dh, device="cuda").bfloat16()
        calls.append(dict(q=q, off=_i32([0, m, 2 * m]), m=m, o=torch.zeros_like(q), w=torch.zeros(nB, 700, device="cuda")))
    ws = B.workspace(max(B.d3tom_attend_cache_workspace_bytes(c.handle, 2 * x["m"], x["m"], 700, H, True) for x in calls))
    tok = torch.arange(700, dtype=torch.int32, device="cuda").repeat(2, 1)
    keep, src, left = _i32([300, 250]), torch.zeros(nB, 700, dtype=torch.int32, device="cuda"), _i32([0, 0])
    ev_ws, w_new, t_new = B.workspace(B.d3tom_cache_evict_workspace_bytes(c.handle, 700)), torch.zeros(nB, 700, device="cuda"), torch.zeros_like(tok)

    def attend(x, o, w):
        B.d3tom_attend_cache(x["q"], c.handle, x["off"], x["m"], 700, 0.1, False, o, ws, weight_out=w)

    def evict(w):
        B.d3tom_cache_evict(c.handle, 700, keep, 2, 9, w, tok, w_new, t_new, left, ev_ws, src=src)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for x in calls:
            attend(x, x["o"], x["w"])
    side.synchronize()
    kept = [c.k_pages.clone(), c.v_pages.clone()]
    graphs = []
    for x in calls:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=side):
            attend(x, x["o"], x["w"])
    for i in range(4):
        want = []
        for x in calls:
            x["q"].normal_()
            want.append((torch.zeros_like(x["o"]), torch.zeros_like(x["w"])))
            attend(x, *want[-1])
        for x in calls:
            x["o"].zero_()
            x["w"].zero_()
        for g in (graphs if i % 2 else graphs[::-1]):
            g.replay()
        torch.cuda.synchronize()
        for x, (o, w) in zip(calls, want):
            assert torch.equal(x["o"], o) and all(torch.equal(x["w"][b, :n], w[b, :n]) for b, n in enumerate(lens)), i
    # the eviction, captured on its own workspace, by other weights at each replay
    w = calls[0]["w"]
    evict(w)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        evict(w)
    for i in range(4):
        w.uniform_()
        c.k_pages.copy_(kept[0])
        c.v_pages.copy_(kept[1])
        graph.replay()
        torch.cuda.synchronize()
        for b, n in enumerate(lens):
            assert np.array_equal(src[b, :int(left[b])].cpu().numpy(), OC.evict(w[b, :n].cpu().numpy(), np.arange(n), int(keep[b]), 2, 9)), i


def test_two_streams_at_once(B):
    # calls on streams, caches and workspaces of their own give what they give alone
    jobs = []
    for i, (m, lens) in enumerate([(1, [5000, 900]), (20, [1500, 2100])]):
        c = Cache(B, lens, 2, 128, 64, "bf16", seed=20 + i)
        q = torch.randn(2 * m, 8, 128, device="cuda").bfloat16()
        n = max(lens)
        job = dict(c=c, q=q, off=_i32([0, m, 2 * m]), m=m, n=n, keep=_i32([x // 2 for x in lens]), ws=B.workspace(B.d3tom_attend_cache_workspace_bytes(c.handle, 2 * m, m, n, 8, True)),
                   ev=B.workspace(B.d3tom_cache_evict_workspace_bytes(c.handle, n)), tok=torch.arange(n, dtype=torch.int32, device="cuda").repeat(2, 1), pages=(c.k_pages.clone(), c.v_pages.clone()),
                   stream=torch.cuda.Stream())
        jobs.append(job)

    def run(j, stream=None):
        out = dict(o=torch.zeros_like(j["q"]), w=torch.zeros(2, j["n"], device="cuda"), w2=torch.zeros(2, j["n"], device="cuda"), t2=torch.zeros_like(j["tok"]),
                   left=_i32([0, 0]), src=torch.zeros_like(j["tok"]))
        torch.cuda.synchronize()
        return out, lambda: (B.d3tom_attend_cache(j["q"], j["c"].handle, j["off"], j["m"], j["n"], 0.1, False, out["o"], j["ws"], weight_out=out["w"], stream=stream),
                             B.d3tom_cache_evict(j["c"].handle, j["n"], j["keep"], 4, 16, out["w"], j["tok"], out["w2"], out["t2"], out["left"], j["ev"], src=out["src"], stream=stream))
    alone, pages = [], []
    for j in jobs:
        out, call = run(j)
        call()
        torch.cuda.synchronize()
        alone.append(out)
        pages.append((j["c"].k_pages.clone(), j["c"].v_pages.clone()))
    for _ in range(3):
        for j in jobs:
            j["c"].k_pages.copy_(j["pages"][0])
            j["c"].v_pages.copy_(j["pages"][1])
        both = [run(j, j["stream"]) for j in jobs]
        for _, call in both:
            call()
        torch.cuda.synchronize()
        for j, (out, _), want, page in zip(jobs, both, alone, pages):
            assert all(torch.equal(out[t], want[t]) for t in ("o", "w", "w2", "t2", "left", "src"))
            assert all(torch.equal(x.view(torch.int16), y.view(torch.int16)) for x, y in zip((j["c"].k_pages, j["c"].v_pages), page))


def test_streams_and_devices(B):
    c = Cache(B, [90], 2, 64, 16, "bf16", seed=2)
    q = torch.randn(1, 4, 64, device="cuda").bfloat16()
    o, o2 = torch.zeros_like(q), torch.zeros_like(q)
    need = B.d3tom_attend_cache_workspace_bytes(c.handle, 1, 1, 90, 4)
    ws = [B.workspace(need) for _ in range(2)]
    B.d3tom_attend_cache(q, c.handle, _i32([0, 1]), 1, 90, 0.1, False, o, ws[0])
    off = _i32([0, 1])
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    B.d3tom_attend_cache(q, c.handle, off, 1, 90, 0.1, False, o2, ws[1], stream=side)
    side.synchronize()
    assert torch.equal(o, o2)
    with pytest.raises(ValueError):
        B.d3tom_attend_cache(q, c.handle, off.cpu(), 1, 90, 0.1, False, o2, ws[1])
    with pytest.raises(B.D3tomError):
        B.d3tom_attend_cache(q, c.handle, off, 1, 10 ** 6, 0.1, False, o2, ws[1])


def test_bindings_check_shapes_types_and_devices(B):
    c = Cache(B, [90, 20], 2, 64, 16, "bf16", seed=2)
    z = lambda *shape, dtype=torch.bfloat16: torch.zeros(shape, dtype=dtype, device="cuda")
    q, k, off, pos = z(5, 4, 64), z(5, 2, 64), _i32([0, 4, 5]), z(5, 2, dtype=torch.int32)
    axes = B.Axes(pos, [16, 16], 10000.0)
    for kw in (dict(q_out=z(5, 4, 32)), dict(q_out=z(5, 4, 64, dtype=torch.float32)), dict(q_out=None), dict(q_out=z(5, 5, 64)[:, :4]), dict(k=z(4, 2, 64)),
               dict(k=z(5, 2, 64, dtype=torch.float32)), dict(q=z(5, 64, 4).transpose(1, 2)), dict(q=z(5, 256)), dict(q=z(5, 4, 64).half()), dict(axes=B.Axes(pos[:4].clone(), [16, 16], 10000.0))):
        with pytest.raises(ValueError):
            B.d3tom_rope_axes(**dict(dict(q=q, k=k, axes=axes, q_out=z(5, 4, 64), k_out=z(5, 2, 64)), **kw))
    slot_t, slot_w = z(2, 100, dtype=torch.int32), z(2, 100, dtype=torch.float32)
    for kw in (dict(k=z(5, 3, 64)), dict(k=z(5, 2, 64, dtype=torch.float32)), dict(v=z(4, 2, 64)), dict(new_off=_i32([0, 5])), dict(new_off=off.float()), dict(tokens=_i32([1, 2])),
               dict(slot_token=z(3, 100, dtype=torch.int32)), dict(slot_weight=z(2, 99, dtype=torch.float32)), dict(slot_weight=z(2, 100)), dict(q=q, q_out=None, axes=axes),
               dict(q=q[:4], q_out=q[:4].clone(), axes=axes)):
        with pytest.raises(ValueError):
            B.d3tom_cache_append(**dict(dict(cache=c.handle, k=k, v=k, new_off=off, max_new=4, tokens=_i32([0] * 5), slot_token=slot_t, slot_weight=slot_w), **kw))
    ws = B.workspace(1 << 22)
    for kw in (dict(q=z(5, 4, 32)), dict(q=q.float()), dict(o=z(4, 4, 64)), dict(o=z(5, 4, 64, dtype=torch.float32)), dict(q_off=_i32([0, 5])), dict(lse=z(5, 3, dtype=torch.float32)),
               dict(weight_out=z(3, 100, dtype=torch.float32)), dict(weight_in=z(2, 90, dtype=torch.float32)), dict(ws=None)):
        with pytest.raises(ValueError):
            B.d3tom_attend_cache(**dict(dict(q=q, cache=c.handle, q_off=off, max_q=4, max_len=90, scale=0.1, causal=False, o=z(5, 4, 64), ws=ws,
                                             weight_in=slot_w, weight_out=slot_w.clone()), **kw))
    for kw in (dict(keep=_i32([3])), dict(keep=_i32([3, 4]).long()), dict(weight_in=slot_t), dict(token_in=slot_w), dict(token_out=z(2, 99, dtype=torch.int32)), dict(len_out=_i32([0])),
               dict(src=z(2, 99, dtype=torch.int32))):
        with pytest.raises(ValueError):
            B.d3tom_cache_evict(**dict(dict(cache=c.handle, max_len=90, keep=_i32([3, 4]), first=0, recent=0, weight_in=slot_w, token_in=slot_t, weight_out=slot_w.clone(),
                                            token_out=slot_t.clone(), len_out=_i32([0, 0]), ws=ws), **kw))
    torch.cuda.synchronize()
