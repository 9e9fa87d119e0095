"""The operators around a key/value cache in pages, followed on their own: each as its plain form (elementary torch operations) and as
the framework's call.

  rope    d3tom_rope_axes     rotary positions with several axes (time, height, width), out of place
  append  d3tom_cache_append  new rows rotated and written into the pages, queries rotated beside them
  attend  d3tom_attend_cache  attention of each sample's newest rows over its pages; weighed: what every slot got is added up
  evict   d3tom_cache_evict   the slots that got the least leave, rows behind the new end move into the holes

Slot j of sample b is row j % page_size of page page_table[b, j // page_size].  A cache's length counts the rows that a call appends or
attends from.  `own` says which of the two a pass computes.
"""
import math
import random

import torch

own = False

SHARED, OWN = 0, 1         # the ladder of rotary frequencies: one over all sections, or one for each axis


# ---- cases -------------------------------------------------------------------------------------------------------------
def _rope(**kw):
    return dict(dict(kind="rope", dtype="bf16", H=32, Hkv=8, dh=128, pairs="24,20,20", ladder=SHARED, stacked=False, sizes=0), **kw)


def _append(**kw):
    return dict(dict(kind="append", dtype="bf16", H=32, Hkv=8, dh=128, pairs="24,20,20", ladder=SHARED, stacked=True, page=16, sizes=0), **kw)


def _attend(**kw):
    return dict(dict(kind="attend", dtype="bf16", H=32, Hkv=8, dh=128, page=16, causal=False, weighed=False, sizes=0), **kw)


def _evict(**kw):
    return dict(dict(kind="evict", dtype="bf16", Hkv=8, dh=128, page=16, first=4, recent=64, sizes=0), **kw)


def listed():
    return [
        # one new token of one sample: launch latency and host work
        _rope(name="rope_one_token", rows=1),
        # the patches of one image crop in a narrow float32 model: two axes, each with its own frequencies, an odd row count
        _rope(name="rope_crop_729_f32", dtype="f32", rows=729, H=16, Hkv=16, dh=64, pairs="16,16", ladder=OWN),
        # a video prompt: twenty frames of 729 patches, three axes, rows that lie in one stacked q | k | v projection
        _rope(name="rope_video_14580", rows=14580, stacked=True),
        # a decoding step of sixteen samples: a row each
        _append(name="append_step_b16", B=16, n_lo=900, n_hi=2688, new_lo=1, new_hi=1),
        # four ragged multimodal prompts that fill an empty cache
        _append(name="append_prompts_b4", B=4, n_lo=1951, n_hi=3773, new_lo=3773, new_hi=3773, page=64),
        # one new token over a full multimodal prompt with as many key heads as query heads
        _attend(name="attend_token_3709", Hkv=32, B=1, n_lo=3709, n_hi=3709, new_lo=1, new_hi=1),
        # the same step for sixteen samples of their own lengths with shared key heads, what every slot got added up for the eviction
        _attend(name="attend_step_b16_weighed", B=16, n_lo=900, n_hi=2688, new_lo=1, new_hi=1, weighed=True),
        # a block of response positions denoised together over the cached prompt: all see all, what they look at added up
        _attend(name="attend_block32_b4_weighed", B=4, n_lo=1951, n_hi=3773, new_lo=32, new_hi=32, page=64, weighed=True),
        # two long conversations, an odd length
        _attend(name="attend_long_131071_b2", B=2, n_lo=131071, n_hi=131071, new_lo=1, new_hi=1, page=64),
        # a small float32 model checking five drafted tokens at once (each sees those in front of it)
        _attend(name="attend_small_f32_causal", dtype="f32", H=4, Hkv=4, dh=64, B=1, n_lo=213, n_hi=213, new_lo=5, new_hi=5, causal=True),
        # a batch's caches cut back to nine tenths
        _evict(name="evict_step_b16", B=16, n_lo=900, n_hi=2688, keep=0.9),
        # one long cache cut to half
        _evict(name="evict_long_65521", B=1, n_lo=65521, n_hi=65521, keep=0.5, page=64),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _heads(rng):
    H = rng.choice([4, 8, 16, 32])
    return H, max(1, H // rng.choice([1, 1, 2, 4, 8]))


def _pairs(rng, dh):
    axes = rng.choice([1, 2, 3, 3, 4])
    left = dh // 2 - (rng.choice([0, 0, 0, dh // 8]))        # sometimes a part of the channels has no position
    cut = sorted(rng.sample(range(1, left), axes - 1))
    return ",".join(str(b - a) for a, b in zip([0] + cut, cut + [left]))


def draw(rng):
    kind = rng.choice(["rope", "append", "attend", "attend", "attend", "evict"])
    sizes = rng.randrange(1, 1 << 20)
    H, Hkv = _heads(rng)
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    dh = rng.choice([64, 128, 128])
    page = rng.choice([16, 32, 64, 128])
    ladder = rng.choice([SHARED, OWN])
    if kind == "rope":
        return _rope(dtype=dtype, rows=_log_int(rng, 1, 14580 if dtype == "bf16" else 7000), H=H, Hkv=Hkv, dh=dh, pairs=_pairs(rng, dh), ladder=ladder,
                     stacked=rng.random() < 0.5, sizes=sizes)
    B = _log_int(rng, 1, 32)
    if kind == "append":
        new = _log_int(rng, 1, max(1, 14000 // B))
        n = new + rng.choice([0, _log_int(rng, 1, 4000)])
        return _append(dtype=dtype, B=B, n_lo=(n + 2) // 3, n_hi=n, new_lo=(new + 1) // 2, new_hi=new, H=H, Hkv=Hkv, dh=dh, pairs=_pairs(rng, dh),
                       ladder=ladder, page=page, stacked=rng.random() < 0.5, sizes=sizes)
    if kind == "evict":
        n = _log_int(rng, 16, 65521 if dtype == "bf16" else 16000)
        B = max(1, min(B, int(1e9 / (n * Hkv * dh * (16 if dtype == "f32" else 8)))))
        return _evict(dtype=dtype, B=B, n_lo=(n + 2) // 3, n_hi=n, keep=rng.uniform(0.25, 0.95), Hkv=Hkv, dh=dh, page=page, first=rng.choice([0, 4]),
                      recent=_log_int(rng, 1, max(1, n // 4)), sizes=sizes)
    new = rng.choice([1, 1, 1, _log_int(rng, 2, 64)])
    n = new - 1 + _log_int(rng, 1, min(131000 if dtype == "bf16" else 16000, int(2.6e8 / (Hkv * dh))))
    most = min(1e9 / (n * Hkv * dh * (8 if dtype == "f32" else 4)), 4e10 / (4.0 * n * new * H * dh))
    if dtype == "f32":
        most = min(most, 4e9 / (4.0 * n * new * H * dh))
    B = max(1, min(B, int(most)))
    while 4.0 * n * new * H * dh > (4e10 if dtype == "bf16" else 4e9) and new > 1:
        new //= 2
    return _attend(dtype=dtype, B=B, n_lo=(n + 2) // 3, n_hi=n, new_lo=(new + 1) // 2, new_hi=new, H=H, Hkv=Hkv, dh=dh, page=page,
                   causal=rng.random() < 0.5, weighed=rng.random() < 0.4, sizes=sizes)


# ---- sizes of a case's samples (part of the case, not of the seed) -------------------------------------------------------
def _samples(c):
    """(lengths, new rows) of the samples; a length counts the new rows"""
    rng = random.Random(c["sizes"])
    n = [rng.randint(c["n_lo"], c["n_hi"]) for _ in range(c["B"])]
    n[0] = c["n_hi"]
    new = [min(v, rng.randint(c.get("new_lo", 0), c.get("new_hi", 0))) for v in n]
    return n, new


def _keeps(c, n):
    return [max(1, math.ceil(c["keep"] * v)) for v in n]


# ---- inputs ----------------------------------------------------------------------------------------------------------------
def _i32(a):
    return torch.tensor(a, dtype=torch.int32, device="cuda")


class _Draw:
    def __init__(self, c, seed):
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(seed)
        self.dt = torch.float32 if c["dtype"] == "f32" else torch.bfloat16

    def normal(self, *shape):
        return torch.empty(shape, dtype=self.dt, device="cuda").normal_(generator=self.g)

    def ints(self, hi, *shape):
        return torch.randint(0, hi, shape, generator=self.g, device="cuda", dtype=torch.int32)

    def uniform(self, *shape):
        return torch.rand(shape, generator=self.g, device="cuda")

    def rows(self, c, rows):
        """q, k and v of new rows: the columns of one stacked projection, or tensors of their own"""
        H, Hkv, dh = c["H"], c["Hkv"], c["dh"]
        if c["stacked"]:
            qkv = self.normal(rows, H + 2 * Hkv, dh)
            return qkv[:, :H], qkv[:, H:H + Hkv], qkv[:, H + Hkv:]
        return self.normal(rows, H, dh), self.normal(rows, Hkv, dh), self.normal(rows, Hkv, dh)

    def positions(self, rows, axes):
        """tokens of images and video: a far first axis (a long conversation's running position), short ones beside it"""
        pos = self.ints(64, rows, axes)
        pos[:, 0] = torch.arange(rows, device="cuda", dtype=torch.int32) + self.ints(100000, 1)
        return pos

    def pages(self, c, n):
        """pages for samples of n tokens, dealt in no order, and the table; entries behind a sample's last page are -1"""
        need = [-(-v // c["page"]) for v in n]
        num = sum(need) + 3
        ids = torch.randperm(num, generator=self.g, device="cuda").to(torch.int32)
        table = torch.full((len(n), max(need) + 1), -1, dtype=torch.int32, device="cuda")
        at = 0
        for b, m in enumerate(need):
            table[b, :m] = ids[at:at + m]
            at += m
        shape = (num, c["page"], c["Hkv"], c["dh"])
        return dict(k_pages=self.normal(*shape), v_pages=self.normal(*shape), page_table=table, kv_len=_i32(n), max_len=max(n))


def _offsets(a):
    out = [0]
    for v in a:
        out.append(out[-1] + v)
    return _i32(out)


def _prepare_rope(c, dr):
    q, k, _ = dr.rows(c, c["rows"])
    return dict(q=q, k=k, pos=dr.positions(c["rows"], c["pairs"].count(",") + 1),
                out=dict(q=torch.zeros(q.shape, dtype=dr.dt, device="cuda"), k=torch.zeros(k.shape, dtype=dr.dt, device="cuda")))


def _prepare_append(c, dr):
    n, new = _samples(c)
    st = dr.pages(c, n)
    q, k, v = dr.rows(c, sum(new))
    W = max(n) + 5
    st.update(q=q, k=k, v=v, pos=dr.positions(sum(new), c["pairs"].count(",") + 1), new_off=_offsets(new), max_new=max(new),
              tokens=torch.cat([torch.arange(a - m, a, dtype=torch.int32) for a, m in zip(n, new)]).cuda(),
              out=dict(q=torch.zeros(q.shape, dtype=dr.dt, device="cuda"), k_pages=st["k_pages"], v_pages=st["v_pages"],
                       token=dr.ints(1 << 20, c["B"], W), weight=dr.uniform(c["B"], W)))
    return st


def _prepare_attend(c, dr):
    n, new = _samples(c)
    st = dr.pages(c, n)
    # a fiftieth of the tokens draws the queries' attention: their logits are 2.5 above the others' on average
    u = dr.normal(c["Hkv"], c["dh"]).float()
    u = u / u.square().sum(1, keepdim=True).sqrt() * math.sqrt(2.5 * math.sqrt(c["dh"]))
    st["k_pages"][dr.uniform(*st["k_pages"].shape[:2]) < 0.02] += u.to(dr.dt)
    q = dr.normal(sum(new), c["H"], c["dh"])
    q += u.to(dr.dt).repeat_interleave(c["H"] // c["Hkv"], 0)
    st.update(q=q, q_off=_offsets(new), max_q=max(new), scale=1.0 / math.sqrt(c["dh"]), causal=c["causal"],
              out=dict(o=torch.zeros_like(q), lse=torch.zeros(q.shape[:2], device="cuda")))
    if c["weighed"]:
        st["weight"] = dr.uniform(c["B"], max(n) + 3) * (8.0 / max(n))       # as much as a few earlier rows gave
        st["out"]["weight"] = torch.zeros_like(st["weight"])
    return st


def _prepare_evict(c, dr):
    n, _ = _samples(c)
    st = dr.pages(c, n)
    B, W = c["B"], max(n)
    # what tokens have got so far is far from even; some slots hold later tokens than their neighbours (an earlier eviction)
    weight = torch.exp(2.0 * torch.empty(B, W, device="cuda").normal_(generator=dr.g) - 4.0)
    token = torch.arange(W, device="cuda", dtype=torch.int32).repeat(B, 1)
    swap = torch.randperm(W, generator=dr.g, device="cuda")[:max(1, W // 16)]
    token[:, swap.sort()[0]] = token[:, swap]
    st.update(weight=weight, token=token, keep=_i32(_keeps(c, n)), first=c["first"], recent=c["recent"],
              out=dict(k_pages=st["k_pages"], v_pages=st["v_pages"], kv_len=torch.zeros(B, dtype=torch.int32, device="cuda"),
                       weight=torch.zeros_like(weight), token=torch.zeros_like(token), src=torch.zeros_like(token)))
    return st


_PREPARE = dict(rope=_prepare_rope, append=_prepare_append, attend=_prepare_attend, evict=_prepare_evict)


def prepare(case, seed):
    st = _PREPARE[case["kind"]](case, _Draw(case, seed))
    st.update(kind=case["kind"], handles={})
    if "pairs" in case:
        st.update(pairs=[int(v) for v in case["pairs"].split(",")], ladder=case["ladder"], theta=10000.0)
    return st


# ---- one pass, plain -----------------------------------------------------------------------------------------------------------
def _angles(s, dh):
    """cos and sin [rows, dh / 2] of the rotary angles (64 bits: positions are far), 32 bits"""
    m = torch.tensor(s["pairs"], device="cuda")
    axis = torch.repeat_interleave(torch.arange(len(s["pairs"]), device="cuda"), m)
    c = torch.arange(axis.numel(), device="cuda", dtype=torch.float64)
    if s["ladder"] == OWN:
        c = (c - (torch.cumsum(m, 0) - m)[axis]) / m[axis]
    else:
        c = 2.0 * c / dh
    a = s["pos"].double()[:, axis] * s["theta"] ** (-c)
    a = torch.cat([a, a.new_zeros(a.shape[0], dh // 2 - axis.numel())], 1)[:, None]
    return torch.cos(a).float(), torch.sin(a).float()


def _turned(x, cos, sin):
    a, b = x.float().chunk(2, -1)
    return torch.cat([a * cos - b * sin, b * cos + a * sin], -1).to(x.dtype)


def _row_sample(off, rows):
    """sample of every row, and the row's place in it"""
    r = torch.arange(rows, device="cuda")
    b = torch.searchsorted(off[1:].long(), r, right=True)
    return b, r - off.long()[b]


def _page_row(s, b, slot):
    ps = s["k_pages"].shape[1]
    return s["page_table"].long()[b, slot // ps], slot % ps


def _plain_append(s):
    out = s["out"]
    cos, sin = _angles(s, s["q"].shape[-1])
    b, i = _row_sample(s["new_off"], s["k"].shape[0])
    slot = (s["kv_len"] - (s["new_off"][1:] - s["new_off"][:-1])).long()[b] + i
    page, row = _page_row(s, b, slot)
    out["k_pages"][page, row] = _turned(s["k"], cos, sin)
    out["v_pages"][page, row] = s["v"]
    out["token"][b, slot] = s["tokens"]
    out["weight"][b, slot] = 0.0
    return dict(out, q=_turned(s["q"], cos, sin))


def _plain_attend(s):
    q, out, L, nq = s["q"], s["out"], s["max_len"], s["max_q"]
    (rows, H, dh), Hkv = q.shape, s["k_pages"].shape[2]
    Bn = s["kv_len"].numel()
    n = s["kv_len"].long()
    j = torch.arange(L, device="cuda")
    page, row = _page_row(s, torch.arange(Bn, device="cuda")[:, None], j[None])
    page = page.clamp(min=0)
    live = j[None] < n[:, None]                                                        # [B, L]
    k = s["k_pages"][page, row].float().permute(0, 2, 3, 1).contiguous()               # [B, Hkv, dh, L]
    v = torch.where(live[:, :, None, None], s["v_pages"][page, row].float(), 0.0).permute(0, 2, 1, 3).contiguous()
    b, i = _row_sample(s["q_off"], rows)
    new = (s["q_off"][1:] - s["q_off"][:-1]).long()
    qp = q.new_zeros(Bn, nq, H, dh, dtype=torch.float32)
    qp[b, i] = q.float() * s["scale"]
    qp = qp.view(Bn, nq, Hkv, H // Hkv, dh).permute(0, 2, 3, 1, 4).reshape(Bn, Hkv, -1, dh)
    logits = torch.matmul(qp, k).view(Bn, Hkv, H // Hkv, nq, L)
    i_all = torch.arange(nq, device="cuda")
    seen = live[:, None, :] & (i_all[None, :, None] < new[:, None, None])              # [B, nq, L]
    if s["causal"]:
        seen = seen & (j[None, None] <= (n - new)[:, None, None] + i_all[None, :, None])
    logits = torch.where(seen[:, None, None], logits, -math.inf)
    top = logits.amax(-1, keepdim=True)
    p = torch.exp(logits - torch.where(top == -math.inf, 0.0, top))
    z = p.sum(-1, keepdim=True)
    lse = (top + torch.log(z)).squeeze(-1)                                             # [B, Hkv, G, nq]
    p = p / torch.where(z == 0, 1.0, z)
    o = torch.matmul(p.view(Bn, Hkv, -1, L), v).view(Bn, Hkv, H // Hkv, nq, dh)
    got = dict(o=o.permute(0, 3, 1, 2, 4).reshape(Bn, nq, H, dh)[b, i].to(q.dtype), lse=lse.permute(0, 3, 1, 2).reshape(Bn, nq, H)[b, i])
    if "weight" in s:
        w = p.sum((1, 2, 3)) / H
        got["weight"] = out["weight"].clone()
        got["weight"][:, :L] = torch.where(live, s["weight"][:, :L] + w, got["weight"][:, :L])
    return got


def _plain_evict(s):
    out, W = s["out"], s["weight"].shape[1]
    n = s["kv_len"].long()[:, None]
    j = torch.arange(W, device="cuda")[None]
    live = j < n
    newest = torch.where(live, s["token"], -1).amax(1, keepdim=True)
    held = live & ((s["token"] < s["first"]) | (s["token"] > newest - s["recent"]))
    value = torch.where(held, math.inf, torch.where(live, s["weight"], -math.inf))
    order = torch.sort(value, dim=1, descending=True, stable=True)[1]
    k = torch.minimum(s["keep"].long()[:, None], n)
    stays = torch.zeros_like(live)
    stays.scatter_(1, order, j < k)
    hb, hj = torch.nonzero((j < k) & ~stays, as_tuple=True)             # as many of either in each sample
    mb, mj = torch.nonzero((j >= k) & stays, as_tuple=True)
    src = torch.where(j < k, j, 0).to(torch.int32)
    src[hb, hj] = mj.to(torch.int32)
    to, frm = _page_row(s, hb, hj), _page_row(s, mb, mj)
    out["k_pages"][to] = out["k_pages"][frm]
    out["v_pages"][to] = out["v_pages"][frm]
    at = src.long()
    return dict(out, kv_len=k[:, 0].to(torch.int32), src=src, weight=torch.where(j < k, s["weight"].gather(1, at), 0.0),
                token=torch.where(j < k, s["token"].gather(1, at), 0))


def _plain(s):
    if s["kind"] == "rope":
        cos, sin = _angles(s, s["q"].shape[-1])
        return dict(q=_turned(s["q"], cos, sin), k=_turned(s["k"], cos, sin))
    return {"append": _plain_append, "attend": _plain_attend, "evict": _plain_evict}[s["kind"]](s)


# ---- one pass, the framework's -------------------------------------------------------------------------------------------------
def _kept(s, name, make):
    """a handle or workspace that the program makes once and keeps"""
    if name not in s["handles"]:
        s["handles"][name] = make()
    return s["handles"][name]


def _own(s):
    from paper_2511_12280_amd import binding as B
    out, kind = s["out"], s["kind"]
    if kind != "rope":
        cache = _kept(s, "cache", lambda: B.PagedCache(s["k_pages"], s["v_pages"], s["page_table"], s["kv_len"]))
    if kind in ("rope", "append"):
        axes = _kept(s, "axes", lambda: B.Axes(s["pos"], s["pairs"], s["theta"], s["ladder"]))
    if kind == "rope":
        B.d3tom_rope_axes(s["q"], s["k"], axes, out["q"], out["k"])
    elif kind == "append":
        B.d3tom_cache_append(cache, s["k"], s["v"], s["new_off"], s["max_new"], axes=axes, q=s["q"], q_out=out["q"], tokens=s["tokens"],
                             slot_token=out["token"], slot_weight=out["weight"])
    elif kind == "attend":
        H, w = s["q"].shape[1], "weight" in s
        ws = _kept(s, "ws", lambda: B.workspace(B.d3tom_attend_cache_workspace_bytes(cache, s["q"].shape[0], s["max_q"], s["max_len"], H, w)))
        B.d3tom_attend_cache(s["q"], cache, s["q_off"], s["max_q"], s["max_len"], s["scale"], s["causal"], out["o"], ws, lse=out["lse"],
                             weight_in=s.get("weight"), weight_out=out.get("weight"))
    else:
        ws = _kept(s, "ws", lambda: B.workspace(B.d3tom_cache_evict_workspace_bytes(cache, s["max_len"])))
        B.d3tom_cache_evict(cache, s["max_len"], s["keep"], s["first"], s["recent"], s["weight"], s["token"], out["weight"], out["token"],
                            out["kv_len"], ws, src=out["src"])
    return out


def run(state):
    return _own(state) if own else _plain(state)


# ---- the definition in 64 bits, sample by sample ---------------------------------------------------------------------------------
def _exact_turn(x, s):
    x, pos = x.double(), s["pos"].double()
    half = x.shape[-1] // 2
    y, at = x.clone(), 0
    for axis, m in enumerate(s["pairs"]):
        for u in range(m):
            f = s["theta"] ** (-(u / m if s["ladder"] == OWN else (at + u) / half))
            co, si = torch.cos(pos[:, axis] * f)[:, None], torch.sin(pos[:, axis] * f)[:, None]
            a, b = x[:, :, at + u], x[:, :, at + u + half]
            y[:, :, at + u], y[:, :, at + u + half] = a * co - b * si, a * si + b * co
        at += m
    return y


def _slots(s, b, n):
    """flat rows of the pages that hold the n slots of sample b"""
    ps = s["k_pages"].shape[1]
    j = torch.arange(n, device="cuda")
    return s["page_table"][b].long()[j // ps] * ps + j % ps


def exact(case, seed):
    if case["kind"] == "evict":
        return None                                     # whole rows and numbers move, nothing is computed
    s = prepare(case, seed)
    if case["kind"] == "rope":
        return dict(q=_exact_turn(s["q"], s), k=_exact_turn(s["k"], s))
    n, new = _samples(case)
    k_flat, v_flat = (s[t].flatten(0, 1) for t in ("k_pages", "v_pages"))
    at = 0
    if case["kind"] == "append":
        k, pages = _exact_turn(s["k"], s), k_flat.double()
        for b, m in enumerate(new):
            pages[_slots(s, b, n[b])[n[b] - m:]] = k[at:at + m]
            at += m
        return dict(q=_exact_turn(s["q"], s), k_pages=pages.view(s["k_pages"].shape), v_pages=None, token=None, weight=None)
    H, Hkv = case["H"], case["Hkv"]
    o, lse = torch.zeros_like(s["q"], dtype=torch.float64), torch.zeros(s["q"].shape[:2], dtype=torch.float64, device="cuda")
    weight = s["out"]["weight"].double() if case["weighed"] else None
    for b, m in enumerate(new):
        rows = _slots(s, b, n[b])
        hidden = torch.zeros(m, n[b], dtype=torch.bool, device="cuda")
        if case["causal"]:
            hidden = torch.triu(torch.ones(m, n[b], dtype=torch.bool, device="cuda"), diagonal=n[b] - m + 1)
        total = torch.zeros(n[b], dtype=torch.float64, device="cuda")
        for h in range(H):
            g = h * Hkv // H
            x = s["q"][at:at + m, h].double() @ k_flat[rows, g].double().t().contiguous() * s["scale"]
            x = x.masked_fill(hidden, -math.inf)
            lse[at:at + m, h] = torch.logsumexp(x, 1)
            p = torch.softmax(x, 1)
            o[at:at + m, h] = p @ v_flat[rows, g].double()
            total += p.sum(0)
        if weight is not None:
            weight[b, :n[b]] = s["weight"][b, :n[b]].double() + total / H
        at += m
    return dict(o=o, lse=lse, **({"weight": weight} if weight is not None else {}))


# ---- what a pass cannot do without -------------------------------------------------------------------------------------------
def work(case):
    eb = 4 if case["dtype"] == "f32" else 2
    row = case["Hkv"] * case["dh"] * eb                  # of k or v
    if case["kind"] == "rope":
        rows, axes = case["rows"], case["pairs"].count(",") + 1
        return {"bytes": rows * (2.0 * (case["H"] + case["Hkv"]) * case["dh"] * eb + 4 * axes), "flops": 3.0 * rows * (case["H"] + case["Hkv"]) * case["dh"]}
    n, new = _samples(case)
    if case["kind"] == "append":
        axes = case["pairs"].count(",") + 1
        return {"bytes": sum(new) * (4.0 * row + 2.0 * case["H"] * case["dh"] * eb + 4 * axes + 12), "flops": 3.0 * sum(new) * (case["H"] + case["Hkv"]) * case["dh"]}
    if case["kind"] == "attend":
        by = sum(2.0 * v * row for v in n) + sum(new) * case["H"] * (2.0 * case["dh"] * eb + 4) + 4.0 * sum(-(-v // case["page"]) for v in n)
        pairs = sum(m * (2 * v - m + 1) / 2 if case["causal"] else m * v for v, m in zip(n, new))
        return {"bytes": by + (8.0 * sum(n) if case["weighed"] else 0.0), "flops": 4.0 * pairs * case["H"] * case["dh"]}
    by = 0.0
    for v, k in zip(n, _keeps(case, n)):
        k = min(k, v)
        by += 8.0 * v + 12.0 * k + 4.0 * row * k * (v - k) / v      # the share of kept slots is the same behind the new end as in front of it
    return {"bytes": by, "flops": 0.0}
