"""The serving operators on the GPU against their fp64 oracle.

Tolerances: eps is torch.finfo(type).eps, a rounding is off by eps / 2 of the
value. Rotation: one rounding of the result, and fp32 errors of the angle
(2^-25 turns of input rounding, 2^-23 of cosine and sine) and of three
operations, below 2^-20 of |a| + |b|. Attention: one rounding of the result and
one of each weight (eps / 2 of sum w |v| together); a score is off by at most
D 2^-24 of its sum |q||k| times the scale plus 2^-22 of its own size (the
products with scale log2 e), a weight by twice that and 2^-20 more from the
exponentials, the sums and the joins. Sampled tokens have to be equal."""
import math

import numpy as np
import pytest
import torch

import paper_2010_02164_amd as sb
from oracle import serving as oracle

pytestmark = pytest.mark.gpu
BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32


def rng(seed):
    return np.random.default_rng(seed)


def dev(a, dtype=None):
    return torch.as_tensor(np.ascontiguousarray(a)).cuda().to(dtype) if dtype else torch.as_tensor(np.ascontiguousarray(a)).cuda()


def i32(a):
    return dev(np.asarray(a, np.int32))


def f64(t):
    return t.double().cpu().numpy()


# -- pages -------------------------------------------------------------------------

def run_plan(lens, add, free, n_pages, table, page, cap, **kw):
    fl = np.full(n_pages, -7, np.int32)
    fl[:len(free)] = free
    tab, fl = i32(table), i32(fl)
    p = sb.plan_pages(i32(lens), i32(add), fl, i32([len(free)]), tab, page_size=page, token_cap=cap, **kw)
    return p, tab, fl


def check_plan(lens, add, free, n_pages, table, page, cap):
    want = oracle.plan_pages(lens, add, free, table, page, cap)
    p, tab, fl = run_plan(lens, add, free, n_pages, table, page, cap)
    got = [x.tolist() for x in (p.lens, p.granted, fl[:int(p.n_free)], tab, p.slots, p.positions, p.q_start)]
    for name, a, b in zip(("lens", "granted", "free", "table", "slots", "positions", "q_start"), got, want):
        assert a == [int(x) for x in b] if name != "table" else a == b.tolist(), name
    return want


@pytest.mark.parametrize("B,page,mode", [(1, 16, "one"), (3, 1, "few"), (7, 5, "mixed"), (64, 16, "one"), (1000, 16, "mixed"), (1025, 8, "one"),
                                         (2049, 3, "mixed"), (8192, 4, "mixed"), (33, 64, "long"), (5, 4096, "long")])
def test_plan(gpu, B, page, mode):
    r = rng(B)
    width = 12 if mode != "long" else 60
    lens = r.integers(0, 6 * page, B)
    add = {"one": np.ones(B, int), "few": r.integers(0, 5, B), "mixed": r.integers(-1, 4 * page, B),
           "long": r.integers(-1, min(50 * page, 3000), B)}[mode]
    held = -(-lens // page)
    n_pages = int(held.sum() + B * 3)
    ids = r.permutation(n_pages)
    table = np.full((B, width), -1)
    table[np.arange(width) < held[:, None]] = ids[:held.sum()]
    free = ids[held.sum():].tolist()
    everything = int(np.maximum(add, 0).sum())
    for cap, some in ((everything + 3, free), (everything // 2, free), (everything + 3, free[:len(free) // 4]), (0, free)):
        want = check_plan(lens, add, some, n_pages, table, page, cap)
        new = [int(x) for b, n in enumerate(lens) if add[b] >= 0 for x in want[3][b, :-(-want[0][b] // page)]]
        assert len(set(new)) == len(new) and not set(new) & set(want[2])   # no page twice


def test_plan_refuses_one_request_without_holding_up_others(gpu):
    want = check_plan([0, 30, 2, 0], [5, 3, 2, 33], [4, 5, 6, 7], 8, np.full((4, 8), 1), 4, 50)
    assert want[1] == [5, 0, 2, 0]


def test_plan_wrong_state_stays_in_bounds(gpu):
    """Lengths and free counts out of range are taken as the nearest in it,
    released pages that do not fit the list are dropped, and slots of page ids
    that are none are -1."""
    p, tab, fl = run_plan([10 ** 9, -5, 4], [-1, 3, 1], list(range(6)), 6, [[9, -3, 7]] * 3, 2, 9)
    assert p.lens.tolist() == [0, 3, 5] and int(p.n_free) == 6 - 3
    assert tab.tolist()[1][:2] == [5, 4]
    p, tab, _ = run_plan([0], [3], [99, -2], 2, [[0, 0]], 2, 4)
    assert p.slots.tolist() == [-1, -1, -1, -1] and p.positions.tolist() == [0, 1, 2, -1]
    lens, table = i32([2]), i32([[0, 1]])   # 2 more fill the row and need a page
    for n_free in (-4, 50):
        p = sb.plan_pages(lens, i32([2]), i32([2, 3]), i32([n_free]), table, page_size=2, token_cap=2)
        assert p.granted.tolist() == ([0] if n_free < 0 else [2])


def test_plan_in_place_and_repeated(gpu):
    """State written over its inputs goes on as the oracle does; state written
    elsewhere leaves the call repeatable."""
    r = rng(3)
    B, page, width, n_pages = 40, 4, 20, 300
    lens, free, table = [0] * B, list(range(n_pages)), np.full((B, width), -1)
    fl, tab = i32(free), i32(table)
    cur = sb.PagePlan(i32([0] * (B + 1)), i32(lens), i32(lens), dev(np.zeros(90, np.int64)), i32([0] * 90), i32([n_pages]))
    for step in range(30):
        add = r.integers(-1, 6, B)
        lens, granted, free, table, slots, pos, q_start = oracle.plan_pages(lens, add, free, table, page, 90)
        apart = [sb.plan_pages(cur.lens, i32(add), fl, cur.n_free, tab, page_size=page, token_cap=90) for _ in range(2)]
        assert all(torch.equal(x, y) for x, y in zip(*apart))
        got = sb.plan_pages(cur.lens, i32(add), fl, cur.n_free, tab, page_size=page, token_cap=90, out=cur)
        assert got is cur and all(torch.equal(x, y) for x, y in zip(got, apart[0]))
        assert cur.lens.tolist() == lens and cur.slots.tolist() == slots and fl[:int(cur.n_free)].tolist() == free


@pytest.mark.parametrize("B,page", [(1, 16), (65, 4), (1024, 16), (1030, 3)])
def test_plan_of_single_tokens(gpu, B, page):
    """Steps in which requests take a token, none, or end; of entries of the
    table that are no pages the slots are -1."""
    r = rng(B + 1)
    lens, add = r.integers(0, 5 * page, B), r.integers(-1, 2, B)
    add[0] = 1
    held = -(-lens // page)
    n_pages = int(held.sum()) + B
    ids = r.permutation(n_pages)
    table = np.full((B, 6), -1)
    table[np.arange(6) < held[:, None]] = ids[:held.sum()]
    free = ids[held.sum():].tolist()
    for cap, some in ((B, free), (B // 2, free), (B + 70, free[:B // 8])):
        check_plan(lens, add, some, n_pages, table, page, cap)
    lens[0], add[:] = 2 * page - 1, 1
    for bad in (-1, -2 ** 31, n_pages, 2 ** 31 - 1):
        table[0, 1] = bad
        p, _, _ = run_plan(lens, add, free, n_pages, table, page, B)
        assert int(p.slots[0]) == -1 and int(p.positions[0]) == 2 * page - 1
        assert bool((p.slots[1:] >= 0).all())


# -- rotary positions and the cache's write --------------------------------------------

def rope_case(T, Hq, Hkv, D, pairs, dtype, seed, page=16, far=10 ** 6):
    r = rng(seed)
    n_pages = T // page + 3
    make = lambda *s: dev(r.standard_normal(s), dtype)   # noqa: E731
    return dict(q=make(T, Hq, D), k=make(T, Hkv, D), v=make(T, Hkv, D), positions=i32(r.integers(0, far, T)),
                slots=dev(r.permutation(n_pages * page)[:T]), k_cache=make(n_pages, page, Hkv, D), v_cache=make(n_pages, page, Hkv, D),
                inv_freq=dev(10000.0 ** (-np.arange(pairs) / max(pairs, 1))))


def check_rope(c, layout, mscale, rotated, before, rows=None):
    """rows: the tokens to look at (None: all)."""
    dtype = rotated.dtype
    eps = torch.finfo(dtype).eps
    inv, pos, slots = f64(c["inv_freq"]), c["positions"].tolist(), c["slots"].tolist()
    page = c["k_cache"].shape[1]
    kb, vb = before[0].clone(), before[1].clone()
    for t in range(len(pos)) if rows is None else rows:
        if not 0 <= slots[t] < kb.shape[0] * page:
            continue
        at = slots[t] // page, slots[t] % page
        for x, got in ((c["q"][t], rotated[t]), (c["k"][t], c["k_cache"][at])):
            for h in range(x.shape[0]):
                want, size = oracle.rotate(f64(x[h]), pos[t], inv, layout, mscale)
                assert np.all(np.abs(f64(got[h]) - want) <= eps / 2 * np.abs(want) + 2.0 ** -20 * size), (t, h)
        assert torch.equal(c["v_cache"][at], c["v"][t])
        kb[at], vb[at] = c["k_cache"][at], c["v"][t]
    if rows is None:   # nothing else was written
        assert torch.equal(kb, c["k_cache"]) and torch.equal(vb, c["v_cache"])


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("T,Hq,Hkv,D,pairs,layout,mscale,page", [
    (1, 4, 1, 64, 32, "half", 1.0, 16), (5, 3, 3, 128, 64, "interleaved", 1.2, 7), (37, 8, 2, 128, 16, "half", 0.7, 1),
    (3, 1, 1, 256, 128, "half", 1.0, 128), (9, 5, 1, 8, 4, "interleaved", 1.0, 3), (4, 2, 2, 512, 256, "half", 1.0, 64),
    (6, 7, 1, 72, 8, "half", 1.1, 5), (2, 2, 1, 64, 0, "half", 1.0, 4), (2, 2, 1, 64, 0, "interleaved", 1.0, 4)])
def test_rope(gpu, T, Hq, Hkv, D, pairs, layout, mscale, page, dtype):
    c = rope_case(T, Hq, Hkv, D, pairs, dtype, T + D, page)
    before = c["k_cache"].clone(), c["v_cache"].clone()
    got = sb.rope_append(**c, layout=layout, mscale=mscale)
    check_rope(c, layout, mscale, got, before)


@pytest.mark.parametrize("layout", ["half", "interleaved"])
def test_rope_many_tokens(gpu, layout):
    """A prompt (several tokens a workgroup, a last one that is not full)."""
    c = rope_case(8195, 4, 2, 64, 16, BF16, 5)
    c["slots"][[0, 4097, 8190]] = torch.tensor([-1, 10 ** 12, c["k_cache"].shape[0] * 16]).cuda()
    before = c["k_cache"].clone(), c["v_cache"].clone()
    out = dev(np.full((8195, 4, 64), 7.0), BF16)
    sb.rope_append(**c, layout=layout, out=out)
    check_rope(c, layout, 1.0, out, before, [1, 2, 3, 4, 5, 4096, 4098, 8189, 8191, 8192, 8193, 8194])
    assert bool((out[[0, 4097, 8190]] == 7).all())          # skipped tokens stay as they were
    one = [sb.rope_append(**{n: (x[t:t + 300] if x.shape[0] == 8195 else x) for n, x in c.items()}, layout=layout)
           for t in range(0, 8195, 300)]                     # and the one-token kernel gives the same bits
    keep = torch.ones(8195, dtype=torch.bool)
    keep[[0, 4097, 8190]] = False
    assert torch.equal(torch.cat(one)[keep], out[keep])


def test_rope_views_in_place(gpu):
    """Slices of one projection's output, turned in place; caches with heads
    before tokens, both in one allocation."""
    T, Hq, Hkv, D, page = 21, 6, 2, 64, 4
    r = rng(8)
    qkv = dev(r.standard_normal((T, Hq + 2 * Hkv, D)), F16)
    c = rope_case(T, Hq, Hkv, D, 32, F16, 9, page)
    pool = torch.zeros(8, 2, Hkv, page, D, dtype=F16, device="cuda")
    q, k, v = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
    c.update(q=q, k=k, v=v, k_cache=pool[:, 0].transpose(1, 2), v_cache=pool[:, 1].transpose(1, 2))
    plain = {n: x.clone() for n, x in c.items()}
    want = sb.rope_append(**{n: x.contiguous() for n, x in plain.items()})
    before = torch.zeros_like(plain["k_cache"]), torch.zeros_like(plain["v_cache"])
    assert sb.rope_append(**c, out=q) is q
    assert torch.equal(q, want)
    check_rope(dict(plain, k_cache=c["k_cache"], v_cache=c["v_cache"]), "half", 1.0, q, before)


def test_rope_slots_given_twice(gpu):
    """The queries are right, and every piece of 8 values in the cache is one of
    the tokens'; nothing else is written."""
    T, D = 600, 64
    c = rope_case(T, 2, 2, D, 32, BF16, 13)
    apart = dict(c, k_cache=c["k_cache"].clone(), v_cache=c["v_cache"].clone())
    want = sb.rope_append(**apart)
    at = [(int(s) // 16, int(s) % 16) for s in c["slots"][:3]]
    own = c["slots"].clone()
    c["slots"] = own[torch.arange(T, device="cuda") % 3]
    before = c["k_cache"].clone(), c["v_cache"].clone()
    assert torch.equal(sb.rope_append(**c), want)
    for cache, held, given in ((c["k_cache"], before[0], apart["k_cache"]), (c["v_cache"], before[1], apart["v_cache"])):
        mine = given.view(-1, 2, D // 8, 8)[own]   # what each token writes
        for i, (page, place) in enumerate(at):
            got = cache[page, place].view(2, D // 8, 8)
            assert bool((mine[i::3] == got).all(-1).any(0).all())
            cache[page, place] = held[page, place]
        assert torch.equal(cache, held)


def test_rope_far_positions(gpu):
    """Positions up to 2^31 - 1: an fp32 angle would be off by whole turns."""
    c = rope_case(4, 1, 1, 64, 32, F16, 11)
    c["positions"] = i32([2 ** 31 - 1, 2 ** 30 + 1, 0, -5])
    before = c["k_cache"].clone(), c["v_cache"].clone()
    check_rope(c, "half", 1.0, sb.rope_append(**c), before)


# -- attention ---------------------------------------------------------------------

def attention_case(B, Hq, Hkv, D, page, q_lens, kv_lens, dtype, seed, pad=0, spread=1.0):
    r = rng(seed)
    q_lens, kv_lens = np.resize(q_lens, B), np.resize(kv_lens, B)
    held = -(-kv_lens // page)
    n_pages = int(held.sum()) + 2
    table = np.full((B, max(int(held.max()), 1) + 1), -1)
    table[np.arange(table.shape[1]) < held[:, None]] = r.permutation(n_pages)[:held.sum()]
    q_start = np.concatenate([[0], np.cumsum(q_lens)])
    T = int(q_start[-1]) + pad
    return dict(q=dev(spread * r.standard_normal((T, Hq, D)), dtype), k_cache=dev(r.standard_normal((n_pages, page, Hkv, D)), dtype),
                v_cache=dev(r.standard_normal((n_pages, page, Hkv, D)), dtype), table=i32(table), lens=i32(kv_lens), q_start=i32(q_start))


def bounds(c, max_q=None, max_kv=None):
    q = (c["q_start"][1:] - c["q_start"][:-1]).max()
    return dict(max_q=int(q) if max_q is None else max_q, max_kv=int(c["lens"].max()) if max_kv is None else max_kv)


def kv_bound(max_q, max_kv):
    """A bound with which the kernel for prompts, which a large max_q takes, splits
    no keys, and workgroups of the other one share them."""
    return 1 if max_q == 1000 else max(max_kv, 5000)


def check_attention(c, got, window=0, sinks=0, scale=None, only=None):
    """only: queries to look at (the oracle runs on those requests' rows)."""
    D = got.shape[2]
    eps = torch.finfo(got.dtype).eps
    scale = 1 / math.sqrt(D) if scale is None else scale
    want, size, big = oracle.attention(f64(c["q"]), f64(c["k_cache"]), f64(c["v_cache"]), c["table"].tolist(), c["lens"].tolist(),
                                       c["q_start"].tolist(), window, sinks, scale)
    score = big * abs(scale) * (D * 2.0 ** -24 + 2.0 ** -22)
    tol = eps / 2 * np.abs(want) + (eps / 2 + 2 * score[..., :1] + 2.0 ** -20) * size + torch.finfo(got.dtype).smallest_normal
    rows = int(c["q_start"][-1])
    d = np.abs(f64(got)[:rows] - want[:rows])
    assert np.all(d <= tol[:rows]), (np.argwhere(~(d <= tol[:rows]))[:5], np.nanmax(d / tol[:rows]))


FORMS = [   # B, Hq, Hkv, page, queries, cached
    (1, 4, 1, 16, [1], [1]), (5, 8, 2, 16, [1], [1, 2, 31, 33, 200]), (3, 5, 5, 7, [1], [64, 500, 13]),
    (2, 16, 1, 1, [1], [40, 97]), (3, 32, 2, 24, [1], [130, 5, 300]), (4, 8, 4, 32, [3, 1, 4, 2], [3, 90, 65, 2]),
    (2, 40, 2, 16, [2], [50, 81]), (3, 4, 2, 16, [40, 1, 97], [40, 260, 150]), (1, 8, 1, 64, [70], [129]), (2, 3, 3, 5, [130, 33], [200, 33]),
]


@pytest.mark.parametrize("dtype,D", [(BF16, 128), (F16, 64), (BF16, 256), (F16, 128)])
@pytest.mark.parametrize("form", range(len(FORMS)))
def test_attention(gpu, form, dtype, D):
    c = attention_case(*FORMS[form][:3], D, *FORMS[form][3:], dtype, form)
    for window, sinks in ((0, 0), (17, 0), (17, 4), (1, 0), (1, 100), (64, 33)):
        got = sb.paged_attention(**c, **bounds(c), window=window, sinks=sinks)
        check_attention(c, got, window, sinks)
        if form < 2 or form > 5:   # by the other kernel: of prompts, or of single tokens
            for max_q, max_kv in ((1000, 1), (0, 1), (0, 5000)):
                got = sb.paged_attention(**c, max_q=max_q, max_kv=max_kv, window=window, sinks=sinks)
                check_attention(c, got, window, sinks)
        got = sb.paged_attention(**c, **bounds(c, max_kv=5000), window=window, sinks=sinks)   # (shared, or split)
        check_attention(c, got, window, sinks)


@pytest.mark.parametrize("form", range(len(FORMS)))
def test_attention_fp16_heads_of_256(gpu, form):
    """Both kernels, whole, shared and split, with and without windows."""
    test_attention(gpu, form, F16, 256)


@pytest.mark.parametrize("q,kv", [([1, 2, 1], [6000, 9, 2500]), ([90, 260, 1], [3000, 2000, 700])])
def test_attention_fp16_heads_of_256_long(gpu, q, kv):
    """Keys in parts, what is hidden not finite, and a key that the last query
    alone sees not a number."""
    c = attention_case(3, 4, 2, 256, 16, q, kv, F16, 17, pad=3)
    for window, sinks in ((0, 0), (1100, 3)):
        check_attention(c, sb.paged_attention(**c, **bounds(c), window=window, sinks=sinks), window, sinks)
    want = sb.paged_attention(**c, **bounds(c))
    last = kv[0] - 1
    at = int(c["table"][0, last // 16]), last % 16
    for j in range(last % 16 + 1, 16):   # behind the first request's last token
        c["k_cache"][at[0], j], c["v_cache"][at[0], j] = math.nan, math.inf
    rows, first = int(c["q_start"][-1]), int(c["q_start"][1]) - 1
    assert torch.equal(sb.paged_attention(**c, **bounds(c))[:rows], want[:rows])
    c["v_cache"][at] = math.nan
    got = sb.paged_attention(**c, **bounds(c))[:rows]
    assert bool(got[first].isnan().all())
    assert torch.equal(got[:first], want[:first]) and torch.equal(got[first + 1:], want[first + 1:rows])


@pytest.mark.parametrize("dtype,D,Hq,Hkv", [(BF16, 128, 4, 1), (F16, 64, 8, 1), (BF16, 256, 2, 1)])
def test_attention_long_cache_in_parts(gpu, dtype, D, Hq, Hkv):
    """Caches long enough to be split over workgroups, short ones beside."""
    c = attention_case(3, Hq, Hkv, D, 16, [1, 2, 1], [6000, 9, 2500], dtype, 5)
    for window, sinks in ((0, 0), (2000, 5)):
        for over in ({}, dict(max_q=1000, max_kv=1)):
            got = sb.paged_attention(**c, **bounds(c, **over), window=window, sinks=sinks)
            check_attention(c, got, window, sinks)


def test_attention_wrong_bounds_only_cost_time(gpu):
    """max_q and max_kv that are too small or too large: the same result up to rounding."""
    for q, kv in (([1], [700, 30]), ([60, 3], [700, 30])):
        c = attention_case(2, 8, 2, 128, 16, q, kv, BF16, 6)
        for max_q, max_kv in ((0, 0), (1, 1), (1, 10 ** 6), (10 ** 6, 700), (2 ** 31 - 1, 2 ** 31 - 1)):
            got = sb.paged_attention(**c, max_q=max_q, max_kv=max_kv, window=300, sinks=2)
            check_attention(c, got, 300, 2)


@pytest.mark.parametrize("max_q", [0, 1, 3, 1000])
def test_attention_of_many_requests(gpu, max_q):
    """More requests than threads, of 0 to 3 queries, some over no tokens; with
    many heads so many that each has a workgroup."""
    for B, Hq, Hkv, D, dtype in ((300, 4, 1, 64, BF16), (700, 20, 1, 64, F16), (1100, 8, 8, 128, BF16)):
        r = rng(B)
        c = attention_case(B, Hq, Hkv, D, 16, r.integers(0, 4, B), r.integers(0, 120, B) * (r.random(B) > 0.1).astype(int), dtype, B)
        for window, sinks in ((0, 0), (20, 2)):
            check_attention(c, sb.paged_attention(**c, max_q=max_q, max_kv=kv_bound(max_q, 120), window=window, sinks=sinks), window, sinks)


@pytest.mark.parametrize("dtype,D,Hq,Hkv,page,q,kv", [
    (BF16, 128, 8, 2, 16, [200], [5000]), (F16, 64, 6, 1, 32, [150, 1, 333], [2600, 900, 4000]), (BF16, 256, 4, 2, 64, [100, 260], [3000, 2000]),
    (F16, 128, 32, 8, 16, [64], [4100])])
def test_attention_prompts_with_split_keys(gpu, dtype, D, Hq, Hkv, page, q, kv):
    """Few long prompts, whose keys are split over workgroups: with windows, pages
    that are none, values that are not finite behind the last key, and rows
    behind the last request."""
    c = attention_case(len(q), Hq, Hkv, D, page, q, kv, dtype, D + len(q), pad=5)
    kw = bounds(c)
    for window, sinks in ((0, 0), (1500, 3), (40, 0)):
        check_attention(c, sb.paged_attention(**c, **kw, window=window, sinks=sinks), window, sinks)
    out = dev(np.full(c["q"].shape, 3.0), dtype)
    clean = sb.paged_attention(**c, **kw)
    last = int(c["lens"][0]) - 1   # a key that the first request's last query alone sees
    at = int(c["table"][0, last // page]), last % page
    held = c["v_cache"][at].clone()
    c["v_cache"][at] = math.nan
    sb.paged_attention(**c, **kw, out=out)
    first, rows = int(c["q_start"][1]) - 1, int(c["q_start"][-1])
    assert torch.equal(out[:first], clean[:first]) and bool(out[first].isnan().all()) and bool((out[rows:] == 3).all())
    c["v_cache"][at] = held
    c["table"][0, 20], c["table"][0, 33] = -1, 10 ** 6
    check_attention(c, sb.paged_attention(**c, **kw))
    c["lens"][0] = 3   # fewer tokens than queries: those before the first see nothing
    got = sb.paged_attention(**c, **kw)
    check_attention(c, got)
    assert bool((got[:int(c["q_start"][1]) - 3] == 0).all())


@pytest.mark.parametrize("max_q", [1, 1000])
def test_attention_windows_of_any_size(gpu, max_q):
    """Up to 2^31 - 1, also for queries before the first cached token."""
    c = attention_case(4, 8, 2, 64, 16, [5, 1, 40, 3], [2, 300, 17, 0], BF16, 14)
    for max_kv in (1, 300, 5000):
        want = sb.paged_attention(**c, max_q=max_q, max_kv=max_kv)
        check_attention(c, want)
        for window in (301, 10 ** 9, 2 ** 31 - 40, 2 ** 31 - 2, 2 ** 31 - 1):
            for sinks in (0, 3, 2 ** 31 - 1):
                got = sb.paged_attention(**c, max_q=max_q, max_kv=max_kv, window=window, sinks=sinks)
                if window > 301:   # (that one may bring another split)
                    assert torch.equal(got, want), (window, sinks)
                check_attention(c, got)
    got = sb.paged_attention(**c, max_q=max_q, max_kv=kv_bound(max_q, 300), window=1, sinks=2 ** 31 - 1)
    check_attention(c, got, 1, 2 ** 31 - 1)


@pytest.mark.parametrize("max_q", [1, 1000])
def test_attention_empty_rows(gpu, max_q):
    """Requests without queries or tokens, queries before the first position,
    rows behind the last request."""
    c = attention_case(6, 4, 2, 64, 8, [0, 2, 1, 0, 5, 1], [9, 2, 0, 0, 3, 6], BF16, 7, pad=4)
    out = dev(np.full(c["q"].shape, 3.0), BF16)
    assert sb.paged_attention(**c, max_q=max_q, max_kv=kv_bound(max_q, 9), out=out) is out
    check_attention(c, out)
    assert bool((out[2] == 0).all()) and bool((out[3:5] == 0).all())   # of a request of 0 tokens; positions -2 and -1
    assert bool((out[-4:] == 3).all())
    out.fill_(3)
    nobody = dict(c, q_start=i32([0] * 7))
    sb.paged_attention(**nobody, max_q=max_q, max_kv=kv_bound(max_q, 9), out=out)
    assert bool((out == 3).all())


@pytest.mark.parametrize("max_q", [1, 1000])
def test_attention_pages_outside_the_cache_are_skipped(gpu, max_q):
    c = attention_case(3, 4, 2, 128, 4, [2, 1, 1], [30, 21, 8], BF16, 8)
    c["table"][0, 3], c["table"][0, 5], c["table"][1, 0] = 10 ** 6, -9, 2 ** 31 - 1
    c["table"][2, :2] = -1
    got = sb.paged_attention(**c, max_q=max_q, max_kv=kv_bound(max_q, 30))
    check_attention(c, got)
    assert bool((got[3] == 0).all())
    c["lens"][1] = 2 ** 31 - 1   # longer than its table row: cut there, whose places behind are -1
    got = sb.paged_attention(**c, max_q=max_q, max_kv=kv_bound(max_q, 30))
    assert bool(torch.isfinite(got).all())


@pytest.mark.parametrize("max_q", [1, 1000])
@pytest.mark.parametrize("Hq", [2, 3, 6])
def test_attention_wrong_starts_stay_in_bounds(gpu, max_q, Hq):
    """Starts that are none: clipped to the rows there are, and a request that
    starts behind the next has none. (m = -1.5e9 queries of 2 heads are 1.29e9
    rows in 32 bits.)"""
    c = attention_case(4, Hq, 1, 64, 8, [2, 0, 3, 0], [9, 5, 20, 7], BF16, 16, pad=3)
    T, kw = 8, dict(max_q=max_q, max_kv=kv_bound(max_q, 20))
    want = sb.paged_attention(**dict(c, q_start=i32([0, 2, 2, T, T])), **kw)
    for last in (0, -5, -2 ** 31, 1_500_000_000):
        for q_start in ([0, 2, 2, 1_500_000_000, last], [-7, 2, 2, 2 ** 31 - 1, last], [0, 2, 2, T, last]):
            out = torch.full_like(want, 3.0)
            sb.paged_attention(**dict(c, q_start=i32(q_start)), **kw, out=out)
            assert torch.equal(out[2:], want[2:]) and (q_start[0] < 0 or torch.equal(out, want)), q_start
    for q_start in ([-2 ** 31, -1, 2 ** 31 - 1, -2 ** 31, 5], [2 ** 31 - 1, 2 ** 31 - 2, -3, 2 ** 30, -2 ** 30]):
        sb.paged_attention(**dict(c, q_start=i32(q_start)), **kw, out=torch.full_like(want, 3.0))
    torch.cuda.synchronize()


@pytest.mark.parametrize("max_q,dtype", [(1, BF16), (1000, BF16), (1000, F16)])
def test_attention_what_is_hidden_does_not_matter(gpu, max_q, dtype):
    """NaN and infinities on pages of nobody, behind the last token, before the
    window, and at positions that other rows of the tile do see."""
    for q, kv, window, sinks in (([1], [50, 77], 20, 3), ([6, 3], [50, 77], 9, 2), ([6, 3], [50, 77], 0, 0)):
        c = attention_case(2, 4, 1, 64, 16, q, kv, dtype, 9)
        clean = sb.paged_attention(**c, max_q=max_q, max_kv=kv_bound(max_q, 77), window=window, sinks=sinks)
        used = torch.zeros(c["k_cache"].shape[:2], dtype=torch.bool, device="cuda")
        m = c["q_start"][1:] - c["q_start"][:-1]
        for b, n in enumerate(kv):
            lo = max(0, n - int(m[b]) + 1 - window) if window else 0
            for j in list(range(min(sinks, lo))) + list(range(lo, n)):
                used[c["table"][b, j // 16], j % 16] = True
        for bad in (math.nan, math.inf, -math.inf):
            c["k_cache"][~used] = bad
            c["v_cache"][~used] = bad
            assert torch.equal(sb.paged_attention(**c, max_q=max_q, max_kv=kv_bound(max_q, 77), window=window, sinks=sinks), clean)
        if q[0] > 1:   # the last position is seen by the last query alone
            at = int(c["table"][0, 49 // 16]), 49 % 16
            c["k_cache"][at], c["v_cache"][at] = 0.0, math.nan
            got = sb.paged_attention(**c, max_q=max_q, max_kv=kv_bound(max_q, 77), window=window, sinks=sinks)
            assert torch.equal(got[:5], clean[:5]) and bool(got[5].isnan().all()) and torch.equal(got[6:], clean[6:])
            c["v_cache"][at] = math.inf
            c["k_cache"][at] = math.nan
            got = sb.paged_attention(**c, max_q=max_q, max_kv=kv_bound(max_q, 77), window=window, sinks=sinks)
            assert torch.equal(got[:5], clean[:5]) and bool(got[5].isnan().all()) and torch.equal(got[6:], clean[6:])


@pytest.mark.parametrize("max_q", [1, 1000])
def test_attention_large_scores(gpu, max_q):
    """Scores of thousands: the running maximum has to move; and a scale of its
    own, also negative and zero."""
    c = attention_case(2, 4, 2, 128, 16, [9, 1], [300, 140], BF16, 10, spread=60.0)
    for scale in (None, -0.02, 0.0):
        got = sb.paged_attention(**c, max_q=max_q, max_kv=kv_bound(max_q, 300), scale=scale)
        check_attention(c, got, scale=scale)


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("max_q", [1, 1000])
def test_attention_many_small_weights(gpu, max_q, dtype):
    """Very many keys of weights around fp16's smallest number (2^-24 of the
    largest one's) next to a large one, which comes first, last, or in between:
    together they are 0.002 to 0.004 of it."""
    n, D = 100_000, 64
    far = [24.4, 24.9, 25.1, 25.6]   # powers of two below the large one's
    for at in (0, n // 2, n - 1):
        c = attention_case(1, 4, 1, D, 128, [1], [n], dtype, 15)
        c["q"].zero_(), c["k_cache"].zero_()
        for h, x in enumerate(far):
            c["q"][0, h, h] = x / 4 * math.log(2)   # in halves: rounded to the type, which both sides take
        c["k_cache"][int(c["table"][0, at // 128]), at % 128, 0, :4] = 4.0
        c["v_cache"] += 1.0
        for max_kv in (1, n):
            check_attention(c, sb.paged_attention(**c, max_q=max_q, max_kv=max_kv, scale=1.0), scale=1.0)


@pytest.mark.parametrize("dtype,D", [(BF16, 64), (BF16, 128), (BF16, 256), (F16, 64), (F16, 128), (F16, 256)])
@pytest.mark.parametrize("n", [2, 700, 6000])
def test_attention_weights_in_two_parts(gpu, n, dtype, D):
    """Up to 16 rows a request: a weight is off by (eps / 2)^2 of itself. Every
    other key is a little less likely and its value the negative one, so that
    weights rounded once would show (their errors add up, the values do not)."""
    c = attention_case(1, 16, 1, D, 16, [1], [n], dtype, n)
    c["q"].zero_(), c["k_cache"].zero_()
    c["q"][0, :, 0] = torch.linspace(0.005, 0.4, 16, device="cuda")
    for j in range(n):
        at = int(c["table"][0, j // 16]), j % 16
        c["v_cache"][at] = 1.0 if j % 2 else -1.0
        c["k_cache"][at][0, 0] = -float(j % 2)
    eps = torch.finfo(dtype).eps
    want, size, big = oracle.attention(f64(c["q"]), f64(c["k_cache"]), f64(c["v_cache"]), c["table"].tolist(), [n], [0, 1], 0, 0, 1.0)
    score = big * (D * 2.0 ** -24 + 2.0 ** -22)
    tol = eps / 2 * np.abs(want) + ((eps / 2) ** 2 + 2 * score + 2.0 ** -20) * size
    for max_kv in (1, 10000):
        d = np.abs(f64(sb.paged_attention(**c, max_q=1, max_kv=max_kv, scale=1.0)) - want)
        assert np.all(d <= tol), np.max(d / tol)


@pytest.mark.parametrize("max_q", [1, 1000])
def test_attention_strides(gpu, max_q):
    """q a slice of a wider projection, caches with heads before tokens in one
    allocation, a table that is part of a wider one, out into a slice."""
    c = attention_case(3, 6, 2, 64, 8, [4, 1, 2], [20, 33, 2], F16, 11)
    want = sb.paged_attention(**c, max_q=max_q, max_kv=kv_bound(max_q, 33), window=9, sinks=1)
    T, P = c["q"].shape[0], c["k_cache"].shape[0]
    wide = torch.randn(T, 10, 64, device="cuda").half()
    wide[:, 2:8] = c["q"]
    pool = torch.empty(P, 2, 2, 8, 64, dtype=F16, device="cuda")
    pool[:, 0], pool[:, 1] = c["k_cache"].transpose(1, 2), c["v_cache"].transpose(1, 2)
    tab = torch.full((3, c["table"].shape[1] + 5), -1, dtype=torch.int32, device="cuda")
    tab[:, :-5] = c["table"]
    out = torch.zeros(6, T, 72, dtype=F16, device="cuda")
    got = sb.paged_attention(wide[:, 2:8], pool[:, 0].transpose(1, 2), pool[:, 1].transpose(1, 2), tab[:, :-5], c["lens"], c["q_start"],
                             max_q=max_q, max_kv=kv_bound(max_q, 33), window=9, sinks=1, out=out[:, :, :64].transpose(0, 1))
    assert torch.equal(got, want) and bool((out[:, :, 64:] == 0).all())


def test_attention_offsets_beyond_32_bits(gpu):
    """A cache of 5 GB, the request's pages at its end."""
    page, Hkv, D = 64, 8, 128
    n_pages = (5 << 30) // (page * Hkv * D * 2)
    k, v = (torch.zeros(n_pages, page, Hkv, D, dtype=BF16, device="cuda") for _ in range(2))
    c = attention_case(1, 16, Hkv, D, page, [1], [150], BF16, 12)
    for max_q in (1, 1000):
        want = sb.paged_attention(**c, max_q=max_q, max_kv=kv_bound(max_q, 150))
        tail = n_pages - c["k_cache"].shape[0]
        k[tail:], v[tail:] = c["k_cache"], c["v_cache"]
        got = sb.paged_attention(c["q"], k, v, torch.where(c["table"] >= 0, c["table"] + tail, -1), c["lens"], c["q_start"],
                                 max_q=max_q, max_kv=kv_bound(max_q, 150))
        assert torch.equal(got, want)


# -- sampling ----------------------------------------------------------------------

def check_sample(z, u, T=None, top_k=None, top_p=None, min_p=None, dtype=F32):
    z = dev(z, F32).to(dtype)
    f = lambda x: None if x is None else dev(np.asarray(x, np.float32))   # noqa: E731
    tok, lp = sb.sample_tokens(z, f(u), temperature=f(T), top_k=None if top_k is None else i32(top_k), top_p=f(top_p), min_p=f(min_p))
    zz = f64(z)
    for r in range(len(zz)):
        val = lambda x, d: d if x is None else np.float32(x[r])   # noqa: E731
        want = oracle.sample(zz[r], np.float64(np.float32(u[r])), float(val(T, 1.0)), 0 if top_k is None else int(top_k[r]),
                             float(val(top_p, 1.0)), float(val(min_p, 0.0)))
        assert int(tok[r]) == want[0], (r, int(tok[r]), want)
        assert float(lp[r]) == pytest.approx(want[1], rel=2.0 ** -22, abs=2.0 ** -36), r
    return tok, lp


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("V", [1, 2, 3, 63, 64, 65, 255, 1000, 1023, 1025, 4097, 32000, 50001])
def test_sample(gpu, V, dtype):
    r = rng(V)
    rows = 24 if V < 2000 else 12
    z = r.standard_normal((rows, V)) * 2.5
    z[np.arange(rows)[:, None], r.integers(0, V, (rows, 5))] += 6 * r.random((rows, 5))
    u, T = r.random(rows), 0.5 + r.random(rows)
    T[3::8] = 0
    k = np.where(np.arange(rows) % 3 == 0, 0, np.exp(r.random(rows) * math.log(max(V, 2))).astype(int))
    p, mp = np.where(np.arange(rows) % 4 == 1, 1.0, 0.5 + 0.5 * r.random(rows)), np.where(np.arange(rows) % 2, 0.0, 0.2 * r.random(rows))
    check_sample(z, u, dtype=dtype)
    check_sample(z, u, T, dtype=dtype)
    check_sample(z, u, T, top_k=k, dtype=dtype)
    check_sample(z, u, T, top_p=p, dtype=dtype)
    check_sample(z, u, None, min_p=mp, dtype=dtype)
    check_sample(z, u, T, k, p, mp, dtype)


@pytest.mark.parametrize("V", [7, 3000])
def test_sample_ties(gpu, V):
    """Equal logits: the lowest indexes are kept, and every border of the draw
    is exact."""
    for z in (np.zeros(V), np.r_[np.zeros(V // 2), np.ones(V - V // 2)], np.tile([1.0, -1.0, 1.0], V)[:V]):
        z = np.tile(z, (16, 1))
        u = np.r_[np.arange(8) / 8, 1 - 2.0 ** -24, 1.0, 0.5, 2.0 ** -24, np.nan, -1.0, 2.0, 0.25]
        check_sample(z, u)
        check_sample(z, u, top_k=np.arange(16) * V // 14)
        check_sample(z, u, top_p=np.arange(16) / 14)
        check_sample(z, u, top_k=np.full(16, V // 2 + 1), top_p=np.arange(16) / 14)
        check_sample(z, u, T=np.full(16, math.log2(math.e)), min_p=np.arange(16) / 14)


@pytest.mark.parametrize("dtype,V", [(F32, 3000), (BF16, 3000), (F32, 9000), (F16, 40000)])
def test_sample_kept_numbers(gpu, dtype, V):
    """top-k around the sizes at which lists are handled another way, without and
    with equal logits across the cut."""
    k = [1, 23, 24, 25, 64, 127, 128, 129, 255, 256, 257, 400, 511, 512, 513, 700]
    r = rng(V)
    z = 2 * r.standard_normal((16, V))
    u = r.random(16)
    for x in (z, np.round(2 * z) / 2):
        check_sample(x, u, top_k=k, dtype=dtype)
        check_sample(x, u, T=np.full(16, 1.5), top_k=k, top_p=np.linspace(0.2, 1, 16), dtype=dtype)
        check_sample(x, u, T=np.linspace(0.3, 3, 16), min_p=np.geomspace(1, 1e-3, 16), dtype=dtype)


def test_sample_captured_with_a_workspace(gpu):
    """Many wide rows captured once; replayed with other logits and filters."""
    r = rng(21)
    rows, V = 40, 50021
    z, u, top_p = (torch.zeros(s, device="cuda") for s in ((rows, V), (rows,), (rows,)))
    top_k = i32([0] * rows)
    graph = torch.cuda.CUDAGraph()
    sb.sample_tokens(z, u, top_k=top_k, top_p=top_p)
    with torch.cuda.graph(graph):
        tok, lp = sb.sample_tokens(z, u, top_k=top_k, top_p=top_p)
    for t in range(6):
        z.copy_(torch.as_tensor(r.standard_normal((rows, V)) * (1 + t)))
        u.copy_(torch.as_tensor(r.random(rows)))
        top_p.copy_(torch.as_tensor(r.random(rows)))
        top_k.copy_(torch.as_tensor(np.where(np.arange(rows) % (t + 2), 0, 40)))
        graph.replay()
        want = sb.sample_tokens(z, u, top_k=top_k, top_p=top_p)
        assert torch.equal(tok, want[0]) and torch.equal(lp, want[1]), t
        torch.cuda.synchronize()


def test_sample_flat_and_wide(gpu):
    """Cuts that keep very many tokens."""
    r = rng(4)
    z = np.concatenate([0.01 * r.standard_normal((6, 20000)), r.standard_normal((6, 20000))])
    u = r.random(12)
    check_sample(z, u, top_p=np.linspace(0.1, 0.999, 12))
    check_sample(z, u, top_k=np.linspace(2, 19999, 12).astype(int))
    check_sample(z, u, top_k=np.linspace(500, 19999, 12).astype(int), top_p=np.linspace(0.999, 0.3, 12), min_p=np.full(12, 0.01))
    check_sample(z, u, T=np.full(12, 100.0))


@pytest.mark.parametrize("dtype,V", [(F32, 16385), (F32, 40003), (F32, 50001), (BF16, 50000), (F16, 131072), (BF16, 262144),
                                     (F32, 262144)])
def test_sample_rows_by_kernels_of_their_own(gpu, dtype, V, monkeypatch):
    """Many wide rows, for whose passes the call brings a workspace: as the
    oracle says (some rows), and every row as without it."""
    r = rng(V)
    rows = 36
    z = r.standard_normal((rows, V)) * r.choice([0.01, 0.5, 1.0, 2.5, 6.0], (rows, 1))
    z[np.arange(rows)[:, None], r.integers(0, V, (rows, 9))] += 12 * r.random((rows, 9))
    z[5] = 1.0                                       # all equal
    z[6] = np.where(np.arange(V) % 3, -1.0, 2.0)     # two values
    z[7] = -np.inf
    z[8, 1:] = -np.inf
    z[9] = np.where(np.arange(V) % 7 == 0, z[9], -np.inf)
    z[10, [3, V - 1]] = np.inf
    z[11, ::2] = np.nan
    z[13] = np.where(np.arange(V) < 5000, 2.0 + 1e-4 * r.random(V), -1.0)   # more in one place than a list takes
    u, T = r.random(rows), 0.4 + r.random(rows)
    u[:4] = 0.0, 1.0, 0.5, 1 - 2.0 ** -24
    T[12::9] = 0
    k = np.where(np.arange(rows) % 4 == 0, np.exp(r.random(rows) * math.log(V)).astype(int), 0)
    p, mp = np.where(np.arange(rows) % 6 == 1, 1.0, 0.3 + 0.7 * r.random(rows)), np.where(np.arange(rows) % 3, 0.0, 0.1 * r.random(rows))
    f = lambda x: dev(np.asarray(x, np.float32))   # noqa: E731
    zd = dev(z, F32).to(dtype)
    kw = dict(u=f(u), temperature=f(T), top_k=i32(k), top_p=f(p), min_p=f(mp))
    for leave in ((), ("top_k",), ("top_k", "top_p"), ("top_k", "min_p"), ("top_k", "top_p", "min_p", "temperature")):
        left = {n: x for n, x in kw.items() if n not in leave}
        tok, lp = sb.sample_tokens(zd, **left)
        for a in range(0, rows, 9):
            with monkeypatch.context() as m:
                m.setattr(sb.decoder.N.lib(), "sb_sample_workspace", lambda args: 0)
                t, q = sb.sample_tokens(zd[a:a + 9], **{n: x[a:a + 9].clone() for n, x in left.items()})
            assert torch.equal(t, tok[a:a + 9]) and torch.equal(q, lp[a:a + 9]), (leave, a)
        if V < 60000:
            for j in range(0, rows, 5):
                want = oracle.sample(f64(zd[j]), float(np.float32(u[j])), float(np.float32(T[j])) if "temperature" in left else 1.0,
                                     int(k[j]) if "top_k" in left else 0, float(np.float32(p[j])) if "top_p" in left else 1.0,
                                     float(np.float32(mp[j])) if "min_p" in left else 0.0)
                assert int(tok[j]) == want[0], (leave, j)
                one = sb.sample_tokens(zd[j:j + 1], **{n: x[j:j + 1].clone() for n, x in left.items()})
                assert int(one[0]) == want[0] and float(one[1]) == float(lp[j])
                assert float(lp[j]) == pytest.approx(want[1], rel=2.0 ** -22, abs=2.0 ** -36)


@pytest.mark.parametrize("dtype,V", [(F32, 49153), (BF16, 49153), (F32, 49159), (F16, 49159), (BF16, 65537)])
def test_sample_last_chunk_of_a_wide_row(gpu, dtype, V, monkeypatch):
    """Rows just long enough for a workspace, the last chunk of 1 or 7 tokens (less
    than 16 bytes): as the oracle says, and as without a workspace."""
    r = rng(V)
    rows = 20
    z = 2 * r.standard_normal((rows, V))
    z[1, -1] = 30.0                                   # the largest last
    z[2, -1] = -np.inf
    z[3] = 1.0                                        # cuts among equals up to the last
    z[4], z[4, -1] = -40.0, 0.0                       # alone
    z[5, -7:] = z[5].max() + 1.0                      # equals at the end
    z[6, :-1] = np.minimum(z[6, :-1], 3.0)
    z[6, -1] = 3.0                                    # equal to the largest of the others
    z[7, -1] = np.nan
    z[8, -1] = np.inf
    u, T = r.random(rows), 0.5 + r.random(rows)
    u[[3, 4, 5, 6, 9]] = 1.0, 0.5, 1.0, 1 - 2.0 ** -24, 1.0
    p, mp = np.where(np.arange(rows) % 5 == 4, 1.0, 0.5 + 0.5 * r.random(rows)), np.where(np.arange(rows) % 3, 0.0, 0.05 * r.random(rows))
    p[[3, 6]] = 0.9999, 0.999
    f = lambda x: dev(np.asarray(x, np.float32))   # noqa: E731
    zd, L = dev(z, F32).to(dtype), sb.decoder.N.lib()
    zz, need = f64(zd), L.sb_sample_workspace
    for kw in (dict(temperature=f(T), top_p=f(p), min_p=f(mp)), dict(temperature=f(T)), dict(top_p=f(p))):
        asked = []
        with monkeypatch.context() as m:
            m.setattr(L, "sb_sample_workspace", lambda args: asked.append(need(args)) or asked[-1])
            tok, lp = sb.sample_tokens(zd, f(u), **kw)
            assert asked[0] > 0
            m.setattr(L, "sb_sample_workspace", lambda args: 0)
            alone = sb.sample_tokens(zd, f(u), **kw)
        assert torch.equal(tok, alone[0]) and torch.equal(lp, alone[1])
        for j in range(rows):
            at = lambda n, d: float(kw[n][j]) if n in kw else d   # noqa: E731
            want = oracle.sample(zz[j], float(np.float32(u[j])), at("temperature", 1.0), 0, at("top_p", 1.0), at("min_p", 0.0))
            assert int(tok[j]) == want[0] and float(lp[j]) == pytest.approx(want[1], rel=2.0 ** -22, abs=2.0 ** -36), j


def test_sample_odd_values(gpu):
    """-inf, NaN, +inf, the largest and smallest numbers, -0; parameters out of
    their range."""
    inf, nan, big = math.inf, math.nan, 3.0e38
    rows = [[-inf, 0, nan, 1, -inf], [nan] * 5, [-inf] * 5, [inf, 0, inf, 1, nan], [big, -big, big, 0, 1], [-big, -big, -inf, -big, nan],
            [-0.0, 0.0, -0.0, 0.0, -inf], [1e-40, 0, -1e-40, 0, 0]]
    n = len(rows)
    for u in (0.0, 0.3, 0.7, 1.0):
        U = [u] * n
        check_sample(rows, U)
        check_sample(rows, U, T=[0.0] * n)
        check_sample(rows, U, T=[nan] * n)
        check_sample(rows, U, T=[-1.0] * n)
        check_sample(rows, U, T=[1e-30] * n)
        check_sample(rows, U, T=[1e30] * n, top_k=[3] * n)
        check_sample(rows, U, top_k=[2] * n, top_p=[0.4] * n, min_p=[0.1] * n)
        check_sample(rows, U, top_k=[-3] * n, top_p=[nan] * n, min_p=[nan] * n)
        check_sample(rows, U, top_k=[2 ** 31 - 1] * n, top_p=[inf] * n, min_p=[inf] * n)
        check_sample(rows, U, top_k=[1] * n, top_p=[-1.0] * n, min_p=[-1.0] * n)
    tok, lp = sb.sample_tokens(dev(np.zeros((1, 4)), F32), dev(np.float32([0.6])), temperature=dev(np.float32([inf])))
    assert int(tok) == 2


@pytest.mark.parametrize("V", [40, 3000, 40000])
def test_sample_weights_of_one_step(gpu, V):
    """Weights around 2^-44 of the largest, which is one: min-p goes by the rounded
    ones. With u = 1 the last kept token is drawn."""
    steps = [2.6, 2.3, 1.55, 1.45, 1.2, 0.95, 0.7, 0.55, 0.45]     # their weights in steps: the last kept is the least
    rows, mins = [], []
    for T in (1.0, 0.5, 3.0):
        for top in (0.0, 21.5, -3.25):
            for mp in (2.0 ** -60, 2.0 ** -45, 2.0 ** -44, 1.4 * 2.0 ** -44, 2.0 ** -43, 2.6 * 2.0 ** -44):
                z = np.full(V, -np.inf)
                z[V // 3] = top
                z[V // 2:V // 2 + len(steps)] = top + T * np.log(np.array(steps) * 2.0 ** -44)
                rows.append((z, T))
                mins.append(mp)
    check_sample([z for z, _ in rows], [1.0] * len(rows), T=[T for _, T in rows], min_p=mins)
    check_sample([z for z, _ in rows], [1.0] * len(rows), T=[T for _, T in rows], min_p=mins, top_k=[7] * len(rows))


def test_sample_views(gpu):
    """Rows of a wider array, at addresses of no alignment, and out tensors."""
    r = rng(6)
    for dtype in (F32, BF16):
        wide = dev(r.standard_normal((5, 3011)), dtype)
        z, u = wide[:, 5:3006], dev(r.random(5).astype(np.float32))
        p = dev(np.full(5, 0.9, np.float32))
        want = sb.sample_tokens(z.contiguous(), u, top_p=p)
        out = torch.full((7,), -9, dtype=torch.int32, device="cuda")[1:6], torch.zeros(5, device="cuda")
        got = sb.sample_tokens(z, u, top_p=p, out=out)
        assert got[0] is out[0] and torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        assert sb.sample_tokens(z[:0], u[:0])[0].shape == (0,)


def test_sample_frequencies(gpu):
    """Draws over a grid of numbers come as often as the weights say."""
    z = dev(np.log([[0.1, 0.2, 0.3, 0.4]]), F32).expand(4096, 4).contiguous()
    u = (torch.arange(4096, device="cuda") / 4096).float()
    assert torch.bincount(sb.sample_tokens(z, u)[0]).tolist() == [410, 819, 1229, 1638]


# -- together ----------------------------------------------------------------------

class Layer:
    """A toy cached decoder of one layer, tokens to logits, on torch products."""

    def __init__(self, seed, V=500, H=256, Hq=8, Hkv=2, D=64):
        g = torch.Generator(device="cuda").manual_seed(seed)
        make = lambda *s: (torch.randn(*s, generator=g, device="cuda") / math.sqrt(s[0])).to(BF16)   # noqa: E731
        self.E, self.qkv, self.o, self.out = make(V, H) * 20, make(H, (Hq + 2 * Hkv) * D), make(Hq * D, H), make(H, V) * 4
        self.Hq, self.Hkv, self.D = Hq, Hkv, D
        self.inv_freq, self.mscale = sb.rope_frequencies(D, scaling="parts", factor=4.0, original_length=64)

    def step(self, tokens, plan, cache, table, **kw):
        x = self.E[tokens]
        qkv = (x @ self.qkv).view(len(tokens), -1, self.D)
        q, k, v = qkv.split([self.Hq, self.Hkv, self.Hkv], 1)
        q = sb.rope_append(q, k, v, plan.positions, plan.slots, *cache, self.inv_freq, mscale=self.mscale)
        a = sb.paged_attention(q, *cache, table, plan.lens, plan.q_start, **kw)
        return (x + a.reshape(len(tokens), -1) @ self.o) @ self.out


def fresh(n_pages, page, layer, B, width, cap):
    cache = [torch.full((n_pages, page, layer.Hkv, layer.D), math.nan, dtype=BF16, device="cuda") for _ in range(2)]
    zero = torch.zeros(B, dtype=torch.int32, device="cuda")
    plan = sb.PagePlan(i32([0] * (B + 1)), zero.clone(), zero.clone(), torch.zeros(cap, dtype=torch.int64, device="cuda"),
                       torch.zeros(cap, dtype=torch.int32, device="cuda"), i32([n_pages]))
    return cache, i32(np.arange(n_pages)), torch.full((B, width), -1, dtype=torch.int32, device="cuda"), plan


@pytest.mark.parametrize("window,sinks", [(0, 0), (24, 3)])
def test_a_run_of_them_together(gpu, window, sinks):
    """Prompts in one step and token by token: caches, attention and draws of a
    batch with a released and reused request follow each request alone."""
    layer, page, width = Layer(1), 8, 16
    r = rng(2)
    prompts = [r.integers(0, 500, n).tolist() for n in (37, 1, 20)]
    kw = dict(max_kv=width * page, window=window, sinks=sinks)

    def generate(prompt, n, us):
        """One request alone, its whole text given anew at each step."""
        text, got = list(prompt), []
        for t in range(n):
            cache, free, table, plan = fresh(width, page, layer, 1, width, len(text))
            plan = sb.plan_pages(plan.lens, i32([len(text)]), free, plan.n_free, table, page_size=page, token_cap=len(text))
            logits = layer.step(torch.tensor(text).cuda(), plan, cache, table, max_q=len(text), **kw)
            tok = sb.sample_tokens(logits[-1:].float(), dev(np.float32(us[t:t + 1])), top_p=dev(np.float32([0.8])))[0]
            got.append((int(tok), logits[-1].float()))
            text.append(int(tok))
        return got

    us = [np.float32(r.random(12)) for _ in range(3)]
    alone = [generate(p, 12 if b != 1 else 6, us[b]) for b, p in enumerate(prompts)]
    cache, free, table, plan = fresh(40, page, layer, 3, width, 64)
    add = i32([len(p) for p in prompts])
    tokens = torch.tensor(sum(prompts, []) + [0] * (64 - sum(map(len, prompts)))).cuda()
    max_q, top_p = 37, dev(np.full(3, 0.8, np.float32))
    used = []
    for t in range(12):
        plan = sb.plan_pages(plan.lens, add, free, plan.n_free, table, page_size=page, token_cap=64, out=plan)
        used.append(40 - int(plan.n_free))
        logits = layer.step(tokens, plan, cache, table, max_q=max_q, **kw)
        last = logits[(plan.q_start[1:].long() - 1).clamp(min=0)].float()
        drawn = sb.sample_tokens(last, dev(np.array([x[t] for x in us], np.float32)), top_p=top_p)[0]
        live = [0, 1, 2] if t < 6 else [0, 2]
        for b in live:
            # (the logits' products round in another order for other batches: the tokens follow the given ones)
            assert torch.allclose(last[b], alone[b][t][1], atol=0.05 * float(alone[b][t][1].abs().max())), (t, b)
        # Each request's next token, in order; request 1 ends after its sixth.
        nxt = [alone[b][t][0] for b in live if not (b == 1 and t == 5)]
        assert drawn.shape == (3,)
        add = i32([1, 1, 1]) if t < 5 else i32([1, -1 if t == 5 else 0, 1])
        tokens = torch.tensor(nxt + [0] * (64 - len(nxt))).cuda()
        max_q = 1
    assert used[6] < used[5] or used[6] <= used[5] + 1   # request 1's pages came back
    assert plan.lens.tolist() == [37 + 11, 0, 20 + 11]


@pytest.mark.parametrize("window,sinks", [(0, 0), (24, 3)])
def test_a_batch_goes_by_its_own_draws(gpu, window, sinks):
    """Every token drawn is the oracle's for that row's logits, and the next step's
    input; at every step each page is in one live request's row or on the free
    list; a released request's row and pages serve the next one."""
    layer, page, width, n_pages, cap = Layer(3), 8, 16, 40, 64
    r = rng(4)
    cache, free, table, plan = fresh(n_pages, page, layer, 3, width, cap)
    top_p, T = dev(np.full(3, 0.8, np.float32)), dev(np.full(3, 1.1, np.float32))
    lens, add, new = [0, 0, 0], [37, 1, 20], [r.integers(0, 500, n).tolist() for n in (37, 1, 20)]
    for t in range(14):
        tokens = torch.tensor(sum(new, []) + [0] * (cap - sum(map(len, new)))).cuda()
        plan = sb.plan_pages(plan.lens, i32(add), free, plan.n_free, table, page_size=page, token_cap=cap, out=plan)
        lens = [0 if n < 0 else x + n for x, n in zip(lens, add)]
        held = [-(-x // page) for x in lens]
        assert plan.lens.tolist() == lens and int(plan.n_free) == n_pages - sum(held), t
        ids = free[:int(plan.n_free)].tolist() + sum((table[b, :n].tolist() for b, n in enumerate(held)), [])
        assert sorted(ids) == list(range(n_pages)), t
        logits = layer.step(tokens, plan, cache, table, max_q=max(add), max_kv=width * page, window=window, sinks=sinks)
        live = [b for b in range(3) if add[b] > 0]
        last = logits[(plan.q_start[1:].long() - 1).clamp(min=0)].float()
        u = r.random(3).astype(np.float32)
        drawn = sb.sample_tokens(last, dev(u), temperature=T, top_p=top_p)[0]
        z = f64(last)
        assert np.isfinite(z[live]).all()
        for b in live:
            assert int(drawn[b]) == oracle.sample(z[b], float(u[b]), float(np.float32(1.1)), 0, float(np.float32(0.8)))[0], (t, b)
        # Request 1 ends after its sixth token; its row stands idle for a step and
        # then takes a prompt of 12.
        add = [1, -1 if t == 5 else 0 if t == 6 else 12 if t == 7 else 1, 1]
        new = [[int(drawn[b])] if add[b] == 1 else r.integers(0, 500, max(add[b], 0)).tolist() for b in range(3)]


def test_captured_steps(gpu):
    """A whole step captured once and replayed, with eager work between: as the
    same steps taken eagerly. Two graphs live at once, each with its workspace."""
    page, width, B = 8, 40, 4
    graphs = []
    for seed in (1, 2):
        layer = Layer(seed)
        state = fresh(100, page, layer, B, width, B)
        shadow = fresh(100, page, layer, B, width, B)
        tokens, u = torch.full((B,), 3 * seed, device="cuda"), torch.zeros(B, device="cuda")
        add = i32([1] * B)
        par = dict(temperature=dev(np.full(B, 0.9, np.float32)), top_k=i32([50] * B), min_p=dev(np.full(B, 0.02, np.float32)))

        def step(state, tokens, u, layer=layer, add=add, par=par):
            cache, free, table, plan = state
            sb.plan_pages(plan.lens, add, free, plan.n_free, table, page_size=page, token_cap=B, out=plan)
            logits = layer.step(tokens, plan, cache, table, max_q=1, max_kv=width * page, window=30, sinks=2)
            new, lp = sb.sample_tokens(logits, u, **par)
            return new.long(), lp

        want_tokens = tokens.clone()
        stream = torch.cuda.Stream()
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream):   # warm-up of torch's own products, on a state of its own
            step(fresh(100, page, layer, B, width, B), tokens, u)
        torch.cuda.current_stream().wait_stream(stream)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            new, lp = step(state, tokens, u)
            tokens.copy_(new)
        graphs.append([graph, state, shadow, tokens, u, lp, want_tokens, step])
    r = rng(5)
    for t in range(40):
        for x in graphs:
            u = torch.as_tensor(r.random(B).astype(np.float32)).cuda()
            x[4].copy_(u)
            x[0].replay()
            new, lp = x[7](x[2], x[6], u)
            x[6] = new
            assert torch.equal(x[3], new) and torch.equal(x[5], lp), t
            assert torch.equal(x[1][3].lens, x[2][3].lens) and torch.equal(x[1][2], x[2][2])
            torch.cuda.synchronize()


def test_other_streams(gpu):
    """Work enqueued on the current stream of the caller, behind what it waits
    for there."""
    c = attention_case(2, 8, 2, 128, 16, [1], [3000, 40], BF16, 13)
    want = sb.paged_attention(**c, **bounds(c))
    stream = torch.cuda.Stream()
    q = torch.zeros_like(c["q"])
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        big = torch.randn(4096, 4096, device="cuda")
        for _ in range(10):
            big = big @ big * 0.01
        q.copy_(c["q"])
        got = sb.paged_attention(**dict(c, q=q), **bounds(c))
    stream.synchronize()
    assert torch.equal(got, want)


def test_python_refusals(gpu):
    c = attention_case(2, 4, 2, 64, 16, [1], [30, 40], BF16, 1)
    kw = bounds(c)
    for name, bad in (("q", c["q"].float()), ("q", c["q"].cpu()), ("q", c["q"].transpose(1, 2)), ("k_cache", c["k_cache"].half()),
                      ("v_cache", c["v_cache"][:-1]), ("table", c["table"].long()), ("lens", c["lens"][:1]), ("q_start", c["q_start"].cpu()),
                      ("q", c["q"][0])):
        with pytest.raises(ValueError):
            sb.paged_attention(**dict(c, **{name: bad}), **kw)
    with pytest.raises(ValueError, match="overlap"):
        sb.paged_attention(**c, **kw, out=c["q"][:1].expand(2, 4, 64))
    with pytest.raises(ValueError, match="backward"):
        sb.paged_attention(**dict(c, q=c["q"].clone().requires_grad_()), **kw)
    with pytest.raises(ValueError, match="argument"):
        sb.paged_attention(**c, **dict(kw, max_kv=2 ** 31))
    for over in (dict(window=-1), dict(max_kv=-1), dict(scale=math.nan)):
        with pytest.raises(sb.decoder.N.StreambeamError):
            sb.paged_attention(**c, **dict(kw, **over))
    odd = torch.zeros(2, 4, 68, dtype=BF16, device="cuda")[:, :, 2:66]   # rows at addresses of 4 bytes
    with pytest.raises(sb.decoder.N.StreambeamError, match="16-byte|multiple of 8"):
        sb.paged_attention(**dict(c, q=odd), **kw)
    r = rope_case(3, 4, 2, 64, 32, BF16, 1)
    for name, bad in (("k", r["k"][:2]), ("v", r["v"][:, :1]), ("positions", r["positions"].long()), ("slots", r["slots"].int()),
                      ("inv_freq", r["inv_freq"].float()), ("k_cache", r["k_cache"][:1].expand(5, 16, 2, 64)), ("q", r["q"].half())):
        with pytest.raises(ValueError):
            sb.rope_append(**dict(r, **{name: bad}))
    with pytest.raises(ValueError, match="layout"):
        sb.rope_append(**r, layout="both")
    z, u = torch.zeros(3, 10, device="cuda"), torch.zeros(3, device="cuda")
    for bad in (dict(top_k=u), dict(top_p=u[:2]), dict(temperature=u.double()), dict(min_p=u.cpu())):
        with pytest.raises(ValueError):
            sb.sample_tokens(z, u, **bad)
    with pytest.raises(ValueError):
        sb.sample_tokens(z.double(), u)
    with pytest.raises(sb.decoder.N.StreambeamError):
        sb.sample_tokens(torch.zeros(1, 262145, device="cuda"), u[:1])
    with pytest.raises(ValueError, match="token_cap"):
        sb.plan_pages(i32([1]), i32([1]), i32([1]), i32([1]), i32([[1]]), page_size=4, token_cap=-1)


def test_no_derivative_is_dropped(gpu):
    """Every floating tensor that a call reads or writes is looked at: those that
    require a gradient, and dual ones of forward mode."""
    from torch.autograd import forward_ad
    a, r = attention_case(2, 4, 2, 64, 16, [1], [30, 40], BF16, 1), rope_case(3, 4, 2, 64, 32, BF16, 1)
    a["out"], r["out"] = torch.empty_like(a["q"]), torch.empty_like(r["q"])
    one = lambda: torch.ones(3, device="cuda")   # noqa: E731
    s = dict(logits=torch.zeros(3, 10, device="cuda"), u=0 * one(), temperature=one(), top_p=one(), min_p=0 * one())
    calls = ((lambda **kw: sb.paged_attention(**kw, **bounds(a)), a), (sb.rope_append, r), (sb.sample_tokens, s))
    for call, args in calls:
        call(**args)
        for name, t in args.items():
            if not t.is_floating_point():
                continue
            with pytest.raises(ValueError, match="backward"):
                call(**dict(args, **{name: t.clone().requires_grad_()}))
            with torch.no_grad():
                call(**dict(args, **{name: t.clone().requires_grad_()}))
            with forward_ad.dual_level(), pytest.raises(ValueError, match="forward"):
                call(**dict(args, **{name: forward_ad.make_dual(t, torch.ones_like(t))}))
    with pytest.raises(ValueError, match="backward"):
        sb.sample_tokens(**s, out=(torch.zeros(3, dtype=torch.int32, device="cuda"), one().requires_grad_()))


def test_writes_are_known_to_autograd(gpu):
    """What a call writes counts as written in place: saved for a backward pass
    before, it is found to have changed."""
    r, a = rope_case(3, 4, 2, 64, 32, BF16, 1), attention_case(2, 4, 2, 64, 16, [1], [30, 40], BF16, 1)
    a["out"] = torch.empty_like(a["q"])
    out = torch.zeros(3, dtype=torch.int32, device="cuda"), torch.zeros(3, device="cuda")
    table, fl, n_free = i32([[0, -1]]), i32([1, 2, 3]), i32([3])
    plan = sb.PagePlan(i32([0, 0]), i32([3]), i32([0]), dev(np.zeros(4, np.int64)), i32([0] * 4), n_free)

    def written(call, *tensors):
        before = [t._version for t in tensors]
        call()
        return all(t._version > v for t, v in zip(tensors, before))

    assert written(lambda: sb.rope_append(**r, out=r["q"]), r["q"], r["k_cache"], r["v_cache"])
    assert written(lambda: sb.rope_append(**r), r["k_cache"], r["v_cache"])
    assert written(lambda: sb.paged_attention(**a, **bounds(a)), a["out"])
    assert written(lambda: sb.sample_tokens(torch.zeros(3, 10, device="cuda"), out[1].clone(), out=out), *out)
    assert written(lambda: sb.plan_pages(plan.lens, i32([2]), fl, n_free, table, page_size=4, token_cap=4, out=plan), table, fl, *plan)
    assert written(lambda: sb.plan_pages(plan.lens, i32([2]), fl, n_free, table, page_size=4, token_cap=4), table, fl)
    w = torch.ones(r["q"].shape, device="cuda", requires_grad=True)
    product = (w * r["q"]).sum()
    with torch.no_grad():
        sb.rope_append(**r, out=r["q"])
    with pytest.raises(RuntimeError, match="in-?place"):
        product.backward()
    with torch.inference_mode():   # tensors without a version
        sb.rope_append(**r)
        sb.paged_attention(**dict(a, out=torch.empty_like(a["q"])), **bounds(a))


def test_strides_of_one_place(gpu):
    """One token, head, page or slot cut out of arrays of odd strides."""
    def cut(t):   # the same values, in rows of an odd stride where there is one
        shape, stride = t.shape, [s if n > 1 else s + 13 for n, s in zip(t.shape, t.stride())]
        flat = torch.zeros(t.numel() + 64, dtype=t.dtype, device="cuda")
        got = flat.as_strided(shape, stride)
        got.copy_(t)
        return got

    for Hq, Hkv, page in ((4, 2, 16), (1, 1, 16), (3, 1, 1)):
        a = attention_case(1, Hq, Hkv, 64, page, [1], [1], BF16, 3)
        a["k_cache"], a["v_cache"], a["table"] = a["k_cache"][:1].contiguous(), a["v_cache"][:1].contiguous(), i32([[0]])
        want = sb.paged_attention(**a, max_q=1, max_kv=1)
        odd = dict(a, **{n: cut(a[n]) for n in ("q", "k_cache", "v_cache")})
        for max_q in (1, 1000):
            assert torch.equal(sb.paged_attention(**odd, max_q=max_q, max_kv=1, out=cut(torch.zeros_like(want))), want)
        r = rope_case(1, Hq, Hkv, 64, 32, F16, 2, page)
        r["k_cache"], r["v_cache"], r["slots"] = r["k_cache"][:1].contiguous(), r["v_cache"][:1].contiguous(), dev(np.zeros(1, np.int64))
        odd = dict(r, **{n: cut(r[n]) for n in ("q", "k", "v", "k_cache", "v_cache")})
        assert torch.equal(sb.rope_append(**odd, out=cut(r["q"])), sb.rope_append(**r))
        assert torch.equal(odd["k_cache"], r["k_cache"]) and torch.equal(odd["v_cache"], r["v_cache"])


def test_plan_takes_whole_numbers_only(gpu):
    args = lambda: (i32([1]), i32([1]), i32([1]), i32([1]), i32([[1]]))   # noqa: E731
    for bad in (dict(page_size=4.5, token_cap=2), dict(page_size=4, token_cap=2.5), dict(page_size=2 ** 40, token_cap=2)):
        with pytest.raises(ValueError):
            sb.plan_pages(*args(), **bad)
    assert sb.plan_pages(*args(), page_size=np.int64(4), token_cap=np.int32(2)).granted.tolist() == [1]


def test_refusals_keep_their_status(gpu):
    """The library's own status, of calls that ask for a workspace first, too."""
    N = sb.decoder.N
    a = attention_case(1, 4, 2, 64, 16, [1], [30], BF16, 1)
    cut = dict(a, q=a["q"][..., :40].contiguous(), k_cache=a["k_cache"][..., :40].contiguous(), v_cache=a["v_cache"][..., :40].contiguous())
    wide, u = torch.zeros(1, 262145, device="cuda"), torch.zeros(1, device="cuda")
    for call, status in ((lambda: sb.paged_attention(**cut, **bounds(a)), N.SB_E_UNSUPPORTED),
                         (lambda: sb.paged_attention(**a, **bounds(a), window=-1), N.SB_E_INVALID_ARG),
                         (lambda: sb.sample_tokens(wide, u), N.SB_E_UNSUPPORTED),
                         (lambda: sb.sample_tokens(wide[:, :0], u), N.SB_E_INVALID_ARG)):
        with pytest.raises(N.StreambeamError) as e:
            call()
        assert e.value.status == status
