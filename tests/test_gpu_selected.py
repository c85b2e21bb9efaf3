"""Selected pages on the GPU against their fp64 oracle: bounds and selections
have to be equal (scores are sums of at most 2 D products of 16-bit values, in
fp64, nearly always exact); attention with the tolerances of test_gpu_serving.py:
one rounding of the result (eps / 2) and one of each weight, scores off by D 2^-24
of their sum |q||k| times the scale plus 2^-22 of themselves, weights by twice
that and 2^-20 more."""
import math

import numpy as np
import pytest
import torch

import paper_2010_02164_amd as sb
from oracle import serving as oracle

pytestmark = pytest.mark.gpu
BF16, F16 = torch.bfloat16, torch.float16


def dev(a, dtype=None):
    t = torch.as_tensor(np.ascontiguousarray(a)).cuda()
    return t.to(dtype) if dtype else t


def i32(a):
    return dev(np.asarray(a, np.int32))


def f64(t):
    return t.double().cpu().numpy()


def case(B, Hq, Hkv, D, page, q_lens, kv_lens, dtype, seed, pad=0, whole=False):
    """whole: keys and queries of small whole numbers, whose scores are often equal."""
    r = np.random.default_rng(seed)
    q_lens, kv_lens = np.resize(q_lens, B), np.resize(kv_lens, B)
    held = -(-kv_lens // page)
    n_pages = int(held.sum()) + 2
    table = np.full((B, max(int(held.max()), 1) + 2), -1)
    table[np.arange(table.shape[1]) < held[:, None]] = r.permutation(n_pages)[:held.sum()]
    q_start = np.concatenate([[0], np.cumsum(q_lens)])
    T = int(q_start[-1]) + pad
    normal = (lambda *s: dev(np.round(r.standard_normal(s)), dtype)) if whole else lambda *s: dev(r.standard_normal(s), dtype)
    c = dict(q=normal(T, Hq, D), k_cache=normal(n_pages, page, Hkv, D), v_cache=normal(n_pages, page, Hkv, D), table=i32(table),
             lens=i32(kv_lens), q_start=i32(q_start))
    c["k_cache"] += normal(n_pages, 1, Hkv, D)
    return c


def max_q(c):
    return int((c["q_start"][1:] - c["q_start"][:-1]).max())


def all_bounds(c):
    """Of every key in the cache: a step of all tokens."""
    n, _, Hkv, D = c["k_cache"].shape
    every = i32(np.concatenate([[0], np.cumsum(c["lens"].tolist())]))
    return sb.page_bounds(c["k_cache"], c["table"], c["lens"], every, torch.zeros(n, 2, Hkv, D, dtype=c["k_cache"].dtype, device="cuda"),
                          max_q=int(c["lens"].max()))


def select(c, bounds, top, first, last, **kw):
    page, max_kv = c["k_cache"].shape[1], kw.pop("max_kv", None)
    max_kv = int(c["lens"].max()) if max_kv is None else max_kv
    return sb.select_pages(c["q"], bounds, c["table"], c["lens"], c["q_start"], page_size=page, top=top, first=first, last=last, max_kv=max_kv, **kw)


def check_select(c, bounds, top, first, last, got):
    pages, kept = oracle.select_pages(f64(c["q"]), f64(bounds), c["table"].tolist(), c["lens"].tolist(), c["q_start"].tolist(),
                                      c["k_cache"].shape[1], top, first, last)
    assert got[1].tolist() == kept.tolist()
    wrong = np.argwhere(got[0].cpu().numpy() != pages)
    assert not len(wrong), (wrong[:5], got[0].cpu().numpy()[tuple(wrong[0][:2])], pages[tuple(wrong[0][:2])])


def check_attention(c, pages, kept, got, scale=None):
    D, eps = got.shape[2], torch.finfo(got.dtype).eps
    scale = 1 / math.sqrt(D) if scale is None else scale
    want, size, big = oracle.selected_attention(f64(c["q"]), f64(c["k_cache"]), f64(c["v_cache"]), pages.tolist(), kept.tolist(), scale)
    score = big * abs(scale) * (D * 2.0 ** -24 + 2.0 ** -22)
    tol = eps / 2 * np.abs(want) + (eps / 2 + 2 * score[..., :1] + 2.0 ** -20) * size + torch.finfo(got.dtype).smallest_normal
    rows = kept.cpu().numpy() >= 0
    d = np.abs(f64(got)[rows] - want[rows])
    assert np.all(d <= tol[rows]), (np.argwhere(~(d <= tol[rows]))[:5], np.nanmax(d / tol[rows]))


# -- bounds ------------------------------------------------------------------------

@pytest.mark.parametrize("dtype,D", [(BF16, 128), (F16, 64), (BF16, 256)])
@pytest.mark.parametrize("B,Hkv,page,q,kv", [(1, 1, 16, [1], [1]), (5, 2, 16, [1], [16, 17, 31, 200, 1]), (3, 3, 7, [3, 0, 9], [9, 50, 10]),
                                             (4, 8, 1, [2, 1], [5, 3]), (2, 5, 64, [130, 1], [130, 65]), (300, 1, 24, [1, 2, 0], [24, 25, 0, 60])])
def test_bounds(gpu, B, Hkv, page, q, kv, dtype, D):
    c = case(B, Hkv, Hkv, D, page, np.minimum(np.resize(q, B), np.resize(kv, B)), kv, dtype, B + page)
    n = c["k_cache"].shape[0]
    start = dev(np.random.default_rng(1).standard_normal((n, 2, Hkv, D)), dtype)
    want = oracle.page_bounds(f64(c["k_cache"]), c["table"].tolist(), c["lens"].tolist(), c["q_start"].tolist(), f64(start))
    for hint in (max_q(c), 0, 10 ** 5, 2 ** 31 - 1):
        bounds = start.clone()
        assert sb.page_bounds(c["k_cache"], c["table"], c["lens"], c["q_start"], bounds, max_q=hint) is bounds
        assert np.array_equal(f64(bounds), want)


def test_bounds_grow_with_the_cache(gpu):
    """Step by step as from the start; values that are not finite; what stands
    behind the last token is not looked at."""
    c = case(3, 2, 2, 64, 8, [1], [40, 33, 25], BF16, 3)
    c["k_cache"][int(c["table"][0, 1]), 3, 0, 5] = math.nan
    c["k_cache"][int(c["table"][1, 0]), 2, 1, 7] = math.inf
    c["k_cache"][int(c["table"][1, 4]), 1:] = math.nan   # behind request 1's 33 tokens
    c["k_cache"][int(c["table"][2, 3]), 1:] = -math.inf
    want = all_bounds(c)
    assert int(want.isnan().sum()) == 2 and int(want.isinf().sum()) == 1
    n = c["k_cache"].shape[0]
    grown = torch.zeros_like(want)
    lens = [0, 0, 0]
    for add in ([8, 5, 1], [1, 0, 24], [31, 28, 0]):
        lens = [a + b for a, b in zip(lens, add)]
        sb.page_bounds(c["k_cache"], c["table"], i32(lens), i32(np.concatenate([[0], np.cumsum(add)])), grown, max_q=1)
    assert lens == [40, 33, 25] and torch.equal(grown.nan_to_num(7.0), want.nan_to_num(7.0))
    # Wrong state: no access outside the arrays.
    for over in (dict(lens=i32([2 ** 31 - 1, -5, 3])), dict(table=c["table"] + 10 ** 6), dict(q_start=i32([0, 2 ** 31 - 1, -2 ** 31, 5]))):
        a = dict(c, **over)
        sb.page_bounds(a["k_cache"], a["table"], a["lens"], a["q_start"], torch.zeros_like(want), max_q=1)
    torch.cuda.synchronize()
    # Heads before tokens, in one allocation with the values.
    pool = torch.empty(n, 2, 2, 8, 64, dtype=BF16, device="cuda")
    pool[:, 0] = c["k_cache"].transpose(1, 2)
    got = all_bounds(dict(c, k_cache=pool[:, 0].transpose(1, 2)))
    assert torch.equal(got.nan_to_num(7.0), want.nan_to_num(7.0))


# -- selection -----------------------------------------------------------------------

FORMS = [   # B, Hq, Hkv, page, queries, cached
    (1, 4, 1, 16, [1], [1]), (3, 8, 2, 16, [1], [900, 33, 300]), (2, 5, 5, 7, [3, 1], [150, 70]), (2, 16, 1, 1, [2], [600, 97]),
    (2, 6, 2, 24, [1, 4], [1300, 500]), (3, 4, 2, 8, [20, 3, 33], [500, 40, 333]), (1, 3, 1, 4, [17], [300]), (5, 2, 2, 8, [1, 0, 2, 9, 1], [400, 90, 64, 65, 0]), (1, 40, 4, 4, [3], [3000]),
]


def test_select_is_the_same_by_either_unit(gpu):
    """A prompt's tokens at once (scored by the matrix unit) and one by one."""
    c = case(2, 8, 2, 128, 16, [70, 45], [3000, 2000], BF16, 15)
    bounds = all_bounds(c)
    pages, kept = select(c, bounds, 20, 1, 2)
    for t in range(0, 115, 7):
        b = 0 if t < 70 else 1
        p = (3000 - 70 + t) if b == 0 else (2000 - 45 + t - 70)
        one = sb.select_pages(c["q"][t:t + 1], bounds, c["table"][b:b + 1], i32([p + 1]), i32([0, 1]), page_size=16, top=20, first=1, last=2,
                              max_kv=3000)
        assert torch.equal(one[0][0], pages[t]) and int(one[1]) == int(kept[t])


@pytest.mark.parametrize("dtype,D", [(BF16, 128), (F16, 64), (BF16, 256), (F16, 256)])
@pytest.mark.parametrize("form", range(len(FORMS)))
@pytest.mark.parametrize("whole", [False, True])
def test_select(gpu, form, dtype, D, whole):
    """whole: many equal scores, of which the lower pages count."""
    c = case(*FORMS[form][:3], D, *FORMS[form][3:], dtype, form, pad=form % 3, whole=whole)
    bounds = all_bounds(c)
    for top, first, last in ((4, 1, 2), (1, 0, 1), (0, 2, 3), (17, 0, 1), (30, 5, 1), (300, 1, 1)):
        for max_kv in (int(c["lens"].max()), 0, 10 ** 6):
            check_select(c, bounds, top, first, last, select(c, bounds, top, first, last, max_kv=max_kv))


def test_select_equal_scores(gpu):
    """More equal scores than fit any list: all, or all but some; the cut among
    them; neighbours in fp64."""
    c = case(1, 4, 2, 64, 1, [1], [5000], BF16, 1)
    bounds = torch.zeros(c["k_cache"].shape[0], 2, 2, 64, dtype=BF16, device="cuda")
    for top in (1, 255, 256, 257, 3000, 4997):
        check_select(c, bounds, top, 1, 1, select(c, bounds, top, 1, 1))
    bounds[c["table"][0, ::7].long().clamp(min=0), 1] = 1.0
    bounds[c["table"][0, 3::50].long().clamp(min=0), 0] = -1.0
    for top in (100, 713, 714, 715, 800, 2500):
        check_select(c, bounds, top, 0, 1, select(c, bounds, top, 0, 1))
    c["q"][:] = 0.0
    c["q"][0, :, 0], c["q"][0, :, 1] = 1.0, 2.0 ** -30   # scores 1 + k 2^-38
    bounds.zero_()
    bounds[:, :, :, 0] = 1.0
    bounds[:, :, :, 1] = (torch.arange(bounds.shape[0], device="cuda") % 200 / 256.0)[:, None, None].to(BF16)
    for top in (3, 40, 1000):
        check_select(c, bounds, top, 0, 1, select(c, bounds, top, 0, 1))


@pytest.mark.parametrize("q", [[1, 2], [30, 21]])
def test_select_odd_values(gpu, q):
    """Bounds and queries that are not finite, pages outside the cache, zeros of
    both signs; single tokens, and so many that the matrix unit scores them."""
    c = case(2, 4, 2, 64, 4, q, [400, 200], F16, 2)
    bounds = all_bounds(c)
    row = c["table"][0].tolist()
    bounds[row[20], 1, 0, 3], bounds[row[30], 0, 0], bounds[row[40], 1] = math.nan, -math.inf, math.inf
    bounds[row[50]], bounds[row[51]] = 0.0, -0.0
    c["table"][0, 60], c["table"][0, 61], c["table"][0, 62] = -1, 10 ** 6, -2 ** 31
    c["q"][0, 0, 9] = 0.0
    for top in (1, 2, 3, 5, 50, 95, 97):
        check_select(c, bounds, top, 1, 2, select(c, bounds, top, 1, 2))
    c["q"][0, 1, 5], c["q"][1, 2, 6] = math.nan, math.inf
    for top in (3, 50, 97):
        check_select(c, bounds, top, 1, 2, select(c, bounds, top, 1, 2))
    for over in (dict(lens=i32([2 ** 31 - 1, -5])), dict(q_start=i32([2 ** 31 - 1, -7, 2])), dict(q_start=i32([-2 ** 31, 2 ** 31 - 1, 1]))):
        select(dict(c, **over), bounds, 5, 1, 1, max_kv=400)   # wrong state: no access outside the arrays
    torch.cuda.synchronize()


@pytest.mark.parametrize("q", [[1, 2], [30, 21]])
@pytest.mark.parametrize("dtype", [BF16, F16])
def test_select_pages_outside_the_cache_come_last(gpu, dtype, q):
    """Behind pages that score minus infinity, too, which stand after them in the table."""
    c = case(2, 4, 2, 64, 4, q, [400, 200], dtype, 5)
    c["q"][:, :, 7] = c["q"][:, :, 7].abs() + 1.0
    bounds = all_bounds(c)
    row = c["table"][0].tolist()
    c["table"][0, 10], c["table"][0, 25], c["table"][0, 40] = -1, 10 ** 6, -2 ** 31
    for col in (20, 30, 55, 90):
        bounds[row[col], 1, :, 7] = -math.inf
    for top in (89, 90, 91, 92, 94, 95, 96):   # of 97 between for request 0's last token, 3 of them not there
        got = select(c, bounds, top, 1, 2)
        check_select(c, bounds, top, 1, 2, got)
        last = got[0][int(c["q_start"][1]) - 1]
        assert int(((last < 0) | (last >= 10 ** 6)).sum()) == 2 * max(0, top - 94)


@pytest.mark.parametrize("q", [[2, 5], [9, 31]])
def test_select_starts_behind_the_tokens(gpu, q):
    """A last start behind n_tokens counts as n_tokens, as in paged_attention: the
    request's queries are its last positions."""
    c = case(2, 4, 2, 64, 4, q, [400, 301], BF16, 23)
    bounds = all_bounds(c)
    want = select(c, bounds, 9, 1, 2)
    check_select(c, bounds, 9, 1, 2, want)
    for behind in (1, 6, 400, 2 ** 31 - 1 - sum(q)):
        got = select(dict(c, q_start=i32([0, q[0], sum(q) + behind])), bounds, 9, 1, 2)
        assert all(torch.equal(a, b) for a, b in zip(got, want)), behind


def test_select_some_tokens_at_a_time(gpu):
    """A table so wide that the scores of all tokens do not fit the workspace."""
    c = case(3, 2, 2, 64, 4, [100, 1, 60], [500, 90, 300], BF16, 6, pad=2)
    wide = torch.full((3, 400000), -1, dtype=torch.int32, device="cuda")
    wide[:, :c["table"].shape[1]] = c["table"]
    bounds = all_bounds(c)
    got = select(dict(c, table=wide), bounds, 9, 1, 2)
    check_select(c, bounds, 9, 1, 2, got)


def test_select_longest_row(gpu):
    """A row of as many pages as there may be, 2^31 - 1024 of one key: a grid's step
    behind the last ones passes 2^31. All pages score the same but three, the last of
    them next to the row's end. And with all but 1100 of them the first ones: so do
    the places of threads behind the last."""
    n = 2 ** 31 - 1024
    q = torch.ones(1, 1, 64, dtype=BF16, device="cuda")
    bounds = torch.zeros(2, 2, 1, 64, dtype=BF16, device="cuda")
    bounds[1, 1] = 1.0
    table = torch.zeros(1, n, dtype=torch.int32, device="cuda")
    table[0, 40], table[0, 2 ** 30], table[0, n - 2] = 1, 1, 1
    torch.cuda.synchronize()
    pages, kept = sb.select_pages(q, bounds, table, i32([n]), i32([0, 1]), page_size=1, top=5, first=1, last=1, max_kv=n)
    assert pages.tolist() == [[[0, 0, 0, 1, 1, 1, 0]]] and int(kept) == 7
    first = n - 1101
    table[0, n - 500:n - 480], table[0, 7] = 1, 1
    pages, kept = sb.select_pages(q, bounds, table, i32([n]), i32([0, 1]), page_size=1, top=22, first=first, last=1, max_kv=n)
    assert torch.equal(pages[0, 0, :first], table[0, :first]) and int(kept) == first + 23
    assert pages[0, 0, first:].tolist() == [0] + [1] * 21 + [0]


def test_select_out_and_strides(gpu):
    c = case(2, 4, 2, 64, 8, [2, 1], [300, 200], BF16, 8, pad=2)
    bounds = all_bounds(c)
    want = select(c, bounds, 5, 1, 2)
    check_select(c, bounds, 5, 1, 2, want)
    T = c["q"].shape[0]
    wide = torch.randn(T, 9, 64, device="cuda").to(BF16)
    wide[:, 3:7] = c["q"]
    tab = torch.full((2, c["table"].shape[1] + 5), -1, dtype=torch.int32, device="cuda")
    tab[:, :-5] = c["table"]
    out = torch.full((T, 2, 8), 9, dtype=torch.int32, device="cuda"), torch.full((T,), 9, dtype=torch.int32, device="cuda")
    got = select(dict(c, q=wide[:, 3:7], table=tab[:, :-5]), bounds, 5, 1, 2, out=out)
    assert got[0] is out[0] and got[1] is out[1]
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and got[1][-2:].tolist() == [-1, -1]


def test_refusals(gpu):
    c = case(1, 4, 2, 64, 8, [2], [100], BF16, 8)
    b = all_bounds(c)
    pages, kept = select(c, b, 3, 1, 1)
    for over, match in ((dict(bounds=b.half()), "bounds"), (dict(bounds=b[:, :1]), "bounds"), (dict(bounds=b.transpose(2, 3)), "bounds"),
                        (dict(top=-1), "top"), (dict(last=0), "last"), (dict(top=2.5), "whole"), (dict(lens=c["lens"].long()), "lens"),
                        (dict(out=(pages[:1], kept)), "pages"), (dict(q=c["q"].float()), "bfloat16"),
                        (dict(q=c["q"].clone().requires_grad_()), "backward")):
        kw = dict(q=c["q"], bounds=b, table=c["table"], lens=c["lens"], q_start=c["q_start"], page_size=8, top=3, max_kv=100)
        with pytest.raises(ValueError, match=match):
            sb.select_pages(**dict(kw, **over))
    kw = dict(q=c["q"], k_cache=c["k_cache"], v_cache=c["v_cache"], pages=pages, kept=kept)
    for over, match in ((dict(pages=pages[:, :1]), "pages"), (dict(pages=pages[0]), "pages"), (dict(kept=kept[:1]), "kept"),
                        (dict(q=c["q"].half()), "k_cache"), (dict(v_cache=c["v_cache"][:2]), "one shape"),
                        (dict(out=torch.empty(2, 3, 64, dtype=BF16, device="cuda")), "heads")):
        with pytest.raises(ValueError, match=match):
            sb.selected_attention(**dict(kw, **over))
    for over, match in ((dict(bounds=b[1:]), "pages"), (dict(lens=c["lens"][:0]), "lens"), (dict(k_cache=c["k_cache"][0]), "k_cache")):
        kw = dict(k_cache=c["k_cache"], table=c["table"], lens=c["lens"], q_start=c["q_start"], bounds=b, max_q=2)
        with pytest.raises(ValueError, match=match):
            sb.page_bounds(**dict(kw, **over))


# -- attention -----------------------------------------------------------------------

@pytest.mark.parametrize("dtype,D", [(BF16, 128), (F16, 64), (BF16, 256), (F16, 128)])
@pytest.mark.parametrize("form", range(len(FORMS)))
def test_selected_attention(gpu, form, dtype, D):
    c = case(*FORMS[form][:3], D, *FORMS[form][3:], dtype, form, pad=2)
    bounds = all_bounds(c)
    for top, first, last in ((4, 1, 2), (0, 0, 1), (30, 2, 1), (300, 1, 1)):
        pages, kept = select(c, bounds, top, first, last)
        out = dev(np.full(c["q"].shape, 3.0), dtype)
        assert sb.selected_attention(c["q"], c["k_cache"], c["v_cache"], pages, kept, out=out) is out
        check_attention(c, pages, kept, out)
        assert bool((out[-2:] == 3).all())


@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (32, 1), (40, 2), (17, 1), (64, 64)])
def test_selected_attention_lists_of_any_kind(gpu, Hq, Hkv):
    """Pages in any order, given twice, outside the cache; kept from none to more
    than there are; many heads of a group and of single ones; a scale of its own."""
    r = np.random.default_rng(Hq)
    T, page, n_pages, width, D = 9, 8, 30, 12, 64
    c = {n: dev(r.standard_normal(s), BF16) for n, s in (("q", (T, Hq, D)), ("k_cache", (n_pages, page, Hkv, D)), ("v_cache", (n_pages, page, Hkv, D)))}
    pages = i32(r.integers(-2, n_pages + 2, (T, Hkv, width)))
    pages[3] = -1
    kept = i32([0, 1, 7, 60, -1, 96, 1000, 2 ** 31 - 1, -2 ** 31])
    for scale in (None, -0.3, 0.0):
        out = dev(np.full((T, Hq, D), 3.0), BF16)
        sb.selected_attention(c["q"], c["k_cache"], c["v_cache"], pages, kept, scale=scale, out=out)
        check_attention(c, pages, kept, out, scale)
        assert bool((out[[0, 3]] == 0).all()) and bool((out[[4, 8]] == 3).all())


@pytest.mark.parametrize("dtype", [BF16, F16])
def test_selected_attention_what_is_hidden_does_not_matter(gpu, dtype):
    """NaN and infinities behind the last key and on pages that are not listed; a
    key that is listed makes its token's head not a number, and no other."""
    c = case(2, 4, 2, 64, 16, [1, 2], [500, 300], dtype, 9)
    pages, kept = select(c, all_bounds(c), 5, 1, 2)
    clean = sb.selected_attention(c["q"], c["k_cache"], c["v_cache"], pages, kept)
    used = torch.zeros(*c["k_cache"].shape[:3], dtype=torch.bool, device="cuda")
    for t, n in enumerate(kept.tolist()):
        for h in range(2):
            for j in range(n):
                used[pages[t, h, j // 16], j % 16, h] = True
    for bad in (math.nan, math.inf, -math.inf):
        c["k_cache"][~used] = bad
        c["v_cache"][~used] = bad
        assert torch.equal(sb.selected_attention(c["q"], c["k_cache"], c["v_cache"], pages, kept), clean)
    c["v_cache"][int(pages[0, 1, -1]), 499 % 16, 1] = math.nan
    got = sb.selected_attention(c["q"], c["k_cache"], c["v_cache"], pages, kept)
    assert torch.equal(got[1:], clean[1:]) and torch.equal(got[0, :2], clean[0, :2]) and bool(got[0, 2:].isnan().all())


def test_all_pages_selected_is_paged_attention(gpu):
    c = case(3, 8, 2, 128, 16, [1, 3, 2], [400, 90, 17], BF16, 4)
    want = sb.paged_attention(**c, max_q=3, max_kv=400)
    pages, kept = select(c, all_bounds(c), 30, 1, 1)
    got = sb.selected_attention(c["q"], c["k_cache"], c["v_cache"], pages, kept)
    check_attention(c, pages, kept, got)
    assert torch.allclose(got.float(), want.float(), rtol=2.0 ** -7, atol=2.0 ** -8)


def test_selected_offsets_beyond_32_bits(gpu):
    """A cache of 5 GB and bounds of 4.6, the pages in use at their ends."""
    page, Hkv, D = 1, 8, 256
    n_pages = (5 << 30) // (page * Hkv * D * 2)
    c = case(1, 8, Hkv, D, page, [1], [400], BF16, 12)
    small = all_bounds(c)
    want = select(c, small, 20, 1, 2)
    out = sb.selected_attention(c["q"], c["k_cache"], c["v_cache"], *want)
    tail = n_pages - c["k_cache"].shape[0]
    k, v = (torch.zeros(n_pages, page, Hkv, D, dtype=BF16, device="cuda") for _ in range(2))
    bounds = torch.zeros(n_pages, 2, Hkv, D, dtype=BF16, device="cuda")
    k[tail:], v[tail:] = c["k_cache"], c["v_cache"]
    far = dict(c, k_cache=k, v_cache=v, table=torch.where(c["table"] >= 0, c["table"] + tail, -1))
    sb.page_bounds(k, far["table"], c["lens"], i32([0, 400]), bounds, max_q=400)
    assert torch.equal(bounds[tail:], small)
    pages, kept = select(far, bounds, 20, 1, 2)
    assert torch.equal(pages, torch.where(want[0] >= 0, want[0] + tail, -1)) and torch.equal(kept, want[1])
    assert torch.equal(sb.selected_attention(c["q"], k, v, pages, kept), out)


def test_selected_captured_and_on_other_streams(gpu):
    c = case(3, 8, 2, 128, 16, [1], [6000, 900, 2500], BF16, 21)
    bounds, other = all_bounds(c), torch.randn_like(c["q"])

    def step():
        sb.page_bounds(c["k_cache"], c["table"], c["lens"], c["q_start"], bounds, max_q=1)
        out = []
        for q in (c["q"], other):
            pages, kept = select(dict(c, q=q), bounds, 20, 1, 2, max_kv=6000)
            out += [pages, kept, sb.selected_attention(q, c["k_cache"], c["v_cache"], pages, kept)]
        return out

    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for t in range(4):
        c["q"].copy_(torch.randn_like(c["q"]))
        c["lens"].copy_(i32([6000 - 300 * t, 900 - t, 2500 - 17 * t]))
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(held, step())), t
        torch.cuda.synchronize()
    want = step()
    torch.cuda.synchronize()
    got = []
    for stream in [torch.cuda.Stream() for _ in range(2)]:
        with torch.cuda.stream(stream):
            pages, kept = select(c, bounds, 20, 1, 2, max_kv=6000)
            got.append((pages, kept, sb.selected_attention(c["q"], c["k_cache"], c["v_cache"], pages, kept)))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for run in got for a, b in zip(run, want))
