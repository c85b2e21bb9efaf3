"""Attention over a shared prefix on the GPU against its fp64 oracle.

Tolerances as in test_gpu_serving.py: eps is torch.finfo(type).eps; one rounding
of the result (eps / 2 of it) and one of each weight (eps / 2 of sum w |v|
together); a score is off by at most D 2^-24 of its sum |q||k| times the scale
plus 2^-22 of its own size, a weight by twice that and 2^-20 more from the
exponentials, the sums and the joins."""
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


def case(members, Hq, Hkv, D, page, prefix, q_lens, kv_lens, dtype, seed, pad=0, spread=1.0, alone=0):
    """members: requests of each group; alone: requests behind the last group."""
    r = np.random.default_rng(seed)
    B = sum(members) + alone
    q_lens, kv_lens, prefix = np.resize(q_lens, B), np.resize(kv_lens, B), np.resize(prefix, len(members))
    held, ahead = -(-kv_lens // page), -(-prefix // page)
    n_pages = int(held.sum() + ahead.sum()) + 2
    ids = r.permutation(n_pages)
    ptab = np.full((len(members), max(int(ahead.max()), 1) + 1), -1)
    ptab[np.arange(ptab.shape[1]) < ahead[:, None]] = ids[:ahead.sum()]
    table = np.full((B, max(int(held.max()), 1) + 2), -1)
    table[np.arange(table.shape[1]) < held[:, None]] = ids[ahead.sum():ahead.sum() + held.sum()]
    q_start = np.concatenate([[0], np.cumsum(q_lens)])
    T = int(q_start[-1]) + pad
    return dict(q=dev(spread * r.standard_normal((T, Hq, D)), dtype), k_cache=dev(r.standard_normal((n_pages, page, Hkv, D)), dtype),
                v_cache=dev(r.standard_normal((n_pages, page, Hkv, D)), dtype), prefix_table=i32(ptab), prefix_lens=i32(prefix),
                group_start=i32(np.concatenate([[0], np.cumsum(members)])), table=i32(table), lens=i32(kv_lens), q_start=i32(q_start))


def bounds(c, **over):
    return dict(dict(max_q=int((c["q_start"][1:] - c["q_start"][:-1]).max()), max_kv=int(c["lens"].max()),
                     max_prefix=int(c["prefix_lens"].max())), **over)


HINTS = [{}, dict(max_q=1), dict(max_q=1000), dict(max_kv=10 ** 6), dict(max_prefix=0), dict(max_prefix=10 ** 6), dict(max_q=0, max_kv=0, max_prefix=0),
         dict(max_q=2 ** 31 - 1, max_kv=2 ** 31 - 1, max_prefix=2 ** 31 - 1)]


def check(c, got, scale=None):
    D, eps = got.shape[2], torch.finfo(got.dtype).eps
    scale = 1 / math.sqrt(D) if scale is None else scale
    args = [f64(c[n]) for n in ("q", "k_cache", "v_cache")]
    args += [c[n].tolist() for n in ("prefix_table", "prefix_lens", "group_start", "table", "lens", "q_start")]
    want, size, big = oracle.shared_attention(*args, scale)
    score = big * abs(scale) * (D * 2.0 ** -24 + 2.0 ** -22)
    tol = eps / 2 * np.abs(want) + (eps / 2 + 2 * score[..., :1] + 2.0 ** -20) * size + torch.finfo(got.dtype).smallest_normal
    rows = int(c["q_start"][-1])
    d = np.abs(f64(got)[:rows] - want[:rows])
    assert np.all(d <= tol[:rows]), (np.argwhere(~(d <= tol[:rows]))[:5], np.nanmax(d / tol[:rows]))


FORMS = [   # members, Hq, Hkv, page, prefix, queries, own tokens, alone
    ([1], 4, 1, 16, [1], [1], [1], 0), ([4], 16, 4, 16, [101], [1], [3, 25], 0), ([5, 5, 5], 4, 4, 7, [64, 200, 13], [1], [1, 40, 33, 90], 0),
    ([3, 1, 4], 32, 2, 24, [130, 5, 300], [1, 2], [31, 64, 2], 2), ([20], 8, 4, 32, [500], [3, 1, 4, 2], [7, 90, 65, 5], 1),
    ([2], 40, 2, 1, [50], [2], [40, 97], 0), ([2, 3], 4, 2, 16, [260, 150], [40, 1, 97], [40, 120, 150], 1), ([1, 1], 8, 1, 64, [129, 64], [70], [70], 0),
    ([40, 1], 3, 3, 5, [333, 1], [1], [2, 70], 5), ([2, 2], 6, 2, 16, [32, 96], [16, 3], [16, 32], 0),
]


@pytest.mark.parametrize("dtype,D", [(BF16, 128), (F16, 64), (BF16, 256), (F16, 128)])
@pytest.mark.parametrize("form", range(len(FORMS)))
def test_shared_attention(gpu, form, dtype, D):
    members, Hq, Hkv, page, prefix, q, kv, alone = FORMS[form]
    c = case(members, Hq, Hkv, D, page, prefix, q, kv, dtype, form, alone=alone)
    for over in HINTS:
        check(c, sb.shared_attention(**c, **bounds(c, **over)))


@pytest.mark.parametrize("dtype,D,Hq,Hkv,members,prefix,q,kv", [
    (BF16, 128, 8, 2, [24], [5000], [1], [900, 1, 2]), (F16, 64, 6, 1, [1, 9, 2], [2600, 900, 4000], [1, 3], [3, 1500]),
    (BF16, 256, 4, 2, [6, 2], [3000, 2000], [1, 5], [20]), (F16, 256, 4, 4, [2, 1], [2500, 3], [30, 2], [1300, 40]),
    (BF16, 64, 4, 4, [2], [6000], [1], [3000, 10])])
def test_shared_attention_in_parts(gpu, dtype, D, Hq, Hkv, members, prefix, q, kv):
    """Long prefixes and long tails, split over workgroups; pages that are none;
    rows behind the last request."""
    c = case(members, Hq, Hkv, D, 16, prefix, q, kv, dtype, D + Hq, pad=3, alone=1)
    out = dev(np.full(c["q"].shape, 3.0), dtype)
    assert sb.shared_attention(**c, **bounds(c), out=out) is out
    check(c, out)
    assert bool((out[-3:] == 3).all())
    c["prefix_table"][0, 3], c["prefix_table"][0, 100], c["table"][0, 0] = -1, 10 ** 6, -2 ** 31
    for over in ({}, dict(max_prefix=0, max_kv=0), dict(max_q=1000)):
        check(c, sb.shared_attention(**c, **bounds(c, **over)))


@pytest.mark.parametrize("max_q", [1, 1000])
def test_shared_attention_empty(gpu, max_q):
    """Groups without requests or tokens, requests without queries or own tokens,
    queries before the first own token, rows behind the last request."""
    c = case([2, 0, 3, 1], 4, 2, 64, 8, [20, 9, 0, 33], [0, 2, 1, 0, 5, 1], [9, 2, 0, 0, 3, 0], BF16, 7, pad=4, alone=2)
    for over in ({}, dict(max_kv=5000), dict(max_prefix=5000)):
        out = dev(np.full(c["q"].shape, 3.0), BF16)
        sb.shared_attention(**c, **bounds(c, max_q=max_q, **over), out=out)
        check(c, out)
        assert bool((out[-4:] == 3).all())
        assert bool((out[2] == 0).all()) and bool((out[3:5] == 0).all())   # of no prefix and no tokens; positions -2 and -1 likewise
        out.fill_(3)
        nobody = dict(c, q_start=i32([0] * 9))
        sb.shared_attention(**nobody, **bounds(c, max_q=max_q, **over), out=out)
        assert bool((out == 3).all())
    none = dict(c, group_start=i32([0] * 5))   # no request has a prefix: as over its own tokens alone
    got = sb.shared_attention(**none, **bounds(c, max_q=max_q))
    check(none, got)


@pytest.mark.parametrize("max_q", [1, 1000])
def test_shared_attention_is_paged_attention_without_a_prefix(gpu, max_q):
    """The same up to the rounding of parts' joins; and with whole pages of prefix,
    as one cache of both."""
    c = case([3, 2], 8, 2, 128, 16, [64, 160], [1, 4, 2], [30, 100, 9], BF16, 3)
    own = {n: c[n] for n in ("q", "k_cache", "v_cache", "lens", "q_start")}
    ahead = [4, 4, 4, 10, 10]
    both = np.full((5, 20), -1)
    for b in range(5):
        g = 0 if b < 3 else 1
        both[b, :ahead[b]] = c["prefix_table"][g, :ahead[b]].cpu().numpy()
        both[b, ahead[b]:ahead[b] + c["table"].shape[1]] = c["table"][b].cpu().numpy()
    want = sb.paged_attention(**dict(own, lens=c["lens"] + i32(ahead) * 16), table=i32(both), max_q=max_q, max_kv=300)
    got = sb.shared_attention(**c, **bounds(c, max_q=max_q))
    assert torch.allclose(got.float(), want.float(), rtol=2 * 2.0 ** -8, atol=2.0 ** -8)
    check(c, got)


@pytest.mark.parametrize("dtype", [BF16, F16])
def test_shared_attention_large_scores_and_scales(gpu, dtype):
    """Scores of thousands, the largest in the prefix or behind it; a scale that is
    negative or 0; weights of the prefix's pass and of the own one meet."""
    for spread, members, q in ((40.0, [9, 2], [1]), (40.0, [2, 1], [9, 1])):
        c = case(members, 4, 2, 128, 16, [300, 140], q, [60, 9, 200], dtype, 10, spread=spread)
        for scale in (None, -0.02, 0.0):
            for over in ({}, dict(max_prefix=5000), dict(max_q=1000)):
                check(c, sb.shared_attention(**c, **bounds(c, **over), scale=scale), scale)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("max_q", [1, 1000])
def test_shared_attention_what_is_hidden_does_not_matter(gpu, max_q, dtype):
    """NaN and infinities on pages of nobody, behind the last tokens, and at
    positions that other rows of the tile do see; in a prefix they reach its group
    and nobody else."""
    c = case([3, 2], 4, 1, 64, 16, [50, 77], [6, 1, 3], [20, 33, 6], dtype, 9)
    kw = bounds(c, max_q=max_q)
    clean = sb.shared_attention(**c, **kw)
    check(c, clean)
    used = torch.zeros(c["k_cache"].shape[:2], dtype=torch.bool, device="cuda")
    for table, lens in ((c["table"], c["lens"]), (c["prefix_table"], c["prefix_lens"])):
        for row, n in zip(table.tolist(), lens.tolist()):
            for j in range(n):
                used[row[j // 16], j % 16] = True
    for bad in (math.nan, math.inf, -math.inf):
        c["k_cache"][~used] = bad
        c["v_cache"][~used] = bad
        assert torch.equal(sb.shared_attention(**c, **kw), clean)
    at = int(c["table"][0, 1]), 19 % 16   # request 0's last token, seen by its last query alone
    held = c["k_cache"][at].clone(), c["v_cache"][at].clone()
    c["k_cache"][at], c["v_cache"][at] = 0.0, math.nan
    got = sb.shared_attention(**c, **kw)
    assert torch.equal(got[:5], clean[:5]) and bool(got[5].isnan().all()) and torch.equal(got[6:], clean[6:])
    c["k_cache"][at], c["v_cache"][at] = held
    c["v_cache"][int(c["prefix_table"][1, 4]), 12] = math.nan   # the last token of the second prefix
    got = sb.shared_attention(**c, **kw)
    first = int(c["q_start"][3])
    assert torch.equal(got[:first], clean[:first]) and bool(got[first:].isnan().all())


@pytest.mark.parametrize("max_q", [1, 1000])
def test_shared_attention_wrong_state_stays_in_bounds(gpu, max_q):
    c = case([2, 2], 6, 2, 64, 8, [30, 9], [2, 0, 3, 1], [9, 5, 20, 7], BF16, 16, pad=3)
    T, kw = c["q"].shape[0], bounds(c, max_q=max_q)
    want = sb.shared_attention(**c, **kw)
    for over in (dict(q_start=i32([0, 2, 2, 2 ** 31 - 1, -5])), dict(q_start=i32([-2 ** 31, -1, 2 ** 31 - 1, -2 ** 31, 5])),
                 dict(group_start=i32([-7, 2 ** 31 - 1, -3])), dict(group_start=i32([4, 1, 0])), dict(prefix_lens=i32([2 ** 31 - 1, -4])),
                 dict(lens=i32([2 ** 31 - 1, -9, 0, 10 ** 9])), dict(prefix_table=c["prefix_table"] + 10 ** 6), dict(table=c["table"] - 10 ** 6)):
        got = sb.shared_attention(**dict(c, **over), **kw)
        assert got.shape == (T, 6, 64)
    torch.cuda.synchronize()
    rows = int(c["q_start"][-1])
    assert torch.equal(sb.shared_attention(**c, **kw)[:rows], want[:rows])
    # group_start beyond the requests is cut off there.
    assert torch.equal(sb.shared_attention(**dict(c, group_start=i32([0, 2, 9])), **kw)[:rows], want[:rows])


def test_shared_attention_groups_over_each_other(gpu):
    """Starts that go back: every other group has all requests, 2^25 units where there
    is room for 2^14. Nothing is written outside the result, and the next call is
    right."""
    c = case([2, 2], 6, 2, 64, 8, [30, 9], [2, 0, 3, 1], [9, 5, 20, 7], BF16, 16)
    want = sb.shared_attention(**c, **bounds(c))
    n, groups = 8192, 8192
    q = torch.randn(n, 16, 64, device="cuda").bfloat16()
    cache = torch.randn(4, 16, 1, 64, device="cuda").bfloat16()
    table, prefix_table = torch.zeros(n, 1, dtype=torch.int32, device="cuda"), torch.zeros(groups, 4096, dtype=torch.int32, device="cuda")
    starts = torch.zeros(groups + 1, dtype=torch.int32, device="cuda")
    starts[1::2] = n
    lens, q_start = torch.ones(n, dtype=torch.int32, device="cuda"), torch.arange(n + 1, dtype=torch.int32, device="cuda")
    long = torch.full((groups,), 65536, dtype=torch.int32, device="cuda")
    held = torch.full((n + 64, 16, 64), 3.0, dtype=BF16, device="cuda")
    sb.shared_attention(q, cache, cache, prefix_table, long, starts, table, lens, q_start, max_q=1, max_kv=1, max_prefix=16, out=held[32:-32])
    assert bool((held[:32] == 3).all()) and bool((held[-32:] == 3).all())
    assert torch.equal(sb.shared_attention(**c, **bounds(c)), want)


@pytest.mark.parametrize("max_q", [1, 1000])
def test_shared_attention_strides(gpu, max_q):
    c = case([2, 1], 6, 2, 64, 8, [40, 21], [4, 1, 2], [20, 33, 2], F16, 11)
    kw = bounds(c, max_q=max_q)
    want = sb.shared_attention(**c, **kw)
    T, P = c["q"].shape[0], c["k_cache"].shape[0]
    wide = torch.randn(T, 10, 64, device="cuda").half()
    wide[:, 2:8] = c["q"]
    pool = torch.empty(P, 2, 2, 8, 64, dtype=F16, device="cuda")
    pool[:, 0], pool[:, 1] = c["k_cache"].transpose(1, 2), c["v_cache"].transpose(1, 2)
    tabs = []
    for name in ("table", "prefix_table"):
        tab = torch.full((c[name].shape[0], c[name].shape[1] + 5), -1, dtype=torch.int32, device="cuda")
        tab[:, :-5] = c[name]
        tabs.append(tab[:, :-5])
    out = torch.zeros(6, T, 72, dtype=F16, device="cuda")
    got = sb.shared_attention(**dict(c, q=wide[:, 2:8], k_cache=pool[:, 0].transpose(1, 2), v_cache=pool[:, 1].transpose(1, 2), table=tabs[0],
                                     prefix_table=tabs[1]), **kw, out=out[:, :, :64].transpose(0, 1))
    assert torch.equal(got, want) and bool((out[:, :, 64:] == 0).all())


def test_shared_attention_many_groups(gpu):
    """More groups and requests than threads."""
    r = np.random.default_rng(5)
    members = r.integers(0, 4, 400)
    c = case(members, 2, 1, 64, 16, r.integers(0, 60, 400), r.integers(0, 3, 50), r.integers(0, 40, 70), BF16, 4, alone=9)
    for over in HINTS[:3]:
        check(c, sb.shared_attention(**c, **bounds(c, **over)))


def test_shared_attention_offsets_beyond_32_bits(gpu):
    """A cache of 5 GB, all pages in use at its end."""
    page, Hkv, D = 64, 8, 128
    n_pages = (5 << 30) // (page * Hkv * D * 2)
    k, v = (torch.zeros(n_pages, page, Hkv, D, dtype=BF16, device="cuda") for _ in range(2))
    c = case([3], 16, Hkv, D, page, [300], [1], [150, 3], BF16, 12)
    for max_q in (1, 1000):
        want = sb.shared_attention(**c, **bounds(c, max_q=max_q))
        tail = n_pages - c["k_cache"].shape[0]
        k[tail:], v[tail:] = c["k_cache"], c["v_cache"]
        moved = {n: torch.where(c[n] >= 0, c[n] + tail, -1) for n in ("table", "prefix_table")}
        assert torch.equal(sb.shared_attention(**dict(c, k_cache=k, v_cache=v, **moved), **bounds(c, max_q=max_q)), want)


def test_shared_attention_refusals(gpu):
    c = case([2, 1], 4, 2, 64, 8, [40, 21], [1], [20, 33, 2], F16, 11)
    for over, match in ((dict(q=c["q"].float()), "bfloat16"), (dict(prefix_lens=c["prefix_lens"][:1]), "prefix_lens"),
                        (dict(group_start=c["group_start"][:2]), "group_start"), (dict(prefix_table=c["prefix_table"].long()), "table"),
                        (dict(lens=c["lens"].long()), "lens"), (dict(v_cache=c["v_cache"][:2]), "one shape"),
                        (dict(q=c["q"].clone().requires_grad_()), "backward")):
        with pytest.raises(ValueError, match=match):
            sb.shared_attention(**dict(c, **over), **bounds(c))


def test_shared_attention_captured_and_on_other_streams(gpu):
    """A graph of two attentions with workspaces of their own, replayed with other
    queries and lengths; two streams at once."""
    c = case([5, 3], 8, 2, 128, 16, [2500, 700], [1], [300, 20], BF16, 21)
    kw = bounds(c)
    other = dict(c, q=torch.randn_like(c["q"]))

    def step():
        return sb.shared_attention(**c, **kw), sb.shared_attention(**other, **kw)

    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for t in range(4):
        c["q"].copy_(torch.randn_like(c["q"]))
        c["lens"].copy_(i32([300 - 40 * t, 20 - t] * 4))
        graph.replay()
        assert all(torch.equal(a, b) for a, b in zip(held, step())), t
        torch.cuda.synchronize()
    want = step()
    torch.cuda.synchronize()
    got = []
    for stream in [torch.cuda.Stream() for _ in range(2)]:
        with torch.cuda.stream(stream):
            got += [step() for _ in range(3)]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for run in got for a, b in zip(run, want))


@pytest.mark.parametrize("dtype,D", [(BF16, 64), (BF16, 128), (BF16, 256), (F16, 64), (F16, 128), (F16, 256)])
@pytest.mark.parametrize("members,q,prefix,own", [
    ([1], [1], [700], [300, 2]), ([2], [1], [700], [30]), ([3], [1], [6000], [2, 70]), ([1, 9], [1], [130, 700], [40]), ([2], [3], [700], [40, 90]),
    ([1], [9], [700], [300])])
def test_shared_attention_weights_in_two_parts(gpu, members, q, prefix, own, dtype, D):
    """By every kind of pass (rows by waves and by workgroups, of the prefix and of
    the own tokens): a weight is off by (eps / 2)^2 of itself, whatever the
    group's size and the bounds that the kernels are chosen by. Every other key is a
    little less likely and its value the negative one, so that weights rounded once
    would show."""
    c = case(members, 16, 1, D, 16, prefix, q, own, dtype, len(members) + D)
    c["q"].zero_()
    c["q"][:, :, 0] = torch.linspace(0.005, 0.4, 16, device="cuda")
    odd = torch.arange(16, device="cuda") % 2   # (pages of 16: a place's parity is its position's)
    c["v_cache"][:] = (2.0 * odd - 1)[:, None, None]
    c["k_cache"].zero_()
    c["k_cache"][..., 0] = -odd[:, None].to(dtype)
    eps = torch.finfo(dtype).eps
    args = [f64(c[n]) for n in ("q", "k_cache", "v_cache")]
    args += [c[n].tolist() for n in ("prefix_table", "prefix_lens", "group_start", "table", "lens", "q_start")]
    want, size, big = oracle.shared_attention(*args, 1.0)
    score = big * (D * 2.0 ** -24 + 2.0 ** -22)
    tol = eps / 2 * np.abs(want) + ((eps / 2) ** 2 + 2 * score[..., :1] + 2.0 ** -20) * size
    for over in HINTS:
        d = np.abs(f64(sb.shared_attention(**c, **bounds(c, **over), scale=1.0)) - want)
        assert np.all(d <= tol), (over, np.max(d / tol))
