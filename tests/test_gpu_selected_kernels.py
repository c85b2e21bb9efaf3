"""Selection of pages by each of its kernels, against the same in 64 bits: lists have
to be equal. Which kernel a call gets is looked at in test_serve_plan_cpu.py."""
import numpy as np
import pytest
import torch

import paper_2010_02164_amd as sb

pytestmark = pytest.mark.gpu
BF16, F16 = torch.bfloat16, torch.float16

PICKS = {   # (threads, pages each keeps in registers): requests, queries each, kv heads, page size, cached, max_kv (None: their largest), whether all are kept
    (256, 4): [(1, 1, 2, 1, [1000], None, True), (1, 1, 2, 1, [1026], None, True), (1, 1, 2, 1, [1027], 0, False), (2, 1, 3, 1, [5000, 900], 0, False)],
    (256, 16): [(64, 1, 4, 1, [2000, 4098], None, True), (130, 1, 2, 1, [1500, 60, 4000], None, True), (64, 1, 4, 1, [5000, 2000], 1500, False),
                (8, 9, 4, 2, [7000, 3000], None, True)],
    (1024, 4): [(1, 1, 2, 1, [2000], None, True), (1, 1, 1, 1, [4098], None, True), (3, 1, 2, 1, [1100, 3000, 1025], None, True),
                (1, 1, 2, 1, [9001], 3000, False)],
    (1024, 16): [(1, 1, 2, 1, [4099], None, True), (2, 1, 1, 1, [16386, 9000], None, True), (1, 1, 2, 1, [20001], None, False),
                 (2, 3, 1, 2, [70001, 40000], None, False)],
}
SCORES = {   # whether 16 tokens at a time are scored by the matrix unit: requests, queries each
    False: [(1, 1), (3, 2), (2, 7)],
    True: [(1, 8), (2, 8), (1, 17), (5, 33)],
}


def case(B, q, Hkv, page, kv, dtype, D, kind, seed):
    """Bounds whose scores are random, whole numbers (many equal), or one of three."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    lens = np.resize(kv, B)
    n_pages, T = 997, B * q
    table = torch.randint(0, n_pages, (B, -(-int(lens.max()) // page) + 3), generator=g, device="cuda", dtype=torch.int32)
    queries, bounds = normal(T, 2 * Hkv, D), normal(n_pages, 2, Hkv, D)
    if kind != "any":
        queries, bounds = queries.round(), bounds.round()
    if kind == "three":
        queries[..., 0], bounds[..., 1:], bounds[..., 0] = 1.0, 0.0, torch.randint(0, 3, (n_pages, 2, Hkv), generator=g, device="cuda").float()
    table[:, 5::41] = -1
    return dict(q=queries.to(dtype), bounds=bounds.to(dtype), table=table, lens=torch.as_tensor(lens).int().cuda(),
                q_start=torch.arange(0, T + 1, q, dtype=torch.int32, device="cuda"))


def check(c, page, tops, max_kv, first=1, last=1):
    """Every list, by a stable sort of scores in fp64."""
    Hkv, n_pages = c["bounds"].shape[2], c["bounds"].shape[0]
    lens, q = c["lens"].tolist(), int(c["q_start"][1])
    heads = c["q"].double().view(len(c["q"]), Hkv, 2, -1)
    up, down = heads.clamp(min=0).sum(2), heads.clamp(max=0).sum(2)
    lo, hi = c["bounds"].double().unbind(1)
    orders = []
    for t in range(len(c["q"])):
        p = lens[t // q] - q + t % q
        row, seen = c["table"][t // q], p // page + 1
        near = row[first:max(seen - last, first)].long()
        score = ((hi * up[t]).sum(-1) + (lo * down[t]).sum(-1))[near.clamp(0, n_pages - 1)]   # [pages, Hkv]
        score[near < 0] = -torch.inf
        orders.append((p, row, seen, torch.sort(score, dim=0, descending=True, stable=True).indices + first))
    for top in tops:
        width = first + top + last
        pages, kept = sb.select_pages(**c, page_size=page, top=top, first=first, last=last, max_kv=max_kv)
        assert pages.shape == (len(c["q"]), Hkv, width)
        want = torch.full_like(pages, -1)
        for t, (p, row, seen, order) in enumerate(orders):
            if seen <= width:
                want[t, :, :seen] = row[:seen]
                assert int(kept[t]) == p + 1
                continue
            cols = torch.cat([torch.arange(first, device="cuda").expand(Hkv, -1), order[:top].sort(0).values.t(),
                              torch.arange(seen - last, seen, device="cuda").expand(Hkv, -1)], 1)
            want[t] = row[cols]
            assert int(kept[t]) == (width - 1) * page + p % page + 1
        assert torch.equal(pages, want), (top, torch.nonzero(pages != want)[:5].tolist())


@pytest.mark.parametrize("kind", ["any", "whole", "three"])
@pytest.mark.parametrize("B,q,Hkv,page,kv,max_kv", [f[:6] for forms in PICKS.values() for f in forms])
def test_select_by_list_kernel(gpu, B, q, Hkv, page, kv, max_kv, kind):
    c = case(B, q, Hkv, page, kv, BF16, 64, kind, B + max(kv))
    most = -(-max(kv) // page) - 2
    check(c, page, (1, 37, 255, 300, most // 3, most - 700, most - 1) if most > 1000 else (1, 37, 300, most - 1), max(kv) if max_kv is None else max_kv)


@pytest.mark.parametrize("dtype,D", [(BF16, 64), (BF16, 128), (BF16, 256), (F16, 64), (F16, 128), (F16, 256)])
@pytest.mark.parametrize("B,q", [f for forms in SCORES.values() for f in forms])
def test_select_by_score_kernel(gpu, B, q, dtype, D):
    """Ends of pieces, of a wave's pages and of chunks; requests that share 16 tokens."""
    for kv in ([1, 17, 66, 67], [700, 1030, 90], [9000, 513]):
        kv = np.maximum(kv, q).tolist()
        check(case(B, q, 3, 4, kv, dtype, D, "any", B + q), 4, (1, 14, 200), max(kv))
