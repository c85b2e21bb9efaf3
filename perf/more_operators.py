"""Operators of a serving step over shared and long contexts, and of its
products in 8-bit integers, as cases to measure.

Three kinds of case, one per operator:

- "linear": a product with a weight matrix in 8-bit integers: the tokens' rows
  are quantised, each with a scale of its own, multiplied by weights with a
  scale for each output channel, and an optional bias is added;
- "shared": attention of a step's queries over a prefix that the requests of
  a group have in common and over each request's own tokens behind it, both
  in the paged cache, grouped heads;
- "sparse": attention over selected pages of long caches: the bounds of the
  pages that a step's tokens went to are brought up to date, pages are ranked
  for every query and key/value head by the largest score that their bounds
  allow, and the query attends to the first and last pages and the best between.

`run` computes them in elementary torch operations, or, with `own` set, makes
the library's calls.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZES = {"f32": 4, "bf16": 2, "f16": 2}


def _linear(name, dtype, M, N, K, out, bias):
    return dict(name=name, kind="linear", dtype=dtype, M=M, N=N, K=K, out=out, bias=bias)


def _shared(name, dtype, groups, members, Hq, Hkv, D, page, prefix, kv, q):
    return dict(name=name, kind="shared", dtype=dtype, groups=groups, members=members, Hq=Hq, Hkv=Hkv, D=D, page=page,
                prefix_lo=prefix[0], prefix_hi=prefix[1], kv_lo=kv[0], kv_hi=kv[1], q_lo=q[0], q_hi=q[1])


def _sparse(name, dtype, B, Hq, Hkv, D, page, kv, q, top, first, last):
    return dict(name=name, kind="sparse", dtype=dtype, B=B, Hq=Hq, Hkv=Hkv, D=D, page=page, kv_lo=kv[0], kv_hi=kv[1],
                q_lo=q[0], q_hi=q[1], top=top, first=first, last=last)


def listed():
    return [
        # One request's next token through a square projection.
        _linear("linear_one_bf16", "bf16", 1, 4096, 4096, "bf16", False),
        # A step of a batch through the joint projection of queries, keys and values.
        _linear("linear_step_bf16", "bf16", 61, 6144, 4096, "bf16", True),
        # Logits of a batch over a translation vocabulary, in fp32 for the sampler.
        _linear("linear_vocab_f16", "f16", 200, 32000, 1000, "f32", False),
        # A long prompt through a wide layer.
        _linear("linear_prompt_bf16", "bf16", 8000, 8192, 4096, "bf16", True),
        # The beam of one input: four hypotheses of a few tokens behind its source.
        _shared("shared_beam_bf16", "bf16", 1, 4, 16, 4, 128, 16, (1001, 1001), (3, 25), (1, 1)),
        # Many beams: each input's hypotheses behind a source of its own.
        _shared("shared_beams_f16", "f16", 40, 5, 16, 4, 64, 16, (200, 3000), (1, 180), (1, 1)),
        # A batch of requests behind one long instruction.
        _shared("shared_step_bf16", "bf16", 1, 64, 32, 8, 128, 16, (8000, 8000), (20, 1500), (1, 1)),
        # Drafts to verify, behind two long documents.
        _shared("shared_drafts_bf16", "bf16", 2, 60, 32, 8, 128, 64, (24000, 33000), (100, 2500), (1, 6)),
        # One request's next token over a cache of some length.
        _sparse("sparse_one_bf16", "bf16", 1, 16, 4, 128, 16, (20001, 20001), (1, 1), 60, 1, 3),
        # A step of a batch over long caches.
        _sparse("sparse_step_bf16", "bf16", 48, 32, 8, 128, 16, (5000, 50000), (1, 1), 120, 1, 7),
        # Drafts over very long caches of small heads and larger pages.
        _sparse("sparse_drafts_f16", "f16", 12, 32, 4, 64, 64, (20000, 120000), (2, 5), 40, 1, 4),
        # A chunk of a prompt behind a long cache.
        _sparse("sparse_prompt_bf16", "bf16", 2, 16, 4, 128, 32, (24000, 30000), (300, 600), 60, 1, 4),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the listed ranges.

    linear: 1 to 8000 rows, 100 to 32000 channels of 64 to 8192 values, three
    types in and out, with and without bias. shared: 1 to 40 groups of 1 to 64
    requests, prefixes of 16 to 33000 tokens, 1 to 2500 tokens of their own, of
    which 1 to 6 are queries, or a chunk of a prompt. sparse: 1 to 48 requests
    over 100 to 120000 tokens, pages of 16 to 128, 4 to 128 of them ranked in,
    single tokens, drafts or chunks of prompts. No drawn case costs more than
    the largest listed one."""
    kind = rng.choice(["linear", "shared", "sparse"])
    if kind == "linear":
        while True:
            M, N, K = _log_int(rng, 1, 8000), _log_int(rng, 100, 32000), _log_int(rng, 64, 8192)
            if M * N * K <= 2 ** 37 and M * N <= 2 ** 26:
                return _linear("", rng.choice(["bf16", "bf16", "f16", "f32"]), M, N, K, rng.choice(["bf16", "bf16", "f16", "f32"]),
                               rng.random() < 0.5)
    dtype = rng.choice(["bf16", "bf16", "f16"])
    D = rng.choice([64, 128, 128, 256])
    group = rng.choice([1, 2, 4, 5, 8])
    Hkv = rng.choice([1, 2, 3, 4, 8]) if D < 256 else rng.choice([1, 2, 4])
    page = rng.choice([16, 16, 24, 32, 64, 128])
    form = rng.choice(["single", "single", "single", "few", "prompt"])
    if kind == "shared":
        while True:
            groups, members = _log_int(rng, 1, 40), _log_int(rng, 1, 64)
            prefix, kv = _log_int(rng, 16, 33000), _log_int(rng, 1, 2500)
            q = (1, 1) if form == "single" else (1, rng.randint(2, 6)) if form == "few" else (10, 100)
            kv = max(kv, q[1])
            if groups * members * (prefix + kv) * q[1] * group * Hkv * D <= 4 * 10 ** 10 and groups * prefix <= 70000 \
                    and groups * members * kv * Hkv * D <= 4 * 10 ** 8:
                return _shared("", dtype, groups, members, group * Hkv, Hkv, D, page, (max(1, prefix // 5), prefix),
                               (max(q[1], kv // 20), kv), q)
    while True:
        B, kv = _log_int(rng, 1, 48), _log_int(rng, 100, 120000)
        q = (1, 1) if form == "single" else (1, rng.randint(2, 6)) if form == "few" else (20, 200)
        kv = max(kv, 2 * q[1])
        top = _log_int(rng, 4, 128)
        if B * kv * Hkv * D <= 13 * 10 ** 8 and B * q[1] * Hkv * (kv // page * 2 + top * page) * D <= 8 * 10 ** 9:
            return _sparse("", dtype, B, group * Hkv, Hkv, D, page, (max(q[1], kv // 10), kv), q, top, rng.choice([0, 1, 2]),
                           rng.choice([1, 2, 4]))


def _spread(lo, hi, n):
    """n whole numbers from lo to hi, evenly spread, the same for every seed."""
    return np.linspace(lo, hi, n).round().astype(np.int64) if n > 1 else np.array([hi], np.int64)


def _lengths(case, g):
    """A request's tokens and the new ones among them, paired the same way for
    every seed and in an order drawn from it."""
    B = case["groups"] * case["members"] if case["kind"] == "shared" else case["B"]
    order = torch.randperm(B, generator=g).numpy()
    new = _spread(case["q_lo"], case["q_hi"], B)[::-1].copy()
    have = np.maximum(_spread(case["kv_lo"], case["kv_hi"], B), new)
    return have[order], new[order]


def _tables(lens, page, ids, extra):
    """Block tables of caches of these lengths, their pages the next of ids."""
    held = -(-lens // page)
    table = np.full((len(lens), int(held.max()) + extra), -1, np.int64)
    table[np.arange(table.shape[1]) < held[:, None]] = ids[:held.sum()]
    return table, ids[held.sum():]


def prepare(case, seed):
    dev = "cuda"
    g = torch.Generator().manual_seed(seed)
    gd = torch.Generator(device=dev).manual_seed(seed)
    kind, dtype = case["kind"], DTYPES[case["dtype"]]

    def normal(*shape, type_=dtype):
        return torch.randn(*shape, generator=gd, device=dev, dtype=torch.float32).to(type_)

    def whole(a):
        return torch.as_tensor(np.ascontiguousarray(a)).to(torch.int32).to(dev)

    if kind == "linear":
        M, N, K = case["M"], case["N"], case["K"]
        # Tokens differ in size, and a few channels stand out in all of them.
        size = torch.exp(0.5 * torch.randn(M, 1, generator=gd, device=dev))
        loud = 1.0 + 9.0 * (torch.rand(K, generator=gd, device=dev) < 0.01)
        x = (torch.randn(M, K, generator=gd, device=dev) * size * loud).to(dtype)
        w = torch.randn(N, K, generator=gd, device=dev) / math.sqrt(K)
        bias = torch.randn(N, generator=gd, device=dev) if case["bias"] else None
        state = dict(kind=kind, x=x, bias=bias, out=DTYPES[case["out"]])
        # The weights are laid out once, as a program that keeps them does: whole
        # multiples of each channel's scale, values rounded up to sixteens with zeros.
        w_scale = w.abs().amax(1) / 127.0
        codes = torch.zeros(N, -(-K // 16) * 16, dtype=torch.int8, device=dev)
        codes[:, :K] = torch.round(w.double() / w_scale.double()[:, None]).to(torch.int8)
        return dict(state, w=codes, w_scale=w_scale)
    lens, new = _lengths(case, g)
    q_start = np.concatenate([[0], np.cumsum(new)])
    Hq, Hkv, D, page = case["Hq"], case["Hkv"], case["D"], case["page"]
    state = dict(kind=kind, q=normal(int(q_start[-1]), Hq, D), lens=whole(lens), q_start=whole(q_start), max_q=int(new.max()),
                 max_kv=int(lens.max()))
    if kind == "shared":
        prefix = _spread(case["prefix_lo"], case["prefix_hi"], case["groups"])
        prefix = prefix[torch.randperm(case["groups"], generator=g).numpy()]
        n_pages = int((-(-lens // page)).sum() + (-(-prefix // page)).sum()) + 3
        prefix_table, ids = _tables(prefix, page, torch.randperm(n_pages, generator=g).numpy(), 1)
        table, _ = _tables(lens, page, ids, 2)
        return dict(state, k_cache=normal(n_pages, page, Hkv, D), v_cache=normal(n_pages, page, Hkv, D), table=whole(table),
                    prefix_table=whole(prefix_table), prefix_lens=whole(prefix), max_prefix=int(prefix.max()),
                    group_start=whole(np.arange(case["groups"] + 1) * case["members"]))
    n_pages = int((-(-lens // page)).sum()) + 3
    table, _ = _tables(lens, page, torch.randperm(n_pages, generator=g).numpy(), 1)
    # Keys of one page resemble each other, those of different pages do not.
    k_cache, v_cache = normal(n_pages, page, Hkv, D), normal(n_pages, page, Hkv, D)
    k_cache += normal(n_pages, 1, Hkv, D)
    # Bounds of the pages that were full before this step; the others as they may be.
    bounds = torch.zeros(n_pages, 2, Hkv, D, dtype=dtype, device=dev)
    full = (lens - new) // page
    done = whole(table[np.arange(table.shape[1]) < full[:, None]]).long()
    for at in done.split(1 << 14):
        bounds[at, 0], bounds[at, 1] = k_cache[at].amin(1), k_cache[at].amax(1)
    return dict(state, k_cache=k_cache, v_cache=v_cache, table=whole(table), bounds=bounds, page=page, top=case["top"],
                first=case["first"], last=case["last"])


def run(s):
    return {"linear": run_linear, "shared": run_shared, "sparse": run_sparse}[s["kind"]](s)


def run_linear(s):
    x, w, w_scale, bias = s["x"], s["w"], s["w_scale"], s["bias"]
    if own:
        from paper_2010_02164_amd import int8_linear, quantize_rows
        codes, x_scale = quantize_rows(x)
        return dict(y=int8_linear(codes, x_scale, w, w_scale, bias=bias, dtype=s["out"]), x_scale=x_scale)
    x_scale = x.float().abs().amax(1) / 127.0
    # (Quotients in 64 bits: many lie next to the border between two whole numbers.)
    codes = torch.round(x.double() / torch.where(x_scale == 0, 1.0, x_scale).double()[:, None]).clamp(-127, 127).float()
    # Products of 1024 values at a time are whole numbers below 2^24.
    K = x.shape[1]
    total = torch.zeros(x.shape[0], w.shape[0], dtype=torch.int32, device=x.device)
    for k in range(0, K, 1024):
        total += (codes[:, k:k + 1024] @ w[:, k:min(k + 1024, K)].float().T).int()
    y = total.double() * x_scale.double()[:, None] * w_scale.double()
    if bias is not None:
        y = y + bias.double()
    return dict(y=y.to(s["out"]), x_scale=x_scale)


def _side_by_side(cache, table, most):
    """Each row's first `most` keys or values, [rows, kv_heads, most, D] in fp32."""
    page = cache.shape[1]
    j = torch.arange(most, device=cache.device)
    at = table[:, j // page].clamp(min=0).long() * page + j % page
    return cache.flatten(0, 1)[at].float().transpose(1, 2).contiguous()


def _batch(q, start, most, Hkv):
    """Queries start[r] .. + most of each row r, [rows, kv_heads, most * group, D] in fp32."""
    T, Hq, D = q.shape
    row = (start[:, None] + torch.arange(most, device=q.device)).clamp(max=T - 1).long()
    return q[row].float().view(len(start), most, Hkv, Hq // Hkv, D).transpose(1, 2).reshape(len(start), Hkv, -1, D)


def _softmax_parts(scores, seen, values):
    """(sum of weights times values, sum of weights, largest score) of each row."""
    scores = scores.masked_fill(~seen, -torch.inf)
    top = scores.amax(-1, keepdim=True)
    w = torch.exp(scores - torch.where(top == -torch.inf, 0.0, top))
    return torch.matmul(w, values), w.sum(-1, keepdim=True), top


def run_shared(s):
    q, k_cache, v_cache, table, lens, q_start = s["q"], s["k_cache"], s["v_cache"], s["table"], s["lens"], s["q_start"]
    prefix_table, prefix_lens, group_start = s["prefix_table"], s["prefix_lens"], s["group_start"]
    if own:
        from paper_2010_02164_amd import shared_attention
        return shared_attention(q, k_cache, v_cache, prefix_table, prefix_lens, group_start, table, lens, q_start,
                                max_q=s["max_q"], max_kv=s["max_kv"], max_prefix=s["max_prefix"])
    T, Hq, D = q.shape
    Hkv, dev, scale = k_cache.shape[2], q.device, 1.0 / math.sqrt(D)
    group, t = Hq // Hkv, torch.arange(T, device=dev)

    def by_token(x, of, first, most):   # [rows, Hkv, most * group, n] -> [T, Hq, n]
        x = x.view(len(x), Hkv, most, group, -1).transpose(1, 2).flatten(2, 3)
        return x[of, t - first[of]]

    # The prefix: all queries of a group's requests over its keys.
    starts = q_start[group_start.long()]
    most = min(s["max_q"] * (len(lens) // len(prefix_lens)), T)
    keys, vals = (_side_by_side(c, prefix_table, s["max_prefix"]) for c in (k_cache, v_cache))
    scores = torch.matmul(_batch(q, starts[:-1], most, Hkv), keys.transpose(2, 3).contiguous()) * scale
    seen = (torch.arange(s["max_prefix"], device=dev) < prefix_lens[:, None])[:, None, None]
    of = torch.searchsorted(starts[1:].contiguous(), t, right=True)
    acc_p, sum_p, top_p = (by_token(x, of, starts, most) for x in _softmax_parts(scores, seen, vals))
    # Each request's own tokens.
    keys, vals = (_side_by_side(c, table, s["max_kv"]) for c in (k_cache, v_cache))
    scores = torch.matmul(_batch(q, q_start[:-1], s["max_q"], Hkv), keys.transpose(2, 3).contiguous()) * scale
    p = (lens - q_start[1:] + q_start[:-1])[:, None] + torch.arange(s["max_q"], device=dev)
    seen = torch.arange(s["max_kv"], device=dev) <= torch.minimum(p, lens[:, None] - 1)[:, :, None]
    seen = seen.repeat_interleave(group, 1)[:, None]
    of = torch.searchsorted(q_start[1:].contiguous(), t, right=True)
    acc_o, sum_o, top_o = (by_token(x, of, q_start, s["max_q"]) for x in _softmax_parts(scores, seen, vals))
    top = torch.maximum(top_p, top_o)
    f, h = torch.exp(top_p - top), torch.exp(top_o - top)
    return ((acc_p * f + acc_o * h) / (sum_p * f + sum_o * h)).to(q.dtype)


def run_sparse(s):
    q, k_cache, v_cache, table, lens, q_start, bounds = (s[n] for n in ("q", "k_cache", "v_cache", "table", "lens", "q_start", "bounds"))
    top, first, last, page = s["top"], s["first"], s["last"], s["page"]
    if own:
        from paper_2010_02164_amd import page_bounds, select_pages, selected_attention
        page_bounds(k_cache, table, lens, q_start, bounds, max_q=s["max_q"])
        pages, kept = select_pages(q, bounds, table, lens, q_start, page_size=page, top=top, first=first, last=last, max_kv=s["max_kv"])
        return dict(out=selected_attention(q, k_cache, v_cache, pages, kept), pages=pages, kept=kept, bounds=bounds)
    T, Hq, D = q.shape
    n_pages, _, Hkv, _ = k_cache.shape
    group, dev = Hq // Hkv, q.device
    # Bounds of the pages that the new tokens went to, over the tokens they hold.
    count = (q_start[1:] - q_start[:-1]).long()
    lo, hi = (lens - count) // page, (lens - 1) // page
    column = lo[:, None] + torch.arange(s["max_q"] // page + 2, device=dev)
    of, col = torch.nonzero((column <= hi[:, None]) & (count > 0)[:, None], as_tuple=True)
    column = column[of, col]
    ids = table[of, column].long()
    held = (torch.arange(page, device=dev) < (lens[of] - column * page)[:, None])[:, :, None, None]
    keys = k_cache[ids]
    bounds[ids, 0] = keys.masked_fill(~held, torch.inf).amin(1)
    bounds[ids, 1] = keys.masked_fill(~held, -torch.inf).amax(1)
    # The largest score a page allows, summed over the heads of a group (in 64
    # bits: pages are ranked by it).
    t = torch.arange(T, device=dev)
    of = torch.searchsorted(q_start[1:].contiguous(), t, right=True)
    p = (lens[of] - q_start[of + 1] + t).long()
    heads = q.double().view(T, Hkv, group, D)
    up, down = heads.clamp(min=0).sum(2), heads.clamp(max=0).sum(2)
    seen_pages = p // page + 1
    P, W = int(-(-s["max_kv"] // page)), first + top + last
    pages = torch.empty(T, Hkv, W, dtype=torch.int32, device=dev)
    out = torch.empty_like(q)
    kept = torch.where(seen_pages <= W, p + 1, (W - 1) * page + p % page + 1).int()
    c, j = torch.arange(P, device=dev), torch.arange(W * page, device=dev)
    step = max(1, min((1 << 28) // (P * 2 * Hkv * D), (1 << 28) // (W * page * Hkv * D)))
    for a in range(0, T, step):
        z = slice(a, min(a + step, T))
        near = bounds[table[of[z], :P].clamp(min=0).long()]                      # [tokens, P, 2, Hkv, D]
        score = (near[:, :, 1].double() * up[z, None]).sum(-1) + (near[:, :, 0].double() * down[z, None]).sum(-1)
        n = seen_pages[z, None, None]
        score = score.transpose(1, 2).masked_fill((c < first) | (c >= n - last), torch.inf).masked_fill(c >= n, -torch.inf)
        order = torch.sort(score, dim=2, descending=True, stable=True).indices[:, :, :W]
        order = order.masked_fill(torch.arange(order.shape[2], device=dev) >= n, P).sort(2).values
        mine = table[of[z]][:, None].expand(-1, Hkv, -1).gather(2, order.clamp(max=P - 1))
        pages[z] = -1
        pages[z, :, :order.shape[2]] = mine.masked_fill(order >= P, -1).int()
        # Attention over them.
        at = pages[z].clamp(min=0).long()[:, :, j // page] * page + j % page       # [tokens, Hkv, keys]
        head = torch.arange(Hkv, device=dev)[:, None]
        keys, vals = (cache.flatten(0, 1)[at, head].float() for cache in (k_cache, v_cache))
        scores = torch.matmul(q[z].float().view(-1, Hkv, group, D), keys.transpose(2, 3).contiguous()) / math.sqrt(D)
        acc, total, _ = _softmax_parts(scores, (j < kept[z, None])[:, None, None], vals)
        out[z] = (acc / total).view(-1, Hq, D).to(q.dtype)
    return dict(out=out, pages=pages, kept=kept, bounds=bounds)


def work(case):
    """Bytes read and written once, and operations, of one pass."""
    if case["kind"] == "linear":
        M, N, K = case["M"], case["N"], case["K"]
        return dict(bytes=M * K * SIZES[case["dtype"]] + N * K + M * N * SIZES[case["out"]] + 4 * (M + N + N * case["bias"]),
                    flops=2 * M * N * K)
    es, Hq, Hkv, D, page = SIZES[case["dtype"]], case["Hq"], case["Hkv"], case["D"], case["page"]
    lens, new = _lengths(case, torch.Generator().manual_seed(0))
    bytes_ = int(2 * new.sum() * Hq * D * es)
    pairs = int(sum(m * n - m * (m - 1) // 2 for n, m in zip(lens.tolist(), new.tolist())))
    if case["kind"] == "shared":
        prefix = _spread(case["prefix_lo"], case["prefix_hi"], case["groups"])
        each = new.reshape(case["groups"], -1).sum(1)   # (the prefixes' order goes by the seed, the average does not)
        pairs += int(prefix.mean() * each.sum())
        return dict(bytes=bytes_ + int(2 * (lens.sum() + prefix.sum()) * Hkv * D * es), flops=4 * pairs * Hq * D)
    flops = 0
    for n, m in zip(lens.tolist(), new.tolist()):
        seen = -(-n // page)
        between = max(seen - case["first"] - case["last"], 0)
        top = min(case["top"], between)
        # Pages that m queries select between them, if they do so independently.
        union = between * (1 - (1 - top / between) ** m) if between else 0
        read = min((union + min(seen, case["first"] + case["last"])) * page, n)
        touched = (n - 1) // page - (n - m) // page + 1
        bytes_ += int(2 * read * Hkv * D * es + seen * 2 * Hkv * D * es + touched * (page + 2) * Hkv * D * es)
        flops += 4 * m * min((top + case["first"] + case["last"]) * page, n) * Hq * D + 4 * m * seen * Hkv * D
    return dict(bytes=bytes_, flops=int(flops))


def exact(case, seed):
    """The outputs in 64 bits from the definitions, request by request."""
    s = prepare(case, seed)
    if case["kind"] == "linear":
        x = s["x"].double()
        scale = (x.abs().max(1).values / 127).float().double()
        codes = torch.nn.functional.pad((x / scale[:, None]).round(), (0, s["w"].shape[1] - x.shape[1]))
        y = torch.cat([c @ s["w"].double().t().contiguous() for c in codes.split(2048)]) * (scale[:, None] * s["w_scale"].double())
        return dict(y=y if s["bias"] is None else y + s["bias"].double(), x_scale=scale)
    page, Hq, Hkv, D = case["page"], case["Hq"], case["Hkv"], case["D"]
    lens, starts = s["lens"].tolist(), s["q_start"].tolist()
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")

    def cached(cache, table, n):
        return cache[table[:-(-n // page)].long()].flatten(0, 1)[:n].double()

    if case["kind"] == "shared":
        for b, n in enumerate(lens):
            g = b // case["members"]
            if b % case["members"] == 0:
                ahead = int(s["prefix_lens"][g])
                prefix = [cached(s[c], s["prefix_table"][g], ahead) for c in ("k_cache", "v_cache")]
            keys, vals = (torch.cat([x, cached(s[c], s["table"][b], n)]) for x, c in zip(prefix, ("k_cache", "v_cache")))
            lo, hi = starts[b], starts[b + 1]
            position = torch.arange(ahead + n - (hi - lo), ahead + n, device="cuda")
            hidden = torch.arange(ahead + n, device="cuda") > position[:, None]
            x = torch.stack([s["q"][lo:hi, h].double() @ keys[:, h * Hkv // Hq].T.contiguous() for h in range(Hq)]) / math.sqrt(D)
            w = torch.softmax(x.masked_fill(hidden, -math.inf), -1)
            for h in range(Hq):
                out[lo:hi, h] = w[h] @ vals[:, h * Hkv // Hq].contiguous()
        return out
    W = case["first"] + case["top"] + case["last"]
    chosen = torch.full((starts[-1], Hkv, W), -1, dtype=torch.int32, device="cuda")
    kept = torch.zeros(starts[-1], dtype=torch.int32, device="cuda")
    bounds = s["bounds"].double()
    if starts[-1] * Hkv > 6000:
        return None
    for b, n in enumerate(lens):
        m = starts[b + 1] - starts[b]
        row = s["table"][b].long()
        for c in range((n - m) // page, -(-n // page)):
            inside = s["k_cache"][row[c], :min(page, n - c * page)].double()
            bounds[row[c], 0], bounds[row[c], 1] = inside.min(0).values, inside.max(0).values
        low, high = bounds[row[:-(-n // page)]].unbind(1)
        keys, vals = cached(s["k_cache"], row, n), cached(s["v_cache"], row, n)
        for h in range(Hkv):
            lo, hi, k, v = low[:, h], high[:, h], keys[:, h].contiguous(), vals[:, h].contiguous()
            for t in range(starts[b], starts[b + 1]):
                p = n - m + t - starts[b]
                seen = p // page + 1
                mine = s["q"][t, h * Hq // Hkv:(h + 1) * Hq // Hkv].double()
                if seen <= W:
                    cols = torch.arange(seen, device="cuda")
                else:
                    between = slice(case["first"], seen - case["last"])
                    score = hi[between] @ mine.clamp(min=0).sum(0) + lo[between] @ mine.clamp(max=0).sum(0)
                    best = torch.topk(score, case["top"]).indices + case["first"]
                    cols = torch.cat([torch.arange(case["first"], device="cuda"), best.sort().values,
                                      torch.arange(seen - case["last"], seen, device="cuda")])
                chosen[t, h, :len(cols)] = row[cols].int()
                at = (cols[:, None] * page + torch.arange(page, device="cuda")).flatten()
                at = at[:len(at) - (page - 1 - p % page)]
                kept[t] = len(at)
                out[t, h * Hq // Hkv:(h + 1) * Hq // Hkv] = torch.softmax(mine @ k[at].T.contiguous() / math.sqrt(D), -1) @ v[at]
    return dict(out=out, pages=chosen, kept=kept, bounds=bounds)
