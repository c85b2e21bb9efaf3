"""The operators of cached decoding with sampled tokens, as cases to measure.

Four kinds of case, one per operator:

- "plan": block tables, slot maps and positions of a step from the requests'
  lengths, with pages taken from and given back to a free list;
- "rope": rotary positions of a step's queries and keys, and the write of its
  keys and values into the paged cache;
- "attend": attention over the paged cache with grouped heads, causal, with an
  optional sliding window and first tokens that stay visible (sinks);
- "sample": one token per row of logits, drawn from a given uniform number
  under temperature, top-k, top-p and min-p.

`run` computes them in elementary torch operations, or, with `own` set, makes
the library's calls.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZES = {"f32": 4, "bf16": 2, "f16": 2}


def _plan(name, B, page, have, add, release=0):
    return dict(name=name, kind="plan", B=B, page=page, have_lo=have[0], have_hi=have[1], add_lo=add[0], add_hi=add[1],
                release=release)


def _rope(name, dtype, T, Hq, Hkv, D, rot, layout, page, far, factor=1.0):
    return dict(name=name, kind="rope", dtype=dtype, T=T, Hq=Hq, Hkv=Hkv, D=D, rot=rot, layout=layout, page=page, far=far,
                factor=factor)


def _attend(name, dtype, B, Hq, Hkv, D, page, q, kv, window=0, sinks=0):
    return dict(name=name, kind="attend", dtype=dtype, B=B, Hq=Hq, Hkv=Hkv, D=D, page=page, q_lo=q[0], q_hi=q[1], kv_lo=kv[0],
                kv_hi=kv[1], window=window, sinks=sinks)


def _sample(name, dtype, rows, V, filters):
    return dict(name=name, kind="sample", dtype=dtype, rows=rows, V=V, filters=filters)


def listed():
    return [
        # A serving step of single tokens: a thousand live requests of very
        # different lengths, every ninth of them finished and released.
        _plan("plan_step_1024", 1024, 16, (1, 4000), (1, 1), release=9),
        # Prompts admitted together: some tens of thousands of tokens.
        _plan("plan_prompts", 37, 64, (0, 900), (300, 2900)),
        # One request's next token, where launches count.
        _rope("rope_one_bf16", "bf16", 1, 16, 4, 128, 128, "half", 16, 5000),
        # A step of a batch, part of the head rotated, interleaved pairs.
        _rope("rope_step_f16", "f16", 301, 32, 8, 64, 32, "interleaved", 16, 30000),
        # A long prompt at far positions, frequencies scaled for it.
        _rope("rope_prompt_bf16", "bf16", 16000, 32, 8, 128, 128, "half", 64, 500000, factor=8.0),
        # One request's next token over a short cache.
        _attend("attend_one_bf16", "bf16", 1, 16, 4, 128, 16, (1, 1), (1001, 1001)),
        # A step of a batch over ordinary to long caches, all of it visible.
        _attend("attend_step_bf16", "bf16", 64, 32, 8, 128, 16, (1, 1), (200, 9000)),
        # A step over very long caches seen through a window with sinks.
        _attend("attend_step_window_f16", "f16", 48, 32, 4, 64, 32, (1, 1), (20000, 100000), window=4096, sinks=4),
        # Prompts in chunks, each behind what is cached already, windowed.
        _attend("attend_prompts_bf16", "bf16", 3, 32, 8, 128, 64, (1500, 4100), (4100, 8200), window=2048, sinks=4),
        # One row: an interactive request's next token.
        _sample("sample_one_f32", "f32", 1, 32000, "mixed"),
        # A batch whose requests each bring their own filters.
        _sample("sample_batch_bf16", "bf16", 320, 64000, "mixed"),
        # The largest: many rows over a large vocabulary in fp32.
        _sample("sample_wide_f32", "f32", 512, 128000, "mixed"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the listed ranges.

    plan: 1 to 2000 requests, pages of 8 to 128 tokens, single tokens or
    prompts, with and without releases. rope: 1 to 16000 tokens, heads of 64
    to 256, a quarter, half or all of them rotated, both layouts. attend:
    single tokens, a few tokens (drafts to verify) or prompts; 1 to 64
    requests, 1 to 32 heads in groups of 1 to 8, any page size of 8 to 128,
    windowed or not. sample: 1 to 512 rows of 300 to 128000 logits in three
    types. No drawn case costs more than the largest listed one."""
    kind = rng.choice(["plan", "rope", "attend", "attend", "sample", "sample"])
    if kind == "plan":
        B = _log_int(rng, 1, 2000)
        long = rng.random() < 0.4
        hi = max(2, min(3000, 80000 // B)) if long else rng.choice([1, 1, 5])
        return dict(_plan("", B, rng.choice([8, 16, 24, 32, 64, 128]), (0, _log_int(rng, 2, 6000)), (1, hi),
                          release=rng.choice([0, 3, 7, 20])))
    page = rng.choice([8, 16, 16, 24, 32, 64, 128])
    dtype = rng.choice(["bf16", "bf16", "f16"])
    D = rng.choice([64, 128, 128, 256])
    group = rng.choice([1, 2, 4, 5, 8])
    Hkv = rng.choice([1, 2, 3, 4])
    if kind == "rope":
        T = _log_int(rng, 1, 16000)
        return _rope("", dtype, T, group * Hkv, Hkv, D, D // rng.choice([1, 2, 4]), rng.choice(["half", "interleaved"]), page,
                     _log_int(rng, 20000, 1000000), factor=rng.choice([1.0, 4.0, 16.0]))
    if kind == "attend":
        form = rng.choice(["single", "single", "few", "prompt"])
        window, sinks = rng.choice([(0, 0), (_log_int(rng, 17, 5000), rng.choice([0, 1, 4, 70]))])
        if form == "prompt":
            q_hi = _log_int(rng, 20, 2500)
            kv_hi = q_hi + _log_int(rng, 1, 2500)
            return _attend("", dtype, rng.choice([1, 2, 3, 5]), group * Hkv, Hkv, D, page, (max(1, q_hi // 4), q_hi),
                           (q_hi, kv_hi), window, sinks)
        q = (1, 1) if form == "single" else (1, rng.randint(2, 9))
        B = _log_int(rng, 1, 64)
        kv_hi = _log_int(rng, 40, max(100, min(90000, 500000 // B)))
        return _attend("", dtype, B, group * Hkv, Hkv, D, page, q, (max(q[1], kv_hi // 20), kv_hi), window, sinks)
    V = _log_int(rng, 300, 128000)
    return _sample("", rng.choice(["f32", "bf16", "f16"]), _log_int(rng, 1, 512), V,
                   rng.choice(["mixed", "mixed", "top_k", "top_p", "min_p", "none"]))


def _spread(lo, hi, n):
    """n whole numbers from lo to hi, evenly spread, the same for every seed."""
    return np.linspace(lo, hi, n).round().astype(np.int64) if n > 1 else np.array([hi], np.int64)


def _frequencies(case):
    """Rotation per position of every pair, base 10000, slowed by `factor`
    as a whole (positions interpolated for longer contexts)."""
    half = case["rot"] // 2
    return 10000.0 ** (-torch.arange(half, dtype=torch.float64) / half) / case["factor"]


def _scale_of(case):
    """The growth of the rotated part's length that goes with `factor`."""
    return 1.0 + 0.1 * math.log(case["factor"])


def _lengths(case, g):
    """A request's cached and new tokens, paired the same way for every
    seed and in an order drawn from it."""
    B = case["B"]
    order = torch.randperm(B, generator=g).numpy()
    if case["kind"] == "plan":
        have, add = _spread(case["have_lo"], case["have_hi"], B), _spread(case["add_lo"], case["add_hi"], B)[::-1].copy()
        if case["release"]:
            add[::case["release"]] = -1
    else:
        add = _spread(case["q_lo"], case["q_hi"], B)
        have = np.maximum(_spread(case["kv_lo"], case["kv_hi"], B), add)
    return have[order], add[order]


def prepare(case, seed):
    dev = "cuda"
    g = torch.Generator().manual_seed(seed)
    gd = torch.Generator(device=dev).manual_seed(seed)
    kind = case["kind"]

    def normal(*shape, dtype):
        return torch.randn(*shape, generator=gd, device=dev, dtype=torch.float32).to(DTYPES[dtype])

    def whole(a, dtype=torch.int32):
        return torch.as_tensor(np.ascontiguousarray(a)).to(dtype).to(dev)

    if kind == "sample":
        rows, V = case["rows"], case["V"]
        z = torch.randn(rows, V, generator=gd, device=dev) * 2.5
        at = torch.randint(V, (rows, 48), generator=gd, device=dev)     # a few likely tokens
        z.scatter_add_(1, at, 10.0 * torch.rand(rows, 48, generator=gd, device=dev))
        f, r = case["filters"], torch.rand(5, rows, generator=g)
        T = 0.5 + 0.8 * r[0]
        top_k = torch.zeros(rows, dtype=torch.int32)
        top_p, min_p = torch.ones(rows), torch.zeros(rows)
        if f in ("mixed", "top_k"):
            top_k = (torch.exp(math.log(min(400, V)) * r[1])).round().to(torch.int32)
        if f in ("mixed", "top_p"):
            top_p = 0.7 + 0.3 * r[2]
        if f in ("mixed", "min_p"):
            min_p = 0.1 * r[3]
        if f == "mixed":   # requests that leave one or the other out, and greedy ones
            n = torch.arange(rows)
            T = torch.where(n % 8 == 7, 0.0, T)
            top_k = torch.where(n % 3 == 2, 0, top_k)
            top_p = torch.where(n % 5 == 4, 1.0, top_p)
            min_p = torch.where(n % 2 == 1, 0.0, min_p)
        return dict(kind=kind, logits=z.to(DTYPES[case["dtype"]]), u=r[4].to(dev), temperature=T.to(dev),
                    top_k=top_k.to(torch.int32).to(dev), top_p=top_p.to(dev), min_p=min_p.to(dev))
    if kind == "plan":
        have, add = _lengths(case, g)
        page, B = case["page"], case["B"]
        held = -(-have // page)
        want = np.maximum(-(-(have + np.maximum(add, 0)) // page), held)
        n_pages = int(want.sum()) + 5
        ids = torch.randperm(n_pages, generator=g).numpy()
        width = int(want.max()) + 3
        table = np.full((B, width), -1, np.int64)
        live = np.arange(width) < held[:, None]
        table[live] = ids[:held.sum()]
        free = np.full(n_pages, -1, np.int64)
        free[:n_pages - held.sum()] = ids[held.sum():]
        return dict(kind=kind, lens=whole(have), add=whole(add), table=whole(table), free_list=whole(free),
                    n_free=whole([n_pages - held.sum()]), page_size=page, token_cap=int(np.maximum(add, 0).sum()) + 7)
    Hq, Hkv, D, page = case["Hq"], case["Hkv"], case["D"], case["page"]
    if kind == "rope":
        T = case["T"]
        n_pages = T // page + 9
        slots = torch.randperm(n_pages * page, generator=g)[:T].to(dev)
        start = int(torch.randint(case["far"] - T, (1,), generator=g))
        return dict(kind=kind, q=normal(T, Hq, D, dtype=case["dtype"]), k=normal(T, Hkv, D, dtype=case["dtype"]),
                    v=normal(T, Hkv, D, dtype=case["dtype"]), slots=slots, layout=case["layout"],
                    positions=(torch.arange(T) + start).to(torch.int32).to(dev), inv_freq=_frequencies(case).to(dev),
                    mscale=_scale_of(case), k_cache=torch.zeros(n_pages, page, Hkv, D, dtype=DTYPES[case["dtype"]], device=dev),
                    v_cache=torch.zeros(n_pages, page, Hkv, D, dtype=DTYPES[case["dtype"]], device=dev))
    lens, new = _lengths(case, g)
    held = -(-lens // page)
    n_pages = int(held.sum()) + 3
    table = np.full((case["B"], int(held.max()) + 1), -1, np.int64)
    table[np.arange(table.shape[1]) < held[:, None]] = torch.randperm(n_pages, generator=g).numpy()[:held.sum()]
    q_start = np.concatenate([[0], np.cumsum(new)])
    return dict(kind=kind, q=normal(int(q_start[-1]), Hq, D, dtype=case["dtype"]), table=whole(table), lens=whole(lens),
                q_start=whole(q_start), k_cache=normal(n_pages, page, Hkv, D, dtype=case["dtype"]),
                v_cache=normal(n_pages, page, Hkv, D, dtype=case["dtype"]), max_q=int(new.max()), max_kv=int(lens.max()),
                window=case["window"], sinks=case["sinks"])


def run(s):
    kind = s["kind"]
    if kind == "plan":
        return run_plan(s)
    if kind == "rope":
        return run_rope(s)
    if kind == "attend":
        return run_attend(s)
    return run_sample(s)


def run_plan(s):
    if own:
        from paper_2010_02164_amd import plan_pages
        p = plan_pages(s["lens"], s["add"], s["free_list"], s["n_free"], s["table"], page_size=s["page_size"],
                       token_cap=s["token_cap"])
        return dict(q_start=p.q_start, lens=p.lens, granted=p.granted, slots=p.slots, positions=p.positions, n_free=p.n_free,
                    table=s["table"], free_list=s["free_list"])
    lens, add, free, table = s["lens"].long(), s["add"].long(), s["free_list"], s["table"]
    page, cap = s["page_size"], s["token_cap"]
    B, width = table.shape
    held = (lens + page - 1) // page
    # Pages of released requests go on top of the stack, in order.
    gone = torch.where(add < 0, held, 0)
    n = s["n_free"].long()
    column = torch.arange(width, device=table.device)
    place = n + (gone.cumsum(0) - gone)[:, None] + column
    on = column < gone[:, None]
    size = free.numel()
    stack = torch.cat([free, free.new_zeros(1)])            # the last place takes what is no page
    stack[torch.where(on, place, size)] = table
    n = n + gone.sum()
    # Requests in order, as long as tokens and pages last.
    tokens = torch.where((add > 0) & (lens + add <= width * page), add, 0)
    need = (lens + tokens + page - 1) // page - held
    need = torch.where(tokens > 0, need, 0)
    fits = (tokens.cumsum(0) <= cap) & (need.cumsum(0) <= n)
    tokens, need = torch.where(fits, tokens, 0), torch.where(fits, need, 0)
    first = need.cumsum(0) - need
    new = (column >= held[:, None]) & (column < (held + need)[:, None])
    popped = stack[(n - 1 - (first[:, None] + column - held[:, None])).clamp(0, size)]
    table.copy_(torch.where(new, popped, table))
    free.copy_(stack[:size])
    after = torch.where(add < 0, 0, lens + tokens)
    q_start = torch.cat([tokens.new_zeros(1), tokens.cumsum(0)])
    t = torch.arange(cap, device=table.device)
    of = torch.searchsorted(q_start[1:].contiguous(), t, right=True).clamp(max=B - 1)
    pos = lens[of] + t - q_start[of]
    real = t < q_start[-1]
    slot = table[of, (pos // page).clamp(0, width - 1)].long() * page + pos % page
    return dict(q_start=q_start.int(), lens=after.int(), granted=tokens.int(), slots=torch.where(real, slot, -1),
                positions=torch.where(real, pos, -1).int(), n_free=(n - need.sum()).int(), table=table, free_list=free)


def run_rope(s):
    q, k, v = s["q"], s["k"], s["v"]
    if own:
        from paper_2010_02164_amd import rope_append
        rotated = rope_append(q, k, v, s["positions"], s["slots"], s["k_cache"], s["v_cache"], s["inv_freq"],
                              layout=s["layout"], mscale=s["mscale"])
        return dict(q=rotated, k_cache=s["k_cache"], v_cache=s["v_cache"])
    angle = s["positions"].double()[:, None] * s["inv_freq"]
    cos, sin = (s["mscale"] * angle.cos()).float()[:, None], (s["mscale"] * angle.sin()).float()[:, None]
    half = s["inv_freq"].numel()

    def rotated(x):
        y = x.float()
        if s["layout"] == "half":
            a, b, rest = y[..., :half], y[..., half:2 * half], y[..., 2 * half:]
            return torch.cat([a * cos - b * sin, a * sin + b * cos, rest], -1).to(x.dtype)
        a, b, rest = y[..., 0:2 * half:2], y[..., 1:2 * half:2], y[..., 2 * half:]
        pairs = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
        return torch.cat([pairs, rest], -1).to(x.dtype)

    s["k_cache"].view(-1, *k.shape[1:])[s["slots"]] = rotated(k)
    s["v_cache"].view(-1, *v.shape[1:])[s["slots"]] = v
    return dict(q=rotated(q), k_cache=s["k_cache"], v_cache=s["v_cache"])


def run_attend(s):
    q, k_cache, v_cache, table, lens, q_start = s["q"], s["k_cache"], s["v_cache"], s["table"], s["lens"], s["q_start"]
    if own:
        from paper_2010_02164_amd import paged_attention
        return paged_attention(q, k_cache, v_cache, table, lens, q_start, max_q=s["max_q"], max_kv=s["max_kv"],
                               window=s["window"], sinks=s["sinks"])
    T, Hq, D = q.shape
    B, Hkv, S, Q = table.shape[0], k_cache.shape[2], s["max_kv"], s["max_q"]
    page = k_cache.shape[1]
    dev = q.device
    # Every request's keys and values side by side, [B, Hkv, S, D].
    j = torch.arange(S, device=dev)
    at = table[:, j // page].clamp(min=0).long() * page + j % page
    keys = k_cache.view(-1, Hkv, D)[at].float().permute(0, 2, 3, 1).contiguous()
    vals = v_cache.view(-1, Hkv, D)[at].float().transpose(1, 2).contiguous()
    # Its queries likewise, [B, Hkv, Q * group, D].
    i = torch.arange(Q, device=dev)
    count = q_start[1:] - q_start[:-1]
    row = (q_start[:-1, None] + i).clamp(max=T - 1)
    queries = q[row.long()].float().view(B, Q, Hkv, Hq // Hkv, D).transpose(1, 2).reshape(B, Hkv, -1, D)
    scores = torch.matmul(queries, keys).view(B, Hkv, Q, Hq // Hkv, S) * (1.0 / math.sqrt(D))
    p = (lens - count)[:, None, None] + i[:, None]
    seen = (j <= p) & (j < lens[:, None, None])
    if s["window"]:
        seen &= (j > p - s["window"]) | (j < s["sinks"])
    scores = scores.masked_fill(~seen[:, None, :, None], -torch.inf)
    top = scores.amax(-1, keepdim=True)
    w = torch.exp(scores - torch.where(top == -torch.inf, 0.0, top))
    total = w.sum(-1, keepdim=True)
    w = w / torch.where(total == 0, 1.0, total)
    got = torch.matmul(w.view(B, Hkv, -1, S), vals).view(B, Hkv, Q, Hq // Hkv, D).transpose(1, 2).reshape(B, Q, Hq, D)
    request = torch.searchsorted(q_start[1:].contiguous(), torch.arange(T, device=dev), right=True)
    return got[request, torch.arange(T, device=dev) - q_start[request]].to(q.dtype)


def run_sample(s):
    if own:
        from paper_2010_02164_amd import sample_tokens
        tokens, logprobs = sample_tokens(s["logits"], s["u"], temperature=s["temperature"], top_k=s["top_k"],
                                         top_p=s["top_p"], min_p=s["min_p"])
        return dict(tokens=tokens, logprobs=logprobs)
    z = s["logits"].double()
    rows, V = z.shape
    top = z.amax(1, keepdim=True)
    T = s["temperature"].double()[:, None]
    greedy = T <= 0
    w = torch.exp((z - top) / torch.where(greedy, 1.0, T))
    z, order = torch.sort(z, dim=1, descending=True, stable=True)
    ws = w.gather(1, order)
    rank = torch.arange(V, device=z.device)
    k = s["top_k"][:, None]
    ws = torch.where((rank < k) | (k <= 0), ws, 0.0)
    before = ws.cumsum(1) - ws
    p = s["top_p"].double()[:, None]
    ws = torch.where((before < p * ws.sum(1, keepdim=True)) | (p >= 1) | (rank == 0), ws, 0.0)
    ws = torch.where(ws >= s["min_p"].double()[:, None].clamp(max=1), ws, 0.0)
    ws = torch.where(greedy & (rank > 0), 0.0, ws)
    w = torch.zeros_like(w).scatter_(1, order, ws)
    mass = w.cumsum(1)
    token = (mass <= s["u"].double()[:, None] * mass[:, -1:]).sum(1)
    token = torch.minimum(token, torch.where(w > 0, rank, 0).amax(1))
    logprob = (w.gather(1, token[:, None])[:, 0] / mass[:, -1]).log()
    return dict(tokens=token.int(), logprobs=logprob.float())


def work(case):
    """Bytes read and written once, and operations, of one pass."""
    kind = case["kind"]
    if kind == "plan":
        have, add = _lengths(case, torch.Generator().manual_seed(0))
        T = int(np.maximum(add, 0).sum())
        return dict(bytes=case["B"] * 20 + T * 12, flops=0)
    es = SIZES[case["dtype"]]
    if kind == "rope":
        per = (case["Hq"] + 2 * case["Hkv"]) * case["D"]
        return dict(bytes=case["T"] * (2 * per * es + 12), flops=case["T"] * (case["Hq"] + case["Hkv"]) * case["rot"] * 3)
    if kind == "sample":
        return dict(bytes=case["rows"] * (case["V"] * es + 28), flops=case["rows"] * case["V"] * 20)
    lens, new = _lengths(case, torch.Generator().manual_seed(0))
    bytes_, pairs = 0, 0
    for n, m in zip(lens.tolist(), new.tolist()):
        p = np.arange(n - m, n)
        low = np.maximum(p + 1 - case["window"], 0) if case["window"] else np.zeros_like(p)
        pairs += int((p + 1 - low + np.minimum(low, case["sinks"])).sum())
        keys = n - int(low[0]) + min(int(low[0]), case["sinks"])
        bytes_ += 2 * m * case["Hq"] * case["D"] * es + 2 * keys * case["Hkv"] * case["D"] * es + -(-keys // case["page"]) * 4
    return dict(bytes=bytes_, flops=4 * pairs * case["Hq"] * case["D"])


def exact(case, seed):
    """The outputs in 64 bits from the definitions, request by request and
    row by row."""
    kind = case["kind"]
    if kind == "plan":
        return None
    s = prepare(case, seed)
    if kind == "sample":
        return _exact_sample(s)
    if kind == "rope":
        angle = s["positions"][:, None].double() * s["inv_freq"]
        turn = s["mscale"] * torch.exp(1j * angle)
        n = 2 * s["inv_freq"].numel()

        def turned(x):
            x = x.double()
            if s["layout"] == "half":
                c = torch.complex(x[..., :n // 2], x[..., n // 2:n]) * turn[:, None]
                return torch.cat([c.real, c.imag, x[..., n:]], -1)
            c = torch.view_as_complex(x[..., :n].unflatten(-1, (-1, 2)).contiguous()) * turn[:, None]
            return torch.cat([torch.view_as_real(c).flatten(-2), x[..., n:]], -1)

        k_cache, v_cache = s["k_cache"].double(), s["v_cache"].double()
        page = k_cache.shape[1]
        k_cache[s["slots"] // page, s["slots"] % page] = turned(s["k"])
        v_cache[s["slots"] // page, s["slots"] % page] = s["v"].double()
        return dict(q=turned(s["q"]), k_cache=k_cache, v_cache=v_cache)
    page, Hq, Hkv, D = case["page"], case["Hq"], case["Hkv"], case["D"]
    lens, starts = s["lens"].tolist(), s["q_start"].tolist()
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    for b, n in enumerate(lens):
        pages = s["table"][b, :-(-n // page)].long()
        keys = s["k_cache"][pages].reshape(-1, Hkv, D)[:n].double()
        vals = s["v_cache"][pages].reshape(-1, Hkv, D)[:n].double()
        lo, hi = starts[b], starts[b + 1]
        far = torch.arange(n - (hi - lo), n, device="cuda")[:, None] - torch.arange(n, device="cuda")
        hidden = far < 0
        if case["window"]:
            hidden |= (far >= case["window"]) & (torch.arange(n, device="cuda") >= case["sinks"])
        for h in range(Hq):
            x = s["q"][lo:hi, h].double() @ keys[:, h * Hkv // Hq].T.contiguous() / math.sqrt(D)
            out[lo:hi, h] = torch.softmax(x.masked_fill(hidden, -math.inf), -1) @ vals[:, h * Hkv // Hq].contiguous()
    return out


def _exact_sample(s):
    z_all, u = s["logits"].double().cpu().numpy(), s["u"].double().cpu().numpy()
    T, top_k, top_p, min_p = (s[n].cpu().numpy() for n in ("temperature", "top_k", "top_p", "min_p"))
    tokens, logprobs = [], []
    for r, z in enumerate(z_all):
        order = np.argsort(-z, kind="stable")
        if T[r] <= 0:
            order = order[:1]
        if top_k[r] > 0:
            order = order[:top_k[r]]
        w = np.exp((z[order] - z[order[0]]) / (np.float64(T[r]) if T[r] > 0 else 1.0))
        keep = len(order)
        if top_p[r] < 1:
            keep = max(1, int(np.searchsorted(np.cumsum(w), np.float64(top_p[r]) * w.sum(), side="left")) + 1)
        keep = min(keep, int((w >= min(np.float64(min_p[r]), 1.0)).sum()))
        back = np.argsort(order[:keep])
        left, mass = order[:keep][back], np.cumsum(w[:keep][back])
        at = min(int(np.searchsorted(mass, u[r] * mass[-1], side="right")), keep - 1)
        tokens.append(int(left[at]))
        logprobs.append(math.log(w[back][at] / mass[-1]))
    return dict(tokens=np.array(tokens, np.int32), logprobs=np.array(logprobs))
