"""The serving operators without a GPU: their oracle's pins, the layout of
their argument structs, and the refusals, which enqueue nothing."""
import math
import os
import re

import numpy as np
import pytest
import torch

import paper_2010_02164_amd as sb
from oracle import serving as oracle
from paper_2010_02164_amd import _native as N

PTR = 0x10000   # never read: every call here is refused first

PLAN = dict(bytes=N.PLAN_ARGS.size, lens=PTR, add=PTR, n_free=PTR, free_list=PTR, table=PTR, lens_out=PTR, n_free_out=PTR, q_start=PTR,
            granted=PTR, slots=PTR, positions=PTR, table_stride=8, n_requests=4, n_pages=32, page_size=16, max_pages=8, token_cap=64,
            reserved=0)
ROPE = dict(bytes=N.ROPE_ARGS.size, q=PTR, k=PTR, v=PTR, q_out=PTR, k_cache=PTR, v_cache=PTR, positions=PTR, slots=PTR, inv_freq=PTR,
            q_token=512, q_head=128, k_token=256, k_head=128, v_token=256, v_head=128, out_token=512, out_head=128, kc_page=4096,
            kc_slot=256, kc_head=128, vc_page=4096, vc_slot=256, vc_head=128, n_tokens=3, q_heads=4, kv_heads=2, head_dim=128, n_pairs=64,
            layout=0, dtype=N.SB_BF16, n_pages=32, page_size=16, mscale=1.0)
ATTN = dict(bytes=N.ATTENTION_ARGS.size, q=PTR, k_cache=PTR, v_cache=PTR, table=PTR, lens=PTR, q_start=PTR, out=PTR, q_token=512,
            q_head=128, out_token=512, out_head=128, kc_page=4096, kc_slot=256, kc_head=128, vc_page=4096, vc_slot=256, vc_head=128,
            table_stride=8, n_tokens=3, n_requests=2, q_heads=4, kv_heads=2, head_dim=128, dtype=N.SB_BF16, n_pages=32, page_size=16,
            max_pages=8, window=0, sinks=0, max_q=2, max_kv=100, scale=0.1)
SAMPLE = dict(bytes=N.SAMPLE_ARGS.size, logits=PTR, u=PTR, temperature=PTR, top_k=PTR, top_p=PTR, min_p=PTR, tokens=PTR, logprobs=PTR,
              row_stride=1000, rows=3, vocab=1000, dtype=N.SB_F32, reserved=0)
STRUCTS = {"sb_plan_args": (N.PLAN_ARGS, PLAN), "sb_rope_args": (N.ROPE_ARGS, ROPE), "sb_attention_args": (N.ATTENTION_ARGS, ATTN),
           "sb_sample_args": (N.SAMPLE_ARGS, SAMPLE)}


@pytest.mark.parametrize("name", sorted(STRUCTS))
def test_packed_arguments_follow_the_header(name):
    """The fields of the header's struct, in their order and types."""
    with open(N.HEADER) as f:
        body = re.search(r"typedef struct \{([^}]*)\} " + name, f.read()).group(1)
    body = re.sub(r"/\*.*?\*/", "", body, flags=re.S)
    fields, codes = [], ""
    for decl in body.split(";"):
        decl = decl.strip()
        if not decl:
            continue
        for part in re.sub(r"^(const )?(void|float|double|int32_t|int64_t) ", "", decl).split(","):
            pointer = "*" in part
            kind = re.match(r"(const )?(\w+)", decl).group(2)
            codes += "P" if pointer else {"int64_t": "q", "int32_t": "i", "float": "f"}[kind]
            fields.append(part.strip(" *"))
    packer, values = STRUCTS[name]
    expanded = "".join(c * int(n or 1) for n, c in re.findall(r"(\d*)([qPif])", packer.format))
    assert codes == expanded
    assert len(fields) == len(values) and ["bytes"] + fields[1:] == list(values)


def _refused(native_lib, call, base, over):
    packer = {id(PLAN): N.PLAN_ARGS, id(ROPE): N.ROPE_ARGS, id(ATTN): N.ATTENTION_ARGS, id(SAMPLE): N.SAMPLE_ARGS}[id(base)]
    assert not set(over) - set(base)
    args = packer.pack(*dict(base, **over).values())
    fn = getattr(native_lib, call)
    status = fn(args, None, 0, None) if call in ("sb_paged_attention", "sb_sample_tokens") else fn(args, None)
    if status != N.SB_OK:
        assert call in native_lib.sb_last_error(None).decode()
    return status


INVALID, UNSUPPORTED = N.SB_E_INVALID_ARG, N.SB_E_UNSUPPORTED


@pytest.mark.parametrize("over,status", [
    (dict(bytes=120), INVALID), (dict(reserved=1), INVALID), (dict(n_requests=0), INVALID), (dict(n_requests=8193), UNSUPPORTED),
    (dict(n_pages=0), INVALID), (dict(page_size=0), INVALID), (dict(page_size=4097), INVALID), (dict(max_pages=0), INVALID),
    (dict(token_cap=-1), INVALID), (dict(table_stride=7), INVALID), (dict(n_pages=1 << 27), UNSUPPORTED),
    (dict(max_pages=1 << 27, table_stride=1 << 27), UNSUPPORTED), (dict(slots=0), INVALID), (dict(lens=0), INVALID),
    (dict(slots=PTR + 4), INVALID), (dict(table=PTR + 2), INVALID)])
def test_plan_refusals(native_lib, over, status):
    assert _refused(native_lib, "sb_plan_pages", PLAN, over) == status


@pytest.mark.parametrize("over,status", [
    (dict(bytes=0), INVALID), (dict(dtype=N.SB_F32), UNSUPPORTED), (dict(layout=2), INVALID), (dict(n_tokens=-1), INVALID),
    (dict(q_heads=0), INVALID), (dict(kv_heads=1025), INVALID), (dict(head_dim=100), UNSUPPORTED), (dict(head_dim=520), UNSUPPORTED),
    (dict(n_pairs=72), INVALID), (dict(n_pairs=-8), INVALID), (dict(n_pairs=12), UNSUPPORTED),
    (dict(n_pairs=6, layout=1), UNSUPPORTED), (dict(n_pages=0), INVALID), (dict(page_size=5000), INVALID),
    (dict(mscale=math.inf), INVALID), (dict(mscale=math.nan), INVALID), (dict(q_token=516), UNSUPPORTED),
    (dict(kc_slot=-256), UNSUPPORTED), (dict(q=PTR + 8), UNSUPPORTED), (dict(v_cache=PTR + 2), UNSUPPORTED), (dict(q_out=0), INVALID),
    (dict(inv_freq=0), INVALID), (dict(inv_freq=PTR + 4), UNSUPPORTED), (dict(n_pages=1 << 28), UNSUPPORTED)])
def test_rope_refusals(native_lib, over, status):
    assert _refused(native_lib, "sb_rope_append", ROPE, over) == status


@pytest.mark.parametrize("over,status", [
    (dict(bytes=8), INVALID), (dict(dtype=N.SB_F32), UNSUPPORTED), (dict(head_dim=96), UNSUPPORTED), (dict(head_dim=512), UNSUPPORTED),
    (dict(n_requests=0), INVALID), (dict(n_tokens=-1), INVALID), (dict(q_heads=5), INVALID), (dict(kv_heads=0), INVALID),
    (dict(page_size=0), INVALID), (dict(max_pages=0), INVALID), (dict(window=-1), INVALID), (dict(sinks=-1), INVALID),
    (dict(max_q=-1), INVALID), (dict(max_kv=-1), INVALID), (dict(scale=math.nan), INVALID), (dict(table_stride=4), INVALID),
    (dict(q_head=124), UNSUPPORTED), (dict(vc_page=-8), UNSUPPORTED), (dict(lens=0), INVALID), (dict(out=0), INVALID),
    (dict(out=PTR + 8), UNSUPPORTED), (dict(n_tokens=1 << 30), UNSUPPORTED), (dict(n_pages=1 << 30), UNSUPPORTED)])
def test_attention_refusals(native_lib, over, status):
    assert _refused(native_lib, "sb_paged_attention", ATTN, over) == status
    if not {"lens", "out"} & set(over):   # (the workspace's size does not look at pointers)
        assert native_lib.sb_attention_workspace(N.ATTENTION_ARGS.pack(*dict(ATTN, **over).values())) == -1


@pytest.mark.parametrize("over,status", [
    (dict(bytes=104), INVALID), (dict(reserved=3), INVALID), (dict(dtype=3), UNSUPPORTED), (dict(rows=-1), INVALID),
    (dict(vocab=0), INVALID), (dict(vocab=262145, row_stride=262145), UNSUPPORTED), (dict(row_stride=999), INVALID),
    (dict(logits=0), INVALID), (dict(u=0), INVALID), (dict(tokens=0), INVALID), (dict(logits=PTR + 2), INVALID),
    (dict(top_k=PTR + 2), INVALID)])
def test_sample_refusals(native_lib, over, status):
    assert _refused(native_lib, "sb_sample_tokens", SAMPLE, over) == status


def test_attention_keys_stay_below_32_bits(native_lib):
    """Tiles of up to 64 keys are looked up four ahead of the last one, numbered in
    32 bits: a table that ends within 320 keys of 2^31 cannot be taken."""
    most = 2 ** 31 - 1024
    for page, fits in ((1, most), (16, most // 16), (4096, most // 4096)):
        for pages in (fits, fits + 1, (2 ** 31 - 1) // page):
            status = N.SB_OK if pages * page <= most else UNSUPPORTED
            over = dict(page_size=page, max_pages=pages, table_stride=pages, n_pages=8)
            assert _refused(native_lib, "sb_paged_attention", ATTN, dict(over, n_tokens=0)) == status, over
            if status != N.SB_OK and pages * page < 2 ** 31:
                assert "MAX_KEYS" in native_lib.sb_last_error(None).decode()


def test_strides_of_one_place_are_not_looked_at(native_lib):
    one = dict(n_tokens=0, q_heads=1, kv_heads=1, n_pages=1, page_size=1)
    names = [n for n in ATTN if n.split("_")[-1] in ("token", "head", "page", "slot")]
    assert len(names) == 10
    odd = {n: 13 for n in names}
    assert _refused(native_lib, "sb_paged_attention", ATTN, dict(one, **odd)) == N.SB_OK
    for n in names:   # but those of several are
        places = dict(one, n_tokens=3, q_heads=2, kv_heads=2, n_pages=2, page_size=2)
        args = N.ATTENTION_ARGS.pack(*dict(ATTN, **places, **{n: 13}).values())
        assert native_lib.sb_attention_workspace(args) == -1 and "stride" in native_lib.sb_last_error(None).decode()
    # (What rope does with its tokens' strides needs a launch: in the tests on a GPU.)
    assert _refused(native_lib, "sb_rope_append", ROPE, dict(one, **odd, k_token=13, k_head=13, v_token=13, v_head=-7)) == N.SB_OK


def test_numbers_that_do_not_fit(native_lib):
    """A scale has to fit fp32 as the power of two that the kernels take; fields of
    whole numbers take no others."""
    for packer, base, over in ((N.PLAN_ARGS, PLAN, dict(page_size=16.5)), (N.SAMPLE_ARGS, SAMPLE, dict(rows=2 ** 31))):
        with pytest.raises(ValueError, match="does not fit"):
            packer.pack(*dict(base, **over).values())
    assert _refused(native_lib, "sb_rope_append", ROPE, dict(mscale=-1e39)) == INVALID
    for scale, status in ((2.35e38, N.SB_OK), (2.4e38, INVALID), (-3.4e38, INVALID), (1e300, INVALID), (0.0, N.SB_OK)):
        assert _refused(native_lib, "sb_paged_attention", ATTN, dict(scale=scale, n_tokens=0)) == status


def test_sample_workspace(native_lib):
    """Only many wide rows, or some with top-p, are faster with one; one that is
    too small is refused."""
    def ask(**over):
        return native_lib.sb_sample_workspace(N.SAMPLE_ARGS.pack(*dict(SAMPLE, **over).values()))
    wide = dict(rows=64, vocab=64000, row_stride=64000)
    assert ask() == 0 and ask(**dict(wide, rows=0)) == 0 and ask(**dict(wide, vocab=32000)) == 0
    assert ask(**dict(wide, rows=1)) > 0 and ask(**dict(wide, rows=1, top_p=0)) == 0
    need = ask(**wide)
    assert 0 < need and ask(**dict(wide, rows=128)) == 2 * need and ask(dtype=9) == -1
    args = N.SAMPLE_ARGS.pack(*dict(SAMPLE, **wide).values())
    assert native_lib.sb_sample_tokens(args, PTR, need - 1, None) == N.SB_E_WORKSPACE
    assert native_lib.sb_sample_tokens(args, PTR + 128, need, None) == N.SB_E_WORKSPACE


def test_missing_arguments(native_lib):
    assert native_lib.sb_plan_pages(None, None) == INVALID
    assert native_lib.sb_rope_append(None, None) == INVALID
    assert native_lib.sb_attention_workspace(None) == -1
    assert native_lib.sb_paged_attention(None, None, 0, None) == INVALID
    assert native_lib.sb_sample_workspace(None) == -1
    assert native_lib.sb_sample_tokens(None, None, 0, None) == INVALID


def test_nothing_to_do_needs_no_gpu(native_lib):
    assert _refused(native_lib, "sb_rope_append", ROPE, dict(n_tokens=0)) == N.SB_OK
    assert _refused(native_lib, "sb_paged_attention", ATTN, dict(n_tokens=0)) == N.SB_OK
    assert _refused(native_lib, "sb_sample_tokens", SAMPLE, dict(rows=0)) == N.SB_OK


def test_tensors_must_be_on_a_gpu():
    x = torch.zeros(2, 1, 64, dtype=torch.bfloat16)
    i = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError, match="GPU"):
        sb.sample_tokens(torch.zeros(2, 5), torch.zeros(2))
    with pytest.raises(ValueError, match="GPU"):
        sb.plan_pages(i, i, i, i, torch.zeros(2, 2, dtype=torch.int32), page_size=4, token_cap=3)
    with pytest.raises(ValueError, match="GPU"):
        sb.rope_append(x, x, x, i, i, x[None], x[None], torch.zeros(4, dtype=torch.float64))
    with pytest.raises(ValueError, match="GPU"):
        sb.paged_attention(x, x[None], x[None], i[None], i, i, max_q=1, max_kv=1)


def test_overlapping_outputs_are_found():
    from paper_2010_02164_amd.serving import _apart
    x = torch.zeros(6, 4, 8)
    for t in (x, x.transpose(0, 1), x[::2], x[:, 1:3], x[:, :, :0], x[:1].expand(1, 4, 8)):
        _apart(t, "x")
    for t in (x[:1].expand(3, 4, 8), torch.as_strided(x, (3, 8), (4, 1))):
        with pytest.raises(ValueError, match="overlap"):
            _apart(t, "x")


def test_gradients_and_tangents_are_refused():
    from torch.autograd import forward_ad

    from paper_2010_02164_amd.serving import _no_grad
    x, y = torch.zeros(3), torch.zeros(3, requires_grad=True)
    _no_grad(x, None)
    with pytest.raises(ValueError, match="backward"):
        _no_grad(x, y)
    with torch.no_grad():
        _no_grad(x, y)
    with forward_ad.dual_level():
        _no_grad(x, None)
        dual = forward_ad.make_dual(x, torch.ones(3))
        for mode in (torch.no_grad(), torch.enable_grad()):
            with mode, pytest.raises(ValueError, match="forward"):
                _no_grad(None, dual)
        _no_grad(forward_ad.unpack_dual(dual).primal)


def test_rope_frequencies():
    f, m = sb.rope_frequencies(8, base=100.0, device="cpu")
    assert f.dtype == torch.float64 and m == 1.0
    assert torch.allclose(f, torch.tensor([1.0, 100 ** -0.25, 0.1, 100 ** -0.75], dtype=torch.float64), rtol=1e-14)
    assert torch.equal(sb.rope_frequencies(8, base=100.0, scaling="linear", factor=4.0, device="cpu")[0], f / 4)
    n, _ = sb.rope_frequencies(8, base=100.0, scaling="ntk", factor=4.0, device="cpu")
    assert n[0] == 1 and math.isclose(n[-1], f[-1] / 4, rel_tol=1e-12)   # the slowest pair is slowed by the factor
    y, m = sb.rope_frequencies(128, scaling="parts", factor=8.0, original_length=4096, device="cpu")
    b = sb.rope_frequencies(128, device="cpu")[0]
    assert math.isclose(m, 1 + 0.1 * math.log(8))
    turns = 4096 * b / (2 * math.pi)
    assert torch.equal(y[turns > 36], b[turns > 36]) and torch.allclose(y[turns < 0.8], b[turns < 0.8] / 8, rtol=1e-12)
    assert bool((y[:-1] > y[1:]).all())
    for bad in (dict(rot_dim=7), dict(rot_dim=0), dict(rot_dim=8, scaling="what"), dict(rot_dim=8, factor=0.5), dict(rot_dim=8, base=1.0)):
        with pytest.raises(ValueError):
            sb.rope_frequencies(device="cpu", **bad)


@pytest.mark.parametrize("rot,base,length,factor", [(128, 10000.0, 131072, 8.0), (64, 10000.0, 65536, 4.0), (128, 500000.0, 8192, 8.0),
                                                    (8, 10000.0, 10 ** 9, 2.0)])
def test_rope_frequencies_in_parts(rot, base, length, factor):
    """Pair i turns length base^(-2 i / rot) / 2 pi times over the original length.
    The blend runs evenly from the whole number below the pair that turns 32 times
    to that above the one that turns once, which may lie behind the last pair:
    none that turns more than once is slowed by the whole factor."""
    got, _ = sb.rope_frequencies(rot, base=base, scaling="parts", factor=factor, original_length=length, device="cpu")
    ends = [rot / 2 * math.log(length / (2 * math.pi * n)) / math.log(base) for n in (32.0, 1.0)]
    lo, hi = max(math.floor(ends[0]), 0), min(math.ceil(ends[1]), rot - 1)
    for i in range(rot // 2):
        plain = base ** (-2 * i / rot)
        slowed = min(max((i - lo) / max(hi - lo, 1e-3), 0.0), 1.0)
        assert math.isclose(float(got[i]), plain * (1 - slowed) + plain / factor * slowed, rel_tol=1e-12), i
        if length * plain / (2 * math.pi) > 1:
            assert float(got[i]) > plain / factor * (1 + 1e-9), i


# -- pins of the oracle ------------------------------------------------------------

def test_oracle_plan_by_hand():
    # Pages of 4. Request 0 (5 cached) wants 4: fills page 7, takes one more;
    # 1 is released (pages 3, 9); 2 wants 1 with room left; 3 wants too much
    # for its row; 4 takes a page.
    table = [[6, 7, -1], [3, 9, -1], [2, -1, -1], [-1, -1, -1], [-1, -1, -1]]
    lens, granted, free, tab, slots, pos, q_start = oracle.plan_pages([5, 6, 2, 0, 0], [4, -1, 1, 13, 2], [1, 0], table, 4, 9)
    assert lens == [9, 0, 3, 0, 2] and granted == [4, 0, 1, 0, 2] and q_start == [0, 4, 4, 5, 5, 7]
    assert free == [1, 0]   # the released pages went out again: 9 to request 0, 3 to request 4
    assert tab.tolist() == [[6, 7, 9], [3, 9, -1], [2, -1, -1], [-1, -1, -1], [3, -1, -1]]
    assert slots == [29, 30, 31, 36, 10, 12, 13, -1, -1] and pos == [5, 6, 7, 8, 2, 0, 1, -1, -1]


def test_oracle_plan_stops_at_the_first_that_does_not_fit():
    table = np.full((3, 4), -1)
    _, granted, free, *_ = oracle.plan_pages([0, 0, 0], [4, 9, 1], [5, 6, 7], table, 4, 100)
    assert granted == [4, 0, 0] and free == [5, 6]   # by pages
    _, granted, *_ = oracle.plan_pages([0, 0, 0], [4, 5, 1], [5, 6, 7, 8], table, 4, 8)
    assert granted == [4, 0, 0]                      # by tokens


def test_oracle_rotation_by_hand():
    x = [1.0, 2.0, 3.0, 4.0, 5.0]
    half, _ = oracle.rotate(x, 1, [math.pi / 2, math.pi], "half", 1.0)
    assert np.allclose(half, [-3, -2, 1, -4, 5])
    pairs, size = oracle.rotate(x, 1, [math.pi / 2, math.pi], "interleaved", 2.0)
    assert np.allclose(pairs, [-4, 2, -6, -8, 5]) and np.allclose(size, [6, 6, 14, 14, 5])


def test_oracle_attention_by_hand():
    # One head of one value; three positions, pages of 2, the second row of
    # the table's page 0 behind the last token.
    k = np.array([[[[0.0]], [[9.0]]], [[[0.0]], [[math.log(3)]]]])
    v = np.array([[[[8.0]], [[9.0]]], [[[1.0]], [[5.0]]]])
    out, *_ = oracle.attention(np.ones((3, 1, 1)), k, v, [[1, 0]], [3], [0, 3], 0, 0, 1.0)
    assert np.allclose(out[:, 0, 0], [1, (1 + 15) / 4, (1 + 15 + 8) / 5])
    out, *_ = oracle.attention(np.ones((1, 1, 1)), k, v, [[1, 0]], [3], [0, 1], 1, 1, 1.0)
    assert np.allclose(out, (1 + 8) / 2)                 # the first token and itself
    out, *_ = oracle.attention(np.ones((2, 1, 1)), k, v, [[1, 0]], [1], [0, 2], 0, 0, 1.0)
    assert np.allclose(out[:, 0, 0], [0, 1])             # a query before the first position
    out, *_ = oracle.attention(np.ones((1, 1, 1)), k, v, [[1, 7]], [3], [0, 1], 1, 0, 1.0)
    assert np.allclose(out, 0)                           # its only key lies on no page


def test_oracle_sample_by_hand():
    z = [0.0, math.log(4), 0.0, math.log(2)]   # weights 1 4 1 2 of 8
    assert [oracle.sample(z, u)[0] for u in (0, 0.12, 0.13, 0.62, 0.63, 0.74, 0.76, 1.0)] == [0, 0, 1, 1, 2, 2, 3, 3]
    assert math.isclose(oracle.sample(z, 0.5)[1], math.log(0.5), abs_tol=1e-12)
    assert oracle.sample(z, 0.0, top_k=2) == (1, pytest.approx(math.log(4 / 6)))
    assert oracle.sample(z, 0.99, top_k=3)[0] == 3 and oracle.sample(z, 0.0, top_k=3)[0] == 0   # of two equals the first
    assert oracle.sample(z, 0.0, top_p=0.49)[0] == 1 and oracle.sample(z, 0.99, top_p=0.6)[0] == 3
    assert oracle.sample(z, 0.99, top_p=0.0)[0] == 1
    assert oracle.sample(z, 0.99, min_p=0.4)[0] == 3 and oracle.sample(z, 0.99, min_p=2.0)[0] == 1
    assert oracle.sample(z, 0.7, T=0.0) == (1, 0.0)
    assert oracle.sample([1.0, math.inf, math.nan, math.inf], 0.6)[0] == 3
    assert oracle.sample([-math.inf, math.nan], 0.5) == (-1, -math.inf)
    # top-k counts before top-p does: of the best two (4, 2 of 6) 0.7 keeps both, of all (8) 0.5 keeps one.
    assert oracle.sample(z, 0.99, top_k=2, top_p=0.7)[0] == 3 and oracle.sample(z, 0.99, top_p=0.5)[0] == 1
