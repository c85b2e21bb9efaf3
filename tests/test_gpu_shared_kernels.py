"""Attention over a shared prefix by each pair of its passes' kernels, with the
tolerances of test_gpu_shared_attention.py. Which pair a step gets is looked at in
test_serve_plan_cpu.py."""
import math

import numpy as np
import pytest
import torch

import paper_2010_02164_amd as sb
from test_gpu_shared_attention import bounds, case, check

pytestmark = pytest.mark.gpu
BF16, F16 = torch.bfloat16, torch.float16

KINDS = {   # (of the prefix, of the own tokens; 1 and 2: 16 and 32 rows by waves, 8: 128 by workgroups): members, Hq, Hkv, queries
    (1, 1): [([1], 16, 1, [1]), ([4, 3], 4, 1, [1]), ([2], 12, 4, [1, 2])],
    (2, 1): [([2], 16, 1, [1]), ([3, 5], 8, 2, [2, 1])],
    (8, 1): [([3], 16, 1, [1]), ([20], 8, 4, [3, 1]), ([40, 1, 9], 6, 2, [1])],
    (2, 2): [([1], 16, 1, [2]), ([1, 1], 16, 2, [4, 3]), ([2], 10, 1, [2, 1])],
    (8, 2): [([2], 16, 1, [3]), ([5, 1], 12, 1, [1, 5]), ([12], 9, 3, [2, 6])],
    (8, 8): [([1], 16, 1, [9]), ([3, 2], 8, 2, [40, 1, 17]), ([2], 3, 3, [65, 130])],
}


@pytest.mark.parametrize("dtype,D", [(BF16, 64), (BF16, 128), (BF16, 256), (F16, 64), (F16, 128), (F16, 256)])
@pytest.mark.parametrize("members,Hq,Hkv,q", [f for forms in KINDS.values() for f in forms])
def test_shared_attention_by_kernel(gpu, members, Hq, Hkv, q, dtype, D):
    """Prefixes of several pieces and of part of a tile; own tokens likewise; then
    with what nobody sees not finite, and with pages that are none."""
    for prefix, own in (([700, 90, 33], [150, 131, 140]), ([2100], [700, 130])):
        c = case(members, Hq, Hkv, D, 24, prefix, q, own, dtype, D + len(members))
        kw = bounds(c)
        clean = sb.shared_attention(**c, **kw)
        check(c, clean)
        used = torch.zeros(c["k_cache"].shape[:2], dtype=torch.bool, device="cuda")
        for table, lens in ((c["table"], c["lens"]), (c["prefix_table"], c["prefix_lens"])):
            j = np.concatenate([np.asarray(row)[np.arange(n) // 24] * 24 + np.arange(n) % 24 for row, n in zip(table.tolist(), lens.tolist())])
            used.view(-1)[torch.as_tensor(j).cuda()] = True
        for bad in (math.nan, -math.inf):
            odd = dict(c, k_cache=c["k_cache"].masked_fill(~used[..., None, None], bad), v_cache=c["v_cache"].masked_fill(~used[..., None, None], bad))
            assert torch.equal(sb.shared_attention(**odd, **kw), clean)
        c["prefix_table"][0, 1], c["table"][0, 2], c["table"][-1, 0] = -1, 10 ** 6, -5
        check(c, sb.shared_attention(**c, **kw))
