"""Products in 8-bit integers by each of their kernels, over depths and remainders
at which it can go wrong, against the same product in 64 bits. Which kernel a size
gets is looked at in test_serve_plan_cpu.py.

Sums of int8 products are whole numbers below 2^53, exact in 64 bits. A result is off
by half a step of its type, and 16-bit ones by the fp32 operations before, 2^-24 each:
three of the product (the sum's rounding, the scales' product, the product of both)
and one of the result with a bias; fp16 results below its normal numbers by half a step
of those, 2^-25."""
import pytest
import torch

import paper_2010_02164_amd as sb

pytestmark = pytest.mark.gpu
BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32

FORMS = {   # (tile, splits, rows' products of a few-row kernel): rows, channels, depths
    "few_16": [(1, 70, 16400), (13, 1001, 8240), (16, 129, 3664), (16, 4096, 4112), (9, 33, 80)],
    "few_32": [(17, 3333, 1008), (20, 4097, 4112), (32, 5000, 2064), (31, 640, 4096), (25, 100, 400), (29, 2000, 6160)],
    "few_64": [(50, 4000, 4096), (61, 6144, 4112), (64, 8192, 4096), (50, 8191, 1616), (47, 3001, 2064), (33, 65, 784), (64, 300, 1616)],
    # 256 x 256: one step of the depth to six, whole and not
    "tiles_256": [(1900, 4700, 16), (2001, 4500, 128), (2049, 4097, 144), (2000, 4500, 256), (1793, 4400, 304), (2100, 4100, 400), (2000, 4500, 512),
                  (1800, 4600, 528), (2050, 4100, 656)],
    "tiles_128": [(65, 257, 16), (300, 5000, 96), (130, 130, 144), (257, 513, 272), (700, 3100, 400), (2048, 4096, 1008), (64, 9000, 2064)],
    "split": [(64, 999, 8192), (129, 257, 6160), (931, 313, 6272), (64, 2500, 6160), (33, 4200, 4112), (29, 2000, 8208), (300, 260, 2064)],
}


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("form,M,N,K", [(f, *s) for f in FORMS for s in FORMS[f]])
def test_linear_by_kernel(gpu, form, M, N, K, dtype):
    """Rows within wider ones that hold other codes, the result's at an odd place."""
    g = torch.Generator(device="cuda").manual_seed(M + N + K)
    x, w = (torch.randint(-128, 128, (n, K + 48), generator=g, device="cuda", dtype=torch.int8)[:, 16:16 + K] for n in (M, N))
    xs, ws = (torch.exp(torch.randn(n, generator=g, device="cuda")) * 1e-3 for n in (M, N))
    bias = torch.randn(N, generator=g, device="cuda")
    sums = x.double() @ w.double().t().contiguous()
    size = sums.abs_().mul_(xs.double()[:, None]).mul_(ws.double())
    plain = (x.double() @ w.double().t().contiguous()).mul_(xs.double()[:, None]).mul_(ws.double())
    eps, before, least = torch.finfo(dtype).eps, 2.0 ** -50 if dtype == F32 else 3 * 2.0 ** -24, 2.0 ** -25 if dtype == F16 else 0.0
    for b in (None, bias):
        want = plain if b is None else plain + b.double()
        tol = want.abs() * (eps / 2 + (0.0 if dtype == F32 or b is None else 2.0 ** -24 * (1 + eps))) + before * size + least
        whole = sb.int8_linear(x, xs, w, ws, bias=b, dtype=dtype)
        d = (whole.double() - want).abs()
        assert bool((d <= tol * (1 + 1e-12)).all()), (torch.nonzero(d > tol)[:5].tolist(), float((d / tol).max()))
        out = torch.full((M, N + 6), 5.0, dtype=dtype, device="cuda")
        sb.int8_linear(x, xs, w, ws, bias=b, out=out[:, 1:1 + N])
        assert torch.equal(out[:, 1:1 + N], whole) and bool((out[:, :1] == 5).all()) and bool((out[:, 1 + N:] == 5).all())
