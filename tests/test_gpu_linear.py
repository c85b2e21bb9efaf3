"""Products in 8-bit integers on the GPU against their fp64 oracle.

Codes and scales have to be equal. Products: the sums are exact, so that a
result is off by one rounding to its type (eps / 2 of the value) and, but for
fp32 results, by the fp32 operations before: the sum's rounding, the scales'
product, the product of both and the bias's addition, 2^-24 of the product (of
the result) each. Results below fp16's or fp32's normal numbers are off by half
a step of those, 2^-25 or 2^-150; fp32 results are computed in fp64."""
import math

import numpy as np
import pytest
import torch

import paper_2010_02164_amd as sb
from oracle import serving as oracle

pytestmark = pytest.mark.gpu
BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32


def f64(t):
    return t.double().cpu().numpy()


def check_quantize(x, got):
    codes, scales = oracle.quantize_rows(f64(x))
    assert np.array_equal(got[1].cpu().numpy(), scales, equal_nan=True)
    assert torch.equal(got[0].cpu().long(), torch.as_tensor(codes))


def check_linear(x, xs, w, ws, bias, got):
    want, size = oracle.linear(x.cpu().numpy(), f64(xs), w.cpu().numpy(), f64(ws), None if bias is None else f64(bias))
    eps, least = torch.finfo(got.dtype).eps, {BF16: 0.0, F16: 2.0 ** -25, F32: 2.0 ** -150}[got.dtype]
    before = 2.0 ** -50 if got.dtype == F32 else 3 * 2.0 ** -24
    tol = eps / 2 * np.abs(want) + before * size + (0 if got.dtype == F32 or bias is None else 2.0 ** -24 * np.abs(want)) * (1 + eps) + least
    d = np.abs(f64(got) - want)
    assert np.all(d <= tol * (1 + 1e-12)), (np.argwhere(~(d <= tol))[:5], np.nanmax(d / tol))


def operands(M, N, K, seed, spread=1.0):
    """K: codes in use, the rest of 16 zeros."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    wide = -(-K // 16) * 16
    x, w = (torch.randint(-128, 128, (n, wide), generator=g, device="cuda", dtype=torch.int8) for n in (M, N))
    x[:, K:] = 0
    xs, ws = (torch.exp(spread * torch.randn(n, generator=g, device="cuda")) * 1e-3 for n in (M, N))
    return x, xs, w, ws, torch.randn(N, generator=g, device="cuda")


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 4096), (3, 15), (5, 16), (4, 17), (7, 100), (9, 1023), (6, 1024), (2, 1025), (3, 1041), (5, 8191),
                                       (2, 8200), (2, 40007), (1, 131056), (1030, 65)])
def test_quantize(gpu, rows, cols, dtype):
    g = torch.Generator(device="cuda").manual_seed(rows + cols)
    x = (torch.randn(rows, cols, generator=g, device="cuda") * torch.exp(2 * torch.randn(rows, 1, generator=g, device="cuda"))).to(dtype)
    got = sb.quantize_rows(x)
    assert got[0].shape == (rows, -(-cols // 16) * 16)
    check_quantize(x, got)


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
def test_quantize_borders(gpu, dtype):
    """Quotients on and next to the borders between two codes, in rows of all
    sizes down to the smallest numbers."""
    tiny = torch.finfo(dtype).smallest_normal
    rows = []
    for scale in (1.0, 2.0, 1 / 127, 3.0, tiny, tiny / 2 ** 5, 127 * tiny, 2.0 ** 7):
        half = (torch.arange(-127, 127, dtype=torch.float64) + 0.5) * scale
        row = torch.cat([half, torch.tensor([127.0 * scale, 0.0, -0.0], dtype=torch.float64)]).to(dtype)
        rows += [row, torch.nextafter(row.float(), torch.tensor(math.inf)).to(dtype), torch.nextafter(row.float(), torch.tensor(0.0)).to(dtype)]
    x = torch.stack(rows).cuda()
    check_quantize(x, sb.quantize_rows(x))
    least = torch.zeros(4, 40, dtype=dtype)   # the smallest numbers there are, the largest
    step = torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps
    least[0, 3], least[1, 7], least[1, 8] = step, -126 * step, 63 * step
    least[2] = torch.finfo(dtype).max
    least[3, 1] = -torch.finfo(dtype).max
    least[3, 2] = torch.finfo(dtype).max / 254
    check_quantize(least.cuda(), sb.quantize_rows(least.cuda()))


@pytest.mark.parametrize("cols", [40, 1500, 5000])
def test_quantize_rows_of_coarse_scales(gpu, cols):
    """fp32 rows whose largest value is a few of the smallest steps: the scale is
    rounded to whole steps, so that quotients lie up to half above 127 and are cut
    off there."""
    tops = torch.cat([torch.arange(60, 260), torch.arange(300, 13000, 97)])
    x = torch.zeros(len(tops), cols, dtype=torch.float64)
    for i, part in enumerate((1.0, -1.0, 0.5, -0.97, 0.9, 0.01)):
        x[:, i * (cols // 7)] = (tops * part).trunc() * 2.0 ** -149
    x = x.float().cuda()
    check_quantize(x, sb.quantize_rows(x))


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("cols", [50, 3000, 9000])
def test_quantize_rows_that_are_not_finite(gpu, cols, dtype):
    x = torch.randn(8, cols, device="cuda").to(dtype)
    x[1, cols - 1], x[2, 0], x[4, cols // 2], x[6] = math.nan, math.inf, -math.inf, 0
    codes, scales = sb.quantize_rows(x)
    check_quantize(x, (codes, scales))
    w = torch.ones(3, codes.shape[1], dtype=torch.int8, device="cuda")
    y = sb.int8_linear(codes, scales, w, torch.ones(3, device="cuda"))
    assert y.isnan().all(1).tolist() == [False, True, True, False, True, False, False, False] and bool((y[6] == 0).all())


def test_quantize_strides_and_out(gpu):
    """Slices at odd places, into a slice."""
    wide = torch.randn(20, 300, device="cuda").half()
    for a, b in ((0, 300), (1, 300), (8, 260), (3, 4)):
        x = wide[::2, a:b]
        want = sb.quantize_rows(x.contiguous())
        check_quantize(x, want)
        codes = torch.full((10, 400), 7, dtype=torch.int8, device="cuda")
        scales = torch.empty(10, device="cuda")
        n = want[0].shape[1]
        got = sb.quantize_rows(x, out=(codes[:, 32:32 + n], scales))
        assert torch.equal(got[0], want[0]) and torch.equal(scales, want[1])
        assert bool((codes[:, :32] == 7).all()) and bool((codes[:, 32 + n:] == 7).all())
    one = wide[:1].expand(5, 300)   # (read only: rows may be one)
    assert torch.equal(sb.quantize_rows(one)[0], sb.quantize_rows(one.contiguous())[0])


SHAPES = [(1, 1, 16), (1, 5, 48), (1, 4096, 4096), (2, 64, 100), (7, 33, 1000), (16, 129, 64), (17, 640, 4096), (31, 100, 272), (33, 65, 500),
          (64, 300, 2064), (65, 257, 128), (100, 96, 5000), (130, 130, 130), (200, 1000, 1000), (257, 513, 1040), (600, 255, 320), (1000, 31, 4000),
          (300, 2200, 96), (1025, 1025, 112),
          # tiles whose depth is split (several rows and channels behind the last), many rounds of steps
          (90, 130, 2048), (31, 200, 8000), (64, 999, 8192), (129, 257, 6160), (931, 313, 6263), (20, 100, 40000), (300, 260, 1030),
          (2000, 4500, 640), (4100, 4200, 272)]


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("M,N,K", SHAPES)
def test_linear(gpu, M, N, K, dtype):
    x, xs, w, ws, bias = operands(M, N, K, M + N + K)
    for b in (None, bias):
        check_linear(x, xs, w, ws, b, sb.int8_linear(x, xs, w, ws, bias=b, dtype=dtype))


@pytest.mark.parametrize("M", [1, 20, 70, 300])
def test_linear_largest_sums(gpu, M):
    """All codes -128 at the greatest depth: 131056 * 2^14 is below 2^31."""
    x, w = (torch.full((n, 131056), -128, dtype=torch.int8, device="cuda") for n in (M, 17))
    w[3] = 127
    one = torch.ones(M, device="cuda"), torch.ones(17, device="cuda")
    got = sb.int8_linear(x, one[0], w, one[1], dtype=F32)
    want = torch.full((M, 17), 131056.0 * 128 * 128, device="cuda")
    want[:, 3] = -131056.0 * 128 * 127
    assert torch.equal(got, want)


@pytest.mark.parametrize("M", [3, 40, 300])
def test_linear_scales_of_all_sizes(gpu, M):
    """Scales whose product with a sum, or with each other, leaves fp32's range
    while the result is within it; zeros, and channels that are not finite."""
    x, xs, w, ws, bias = operands(M, 50, 200, 7)
    for a, b in ((1e30, 1e-30), (1e-38, 1e36), (1e-42, 1e38), (3e38, 1e-40), (0.0, 1.0)):
        xs[:], ws[:] = a, b
        for dtype in (BF16, F32):
            check_linear(x, xs, w, ws, bias, sb.int8_linear(x, xs, w, ws, bias=bias, dtype=dtype))
    xs[:], ws[:] = 1e-3, 1e-3
    ws[4], bias[9], xs[1] = math.nan, math.inf, math.nan
    y = sb.int8_linear(x, xs, w, ws, bias=bias)
    assert bool(y[:, 4].isnan().all()) and bool(y[1].isnan().all())
    assert bool((y[0, 9] == math.inf)) and int((~torch.isfinite(y[0])).sum()) == 2


@pytest.mark.parametrize("M,N,K", [(5, 70, 160), (50, 131, 1024), (140, 150, 336), (100, 150, 4112)])
@pytest.mark.parametrize("dtype", [BF16, F32])
def test_linear_strides(gpu, M, N, K, dtype):
    """Rows within wider ones, which hold other codes behind their ends, into a
    slice at an odd place."""
    x, xs, w, ws, bias = operands(M, N, K, 3)
    want = sb.int8_linear(x, xs, w, ws, bias=bias, dtype=dtype)
    check_linear(x, xs, w, ws, bias, want)
    wx, ww = torch.full((M, K + 48), 99, dtype=torch.int8, device="cuda"), torch.full((N, K + 32), -99, dtype=torch.int8, device="cuda")
    wx[:, 16:16 + K], ww[:, 32:] = x, w
    for at in (0, 1, 8):
        out = torch.full((M, N + 13), 5.0, dtype=dtype, device="cuda")
        got = sb.int8_linear(wx[:, 16:16 + K], xs, ww[:, 32:], ws, bias=bias, out=out[:, at:at + N])
        assert torch.equal(got, want)
        assert bool((out[:, :at] == 5).all()) and bool((out[:, at + N:] == 5).all())


def test_linear_workspace(gpu):
    """Asked for where the depth is split, refused where it is too small; what stands
    in it before the call does not matter."""
    N = sb.decoder.N
    x, xs, w, ws, _ = operands(100, 150, 4112, 5)
    out = torch.empty(100, 150, device="cuda")
    args = N.LINEAR_ARGS.pack(N.LINEAR_ARGS.size, x.data_ptr(), w.data_ptr(), xs.data_ptr(), ws.data_ptr(), 0, out.data_ptr(), 4112, 4112, 150,
                              100, 150, 4112, N.SB_F32)
    L = N.lib()
    need = L.sb_linear_workspace(args)
    assert need > 0
    work = torch.full((need + 256,), 0x7F, dtype=torch.uint8, device="cuda")
    stream = torch.cuda.current_stream().cuda_stream
    assert L.sb_quantized_linear(args, None, 0, stream) == N.SB_E_WORKSPACE
    assert L.sb_quantized_linear(args, work.data_ptr(), need - 1, stream) == N.SB_E_WORKSPACE
    assert L.sb_quantized_linear(args, work.data_ptr() + 64, need, stream) == N.SB_E_WORKSPACE
    assert L.sb_quantized_linear(args, work.data_ptr(), need, stream) == N.SB_OK
    check_linear(x, xs, w, ws, None, out)
    assert bool((work[need:] == 0x7F).all())


def test_linear_refusals(gpu):
    x, xs, w, ws, bias = operands(4, 8, 64, 1)
    for over, match in ((dict(w=w[:, :48]), "columns"), (dict(x_scale=xs[:3]), "x_scale"), (dict(w_scale=ws.double()), "w_scale"),
                        (dict(bias=bias[:7]), "bias"), (dict(dtype=torch.float64), "dtype"), (dict(x=x.int()), "x must"),
                        (dict(out=torch.empty(4, 9, device="cuda")), "columns"), (dict(out=torch.empty(3, 8, device="cuda")), "rows"),
                        (dict(w=w.cpu()), "w must"), (dict(bias=bias.clone().requires_grad_()), "backward"),
                        (dict(out=torch.empty(1, 8, device="cuda").expand(4, 8)), "overlap")):
        with pytest.raises(ValueError, match=match):
            sb.int8_linear(**dict(dict(x=x, x_scale=xs, w=w, w_scale=ws, bias=bias), **over))
    with pytest.raises(sb.decoder.N.StreambeamError, match="multiple of 16"):
        sb.int8_linear(x[:, :40], xs, w[:, :40], ws)
    with pytest.raises(ValueError, match="backward"):
        sb.quantize_rows(torch.randn(3, 4, device="cuda", requires_grad=True))
    with pytest.raises(ValueError, match="matrix"):
        sb.quantize_rows(torch.randn(3, 4, device="cuda").t())


def test_linear_of_no_rows(gpu):
    w = torch.ones(5, 32, dtype=torch.int8, device="cuda")
    codes, scales = sb.quantize_rows(torch.empty(0, 20, device="cuda"))
    assert codes.shape == (0, 32) and scales.shape == (0,)
    assert sb.int8_linear(codes, scales, w, torch.ones(5, device="cuda")).shape == (0, 5)


def test_linear_captured_and_on_other_streams(gpu):
    """Several products in one graph, replayed with other rows; two streams at once."""
    layers = [operands(24, n, k, n) for n, k in ((500, 256), (300, 4096), (33, 64))]
    xs = [torch.randn(24, layer[0].shape[1], device="cuda").to(BF16) for layer in layers]

    def step():
        out = []
        for x, (_, _, w, ws, bias) in zip(xs, layers):
            codes, scales = sb.quantize_rows(x)
            out.append(sb.int8_linear(codes, scales, w, ws, bias=bias, dtype=F32))
        return out

    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for t in range(4):
        for x in xs:
            x.copy_(torch.randn(x.shape, device="cuda") * (t + 1))
        graph.replay()
        for a, b in zip(held, step()):
            assert torch.equal(a, b), t
        torch.cuda.synchronize()
    want = step()
    side = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = []
    for stream in side:
        with torch.cuda.stream(stream):
            got.append([step() for _ in range(3)])
    torch.cuda.synchronize()
    for runs in got:
        for one in runs:
            assert all(torch.equal(a, b) for a, b in zip(one, want))
