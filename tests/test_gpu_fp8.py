"""8-bit output head on the GPU against the float64 oracle: codes and orders exact, scales, products and log probabilities within
bounds made of their roundings."""
import numpy as np
import pytest
import torch

from oracle import fp8

pytestmark = pytest.mark.gpu

U = 2.0 ** -24         # half a step of fp32
HALF_BF16 = 2.0 ** -8
DT = {"fp32": torch.float32, "bf16": torch.bfloat16}


def bits(codes):
    return codes.view(torch.uint8).cpu().numpy()


def check_scale(got, want, tol):
    got = got.double().cpu().numpy()
    assert np.array_equal(np.isnan(got), np.isnan(want))
    fine = ~np.isnan(want)
    assert np.all(np.abs(got - want)[fine] <= tol * np.abs(want[fine]) + 2.0 ** -149)


def norm_tol(K):
    """The sum of K squares in a thread's part and over threads (all terms positive), its half as a root, the reciprocal root of 2
    units (2^-22 each), the factor 1 / 448, and three products."""
    return (K / 512 + 40) / 2 * U + 2.0 ** -22 * 2 + 6 * U


# ------------------------------------------------------------------------------------------------ quantisers
@pytest.mark.parametrize("x", ["fp32", "bf16"])
@pytest.mark.parametrize("norm", [False, True])
@pytest.mark.parametrize("M,K", [(1, 16), (3, 64), (2, 128), (5, 144), (7, 1040), (33, 3200), (300, 4096), (4, 11008), (2, 16400), (3, 20000)])
def test_quant_rows(a48, cuda_dev, M, K, norm, x):
    rng = np.random.default_rng(M * K)
    v = rng.standard_normal((M, K)) * np.exp(rng.standard_normal((M, 1))) * np.where(rng.random(K) < 0.01, 20, 1)
    t = torch.tensor(v, dtype=torch.float32).to(DT[x])
    gain = torch.tensor(rng.uniform(0.5, 1.5, K), dtype=torch.float32) if norm else None
    codes, scale = a48.quant_fp8(t.to(cuda_dev), gain.to(cuda_dev) if norm else None, 1e-5)
    want, want_scale = fp8.quant_rows(t.double().numpy(), gain.double().numpy() if norm else None, float(np.float32(1e-5)))
    assert np.array_equal(bits(codes), want)
    check_scale(scale, want_scale, norm_tol(K) if norm else 2 * U)


@pytest.mark.parametrize("x", ["fp32", "bf16"])
@pytest.mark.parametrize("M,K", [(19003, 256), (19001, 272), (4802, 2048), (2403, 4096), (2401, 8208), (2402, 11008), (4001, 4112), (3701, 8208), (3601, 16384), (3601, 16400)])
def test_quant_many_rows_are_what_few_are(a48, cuda_dev, M, K, x):
    torch.manual_seed(M)
    h = torch.randn(M, K, device=cuda_dev) * torch.logspace(-12, 12, M, device=cuda_dev)[torch.randperm(M, device=cuda_dev), None]
    h = h.bfloat16() if x == "bf16" else h
    h[M // 2] = 0
    h[-1] = 1e-25  # its squares are none in fp32
    h[-2, K // 2] = float("nan")
    gain = torch.rand(K, device=cuda_dev) + 0.5
    codes, scale = a48.quant_fp8(h, gain)
    for first in range(0, M, 113):
        rows = slice(first, min(M, first + 113))
        c, s = a48.quant_fp8(h[rows], gain)
        assert torch.equal(c.view(torch.uint8), codes[rows].view(torch.uint8)) and torch.equal(s.view(torch.int32), scale[:, rows].contiguous().view(torch.int32))


@pytest.mark.parametrize("x", ["fp32", "bf16"])
@pytest.mark.parametrize("norm", [False, True])
def test_quant_ties_go_to_the_even_code(a48, cuda_dev, x, norm):
    """The largest entry is 448, 1.75 and 21 / 16 times powers of two, so that entries halfway between two codes are exact."""
    ties = np.concatenate([(fp8.GRID[1:] + fp8.GRID[:-1]) / 2, fp8.GRID])
    rows = []
    for peak in (448.0, 1.75, 448.0 * 21 / 16 / 7 * 4, 448 * 2.0 ** -20):
        row = np.zeros(384)
        row[:ties.size] = ties * peak / 448
        row[::2] *= -1
        row[[127, 255, 383]] = peak
        rows.append(row)
    t = torch.tensor(np.array(rows), dtype=torch.float32).to(DT[x])
    gain = torch.ones(384) if norm else None
    codes, _ = a48.quant_fp8(t.to(cuda_dev), gain.to(cuda_dev) if norm else None)
    assert np.array_equal(bits(codes), fp8.quant_rows(t.double().numpy())[0])


@pytest.mark.parametrize("norm", [False, True])
def test_quant_bf16_every_quotient(a48, cuda_dev, norm):
    """All pairs of an 8-bit mantissa of the largest entry and of another one, in the normal and the subnormal codes."""
    m = np.arange(128, 256) / 128.0
    rows = np.zeros((128 * 9, 128))
    for i, peak in enumerate(m):
        for j, down in enumerate((0, 1, 4, 6, 12, 13, 14, 16, 18)):  # exponents below the largest one's
            rows[9 * i + j, :127] = m[:127] * 2.0 ** -down * np.where(np.arange(127) % 2, 1, -1)
            rows[9 * i + j, :127][np.abs(rows[9 * i + j, :127]) > peak] = 0
            rows[9 * i + j, 127] = peak
    t = torch.tensor(rows, dtype=torch.float32).bfloat16()
    gain = torch.ones(128) if norm else None
    codes, _ = a48.quant_fp8(t.to(cuda_dev), gain.to(cuda_dev) if norm else None)
    want, _ = fp8.quant_rows(t.double().numpy())
    assert np.array_equal(bits(codes), want)
    codes, _ = a48.quant_fp8_weight(t.to(cuda_dev))
    assert np.array_equal(bits(codes), fp8.quant_weight(t.double().numpy())[0])


@pytest.mark.parametrize("x", ["fp32", "bf16"])
@pytest.mark.parametrize("norm", [False, True])
def test_quant_extremes(a48, cuda_dev, x, norm):
    """Zeros, the smallest and the largest numbers, and what is no number, each in a block of its own."""
    rng = np.random.default_rng(5)
    v = rng.standard_normal((9, 384)).astype(np.float32)
    v[0] = 0
    v[1, :128] = 0
    v[2] *= np.float32(1e-37)
    v[3] *= np.float32(2e-41)
    v[4] *= np.float32(3e37 / 4)
    v[5] = np.where(np.arange(384) % 3, 2.0 ** -149, 0) if x == "fp32" else np.where(np.arange(384) % 3, 2.0 ** -133, 0)
    v[6, 130] = np.nan
    v[7, 5] = np.inf
    v[8, 383] = -np.inf
    t = torch.tensor(v).to(DT[x])
    gain = torch.tensor(rng.uniform(0.5, 2.0, 384), dtype=torch.float32) if norm else None
    codes, scale = a48.quant_fp8(t.to(cuda_dev), gain.to(cuda_dev) if norm else None)
    d = t.double().numpy()
    want, want_scale = fp8.quant_rows(d, gain.double().numpy() if norm else None, float(np.float32(1e-5)))
    if norm:  # a row's size is no number, or infinite, with one of its entries
        want_scale[:, 6] = np.nan
        want_scale[:, 7:] = np.where(np.isnan(want_scale[:, 7:]), np.nan, 0)
    assert np.array_equal(bits(codes), want)
    scale = scale.double().cpu().numpy()
    assert np.array_equal(np.isnan(scale), np.isnan(want_scale))
    fine = ~np.isnan(want_scale)
    assert np.all(np.abs(scale - want_scale)[fine] <= (norm_tol(384) * np.abs(want_scale) + 2.0 ** -148)[fine])


@pytest.mark.parametrize("x", ["fp32", "bf16"])
@pytest.mark.parametrize("M,K", [(6, 384), (3, 20000)])
def test_quant_with_nothing_added_to_the_mean(a48, cuda_dev, M, K, x):
    v = np.random.default_rng(K).standard_normal((M, K)).astype(np.float32)
    v[0] = 0
    v[1] *= np.float32(1e-25)
    v[2] = np.where(np.arange(K) % 3, 2.0 ** -133, 0)
    t, gain = torch.tensor(v).to(DT[x]), torch.linspace(0.5, 2.0, K)
    codes, scale = a48.quant_fp8(t.to(cuda_dev), gain.to(cuda_dev), 0.0)
    with np.errstate(divide="ignore", invalid="ignore"):
        want, want_scale = fp8.quant_rows(t.double().numpy(), gain.double().numpy(), 0.0)
    want_scale[:, 0] = 0
    assert np.array_equal(bits(codes), want)
    check_scale(scale, want_scale, norm_tol(K))


def test_rows_past_two_to_the_31_entries(a48, cuda_dev):
    M, N, few = 70001, 32000, 2000
    torch.manual_seed(1)
    wc, ws = a48.quant_fp8_weight(torch.randn(N, 16, device=cuda_dev))
    h = torch.randn(M, 16, device=cuda_dev)
    end = slice(M - few, M)
    for dtype in (torch.float32, torch.bfloat16):
        y = a48.linear_fp8(*a48.quant_fp8(h), wc, ws, dtype=dtype)
        assert torch.equal(y[end], a48.linear_fp8(*a48.quant_fp8(h[end]), wc, ws, dtype=dtype))
        tokens = torch.randint(N, (M,), device=cuda_dev)
        for all_of, of_end in zip(a48.logprobs(y, tokens, top=2), a48.logprobs(y[end], tokens[end], top=2)):
            assert torch.equal(all_of[end], of_end)
        codes, scale = a48.quant_fp8(y, torch.ones(N, device=cuda_dev))
        c, s = a48.quant_fp8(y[end], torch.ones(N, device=cuda_dev))
        assert torch.equal(codes[end].view(torch.uint8), c.view(torch.uint8)) and torch.equal(scale[:, end].contiguous(), s)
        del y, codes


def test_quant_rows_may_be_strided_and_outputs_given(a48, cuda_dev):
    wide = torch.randn(40, 512, device=cuda_dev).bfloat16()
    part = wide[:, 128:384]
    codes, scale = torch.zeros(41, 256, dtype=torch.float8_e4m3fn, device=cuda_dev), torch.full((2, 40), -1.0, device=cuda_dev)
    c, s = a48.quant_fp8(part, codes=codes[:40], scale=scale)
    assert c.data_ptr() == codes.data_ptr() and s.data_ptr() == scale.data_ptr()
    want, want_scale = fp8.quant_rows(part.double().cpu().numpy())
    assert np.array_equal(bits(codes[:40]), want) and bits(codes[40:]).max() == 0
    check_scale(scale, want_scale, 2 * U)


@pytest.mark.parametrize("x", ["fp32", "bf16"])
@pytest.mark.parametrize("N,K", [(1, 16), (127, 128), (128, 144), (129, 64), (300, 1040), (700, 3200)])
def test_quant_weight(a48, cuda_dev, N, K, x):
    w = (torch.randn(N, K + 16, generator=torch.Generator().manual_seed(N)) * 0.02).to(DT[x])
    w[0, :min(K, 128)] *= 50
    if N > 128:
        w[128:, :64] = 0
    w = w[:, :K] if K % 16 == 0 and x == "fp32" else w[:, :K].contiguous()
    codes, scale = a48.quant_fp8_weight(w.to(cuda_dev) if w.is_contiguous() else torch.nn.functional.pad(w, (0, 16)).to(cuda_dev)[:, :K])
    want, want_scale = fp8.quant_weight(w.double().numpy())
    assert np.array_equal(bits(codes), want)
    check_scale(scale, want_scale, 2 * U)


def test_quant_weight_blocks_do_not_touch_one_another(a48, cuda_dev):
    w = torch.randn(256, 256)
    w[3, 200], w[200, 3] = float("nan"), 1e38
    w[128:, 128:] *= 1e-40
    for t in (w, w.bfloat16()):
        codes, scale = a48.quant_fp8_weight(t.to(cuda_dev))
        want, want_scale = fp8.quant_weight(t.double().numpy())
        assert np.array_equal(bits(codes), want)
        s = scale.double().cpu().numpy()
        assert np.isnan(s[0, 1]) and np.isnan(s).sum() == 1
        fine = ~np.isnan(s)
        assert np.all(np.abs(s - want_scale)[fine] <= 2 * U * want_scale[fine] + 2.0 ** -149)


def borders(peak):
    """253 entries: the numbers halfway between two codes, and the codes' own, of a block whose largest entry is `peak`."""
    row = np.concatenate([(fp8.GRID[1:] + fp8.GRID[:-1]) / 2, fp8.GRID]) * (peak / 448.0)
    row[::2] *= -1
    return row


PEAKS = [m * 2.0 ** e for e in range(-126, 128) for m in (1.75, 1.3359375)]


@pytest.mark.parametrize("x", ["fp32", "bf16"])
@pytest.mark.parametrize("norm", [False, True])
def test_quant_blocks_of_every_size(a48, cuda_dev, norm, x):
    """Codes stay exact up to the largest and down to the smallest numbers; so do those of entries halfway between two codes."""
    v = np.zeros((len(PEAKS), 256), np.float64)
    for row, peak in zip(v, PEAKS):
        row[:253] = borders(peak)
        row[127] = row[255] = peak
    t = torch.tensor(v, dtype=torch.float32).to(DT[x])
    codes, scale = a48.quant_fp8(t.to(cuda_dev), torch.ones(256, device=cuda_dev) if norm else None)
    want, want_scale = fp8.quant_rows(t.double().numpy(), np.ones(256) if norm else None, float(np.float32(1e-5)))
    assert np.array_equal(bits(codes), want)
    check_scale(scale, want_scale, norm_tol(256) if norm else 2 * U)


@pytest.mark.parametrize("x", ["fp32", "bf16"])
def test_quant_weight_blocks_of_every_size(a48, cuda_dev, x):
    peaks = PEAKS[::7]
    w = np.zeros((128 * len(peaks), 128))
    for i, peak in enumerate(peaks):
        w[128 * i + 3:128 * i + 5] = np.append(borders(peak), [peak, 0, 0]).reshape(2, 128)
    t = torch.tensor(w, dtype=torch.float32).to(DT[x])
    codes, scale = a48.quant_fp8_weight(t.to(cuda_dev))
    want, want_scale = fp8.quant_weight(t.double().numpy())
    assert np.array_equal(bits(codes), want)
    check_scale(scale, want_scale, 2 * U)


@pytest.mark.parametrize("x", ["fp32", "bf16"])
def test_quant_gains_of_every_size(a48, cuda_dev, x):
    """Blocks whose products are tiny or huge though an entry or its gain is neither, zeros among the gains, and gains that bring
    all of a block's products below fp32's range (a block of zeros then)."""
    rng = np.random.default_rng(11)
    g = rng.uniform(0.5, 2.0, (9, 128)) * np.where(rng.random((9, 128)) < 0.3, -1, 1)
    v = rng.standard_normal((5, 9, 128))
    v[:, 0] *= 1e10
    g[0] *= 1e-42          # products 1e-32
    v[:, 1] *= 1e-33
    v[:, 1, 5::16], g[1, 5::16] = 1e36, 0.0   # nothing but the channels without a gain are large
    v[:, 2] *= 1e-38
    g[2] *= 1e38
    v[:, 3] *= 1e-38
    g[3] *= 1e4
    v[:, 4] *= 1e30
    g[4] *= 5e6            # up to 3e37
    g[5] = 0.0
    v[:, 6] *= 1e-30
    g[6] *= 1e-25          # products of 0 in fp32
    g[7] = np.where(np.arange(128) % 3, 0.0, 1.0)
    v[:, 8] *= 1e-4
    v[:, 8, 7] = 3e8
    g[8] *= 1e-35          # 3e8 * 2^100 would be infinite
    t, gain = torch.tensor(v.reshape(5, -1), dtype=torch.float32).to(DT[x]), torch.tensor(g.reshape(-1), dtype=torch.float32)
    codes, scale = a48.quant_fp8(t.to(cuda_dev), gain.to(cuda_dev), 1e-5)
    d = t.double().numpy()
    d[:, 6 * 128:7 * 128] = 0
    want, want_scale = fp8.quant_rows(d, gain.double().numpy(), float(np.float32(1e-5)))
    assert np.array_equal(bits(codes), want)
    check_scale(scale, want_scale, norm_tol(9 * 128))
    codes, scale = a48.quant_fp8(t[:, 128 * 8:].contiguous().to(cuda_dev), gain[128 * 8:].contiguous().to(cuda_dev), 0.0)
    want, want_scale = fp8.quant_rows(d[:, 128 * 8:], gain[128 * 8:].double().numpy(), 0.0)
    assert np.array_equal(bits(codes), want)
    check_scale(scale, want_scale, norm_tol(128))


# Factors of a block's largest product, and x 2^e and g of one next to the border between two codes: nearer than 2^-47 of it.
NEAR_BORDERS = [(15524161, 13731829, 15155671, -14, 11553968), (12255099, 16753811, 15555131, -1, 14613708), (16166145, 11826467, 11563907, -1, 15942728),
                (11866993, 10753029, 14909512, -5, 12838058), (16547609, 11469091, 12663397, -10, 16592724), (12604235, 12582685, 15283787, -12, 10747286),
                (10712629, 9457341, 12678437, -7, 13128019), (15317239, 15067483, 16015965, -11, 14924784), (14480513, 14705649, 15924659, -6, 14804770),
                (9987623, 16761003, 16324057, -3, 13917448), (8957797, 9663743, 13162533, -6, 15971952), (12181003, 12295769, 11348118, -4, 16026393)]


@pytest.mark.parametrize("of_x,of_gain", [(0, 0), (-64, -60), (-70, -74), (-100, -40), (-20, -149), (40, 26), (38, 38)])
def test_quant_products_next_to_a_border(a48, cuda_dev, of_x, of_gain):
    """Products of an entry and its gain have 48 bits, all of which may count."""
    from fractions import Fraction
    x, gain, want = np.zeros((len(NEAR_BORDERS), 128)), np.ones((len(NEAR_BORDERS), 128)), np.zeros((len(NEAR_BORDERS), 128), np.uint8)
    for i, (xa, ga, xb, e, gb) in enumerate(NEAR_BORDERS):
        x[i, [5, 6, 100]], gain[i, [5, 6, 100]] = (xa, xb * 2.0 ** e, -xb * 2.0 ** e), (ga, gb, gb)
        t = Fraction(448 * xb * gb, xa * ga) * Fraction(2) ** e
        off = [abs(Fraction(float(v)) - t) for v in fp8.GRID]
        code = min(range(127), key=lambda c: (off[c], c % 2))
        other = sorted(off)[1]
        assert 0 < other - off[code] < other * Fraction(1, 2 ** 40)
        want[i, [5, 6, 100]] = 126, code, code | 128
    x, gain = x.reshape(1, -1) * 2.0 ** of_x, gain.reshape(-1) * 2.0 ** of_gain
    t, g = torch.tensor(x, dtype=torch.float32), torch.tensor(gain, dtype=torch.float32)
    assert np.array_equal(t.double().numpy(), x) and np.array_equal(g.double().numpy(), gain)
    codes, _ = a48.quant_fp8(t.to(cuda_dev), g.to(cuda_dev))
    assert np.array_equal(bits(codes).reshape(want.shape), want)


def least_time(call, n=12):
    """Least of n times in us, the call replayed from a graph."""
    call()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    times = []
    for _ in range(n):
        begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        torch.cuda.synchronize()
        begin.record()
        graph.replay()
        end.record()
        torch.cuda.synchronize()
        times.append(begin.elapsed_time(end) * 1e3)
    return min(times)


@pytest.mark.parametrize("x", ["fp32", "bf16"])
@pytest.mark.parametrize("K", [4096, 16384, 20000])
def test_quant_rows_whose_squares_are_out_of_range_hold_nobody_up(a48, cuda_dev, K, x):
    """The squares of such a row are added once more in 64 bits, by many threads at once (by one for each block of channels the
    call took tens of times as long); those of a row with a NaN are not."""
    h, gain = torch.randn(64, K, device=cuda_dev).to(DT[x]), torch.ones(K, device=cuda_dev)
    codes, scale = torch.empty(64, K, dtype=torch.float8_e4m3fn, device=cuda_dev), torch.empty((K + 127) // 128, 64, device=cuda_dev)
    usual = least_time(lambda: a48.quant_fp8(h, gain, codes=codes, scale=scale))
    for odd, most in ((float("nan"), 1.5), (1e25, 4.0), (float("inf"), 4.0)):
        h[9, 100] = odd
        assert least_time(lambda: a48.quant_fp8(h, gain, codes=codes, scale=scale)) <= most * usual + 2.0, odd
        want, want_scale = fp8.quant_rows(h.double().cpu().numpy(), np.ones(K), float(np.float32(1e-5)))
        if odd == float("inf"):
            want_scale[1:, 9] = 0
        assert np.array_equal(bits(codes), want)
        check_scale(scale, want_scale if odd == odd else np.where(np.arange(64) == 9, np.nan, want_scale), norm_tol(K))


# ------------------------------------------------------------------------------------------------ product
def operands(M, N, K, seed=0):
    g = torch.Generator().manual_seed(seed + M * 7 + N * 3 + K)
    x = (torch.randn(M, K, generator=g) * 60).to(torch.float8_e4m3fn)
    w = (torch.randn(N, K, generator=g) * 60).to(torch.float8_e4m3fn)
    kb, nb = (K + 127) // 128, (N + 127) // 128
    return x, torch.rand(kb, M, generator=g) + 0.5, w, (torch.rand(nb, kb, generator=g) + 0.5) * 1e-3


def product_bound(mag, K, y, want):
    """Each term is exact; the sums of a block (128 additions), its scale (two roundings), its addition: fp32, each taken as a whole
    step because how the tensor core rounds inside a block is not told."""
    kb = (K + 127) // 128
    return mag * (128 + kb + 4) * 2 * U + (HALF_BF16 * np.abs(want) if y == "bf16" else 0) + 1e-30


def check_product(a48, dev, M, N, K, y, out=None):
    x, xs, w, ws = operands(M, N, K)
    got = a48.linear_fp8(x.to(dev), xs.to(dev), w.to(dev), ws.to(dev), dtype=DT[y], Y=out)
    want, mag = fp8.linear(x.view(torch.uint8).numpy(), xs.numpy(), w.view(torch.uint8).numpy(), ws.numpy())
    err = np.abs(got.double().cpu().numpy() - want)
    assert np.all(err <= product_bound(mag, K, y, want)), float((err / product_bound(mag, K, y, want)).max())
    assert a48.kernel_status()[0] == 0
    return got


@pytest.mark.parametrize("y", ["fp32", "bf16"])
@pytest.mark.parametrize("M,N,K", [
    (1, 1, 16), (1, 100, 64), (1, 4111, 1040), (2, 257, 144), (7, 3000, 128), (8, 2500, 3200), (9, 333, 2048), (16, 2400, 272), (17, 999, 1040),
    (32, 1000, 1536), (1, 130, 22016), (32, 300, 11008),                 # streamed weights; the last one does not fit and takes tiles
    (33, 100, 16), (33, 4111, 1040), (64, 9500, 272), (100, 500, 1536), (128, 257, 4096), (129, 64, 144), (200, 3000, 528), (257, 1001, 272),
    (512, 2500, 256), (1025, 300, 384), (1999, 777, 1040), (2500, 130, 16),
])
def test_linear(a48, cuda_dev, M, N, K, y):
    check_product(a48, cuda_dev, M, N, K, y)


@pytest.mark.parametrize("y", ["fp32", "bf16"])
@pytest.mark.parametrize("M", [1, 5, 40, 300])
@pytest.mark.parametrize("left,right", [(0, 1), (1, 2), (8, 8), (3, 0)])
def test_linear_into_part_of_a_wider_matrix(a48, cuda_dev, M, left, right, y):
    N = 273
    wide = torch.full((M + 1, left + N + right), 7.0, dtype=DT[y], device=cuda_dev)
    got = check_product(a48, cuda_dev, M, N, 272, y, out=wide[:M, left:left + N])
    assert got.data_ptr() == wide[:, left:].data_ptr()
    rest = wide.clone()
    rest[:M, left:left + N] = 7.0
    assert torch.all(rest == 7.0)


@pytest.mark.parametrize("M", [3, 20, 70, 400])
def test_linear_scales_of_zero_and_nan(a48, cuda_dev, M):
    """A token whose scale is no number gives a row of NaN and touches no other; one of zeros gives zeros."""
    N, K = 400, 528
    x, xs, w, ws = operands(M, N, K)
    xs[:, 1] = 0
    xs[2, 0] = float("nan")
    ws[1, 3] = float("nan")
    got = a48.linear_fp8(x.to(cuda_dev), xs.to(cuda_dev), w.to(cuda_dev), ws.to(cuda_dev)).cpu()
    assert torch.isnan(got[0]).all() and torch.isnan(got[:, 128:256]).all()
    assert torch.all(got[1, :128] == 0) and torch.isfinite(got[1:, :128]).all() and torch.isfinite(got[1:, 256:]).all()
    want, mag = fp8.linear(x.view(torch.uint8).numpy()[1:], xs.numpy()[:, 1:], w.view(torch.uint8).numpy()[256:], ws.numpy()[2:])
    assert np.all(np.abs(got[1:, 256:].double().numpy() - want) <= product_bound(mag, K, "fp32", want))


def test_linear_is_the_same_every_time(a48, cuda_dev):
    for M in (4, 30, 64, 700):
        args = [t.to(cuda_dev) for t in operands(M, 3000, 1040)]
        first = a48.linear_fp8(*args)
        assert all(torch.equal(first, a48.linear_fp8(*args)) for _ in range(3))


# ------------------------------------------------------------------------------------------------ log probabilities
def logprob_bound(o, V, lp):
    """fp32: the difference, its factor and the factor's own rounding act on an exponent of up to the row's spread, 2^x has two units,
    a thread adds V / 256 terms and the threads' sums a dozen more; then a logarithm, a difference and a product."""
    return U * (8 * o["spread"] + V / 256 + 64 + 8 * np.abs(np.where(np.isfinite(lp), lp, 0)))


def check_logprobs(a48, dev, x, tokens, top=0, temperature=1.0):
    got = a48.logprobs(x.to(dev), tokens.to(dev), top=top, temperature=temperature)
    o = fp8.logprobs(x.double().numpy(), tokens.numpy(), top, float(np.float32(temperature)))
    V = x.shape[1]
    for name in ("logprob", "entropy"):
        g, want = getattr(got, name).double().cpu().numpy(), o[name]
        assert np.array_equal(np.isnan(g), np.isnan(want)), name
        assert np.array_equal(np.isinf(g), np.isinf(want)), name
        fine = np.isfinite(want)
        tol = logprob_bound(o, V, want) * (1 if name == "logprob" else 2 + o["mean"])
        assert np.all(np.abs(g - want)[fine] <= tol[fine]), (name, float((np.abs(g - want)[fine] / tol[fine]).max()))
    assert np.array_equal(got.rank.cpu().numpy(), o["rank"])
    if top:
        assert np.array_equal(got.top_ids.cpu().numpy(), o["top_ids"])
        g, want = got.top_logprobs.double().cpu().numpy(), o["top_logprobs"]
        assert np.array_equal(np.isnan(g), np.isnan(want)) and np.array_equal(np.isinf(g), np.isinf(want))
        fine = np.isfinite(want)
        assert np.all(np.abs(g - want)[fine] <= np.broadcast_to(logprob_bound(o, V, o["logprob"] * 0)[:, None], want.shape)[fine] + 8 * U * np.abs(want[fine]))
    return got


def rows_of(kind, M, V, rng):
    x = rng.standard_normal((M, V)) * 2
    if kind == "peaked":
        x[np.arange(M), rng.integers(0, V, M)] += 25
    elif kind == "equal":
        x[:] = 1.5
    elif kind == "rising":
        x = np.sort(x, 1)
    elif kind == "falling":
        x = -np.sort(-x, 1)
    elif kind == "masked":
        x[rng.random((M, V)) > 0.01] = -np.inf
        x[:, V // 2] = 0.5
    elif kind == "lowest":  # masks of the type's lowest value
        x[rng.random((M, V)) > 0.01] = float(torch.finfo(torch.bfloat16).min)
    elif kind == "all lowest":
        x[:] = float(torch.finfo(torch.bfloat16).min)
    elif kind == "one":
        x[:] = -np.inf
        x[np.arange(M), rng.integers(0, V, M)] = -3.0
    elif kind == "coarse":
        x = np.round(x)
    elif kind == "cluster":  # a stretch of large ones among small ones, more than the list holds
        x[:, V // 3:V // 3 + V // 4] += 50
    elif kind == "far":
        x += 30000
    return x


KINDS = ["random", "peaked", "equal", "rising", "falling", "masked", "lowest", "all lowest", "one", "coarse", "cluster", "far"]


@pytest.mark.parametrize("x", ["fp32", "bf16"])
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("M,V,top", [(3, 32000, 20), (160, 8201, 64), (4, 50021, 5), (3, 1 << 20, 64)])
def test_logprobs(a48, cuda_dev, M, V, top, kind, x):
    rng = np.random.default_rng(V + KINDS.index(kind))
    v = torch.tensor(rows_of(kind, M, V, rng), dtype=torch.float32).to(DT[x])
    tokens = torch.tensor(rng.integers(0, V, M))
    tokens[1] = -1
    tokens[2] = int(v[2].float().argmax())
    check_logprobs(a48, cuda_dev, v, tokens, top)


@pytest.mark.parametrize("x", ["fp32", "bf16"])
@pytest.mark.parametrize("V", [1, 2, 3, 7, 8, 9, 63, 64, 100, 1023, 1025, 2049, 8191, 8193])
def test_logprobs_small_and_odd(a48, cuda_dev, V, x):
    rng = np.random.default_rng(V)
    v = torch.tensor(rng.standard_normal((13, V)) * 3, dtype=torch.float32).to(DT[x])
    check_logprobs(a48, cuda_dev, v, torch.tensor(rng.integers(0, V, 13)), min(V, 64))
    check_logprobs(a48, cuda_dev, v, torch.tensor(rng.integers(0, V, 13), dtype=torch.int32), 1, temperature=0.3)


def test_logprobs_rows_without_a_distribution(a48, cuda_dev):
    nan, inf = float("nan"), float("inf")
    for M, V in ((8, 9000), (200, 300)):
        x = torch.randn(M, V)
        x[0, V - 1], x[1, 0], x[2] = nan, inf, -inf
        x[3, ::2] = -inf
        x[4] = nan
        tokens = torch.arange(M) % V
        got = check_logprobs(a48, cuda_dev, x, tokens, 3)
        assert torch.isnan(got.entropy[[0, 1, 2, 4]].cpu()).all() and torch.isfinite(got.entropy[5:].cpu()).all()
        assert got.top_ids[4].tolist() == [-1] * 3


def test_logprobs_more_alternatives_than_possible_tokens(a48, cuda_dev):
    """Behind the possible tokens come the others, the lowest index first."""
    for V in (70, 9001):
        x = torch.full((2, V), -float("inf"))
        x[:, 33], x[:, 5] = 1.0, 2.0
        got = check_logprobs(a48, cuda_dev, x, torch.tensor([7, 33]), 12)
        assert got.top_ids[0].tolist() == [5, 33, 0, 1, 2, 3, 4, 6, 7, 8, 9, 10] and got.rank.tolist() == [8, 1]
        assert got.logprob[0].item() == -float("inf")


def test_logprobs_tokens_outside_the_vocabulary(a48, cuda_dev):
    x = torch.randn(4, 500)
    for dtype in (torch.int64, torch.int32):
        got = a48.logprobs(x.to(cuda_dev), torch.tensor([-1, 500, -(2 ** 31), 499], dtype=dtype).to(cuda_dev))
        assert got.rank[:3].tolist() == [-1] * 3 and got.logprob[:3].tolist() == [0.0] * 3 and got.rank[3].item() >= 0
    got = a48.logprobs(x.to(cuda_dev), torch.tensor([2 ** 32, 2 ** 40, -(2 ** 40), 0]).to(cuda_dev))
    assert got.rank[:3].tolist() == [-1] * 3


@pytest.mark.parametrize("x", ["fp32", "bf16"])
def test_logprobs_rows_may_be_strided_and_start_anywhere(a48, cuda_dev, x):
    wide = (torch.randn(20, 9100) * 2).to(DT[x])
    for first in range(0, 9):
        part = wide[:, first:first + 9013]
        tokens = torch.randint(0, 9013, (20,))
        dev = wide.to(cuda_dev)[:, first:first + 9013]
        got = a48.logprobs(dev, tokens.to(cuda_dev), top=4)
        o = fp8.logprobs(part.double().numpy(), tokens.numpy(), 4)
        assert np.array_equal(got.top_ids.cpu().numpy(), o["top_ids"]) and np.array_equal(got.rank.cpu().numpy(), o["rank"])
        assert np.all(np.abs(got.logprob.double().cpu().numpy() - o["logprob"]) <= logprob_bound(o, 9013, o["logprob"]))


def test_logprobs_without_tokens_and_twice_the_same(a48, cuda_dev):
    x = (torch.randn(300, 20011) * 2).to(cuda_dev)
    first = a48.logprobs(x, top=30)
    assert first.logprob is None and first.rank is None
    for _ in range(3):
        again = a48.logprobs(x, top=30)
        assert all(torch.equal(p, q) for p, q in zip(first[1:2] + first[3:], again[1:2] + again[3:]))
    assert a48.logprobs(x).top_ids is None


@pytest.mark.parametrize("temperature", [1e-3, 0.5, 2.0, 1e3])
def test_logprobs_temperature(a48, cuda_dev, temperature):
    x = torch.randn(5, 9000) * 3
    check_logprobs(a48, cuda_dev, x, torch.arange(5), 7, temperature)


@pytest.mark.parametrize("x", ["fp32", "bf16"])
@pytest.mark.parametrize("M,V", [(200, 32000), (100, 32000), (160, 128001)])
def test_logprobs_of_a_token_that_is_nearly_certain(a48, cuda_dev, M, V, x):
    """A peak anywhere in the row, 15 to 40 above the rest: no log probability above 0, no entropy below it, and errors that are small
    beside the tail.  What is added to the peak's own 1 rounds to a unit at most for a term of that size and to the term itself below
    (V / 256 of them in a thread, a dozen sums that are joined, a logarithm and two products); the terms' own relative errors are those of
    `logprob_bound` and act on the tail."""
    rng = np.random.default_rng(V + M)
    v = rng.standard_normal((M, V))
    at, height = rng.integers(0, V, M), rng.uniform(15, 40, M)
    v[np.arange(M), at] = v.max(1) + height
    v = torch.tensor(v, dtype=torch.float32).to(DT[x])
    got = a48.logprobs(v.to(cuda_dev), torch.tensor(at).to(cuda_dev), top=2)
    o = fp8.logprobs(v.double().numpy(), at, 2)
    lp, ent, best = (t.double().cpu().numpy() for t in (got.logprob, got.entropy, got.top_logprobs))
    assert np.all(lp <= 0) and np.all(ent >= 0) and np.array_equal(best[:, 0], lp)
    tail, second = -np.expm1(o["logprob"]), np.exp(o["top_logprobs"][:, 1])
    tol = U * 24 + V / 256 * np.minimum(U, second) + tail * U * (8 * o["spread"] + 64)
    assert np.all(np.abs(lp - o["logprob"]) <= tol), float((np.abs(lp - o["logprob"]) / tol).max())
    tol_ent = 2 * tol + tail * o["spread"] * U * (8 * o["spread"] + V / 256 + 64)  # the products' sum is at most tail * spread
    assert np.all(np.abs(ent - o["entropy"]) <= tol_ent), float((np.abs(ent - o["entropy"]) / tol_ent).max())
    assert np.array_equal(got.rank.cpu().numpy(), np.zeros(M)) and np.array_equal(got.top_ids.cpu().numpy(), o["top_ids"])


@pytest.mark.parametrize("x", ["fp32", "bf16"])
def test_logprobs_keeps_a_tail_of_terms_that_are_nothing_beside_the_peak(a48, cuda_dev, x):
    """Each of a million equal logits 17.5 below the peak is less than half a unit beside its 1.  Sixteen terms or more of a thread are
    added together: V / 4096 roundings of half a unit (U) at most, and a few dozen of sums that are joined."""
    M, V, below = 160, 1 << 20, 17.5
    v = torch.zeros(M, V, dtype=DT[x], device=cuda_dev)
    at = torch.arange(M, device=cuda_dev) * 6001
    v[torch.arange(M, device=cuda_dev), at] = below
    got = a48.logprobs(v, at)
    tail = (V - 1) * np.exp(-below)
    assert np.all(np.abs(got.logprob.double().cpu().numpy() + np.log1p(tail)) <= U * (V / 4096 + 64 + tail * 8 * below))
    entropy = np.log1p(tail) + tail * below / (1 + tail)  # the sum of its products has V / 256 roundings in a thread
    assert np.all(np.abs(got.entropy.double().cpu().numpy() - entropy) <= U * (V / 4096 + 64 + tail * below * (8 * below + V / 256 + 64)))


@pytest.mark.parametrize("x", ["fp32", "bf16"])
def test_logprobs_of_logits_further_apart_than_the_largest_number(a48, cuda_dev, x):
    """At a temperature that makes such a difference a number again, a logit of the lowest value is still a token that can be."""
    most = float(torch.finfo(DT[x]).max)
    for M, V in ((3, 9000), (200, 500)):
        v = torch.full((M, V), -most)
        v[:, 100] = most
        tokens = torch.arange(M) % 90
        check_logprobs(a48, cuda_dev, v.to(DT[x]), tokens, 5, 1e30)
    h = torch.full((40, 128), 1.0, device=cuda_dev)
    w = torch.full((256, 128), -1.0, device=cuda_dev)
    w[7] = 1.0
    wc, ws = a48.quant_fp8_weight(w * 2.6e36)  # logits of 3.3e38 either way
    for M in (5, 40):
        lp, ent = a48.score(h[:M], None, wc, ws, torch.arange(M, device=cuda_dev), temperature=1e30)
        logits = a48.linear_fp8(*a48.quant_fp8(h[:M]), wc, ws).double().cpu().numpy()
        o = fp8.logprobs(logits, np.arange(M), 0, float(np.float32(1e30)))
        assert np.all(np.abs(lp.double().cpu().numpy() - o["logprob"]) <= 8 * U * np.abs(o["logprob"])) and torch.all(ent == 0)


# ------------------------------------------------------------------------------------------------ scores
@pytest.mark.parametrize("M,N,K,x,norm,temperature", [
    (1, 32000, 256, "bf16", True, 1.0), (5, 1003, 208, "fp32", True, 0.8), (32, 500, 1040, "bf16", False, 1.0), (33, 2003, 528, "bf16", True, 1.0),
    (61, 9500, 272, "fp32", True, 1.5), (128, 130, 256, "bf16", True, 1.0), (300, 5003, 272, "bf16", True, 1.0), (1100, 1000, 400, "fp32", True, 0.7),
    (2000, 3001, 256, "bf16", True, 1.0)])
def test_score(a48, cuda_dev, M, N, K, x, norm, temperature):
    rng = np.random.default_rng(M + N)
    h = torch.tensor(rng.standard_normal((M, K)), dtype=torch.float32).to(DT[x])
    gain = torch.tensor(rng.uniform(0.5, 1.5, K), dtype=torch.float32) if norm else None
    w = torch.tensor(rng.standard_normal((N, K)) * 0.1, dtype=torch.float32)
    wc, ws = a48.quant_fp8_weight(w.to(cuda_dev))
    tokens = torch.tensor(rng.integers(0, N, M))
    tokens[M // 2] = -1
    lp, ent = a48.score(h.to(cuda_dev), gain.to(cuda_dev) if norm else None, wc, ws, tokens.to(cuda_dev), temperature=temperature)
    assert a48.kernel_status()[0] == 0
    codes, scale = fp8.quant_rows(h.double().numpy(), gain.double().numpy() if norm else None, float(np.float32(1e-5)))
    logits, mag = fp8.linear(codes, scale, bits(wc), ws.double().cpu().numpy())
    o = fp8.logprobs(logits, tokens.numpy(), 0, float(np.float32(temperature)))
    # errors of the logits, and of the scales that they share; an entropy moves by the spread of what it averages
    off = ((product_bound(mag, K, "fp32", logits) + norm_tol(K) * mag).max(1)) / temperature
    assert np.all(np.abs(lp.double().cpu().numpy() - o["logprob"]) <= 2 * off + logprob_bound(o, N, o["logprob"]))
    assert np.all(np.abs(ent.double().cpu().numpy() - o["entropy"]) <= (2 * off + logprob_bound(o, N, o["entropy"])) * (2 + 2 * o["mean"]))


def test_score_takes_a_workspace_and_refuses_a_small_one(a48, cuda_dev):
    for M in (8, 200):
        h, w = torch.randn(M, 256, device=cuda_dev), torch.randn(700, 256, device=cuda_dev)
        wc, ws = a48.quant_fp8_weight(w)
        tokens = torch.randint(0, 700, (M,), device=cuda_dev, dtype=torch.int32)
        need = a48.score_workspace_bytes(M, 700, 256)
        space = torch.full((need,), 255, dtype=torch.uint8, device=cuda_dev)  # what lies in it does not matter
        first, again = a48.score(h, None, wc, ws, tokens), a48.score(h, None, wc, ws, tokens, workspace=space)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])
        with pytest.raises(a48.A48Error):
            a48.score(h, None, wc, ws, tokens, workspace=space[:need - 256])


@pytest.mark.parametrize("M", [6, 300])
def test_score_with_tokens_that_are_no_numbers(a48, cuda_dev, M):
    """A hidden state with a NaN makes its own row NaN and no other."""
    h, w = torch.randn(M, 256, device=cuda_dev), torch.randn(700, 256, device=cuda_dev)
    wc, ws = a48.quant_fp8_weight(w)
    tokens = torch.arange(M, device=cuda_dev)
    clean = a48.score(h, torch.ones(256, device=cuda_dev), wc, ws, tokens)
    h[3, 17] = float("nan")
    lp, ent = a48.score(h, torch.ones(256, device=cuda_dev), wc, ws, tokens)
    others = torch.arange(M, device=cuda_dev) != 3
    assert torch.isnan(lp[3]) and torch.isnan(ent[3])
    assert torch.equal(lp[others], clean[0][others]) and torch.equal(ent[others], clean[1][others])


@pytest.mark.parametrize("M", [33, 97, 129, 260, 1030, 1281])
def test_score_of_a_last_warp_that_is_not_full(a48, cuda_dev, M):
    """Rows are scored alike whichever rows share a tile with them, over many tiles of features, the tokens in any of them."""
    N, K = 20001, 272
    torch.manual_seed(M)
    h, gain = torch.randn(M, K, device=cuda_dev), torch.rand(K, device=cuda_dev) + 0.5
    wc, ws = a48.quant_fp8_weight(torch.randn(N, K, device=cuda_dev))
    tokens = torch.randint(N, (M,), device=cuda_dev)
    tokens[::5] = torch.arange(N - 1, -1, -1, device=cuda_dev)[: tokens[::5].numel()]
    lp, ent = a48.score(h, gain, wc, ws, tokens)
    r = a48.logprobs(a48.linear_fp8(*a48.quant_fp8(h, gain), wc, ws), tokens)
    assert a48.kernel_status()[0] == 0
    assert torch.allclose(lp, r.logprob, rtol=0, atol=1e-4) and torch.allclose(ent, r.entropy, rtol=0, atol=1e-4)


@pytest.mark.parametrize("M", [20, 100, 300, 1300])
def test_score_keeps_a_tail_of_terms_that_are_nothing_beside_the_peak(a48, cuda_dev, M):
    """One logit of 17.5, ahead of the others in its tile, among zeros.  At most 15 terms of less than half a unit (U) are lost beside its 1, and what is joined with it is
    rounded some 25 times."""
    N, K, below = 32000, 128, 17.5
    w = torch.zeros(N, K, device=cuda_dev)
    w[12288] = below / K
    lp, ent = a48.score(torch.ones(M, K, device=cuda_dev), None, *a48.quant_fp8_weight(w), torch.full((M,), 12288, device=cuda_dev))
    tail = (N - 1) * np.exp(-below)
    assert np.all(np.abs(lp.double().cpu().numpy() + np.log1p(tail)) <= U * (40 + tail * 16 * below))
    entropy = np.log1p(tail) + tail * below / (1 + tail)
    assert np.all(np.abs(ent.double().cpu().numpy() - entropy) <= U * (40 + tail * below * (16 * below + 256)))


# ------------------------------------------------------------------------------------------------ together, streams, graphs
def test_a_blocks_output_through_the_head(a48, cuda_dev):
    """One transformer block, then scores of a prompt and the logits of its last token: the head on what the framework computes."""
    from paper_2411_04965_b200 import synth
    H, F, V, T = 256, 768, 1000, 40
    names = (("q", H, H), ("k", H, H), ("v", H, H), ("o", H, H), ("gate", F, H), ("up", F, H), ("down", H, F))
    packed = {n: a48.pack_ternary(synth.latent_weights(r, c, seed=30 + i).to(cuda_dev), 1e-5, a48.LAYOUT_ALL) for i, (n, r, c) in enumerate(names)}
    block = a48.Block(packed, synth.norm_gains(H, 1).to(cuda_dev), synth.norm_gains(H, 2).to(cuda_dev), n_heads=4, k_o=H // 2, k_down=F // 2)
    h = block.forward(synth.gaussian_outlier_activations(T, H, seed=3, count=2).to(cuda_dev), 1, T)
    gain = synth.norm_gains(H, 4).to(cuda_dev)
    wc, ws = a48.quant_fp8_weight(synth.latent_weights(V, H, seed=5).to(cuda_dev))
    tokens = torch.arange(T, device=cuda_dev) * 7 % V
    lp, ent = a48.score(h, gain, wc, ws, tokens)
    codes, scale = a48.quant_fp8(h, gain)
    logits = a48.linear_fp8(codes, scale, wc, ws)
    r = a48.logprobs(logits, tokens, top=5)
    assert torch.allclose(lp, r.logprob, rtol=0, atol=1e-4) and torch.allclose(ent, r.entropy, rtol=0, atol=1e-4)
    last = a48.logprobs(a48.linear_fp8(*a48.quant_fp8(h[-1:], gain), wc, ws), tokens[-1:], top=5)
    o = fp8.quant_rows(h.double().cpu().numpy(), gain.double().cpu().numpy(), float(np.float32(1e-5)))
    want, mag = fp8.linear(o[0], o[1], bits(wc), ws.double().cpu().numpy())
    assert np.array_equal(bits(codes), o[0])
    tol = product_bound(mag, H, "fp32", want) + norm_tol(H) * mag
    assert np.all(np.abs(logits.double().cpu().numpy() - want) <= tol)
    assert np.abs(last.logprob.item() - fp8.logprobs(want[-1:], [int(tokens[-1])])["logprob"][0]) <= 1e-4


@pytest.mark.parametrize("M", [4, 48, 300])
def test_captured_and_replayed_with_other_contents(a48, cuda_dev, M):
    K, V = 272, 9000
    gain = torch.rand(K, device=cuda_dev) + 0.5
    wc, ws = a48.quant_fp8_weight(torch.randn(V, K, device=cuda_dev))
    h, tokens = torch.randn(M, K, device=cuda_dev).bfloat16(), torch.randint(0, V, (M,), device=cuda_dev)

    def step():
        logits = a48.linear_fp8(*a48.quant_fp8(h, gain), wc, ws)
        return (*a48.logprobs(logits, tokens, top=4), *a48.score(h, gain, wc, ws, tokens))

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = step()
    for seed in range(3):
        torch.manual_seed(seed)
        h.copy_(torch.randn(M, K))
        tokens.copy_(torch.randint(0, V, (M,)))
        graph.replay()
        for got, want in zip(captured, step()):
            assert torch.equal(got, want)


def test_two_streams_at_once(a48, cuda_dev):
    args = [[t.to(cuda_dev) for t in operands(M, 5000, 1040, seed=M)] for M in (600, 40, 5, 700)]
    want = [a48.linear_fp8(*a) for a in args]
    wanted = [a48.logprobs(y, top=9) for y in want]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in args]
    got = []
    for _ in range(3):
        for s, a in zip(streams, args):
            y = a48.linear_fp8(*a, stream=s)
            got.append((y, a48.logprobs(y, top=9, stream=s)))
    torch.cuda.synchronize()
    for i, (y, r) in enumerate(got):
        assert torch.equal(y, want[i % 4]) and torch.equal(r.top_ids, wanted[i % 4].top_ids) and torch.equal(r.entropy, wanted[i % 4].entropy)


def test_binding_refuses(a48, cuda_dev):
    x, xs, w, ws = (t.to(cuda_dev) for t in operands(4, 100, 256))
    h, tokens = torch.randn(4, 256, device=cuda_dev), torch.zeros(4, dtype=torch.int64, device=cuda_dev)
    for bad in (lambda: a48.quant_fp8(h.half()), lambda: a48.quant_fp8(h.t()), lambda: a48.quant_fp8(h.cpu()), lambda: a48.quant_fp8(h, gain=h[0, :128]),
                lambda: a48.quant_fp8(h, gain=h[0].double()), lambda: a48.quant_fp8(h, codes=x[:3]), lambda: a48.linear_fp8(x.view(torch.uint8), xs, w, ws),
                lambda: a48.linear_fp8(x, xs[:1], w, ws), lambda: a48.linear_fp8(x, xs, w[:, :128], ws), lambda: a48.linear_fp8(x, xs, w, ws.t()),
                lambda: a48.linear_fp8(x, xs, w, ws, dtype=torch.float16), lambda: a48.linear_fp8(x, xs, w.cpu(), ws),
                lambda: a48.linear_fp8(x, xs, w, ws, Y=torch.empty(4, 99, device=cuda_dev)), lambda: a48.logprobs(h, tokens[:3]),
                lambda: a48.logprobs(h, tokens.float()), lambda: a48.logprobs(h.cpu(), tokens), lambda: a48.score(h, None, w, ws[:, :1], tokens)):
        with pytest.raises((AssertionError, a48.A48Error)):
            bad()
    for bad in (lambda: a48.quant_fp8(h[:, :250]), lambda: a48.quant_fp8(h[:0]), lambda: a48.logprobs(h, tokens, top=65), lambda: a48.logprobs(h, tokens, temperature=0.0),
                lambda: a48.quant_fp8(h[:1].expand(4, 256))):
        with pytest.raises(a48.A48Error):
            bad()
    torch.cuda.synchronize()
