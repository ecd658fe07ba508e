"""8-bit output head without a GPU: the oracle's own numbers, the C ABI's refusals, workspace sizes."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import fp8

P = ctypes.c_void_p


def test_grid_is_e4m3():
    codes = np.arange(127, dtype=np.uint8)
    assert np.array_equal(fp8.GRID, torch.from_numpy(codes).view(torch.float8_e4m3fn).double().numpy())
    assert fp8.GRID[-1] == 448.0


def test_nearest_code_is_the_types_own_rounding():
    rng = np.random.default_rng(1)
    t = rng.uniform(-448, 448, 20000) * 2.0 ** rng.integers(-18, 1, 20000)
    ties = (fp8.GRID[1:] + fp8.GRID[:-1]) / 2
    t = np.concatenate([t.astype(np.float32), ties, -ties, fp8.GRID, -fp8.GRID]).astype(np.float32)
    assert np.array_equal(fp8.nearest_code(t.astype(np.float64)), torch.from_numpy(t).to(torch.float8_e4m3fn).view(torch.uint8).numpy())


def test_largest_entry_becomes_448_and_error_is_half_a_step():
    x = np.random.default_rng(2).standard_normal((5, 300))
    codes, scale = fp8.quant_rows(x)
    for b in range(3):
        part = np.s_[:, b * 128:(b + 1) * 128]
        assert np.all(np.abs(fp8.value(codes[part])).max(1) == 448.0)
        back = fp8.value(codes[part]) * scale[b][:, None]
        step = np.maximum(np.abs(x[part]) * 2.0 ** -4, scale[b][:, None] * 2.0 ** -10)  # eps / 2, and half of the smallest number
        assert np.all(np.abs(back - x[part]) <= step * (1 + 1e-12))


def test_gain_only_changes_scales_by_the_rows_size():
    rng = np.random.default_rng(3)
    x, gain = rng.standard_normal((4, 256)), rng.uniform(0.5, 2, 256)
    c0, s0 = fp8.quant_rows(x * gain)
    c1, s1 = fp8.quant_rows(x, gain, 0.0)
    assert np.array_equal(c0, c1)
    assert np.allclose(s1, s0 / np.sqrt((x * x).mean(1)), rtol=1e-14)


def test_logprobs_of_a_known_row():
    x = np.log([[0.5, 0.25, 0.125, 0.125]])
    r = fp8.logprobs(x, [2], top=4)
    assert np.allclose(r["logprob"], np.log(0.125)) and np.allclose(r["entropy"], 1.75 * np.log(2))
    assert r["rank"][0] == 2 and r["top_ids"][0].tolist() == [0, 1, 2, 3]
    r = fp8.logprobs(x, [-1], top=2, temperature=0.5)
    assert r["logprob"][0] == 0 and r["rank"][0] == -1
    assert np.allclose(np.exp(r["top_logprobs"][0]), np.array([0.25, 0.0625]) / 0.34375)


def test_rows_without_a_distribution():
    inf = np.inf
    r = fp8.logprobs(np.array([[0.0, np.nan], [inf, 0.0], [-inf, -inf], [-inf, 1.0]]), [0, 0, 0, 1], top=1)
    assert np.isnan(r["entropy"][:3]).all() and r["top_ids"][:3].tolist() == [[-1]] * 3 and r["rank"].tolist() == [-1, -1, -1, 0]
    assert r["entropy"][3] == 0 and r["logprob"][3] == 0


# ------------------------------------------------------------------------------------------------ refusals
OK, INVALID, SHAPE, ALIGN, CUDA, NOMEM, LIMIT = 0, 1, 2, 3, 5, 7, 8
p, odd, null = P(4096), P(4100), P(0)


def _status(call, base, changes):
    args = dict(base)
    args.update(changes)
    return call(*args.values())


@pytest.fixture()
def lib(a48):
    return a48.lib()


QUANT = dict(X=p, stride=256, bf16=0, M=4, K=256, gain=p, eps=1e-5, codes=p, scale=p, st=null)
QUANT_BAD = [(dict(X=null), INVALID), (dict(codes=null), INVALID), (dict(scale=null), INVALID), (dict(M=0), SHAPE), (dict(M=-3), SHAPE), (dict(M=(1 << 30) + 1), LIMIT),
             (dict(K=0), SHAPE), (dict(K=24), SHAPE), (dict(K=1 << 21), SHAPE), (dict(stride=255), SHAPE), (dict(stride=258), ALIGN),
             (dict(stride=260, bf16=1), ALIGN), (dict(X=odd), ALIGN), (dict(gain=odd), ALIGN), (dict(codes=odd), ALIGN), (dict(scale=odd), ALIGN),
             (dict(eps=-1.0), INVALID), (dict(eps=float("nan")), INVALID), (dict(eps=float("inf")), INVALID)]


@pytest.mark.parametrize("change,status", QUANT_BAD)
def test_quant_refuses(lib, change, status):
    assert _status(lib.bitnet_a48_quant_fp8, QUANT, change) == status


WEIGHT = dict(W=p, stride=256, bf16=0, N=4, K=256, codes=p, scale=p, st=null)


@pytest.mark.parametrize("change,status", [(dict(W=null), INVALID), (dict(N=0), SHAPE), (dict(N=(1 << 20) + 1), SHAPE), (dict(K=40), SHAPE),
                                           (dict(stride=128), SHAPE), (dict(W=odd), ALIGN), (dict(scale=odd), ALIGN)])
def test_quant_weight_refuses(lib, change, status):
    assert _status(lib.bitnet_a48_quant_fp8_weight, WEIGHT, change) == status


LINEAR = dict(x=p, xs=p, M=4, w=p, ws=p, N=100, K=256, Y=p, stride=100, bf16=0, st=null)


@pytest.mark.parametrize("change,status", [(dict(x=null), INVALID), (dict(xs=null), INVALID), (dict(w=null), INVALID), (dict(ws=null), INVALID),
                                           (dict(Y=null), INVALID), (dict(M=0), SHAPE), (dict(M=(1 << 30) + 1), LIMIT), (dict(N=0), SHAPE), (dict(K=8), SHAPE), (dict(K=130), SHAPE),
                                           (dict(N=(1 << 20) + 1), SHAPE), (dict(stride=99), SHAPE), (dict(x=odd), ALIGN), (dict(w=odd), ALIGN),
                                           (dict(Y=P(4098)), ALIGN), (dict(Y=P(4097), bf16=1), ALIGN)])
def test_linear_refuses(lib, change, status):
    assert _status(lib.bitnet_a48_linear_fp8, LINEAR, change) == status


LOGPROBS = dict(x=p, stride=100, bf16=0, M=4, V=100, temperature=1.0, tokens=p, i64=1, logprob=p, entropy=p, rank=p, top=5, ids=p, best=p, st=null)


@pytest.mark.parametrize("change,status", [(dict(x=null), INVALID), (dict(tokens=null), INVALID), (dict(tokens=null, rank=null), INVALID),
                                           (dict(ids=null), INVALID), (dict(best=null), INVALID), (dict(top=-1), INVALID), (dict(top=101), SHAPE),
                                           (dict(top=65), LIMIT), (dict(M=0), SHAPE), (dict(M=(1 << 30) + 1), LIMIT), (dict(V=0, top=0), SHAPE), (dict(stride=99), SHAPE),
                                           (dict(V=(1 << 20) + 1, stride=1 << 21), LIMIT), (dict(temperature=0.0), INVALID), (dict(temperature=-1.0), INVALID),
                                           (dict(temperature=float("nan")), INVALID), (dict(temperature=float("inf")), INVALID),
                                           (dict(logprob=null, entropy=null, rank=null, top=0), INVALID), (dict(x=P(4097), bf16=1), ALIGN),
                                           (dict(x=P(4098)), ALIGN), (dict(tokens=odd), ALIGN), (dict(logprob=P(4098)), ALIGN), (dict(ids=P(4098)), ALIGN)])
def test_logprobs_refuses(lib, change, status):
    assert _status(lib.bitnet_a48_logprobs, LOGPROBS, change) == status


SCORE = dict(X=p, stride=256, bf16=0, M=4, gain=p, eps=1e-5, w=p, ws=p, N=100, K=256, temperature=1.0, tokens=p, i64=1, logprob=p, entropy=p,
             space=p, bytes=1 << 30, st=null)


@pytest.mark.parametrize("change,status", [(dict(X=null), INVALID), (dict(w=null), INVALID), (dict(tokens=null), INVALID), (dict(logprob=null), INVALID),
                                           (dict(entropy=null), INVALID), (dict(space=null), INVALID), (dict(M=0), SHAPE), (dict(N=0), SHAPE),
                                           (dict(K=100, stride=112), SHAPE), (dict(temperature=0.0), INVALID), (dict(eps=-1.0), INVALID), (dict(X=odd), ALIGN),
                                           (dict(space=odd), ALIGN), (dict(w=odd), ALIGN), (dict(tokens=odd), ALIGN), (dict(bytes=100), NOMEM)])
def test_score_refuses(lib, change, status):
    assert _status(lib.bitnet_a48_score, SCORE, change) == status


def test_limits_in_range_reach_the_device_check(lib):
    if torch.cuda.is_available():
        pytest.skip("this check is for machines without a GPU")
    assert _status(lib.bitnet_a48_quant_fp8, QUANT, dict(M=1, stride=0, gain=null)) == CUDA  # a stride of one row does not count
    assert _status(lib.bitnet_a48_linear_fp8, LINEAR, dict(M=1, stride=0, K=16)) == CUDA
    assert _status(lib.bitnet_a48_logprobs, LOGPROBS, dict(top=64)) == CUDA
    assert _status(lib.bitnet_a48_logprobs, LOGPROBS, dict(x=odd, tokens=null, logprob=null, rank=null, i64=0)) == CUDA
    assert _status(lib.bitnet_a48_score, SCORE, {}) == CUDA


def test_workspace_sizes(a48):
    size = a48.score_workspace_bytes
    assert size(0, 100, 256) == size(4, 0, 256) == size(4, 100, 100) == size(4, 1 << 21, 256) == 0
    assert size(4, 1000, 256) >= 4 * 256 + 2 * 4 * 4 + 4 * 1000 * 4  # few tokens keep their logits
    M, N, K = 4096, 32000, 4096
    assert M * K < size(M, N, K) < M * K + M * 32 * 4 + M * (250 * 16 + 4) + 4096  # sums of 128 columns instead of logits
    assert size(1 << 20, 32000, 4096) > 1 << 32  # no overflow
    assert size((1 << 30) + 1, 100, 256) == 0
    for N in (1, 64, 65, 128, 300):  # whichever tiles the product takes
        assert size(700, N, 256) >= 700 * (256 + 8 + 4) + 700 * 16 * max(2 * ((N + 255) // 256), (N + 63) // 64)
