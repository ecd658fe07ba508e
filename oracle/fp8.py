"""float64 oracle of the 8-bit output head: e4m3 rounding with block scales, the product, what is read off logits.

numpy only; shares nothing with the kernels.  Layouts as in ``include/bitnet_a48.h``."""
import numpy as np

BLOCK = 128
GRID = np.array([(m / 8.0) * 2.0 ** -6 if e == 0 else (1 + m / 8.0) * 2.0 ** (e - 7) for e in range(16) for m in range(8)][:127])  # code -> value


def nearest_code(t):
    """Codes (uint8) of the e4m3 numbers nearest to |t| <= 448, ties to the even code; the sign bit kept for -0 too."""
    a = np.minimum(np.abs(t), 448.0)
    hi = np.clip(np.searchsorted(GRID, a), 0, 126)
    lo = np.maximum(hi - 1, 0)
    up, down = GRID[hi] - a, a - GRID[lo]
    code = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    return (code | np.where(np.signbit(t), 128, 0)).astype(np.uint8)


def value(codes):
    c = np.asarray(codes, np.uint8)
    v = np.append(GRID, np.nan)[c & 127]
    return np.where(c & 128, -v, v)


def quant_rows(x, gain=None, eps=1e-5):
    """(codes uint8 [M, K], scales float64 [blocks, M])."""
    x = np.asarray(x, np.float64)
    M, K = x.shape
    size = np.ones(M)
    if gain is not None:
        size = 1.0 / np.sqrt((x * x).mean(1) + eps)
        x = x * np.asarray(gain, np.float64)
    codes, scale = np.zeros((M, K), np.uint8), np.zeros(((K + BLOCK - 1) // BLOCK, M))
    for b in range(scale.shape[0]):
        part = x[:, b * BLOCK:(b + 1) * BLOCK]
        peak = np.abs(part).max(1)
        fine = np.isfinite(peak)
        p = np.where(fine & (peak > 0), peak, 1.0)
        got = nearest_code(np.where(fine[:, None], part, 0.0) * 448.0 / p[:, None])
        codes[:, b * BLOCK:(b + 1) * BLOCK] = np.where((fine & (peak > 0))[:, None], got, 0)
        scale[b] = np.where(fine, peak / 448.0 * size, np.nan)
    return codes, scale


def quant_weight(w):
    """(codes uint8 [N, K], scales float64 [row blocks, channel blocks])."""
    w = np.asarray(w, np.float64)
    N, K = w.shape
    nb, kb = (N + BLOCK - 1) // BLOCK, (K + BLOCK - 1) // BLOCK
    codes, scale = np.zeros((N, K), np.uint8), np.zeros((nb, kb))
    for i in range(nb):
        for j in range(kb):
            at = np.s_[i * BLOCK:(i + 1) * BLOCK, j * BLOCK:(j + 1) * BLOCK]
            peak = np.abs(w[at]).max()
            scale[i, j] = peak / 448.0 if np.isfinite(peak) else np.nan
            if np.isfinite(peak) and peak > 0:
                codes[at] = nearest_code(w[at] * 448.0 / peak)
    return codes, scale


def linear(codes, scale, w_codes, w_scale):
    """(y, sum of the absolute terms), float64 [M, N]."""
    M, K = codes.shape
    N = w_codes.shape[0]
    xv = value(codes) * np.repeat(np.asarray(scale, np.float64).T, BLOCK, 1)[:, :K]
    wv = value(w_codes) * np.repeat(np.repeat(np.asarray(w_scale, np.float64), BLOCK, 0)[:N], BLOCK, 1)[:, :K]
    return xv @ wv.T, np.abs(xv) @ np.abs(wv).T


def logprobs(x, tokens, top=0, temperature=1.0):
    """dict of logprob, entropy, rank, top_ids, top_logprobs of rows of logits, and the spread |d| that errors grow with."""
    x = np.asarray(x, np.float64)
    M, V = x.shape
    out = {"logprob": np.full(M, np.nan), "entropy": np.full(M, np.nan), "rank": np.full(M, -1), "top_ids": np.full((M, top), -1),
           "top_logprobs": np.full((M, top), np.nan), "mean": np.zeros(M), "spread": np.zeros(M)}
    for m in range(M):
        row, t = x[m], int(tokens[m])
        peak = row.max()
        if np.isnan(row).any() or peak == np.inf or peak == -np.inf:
            continue
        d = np.float64(1.0 / temperature) * (row - peak)
        e = np.exp(d)
        total = e.sum()
        logp = d - np.log(total)
        live = e > 0
        out["entropy"][m] = np.log(total) - (e[live] * d[live]).sum() / total
        out["mean"][m] = -(e[live] * d[live]).sum() / total
        out["spread"][m] = min(110.0, float(-d[np.isfinite(d)].min()))
        order = np.lexsort((np.arange(V), -row))
        if 0 <= t < V:
            out["logprob"][m] = logp[t]
            out["rank"][m] = int(np.flatnonzero(order == t)[0])
        else:
            out["logprob"][m] = 0.0
        out["top_ids"][m] = order[:top]
        out["top_logprobs"][m] = logp[order[:top]]
    return out
