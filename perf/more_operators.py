"""Cases for measuring the 8-bit output head: the matrix that stays out of the ternary layers, and what is read off its logits.

Four operators: `quant` rounds token rows (optionally RMS-normalised first) or a weight matrix to e4m3 with a scale for each
block of 128 channels (of 128 x 128 entries for a weight); `linear` is the product of two such matrices; `logprobs` gives, for
rows of logits, the log probability of a given token, its place in the order of all tokens, the row's entropy and the most
likely tokens; `score` goes from hidden states to the log probability of the given tokens and the entropy, without logits.

`run` computes them in plain torch operations (`own` false) or through the framework's calls (`own` true); `exact` evaluates
the same definitions in 64 bits.

Layouts: codes e4m3 [rows, K]; the scales of token rows fp32 [ceil(K / 128), rows] (a block's scales of all tokens side by
side), those of a weight [N, K] fp32 [ceil(N / 128), ceil(K / 128)].  An entry stands for scale * code, scale = amax / 448.
A block of zeros has scale 0.  A token of -1 stands for no token (padding): log probability 0, place -1.  A row whose logits
give no distribution (a NaN, +inf, or nothing but -inf) has NaN everywhere and -1 for places and tokens.
"""
import math
import random

import torch

own = False

BLOCK, TOP_CODE, NORM_EPS = 128, 448.0, 1e-5


# ------------------------------------------------------------------------------------------------ cases
def listed():
    """Hidden sizes 4096, 3200 and 1536 are the 7B, 3B and 700M models', 11008 the 7B feed-forward's, batches 1, 8 and 64 the
    decode benchmark's, 2048, 4096 and 16384 tokens the prefill benchmark's; vocabularies of 32000 and 128000 are generic."""
    return [
        # hidden states of one decoding step on their way into the head: all latency
        _case("quant_decode_b8", "quant", rows=8, k=3200, x="bf16", norm=True),
        # four prompts of the 7B shape, as the last block leaves them
        _case("quant_prompts_7b", "quant", rows=16384, k=4096, x="fp32", norm=True),
        # a head's matrix, once at loading
        _case("quant_weight_7b", "quant_weight", rows=32000, k=4096, x="bf16"),
        # one token of one sequence through the 7B head: the matrix is read once, nothing else counts
        _case("head_decode_b1", "linear", rows=1, n=32000, k=4096, y="fp32"),
        # a batch of single tokens through the 3B head
        _case("head_decode_b64_3b", "linear", rows=64, n=32000, k=3200, y="fp32"),
        # a projection of a 7B layer kept in 8 bits, ragged packed prompts
        _case("linear_ragged_7b", "linear", rows=1999, n=11008, k=4096, y="bf16"),
        # all logits of a prompt of 4096 tokens, 7B head: the largest product
        _case("head_prompt_7b", "linear", rows=4096, n=32000, k=4096, y="fp32"),
        # logits of a decoding step with twenty alternatives, as a serving interface returns them
        _case("logprobs_decode_b8", "logprobs", rows=8, n=32000, top=20, x="fp32"),
        # scoring whole prompts, some of it padding
        _case("logprobs_prompts", "logprobs", rows=4096, n=32000, top=1, x="fp32", padded=0.1),
        # a large odd vocabulary in bf16 where a grammar allows few tokens, above temperature one
        _case("logprobs_masked_wide", "logprobs", rows=517, n=128001, top=5, x="bf16", allowed=0.02, temperature=1.3),
        # likelihood of the four endings of one question, the 3B head
        _case("score_endings_3b", "score", rows=61, n=32000, k=3200, x="bf16"),
        # perplexity of a prompt of 4096 tokens, the 7B head
        _case("score_prompt_7b", "score", rows=4096, n=32000, k=4096, x="bf16", padded=0.05),
    ]


def _case(name, op, *, rows, n=0, k=0, x="bf16", y="fp32", norm=False, top=0, padded=0.0, allowed=1.0, temperature=1.0):
    """rows: tokens, or rows of the weight; n: output features or vocabulary; k: channels; padded: share of rows without a
    token; allowed: share of the vocabulary that is not masked."""
    case = {"op": op, "rows": rows, "n": n, "k": k, "x": x, "y": y, "norm": norm, "top": top, "padded": padded,
            "allowed": allowed, "temperature": temperature}
    return dict(case, name=name) if name else case


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    while True:
        op = rng.choice(["quant", "quant", "quant_weight", "linear", "linear", "linear", "logprobs", "logprobs", "score", "score"])
        k = rng.choice([1536, 2048, 3200, 4096, 16 * _log_int(rng, 4, 688)])
        x = rng.choice(["bf16", "fp32"])
        if op == "quant":
            case = _case("", op, rows=_log_int(rng, 1, 16384), k=k, x=x, norm=rng.random() < 0.6)
        elif op == "quant_weight":
            case = _case("", op, rows=_log_int(rng, 64, 32000), k=k, x=x)
        elif op == "linear":
            case = _case("", op, rows=_log_int(rng, 1, 4096), n=_log_int(rng, 100, 32000), k=k, y=rng.choice(["bf16", "fp32"]))
        elif op == "logprobs":
            case = _case("", op, rows=_log_int(rng, 1, 4096), n=_log_int(rng, 100, 128000), top=rng.choice([0, 1, 5, 20, 64]), x=x,
                         padded=rng.choice([0.0, 0.1]), allowed=rng.choice([1.0, 1.0, 0.3, 0.01]), temperature=rng.choice([1.0, 1.0, 0.7, 1.5]))
        else:
            case = _case("", op, rows=_log_int(rng, 1, 4096), n=_log_int(rng, 1000, 32000), k=k, x=x,
                         padded=rng.choice([0.0, 0.1]), temperature=rng.choice([1.0, 0.8]))
        w = work(case)
        if w["flops"] <= 1.08e12 and w["bytes"] <= 7e8:
            return case


def _blocks(n):
    return (n + BLOCK - 1) // BLOCK


def work(case):
    rows, n, k, op = case["rows"], case["n"], case["k"], case["op"]
    x, y = (4 if case[t] == "fp32" else 2 for t in "xy")
    if op == "quant":
        return {"bytes": rows * (k * (x + 1) + 4 * _blocks(k)) + (4 * k if case["norm"] else 0), "flops": rows * k * (6 if case["norm"] else 3)}
    if op == "quant_weight":
        return {"bytes": rows * k * (x + 1) + 4 * _blocks(rows) * _blocks(k), "flops": rows * k * 3}
    weight = n * k + 4 * _blocks(n) * _blocks(k)
    if op == "linear":
        return {"bytes": rows * (k + 4 * _blocks(k)) + weight + rows * n * y, "flops": 2 * rows * n * k}
    if op == "logprobs":
        return {"bytes": rows * (n * x + 8 + 12 + 8 * case["top"]), "flops": rows * n * 6}
    return {"bytes": rows * (k * x + 8 + 8) + 4 * k + weight, "flops": 2 * rows * n * k}


# ------------------------------------------------------------------------------------------------ inputs
_TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    op, rows, n, k = case["op"], case["rows"], case["n"], case["k"]
    state = {"case": case}
    if op in ("quant", "score"):
        state["x"] = _hidden(rows, k, g).to(_TYPES[case["x"]])
        state["gain"] = 1.0 + 0.1 * _randn(g, k) if op == "score" or case["norm"] else None
    elif op == "quant_weight":
        state["w"] = (0.02 * _randn(g, rows, k)).to(_TYPES[case["x"]])
    elif op == "linear":
        state["x"] = _quantise_rows(_hidden(rows, k, g).double())
    else:
        x = 2.0 * _randn(g, rows, n)
        x[torch.arange(rows, device="cuda"), _randint(g, n, rows)] += 4.0  # mostly one token stands out
        if case["allowed"] < 1.0:
            x[torch.rand(rows, n, generator=g, device="cuda") >= case["allowed"]] = -math.inf
        state["logits"] = x.to(_TYPES[case["x"]])
    if op in ("linear", "score"):
        w = torch.empty(n, k, device="cuda", dtype=torch.bfloat16)
        w.normal_(0.0, 0.02, generator=g)
        state["w"] = _quantise_blocks(w)
    if op in ("logprobs", "score"):
        tokens = _randint(g, n, rows)
        if op == "logprobs":  # a token that was taken is an allowed one
            likely = state["logits"].argmax(-1)
            tokens = torch.where(torch.isfinite(state["logits"].gather(1, tokens[:, None])[:, 0]), tokens, likely)
        state["tokens"] = torch.where(torch.rand(rows, generator=g, device="cuda") < case["padded"], -1, tokens)
    return state


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda")


def _randint(g, n, rows):
    return torch.randint(0, n, (rows,), generator=g, device="cuda")


def _hidden(rows, k, g):
    """Hidden states: tokens of different size, one channel in a hundred far larger than the others."""
    x = _randn(g, rows, k)
    x *= torch.where(torch.rand(k, generator=g, device="cuda") < 0.01, 20.0, 1.0)
    x *= torch.exp(0.5 * _randn(g, rows, 1))
    return x


# ------------------------------------------------------------------------------------------------ one pass
def run(state):
    if own:
        return _run_own(state)
    return {"quant": _plain_quant, "quant_weight": _plain_quant_weight, "linear": _plain_linear, "logprobs": _plain_logprobs,
            "score": _plain_score}[state["case"]["op"]](state)


def _run_own(state):
    from paper_2411_04965_b200 import binding as a48

    case = state["case"]
    if case["op"] == "quant":
        codes, scale = a48.quant_fp8(state["x"], gain=state["gain"], norm_eps=NORM_EPS)
        return {"codes": codes, "scale": scale}
    if case["op"] == "quant_weight":
        codes, scale = a48.quant_fp8_weight(state["w"])
        return {"codes": codes, "scale": scale}
    if case["op"] == "linear":
        return {"y": a48.linear_fp8(*state["x"], *state["w"], dtype=_TYPES[case["y"]])}
    if case["op"] == "logprobs":
        r = a48.logprobs(state["logits"], state["tokens"], top=case["top"], temperature=case["temperature"])
        out = {"logprob": r.logprob, "entropy": r.entropy, "rank": r.rank}
        return dict(out, top_ids=r.top_ids, top_logprobs=r.top_logprobs) if case["top"] else out
    logprob, entropy = a48.score(state["x"], state["gain"], *state["w"], state["tokens"], norm_eps=NORM_EPS, temperature=case["temperature"])
    return {"logprob": logprob, "entropy": entropy}


def _to_grid(t):
    """The nearest e4m3 numbers (ties to even) of 64-bit numbers of at most 448, in 64 bits."""
    step = torch.exp2(torch.frexp(t).exponent.clamp(min=-5).double() - 4)
    return torch.round(t / step) * step


def _quantise_rows(x):
    """Codes and scales of token rows in 64 bits: a block's largest entry becomes 448, a code does not depend on the row's size."""
    rows, k = x.shape
    blocks = torch.nn.functional.pad(x, (0, -k % BLOCK)).unflatten(1, (-1, BLOCK))
    amax = blocks.abs().amax(-1)
    t = blocks * TOP_CODE / torch.where(amax == 0, 1.0, amax)[..., None]
    return _to_grid(t).flatten(1)[:, :k].to(torch.float8_e4m3fn), (amax / TOP_CODE).float().t().contiguous()


def _quantise_blocks(w):
    n, k = w.shape
    nb, kb = _blocks(n), _blocks(k)
    tiles = torch.nn.functional.pad(w, (0, -k % BLOCK, 0, -n % BLOCK)).unflatten(1, (kb, BLOCK)).unflatten(0, (nb, BLOCK))
    amax = tiles.abs().amax((1, 3)).double()
    t = tiles.double() * TOP_CODE / torch.where(amax == 0, 1.0, amax)[:, None, :, None]
    codes = _to_grid(t).to(torch.float8_e4m3fn).reshape(nb * BLOCK, kb * BLOCK)[:n, :k].contiguous()
    return codes, (amax / TOP_CODE).float()


def _normalised(x, gain):
    """(numbers to round to codes, factor of the scales): the row's size is a factor of the scale alone."""
    x = x.double()
    if gain is None:
        return x, None
    return x * gain.double(), torch.rsqrt(x.square().mean(-1) + NORM_EPS)


def _quantised_hidden(state):
    v, size = _normalised(state["x"], state["gain"])
    codes, scale = _quantise_rows(v)
    if size is not None:
        amax = torch.nn.functional.pad(v, (0, -v.shape[1] % BLOCK)).unflatten(1, (-1, BLOCK)).abs().amax(-1)
        scale = (amax / TOP_CODE * size[:, None]).float().t().contiguous()
    return codes, scale


def _plain_quant(state):
    codes, scale = _quantised_hidden(state)
    return {"codes": codes, "scale": scale}


def _plain_quant_weight(state):
    codes, scale = _quantise_blocks(state["w"])
    return {"codes": codes, "scale": scale}


def _product(x, w):
    """fp32 product of (codes, scales of rows) and (codes, scales of blocks)."""
    (xc, xs), (wc, ws) = x, w
    k = xc.shape[1]
    xf = xc.float() * xs.t().repeat_interleave(BLOCK, 1)[:, :k]
    wf = wc.float() * ws.repeat_interleave(BLOCK, 0)[:wc.shape[0]].repeat_interleave(BLOCK, 1)[:, :k]
    return xf @ wf.t()


def _plain_linear(state):
    return {"y": _product(state["x"], state["w"]).to(_TYPES[state["case"]["y"]])}


def _distribution(x, tokens, temperature):
    """log probabilities of `tokens`, entropies, and what turns a logit into a log probability: max and log of the sum."""
    x = x / temperature if temperature != 1.0 else x
    m = x.amax(-1, keepdim=True)
    d = x - m
    e = torch.exp(d)
    total = e.sum(-1)
    entropy = torch.log(total) - (e * torch.where(d == -math.inf, 0.0, d)).sum(-1) / total
    taken = d.gather(1, tokens.clamp(min=0)[:, None])[:, 0] - torch.log(total)
    return torch.where((tokens < 0) & ~torch.isnan(total), 0.0, taken), entropy, m, torch.log(total)


def _plain_logprobs(state):
    case, tokens = state["case"], state["tokens"]
    x = state["logits"].float()
    logprob, entropy, m, log_total = _distribution(x, tokens, case["temperature"])
    at = torch.arange(case["n"], device=x.device)
    own_logit = x.gather(1, tokens.clamp(min=0)[:, None])
    rank = (x > own_logit).sum(-1) + ((x == own_logit) & (at < tokens[:, None])).sum(-1)
    bad = torch.isnan(log_total)
    out = {"logprob": logprob, "entropy": entropy, "rank": torch.where((tokens < 0) | bad, -1, rank).int()}
    if case["top"]:
        bits = (x + 0.0).view(torch.int32).long()  # -0 counts as 0
        order = torch.where(bits < 0, -2147483648 - bits, bits) * 2 ** 32 + (case["n"] - 1 - at)  # equal logits: the lower index first
        ids = case["n"] - 1 - (order.topk(case["top"], -1).values & 0xFFFFFFFF)
        out["top_ids"] = torch.where(bad[:, None], -1, ids).int()
        taken = x.gather(1, ids)
        out["top_logprobs"] = (taken / case["temperature"] if case["temperature"] != 1.0 else taken) - m - log_total[:, None]
    return out


def _plain_score(state):
    logits = _product(_quantised_hidden(state), state["w"])
    logprob, entropy, _, _ = _distribution(logits, state["tokens"], state["case"]["temperature"])
    return {"logprob": logprob, "entropy": entropy}


# ------------------------------------------------------------------------------------------------ in 64 bits
def exact(case, seed):
    state = prepare(case, seed)
    op = case["op"]
    if op == "quant":
        codes, scale = _exact_rows(state["x"].double(), state["gain"])
        return {"codes": codes, "scale": scale}
    if op == "quant_weight":
        w = state["w"]
        codes, scale = torch.empty(w.shape, dtype=torch.float64, device=w.device), []
        for r in range(0, w.shape[0], BLOCK):  # a stretch of 128 rows at a time
            rows = w[r:r + BLOCK].double()
            peak = torch.stack([c.abs().max() for c in rows.split(BLOCK, 1)])
            codes[r:r + BLOCK] = _nearest(rows * 448.0 / torch.where(peak > 0, peak, 1.0).repeat_interleave(BLOCK)[:w.shape[1]])
            scale.append(peak / 448.0)
        return {"codes": codes, "scale": torch.stack(scale)}
    if op == "linear":
        return {"y": _exact_product(state["x"][0].double(), state["x"][1].double(), state["w"])}
    if op == "logprobs":
        return _exact_logprobs(state["logits"].double(), state["tokens"], case)
    logits = _exact_product(*_exact_rows(state["x"].double(), state["gain"]), state["w"])
    out = _exact_logprobs(logits, state["tokens"], dict(case, top=0))
    return {"logprob": out["logprob"], "entropy": out["entropy"]}


def _nearest(t):
    """Nearest of the e4m3 numbers by looking them up; a tie goes to the even mantissa."""
    grid = torch.arange(127, dtype=torch.uint8, device=t.device).view(torch.float8_e4m3fn).double()  # 0 .. 448
    a = t.abs().clamp(max=448.0).contiguous()
    hi = torch.searchsorted(grid, a).clamp(max=126)
    lo = (hi - 1).clamp(min=0)
    up, down = grid[hi] - a, a - grid[lo]
    take = torch.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    return grid[take] * torch.sign(t)


def _exact_rows(x, gain):
    rows, k = x.shape
    size = torch.ones(rows, dtype=torch.float64, device=x.device)
    if gain is not None:
        size = 1.0 / torch.sqrt((x * x).sum(1) / k + NORM_EPS)
        x = x * gain.double()[None]
    codes, scale = torch.empty_like(x), []
    for c in range(0, k, BLOCK):  # a block of channels at a time
        part = x[:, c:c + BLOCK]
        peak = part.abs().max(1).values
        codes[:, c:c + BLOCK] = _nearest(part * 448.0 / torch.where(peak > 0, peak, 1.0)[:, None])
        scale.append(peak / 448.0 * size)
    return codes, torch.stack(scale)


def _exact_product(codes, scale, w):
    wc, ws = w
    y = torch.zeros(codes.shape[0], wc.shape[0], dtype=torch.float64, device=codes.device)
    rows_of = torch.arange(wc.shape[0], device=codes.device) // BLOCK
    for b in range(scale.shape[0]):
        part = slice(b * BLOCK, (b + 1) * BLOCK)
        y.addmm_(codes[:, part] * scale[b][:, None], (wc[:, part].double() * ws[rows_of, b].double()[:, None]).t())
    return y


def _exact_logprobs(x, tokens, case):
    rows = torch.arange(x.shape[0], device=x.device)
    logp = torch.log_softmax(x / case["temperature"], -1)
    none, bad = tokens < 0, torch.isnan(logp[:, 0])
    p = torch.exp(logp)
    out = {"logprob": torch.where(none & ~bad, 0.0, logp[rows, tokens.clamp(min=0)]),
           "entropy": -torch.where(p > 0, p * logp, torch.where(torch.isnan(p), p, 0.0)).sum(-1)}
    del p
    if case["op"] == "logprobs":
        mine = x[rows, tokens.clamp(min=0)][:, None]
        before = torch.arange(x.shape[1], device=x.device)[None] < tokens[:, None]
        rank = torch.where(before, x >= mine, x > mine).sum(-1)
        out["rank"] = torch.where(none | bad, -1, rank).int()
    if case["top"]:
        left, ids = x.clone(), []
        gone = torch.zeros_like(x, dtype=torch.bool)
        for _ in range(case["top"]):  # the first of the largest that are left, one after the other
            best = left.masked_fill(gone, -math.inf).max(-1, keepdim=True).values
            at = ((left == best) & ~gone).int().argmax(-1)
            gone[rows, at] = True
            ids.append(at)
        ids = torch.stack(ids, 1)
        out["top_logprobs"] = logp.gather(1, ids)
        out["top_ids"] = torch.where(bad[:, None], -1, ids).int()
    return out
