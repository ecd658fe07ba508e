"""Cases for measuring the paged low-bit key/value cache and the attention over it.

Three operators: `write` rotates the queries and keys of new tokens (RoPE), quantises keys and values per head vector to
8, 4 or 3 bits and stores them in the pages of a cache, from where they are read back; `read` dequantises positions of
many sequences out of the pages; `attend` is causal attention of new tokens (one per sequence while decoding, many while
prefilling) over the pages, with an optional sliding window beside which the first tokens stay visible (sinks).

`run` computes them in plain torch operations (`own` false) or through the framework's calls (`own` true); `exact`
evaluates the same definitions in 64 bits.

Cache layout, the one the framework's calls read and write: pool uint8 [pages, kv heads, chunk]; a chunk holds, for the
`page` positions of the page,
    key codes [page, row] | value codes [page, row] | key scales fp32 [page] | value scales fp32 [page]
    | 3 bits only: 4-bit codes of the key and of the value at position 0 of a sequence (its bos token) [2, P / 2]
where P is the head dimension padded to a multiple of 32 and row = P * bits / 8.  An entry is u = q + L + 1 >= 0 with
L = 2^(bits-1) - 1 and stands for scale * q.  8 bits: one byte per entry; 4 bits: entry 2i in the low half of byte i;
3 bits: 32 entries in three 32-bit words, entries 5j..5j+4 in bits 0..14 of word j's low half, entry 15 in the top bits
of the three low halves, entries 16..31 the same way in the high halves.
"""
import math
import random

import torch

own = False

EPS, ROPE_BASE = 1e-5, 10000.0


# ------------------------------------------------------------------------------------------------ cases
def listed():
    """Head shapes are the 7B (32 heads of 128), 3B (32 of 100) and 700M (16 of 96) models', the same with shared
    key/value heads, and heads of 64; batches 1, 8, 32 and 64 and contexts of 2048 are the decode benchmark's, prompts
    of 4096 and 2048 tokens the prefill benchmark's."""
    return [
        # one decoding step of eight sequences of the 7B shape: the smallest write, all latency
        _case("write_decode_b8", "write", bits=3, heads=32, kv_heads=32, hd=128, page=64, seqs=8, q=1, kv=2048, kv_min=301, x="fp32"),
        # a ragged prompt batch, q, k and v side by side in one bf16 projection
        _case("write_prompts", "write", bits=4, heads=32, kv_heads=8, hd=128, page=64, seqs=5, q=4096, q_min=37, kv=4096, x="bf16", fused=True),
        # the prompts of the 700M shape, fp32 as the contraction leaves them
        _case("write_prompt_700m", "write", bits=8, heads=16, kv_heads=16, hd=96, page=16, seqs=1, q=2048, kv=2048, x="fp32"),
        # the cached prefix of a batch brought back, e.g. to be handed to another worker
        _case("read_prefix", "read", bits=4, heads=32, kv_heads=8, hd=128, page=64, seqs=32, q=4096, q_min=511, kv=4096, x="bf16"),
        # one 3B-shape context in full precision
        _case("read_one_3b", "read", bits=3, heads=32, kv_heads=32, hd=100, page=32, seqs=1, q=2047, kv=2048, x="fp32"),
        # one token of one 7B sequence: the smallest attention, all latency
        _case("decode_b1", "attend", bits=3, heads=32, kv_heads=32, hd=128, page=64, seqs=1, q=1, kv=2048),
        # a serving batch with shared key/value heads at ragged lengths
        _case("decode_b64_shared", "attend", bits=4, heads=32, kv_heads=8, hd=128, page=64, seqs=64, q=1, kv=8192, kv_min=130),
        # long contexts through a window with sinks, several tokens per sequence (drafted tokens being verified)
        _case("verify_window", "attend", bits=8, heads=32, kv_heads=8, hd=64, page=32, seqs=8, q=4, kv=32768, kv_min=9001, window=4096, sinks=4),
        # decoding the 3B shape at batch 32
        _case("decode_b32_3b", "attend", bits=4, heads=32, kv_heads=32, hd=100, page=128, seqs=32, q=1, kv=2048, kv_min=1500),
        # a scheduler's mixed step: two chunks of prompts beside thirty decoding sequences
        _case("mixed_step", "attend", bits=4, heads=32, kv_heads=8, hd=128, page=64, seqs=32, q=513, q_min=1, long=2, kv=4100, kv_min=517),
        # the 7B prefill, four prompts at once
        _case("prefill_7b", "attend", bits=3, heads=32, kv_heads=32, hd=128, page=64, seqs=4, q=4096, kv=4096),
        # a chunk of a long prompt behind its cached part, window and sinks
        _case("chunk_window", "attend", bits=8, heads=32, kv_heads=8, hd=128, page=64, seqs=2, q=2048, q_min=1333, kv=16384, kv_min=12345, window=2048, sinks=4),
    ]


def _case(name, op, *, bits, heads, kv_heads, hd, page, seqs, q, kv, x="bf16", q_min=None, kv_min=None, long=0, window=0, sinks=0, fused=False):
    """q, kv: the largest number of new tokens and of positions per sequence, q_min, kv_min the smallest; long: so many
    sequences have q new tokens and the others q_min (0: spread evenly)."""
    case = {"op": op, "bits": bits, "heads": heads, "kv_heads": kv_heads, "hd": hd, "page": page, "seqs": seqs, "q": q,
            "q_min": q if q_min is None else q_min, "kv": kv, "kv_min": kv if kv_min is None else kv_min, "long": long,
            "window": window, "sinks": sinks, "x": x, "fused": fused}
    return dict(case, name=name) if name else case


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    while True:
        op = rng.choice(["write", "read", "attend", "attend", "attend"])
        heads, kv_heads = rng.choice([(32, 32), (16, 16), (32, 8), (32, 4), (24, 8), (28, 4), (16, 1), (8, 8)])
        hd = rng.choice([64, 96, 100, 128, 128, 128])
        seqs = _log_int(rng, 1, 64)
        kv = _log_int(rng, 1, 32768)
        kv_min = rng.randint(max(1, kv // 8), kv)
        window = sinks = long = q_min = 0
        if op == "attend":
            form = rng.choice(["decode", "verify", "chunk", "mixed"])
            q = {"decode": 1, "verify": rng.randint(2, 8)}.get(form) or _log_int(rng, 9, 4096)
            q_min = q if form in ("decode", "verify") else 1 if form == "mixed" else rng.randint(max(1, q // 2), q)
            long = rng.randint(1, max(1, seqs // 8)) if form == "mixed" else 0
            if rng.random() < 0.4:
                window, sinks = _log_int(rng, 64, 8192), rng.choice([0, 1, 4, 16])
        elif op == "write":
            q = _log_int(rng, 1, 4096)
            q_min = rng.randint(max(1, q // 8), q)
        else:
            q = kv
            q_min = rng.randint(max(1, q // 8), q)
        kv, kv_min = max(kv, q), max(kv_min, q)
        case = _case("", op, bits=rng.choice([3, 4, 8]), heads=heads, kv_heads=kv_heads, hd=hd, page=rng.choice([16, 32, 64, 64, 128]),
                     seqs=seqs, q=q, q_min=q_min, kv=kv, kv_min=kv_min, long=long, window=window, sinks=sinks,
                     x=rng.choice(["bf16", "fp32"]) if op != "attend" else "bf16", fused=op == "write" and rng.random() < 0.5)
        w = work(case)
        if w["flops"] > 4.5e11 or w["bytes"] > 1.3e9 or seqs * kv * kv_heads > 4.2e6:
            continue  # no larger than the largest listed ones
        if op == "attend" and seqs * heads * q * kv > 2.1e9:
            continue  # the plain form's padded scores
        return case


def _lengths(case):
    """(new tokens, positions) of every sequence: spread evenly between the case's limits, in a fixed order."""
    n, order = case["seqs"], random.Random(case["seqs"] * 1000003 + case["kv"])

    def spread(lo, hi):
        v = [hi - (hi - lo) * i // max(1, n - 1) for i in range(n)]
        order.shuffle(v)
        return v

    q = [case["q"]] * case["long"] + [case["q_min"]] * (n - case["long"]) if case["long"] else spread(case["q_min"], case["q"])
    kv = [max(a, b) for a, b in zip(q, spread(case["kv_min"], case["kv"]))]
    return q, kv


def work(case):
    q, kv = _lengths(case)
    tokens, hd, row = sum(q), case["hd"], _padded(case["hd"]) * case["bits"] // 8 + 4
    x = 4 if case["x"] == "fp32" else 2
    packed = 2 * case["kv_heads"] * row  # of one position
    if case["op"] == "write":
        new = (case["heads"] + 2 * case["kv_heads"]) * hd
        back = 2 * case["kv_heads"] * hd * 4
        return {"bytes": tokens * (new * x + case["heads"] * hd * 2 + 2 * packed + back), "flops": tokens * new * 6}
    if case["op"] == "read":
        return {"bytes": tokens * (packed + 2 * case["kv_heads"] * hd * x), "flops": tokens * 2 * case["kv_heads"] * hd}
    pairs = seen = 0
    for t, n in zip(q, kv):
        first = n - t  # position of the first new token
        if case["window"]:
            w, s = case["window"], case["sinks"]
            for p in range(first, n):
                lo = max(0, p + 1 - w)
                pairs += p + 1 - lo + min(s, lo)
            lo = max(0, first + 1 - w)
            seen += n - lo + min(s, lo)
        else:
            pairs += t * first + t * (t + 1) // 2
            seen += n
    return {"bytes": tokens * case["heads"] * hd * 4 + seen * packed, "flops": 4 * hd * case["heads"] * pairs}


# ------------------------------------------------------------------------------------------------ layout
def _padded(hd):
    return (hd + 31) // 32 * 32


def _sections(case):
    """Byte offsets in a chunk: key codes, value codes, key scales, value scales, position 0's codes, end."""
    row, page, P = _padded(case["hd"]) * case["bits"] // 8, case["page"], _padded(case["hd"])
    at = [0]
    for n in (page * row, page * row, page * 4, page * 4, P if case["bits"] == 3 else 0):
        at.append(at[-1] + n)
    return at


def _pack(u, bits):
    """Entries [..., P] (int32, unsigned codes) -> bytes [..., P * bits / 8]."""
    if bits == 8:
        return u.to(torch.uint8)
    if bits == 4:
        return (u[..., 0::2] | (u[..., 1::2] << 4)).to(torch.uint8)
    h = u.unflatten(-1, (-1, 2, 16))  # granule, half, entry
    at = torch.arange(5, device=u.device, dtype=torch.int32) * 3
    words = [(h[..., 5 * j:5 * j + 5] << at).sum(-1, dtype=torch.int32) | (((h[..., 15] >> j) & 1) << 15) for j in range(3)]
    w = torch.stack(words, -2)  # granule, word, half
    return torch.where(w >= 32768, w - 65536, w).to(torch.int16).contiguous().view(torch.uint8).flatten(-3)


def _unpack(b, bits):
    """Bytes [..., P * bits / 8] -> entries [..., P], int32."""
    if bits == 8:
        return b.to(torch.int32)
    if bits == 4:
        return torch.stack((b & 15, b >> 4), -1).flatten(-2).to(torch.int32)
    w = b.contiguous().view(torch.int16).to(torch.int32).unflatten(-1, (-1, 3, 2)) & 0xFFFF  # granule, word, half
    at = torch.arange(5, device=b.device, dtype=torch.int32) * 3
    five = (w.unsqueeze(-1) >> at) & 7  # granule, word, half, entry
    top = ((w >> 15) << torch.arange(3, device=b.device, dtype=torch.int32)[:, None]).sum(-2, dtype=torch.int32)
    return torch.cat((five.transpose(-3, -2).flatten(-2), top.unsqueeze(-1)), -1).flatten(-3)


def _part(pool, case, i):
    """Codes (i = 0 keys, 1 values) [pages, kv heads, page, row] or scales (2, 3) [pages, kv heads, page], as views."""
    at = _sections(case)
    part = pool[:, :, at[i]:at[i + 1]]
    return part.unflatten(-1, (case["page"], -1)) if i < 2 else part.view(torch.float32)


def _bos(pool, case):
    """Codes of position 0 in a 3-bit cache, [pages, kv heads, 2, P / 2]."""
    at = _sections(case)
    return pool[:, :, at[4]:at[5]].unflatten(-1, (2, -1))


# ------------------------------------------------------------------------------------------------ inputs
def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    q_len, kv_len = _lengths(case)
    tokens, kvh, hd, page, bits = sum(q_len), case["kv_heads"], case["hd"], case["page"], case["bits"]
    counts = [(n + page - 1) // page for n in kv_len]
    total, width = sum(counts), max(counts)
    n_pages = total + 3
    order = torch.randperm(n_pages, generator=g, device=dev)[:total].to(torch.int32)  # pages in no order, as after some service
    table = torch.full((case["seqs"], width), -1, dtype=torch.int32, device=dev)
    counts_dev = torch.tensor(counts, device=dev)
    table[torch.arange(width, device=dev)[None, :] < counts_dev[:, None]] = order
    state = {
        "case": case, "table": table, "tokens": tokens,
        "q_start": torch.tensor([0] + q_len, device=dev).cumsum(0).to(torch.int32),
        "kv_len": torch.tensor(kv_len, device=dev, dtype=torch.int32),
        "pool": torch.zeros(n_pages, kvh, _sections(case)[-1], dtype=torch.uint8, device=dev),
    }
    xt = torch.float32 if case["x"] == "fp32" else torch.bfloat16
    if case["op"] == "write":  # what the projections give: a few channels carry larger values
        shapes = [case["heads"] * hd, kvh * hd, kvh * hd]
        x = torch.randn(tokens, sum(shapes), generator=g, device=dev)
        x *= torch.where(torch.rand(sum(shapes), generator=g, device=dev) < 0.01, 8.0, 1.0)
        x = x.to(xt)
        state["qkv"] = list(x.split(shapes, 1)) if case["fused"] else [t.contiguous() for t in x.split(shapes, 1)]
        return state
    # a cache in service: every slot of its pages has been written at some time, those behind a sequence's end too
    first = table[:, 0].long()
    for i in range(2):
        head = torch.randn(n_pages, kvh, page, hd, generator=g, device=dev)
        if i == 1:
            head[first, :, 0] *= 0.1  # values of a first token are small where it serves as a sink
        codes, scale = _quantise(head, bits)
        _part(state["pool"], case, i).copy_(_pack(_padding(codes, hd, bits), bits))
        _part(state["pool"], case, 2 + i).copy_(scale)
        if bits == 3:
            codes, scale = _quantise(head[:, :, 0], 4)
            _bos(state["pool"], case)[:, :, i].copy_(_pack(_padding(codes, hd, 4), 4))
            _part(state["pool"], case, 2 + i)[first, :, 0] = scale[first]
    if case["op"] == "attend":
        state["q"] = (1.5 * torch.randn(tokens, case["heads"] * hd, generator=g, device=dev)).to(torch.bfloat16)
    return state


def _padding(u, hd, bits):
    return torch.nn.functional.pad(u, (0, _padded(hd) - hd), value=2 ** (bits - 1))  # the code of 0


def _quantise(x, bits):
    """Unsigned codes (int32) and scales of head vectors [..., hd]; in the type of x."""
    L = 2 ** (bits - 1) - 1
    gamma = x.abs().amax(-1, keepdim=True)
    q = torch.clamp(torch.round(L / (gamma + EPS) * x), -(L + 1), L)
    return q.to(torch.int32) + (L + 1), (gamma[..., 0] / L).to(torch.float32)


# ------------------------------------------------------------------------------------------------ one pass
def run(state):
    if own:
        return _run_own(state)
    return {"write": _plain_write, "read": _plain_read, "attend": _plain_attend}[state["case"]["op"]](state)


def _run_own(state):
    from paper_2411_04965_b200 import binding as a48

    case = state["case"]
    if "cache" not in state:  # a serving program makes the handle with the pool, once
        state["cache"] = a48.PagedCache(case["bits"], case["kv_heads"], case["hd"], case["page"], state["pool"].shape[0], pool=state["pool"])
    cache = state["cache"]
    batch = a48.PagedBatch(state["q_start"], state["kv_len"], state["table"], state["tokens"], case["q"], case["kv"])
    if case["op"] == "write":
        q, k, v = state["qkv"]
        q = a48.paged_write(cache, batch, k, v, q=q, rope_base=ROPE_BASE, eps=EPS)
        k, v = a48.paged_read(cache, batch, dtype=torch.float32)
        return {"q": q, "k": k, "v": v}
    if case["op"] == "read":
        k, v = a48.paged_read(cache, batch, dtype=torch.float32 if case["x"] == "fp32" else torch.bfloat16)
        return {"k": k, "v": v}
    return {"out": a48.attention_paged(cache, batch, state["q"], window=case["window"], sinks=case["sinks"])}


def _places(state):
    """Sequence, index among its new tokens, position, page and slot of every new token."""
    case = state["case"]
    row = torch.arange(state["tokens"], device=state["pool"].device)
    starts = state["q_start"].long()
    b = torch.searchsorted(starts, row, right=True) - 1
    i = row - starts[b]
    pos = state["kv_len"].long()[b] - (starts[b + 1] - starts[b]) + i
    page = state["table"].long()[b, pos // case["page"]]
    return b, i, pos, page, pos % case["page"]


def _rotate(x, cos, sin):
    lo, hi = x.chunk(2, -1)
    return torch.cat((lo * cos - hi * sin, hi * cos + lo * sin), -1)


def _plain_write(state):
    case, pool = state["case"], state["pool"]
    hd, bits = case["hd"], case["bits"]
    _, _, pos, page, slot = _places(state)
    q, k, v = (x.double().unflatten(-1, (-1, hd)) for x in state["qkv"])
    freq = ROPE_BASE ** (-torch.arange(hd // 2, device=pool.device, dtype=torch.float64) / (hd // 2))
    angle = (pos.double()[:, None] * freq)[:, None, :]
    cos, sin = angle.cos(), angle.sin()
    q, k = _rotate(q, cos, sin), _rotate(k, cos, sin)
    for i, x in enumerate((k, v)):
        codes, scale = _quantise(x, bits)
        rows = _pack(_padding(codes, hd, bits), bits)
        if bits == 3:
            zero = pos == 0
            four, four_scale = _quantise(x, 4)
            _bos(pool, case)[page[zero], :, i] = _pack(_padding(four, hd, 4), 4)[zero]
            scale = torch.where(zero[:, None], four_scale, scale)
        _part(pool, case, i)[page, :, slot] = rows
        _part(pool, case, 2 + i)[page, :, slot] = scale
    return {"q": q.flatten(1).to(torch.bfloat16), **_plain_read(state)}


def _plain_read(state):
    case, pool = state["case"], state["pool"]
    hd, bits = case["hd"], case["bits"]
    _, _, pos, page, slot = _places(state)
    out = {}
    for i, name in enumerate(("k", "v")):
        value = _unpack(_part(pool, case, i)[page, :, slot], bits)[..., :hd].float() - 2 ** (bits - 1)
        if bits == 3:
            four = _unpack(_bos(pool, case)[page, :, i], 4)[..., :hd].float() - 8
            value = torch.where((pos == 0)[:, None, None], four, value)
        out[name] = (value * _part(pool, case, 2 + i)[page, :, slot][..., None]).to(torch.float32 if case["x"] == "fp32" or case["op"] == "write" else torch.bfloat16)
    return out


def _plain_attend(state):
    case, pool = state["case"], state["pool"]
    hd, bits, kvh, B = case["hd"], case["bits"], case["kv_heads"], case["seqs"]
    group = case["heads"] // kvh
    b, i, pos, _, _ = _places(state)
    Q = torch.zeros(B, case["q"], kvh, group, hd, device=pool.device)
    Q[b, i] = state["q"].float().unflatten(-1, (kvh, group, hd))
    Q = Q.permute(0, 2, 1, 3, 4).flatten(2, 3)  # [B, kv heads, tokens * group, hd]
    chunks = pool[state["table"].long().clamp(min=0)]  # [B, pages, kv heads, chunk]
    heads = []
    for n in range(2):
        codes = _unpack(_part(chunks.flatten(0, 1), case, n), bits)[..., :hd].float() - 2 ** (bits - 1)
        codes = codes.unflatten(0, (B, -1))  # [B, pages, kv heads, page, hd]
        if bits == 3:
            codes[:, 0, :, 0] = _unpack(_bos(chunks[:, 0], case)[:, :, n], 4)[..., :hd].float() - 8
        codes *= _part(chunks.flatten(0, 1), case, 2 + n).unflatten(0, (B, -1))[..., None]
        heads.append(codes.permute(0, 2, 1, 3, 4).flatten(2, 3))  # [B, kv heads, positions, hd]
    K, V = heads
    j = torch.arange(K.shape[2], device=pool.device)
    first = state["kv_len"].long() - (state["q_start"][1:] - state["q_start"][:-1]).long()
    at = (first[:, None] + torch.arange(case["q"], device=pool.device)).repeat_interleave(group, 1)[..., None]  # [B, rows, 1]
    live = (j < state["kv_len"][:, None])[:, None, :] & (j <= at)
    if case["window"]:
        live &= (j > at - case["window"]) | (j < case["sinks"])
    S = (Q @ K.transpose(-1, -2)) / math.sqrt(hd)
    S.masked_fill_(~live[:, None], -math.inf)
    m = S.amax(-1, keepdim=True)
    S = torch.exp(S.sub_(torch.where(m == -math.inf, 0.0, m)))
    V = torch.where((j < state["kv_len"][:, None])[:, None, :, None], V, 0.0)
    total = S.sum(-1, keepdim=True)
    O = (S @ V) / torch.where(total == 0, 1.0, total)
    O = O.unflatten(2, (case["q"], group)).permute(0, 2, 1, 3, 4)  # [B, tokens, kv heads, group, hd]
    return {"out": O[b, i].flatten(1).to(torch.bfloat16)}


# ------------------------------------------------------------------------------------------------ in 64 bits
def exact(case, seed):
    state = prepare(case, seed)
    starts, lens, table = state["q_start"].tolist(), state["kv_len"].tolist(), state["table"].long()
    dev, hd, kvh, heads = state["pool"].device, case["hd"], case["kv_heads"], case["heads"]
    if case["op"] == "write":
        q, k, v = (x.double() for x in state["qkv"])
        place = torch.cat([torch.arange(n - (e - s), n, device=dev, dtype=torch.float64) for s, e, n in zip(starts, starts[1:], lens)])
        rates = torch.tensor([ROPE_BASE ** (-2.0 * i / hd) for i in range(hd // 2)], device=dev, dtype=torch.float64)
        turn = torch.polar(torch.ones_like(place[:, None] * rates), place[:, None] * rates)  # the pair (i, i + hd/2) as a complex number

        def turned(x):
            x = x.reshape(x.shape[0], -1, 2, hd // 2)
            z = torch.complex(x[:, :, 0], x[:, :, 1]) * turn[:, None]
            return torch.cat((z.real, z.imag), -1)

        def stored(x):
            gamma = x.abs().max(-1).values[..., None]
            wide = torch.full_like(place, 4.0 if case["bits"] == 3 else case["bits"])  # bits of every position
            bits = torch.where(place == 0, wide, torch.full_like(place, case["bits"]))[:, None, None]
            L = 2.0 ** (bits - 1) - 1
            code = torch.minimum(torch.maximum((L / (gamma + EPS) * x).round(), -(L + 1)), L)
            return gamma / L * code

        return {"q": turned(q).reshape(q.shape), "k": stored(turned(k)), "v": stored(v.reshape(v.shape[0], -1, hd))}

    def head(b, n, i):
        """Keys (i = 0) or values (1) of positions 0 .. n - 1 of sequence b, [n, kv heads, hd]."""
        held = table[b, :(n + case["page"] - 1) // case["page"]]
        pages = state["pool"][held]
        at, bits, P = _sections(case), case["bits"], _padded(hd)
        raw = pages[:, :, at[i]:at[i + 1]].reshape(len(held), kvh, case["page"], -1)
        scale = pages[:, :, at[2 + i]:at[3 + i]].contiguous().view(torch.float32).double()
        u = torch.empty(len(held), kvh, case["page"], P, dtype=torch.float64, device=dev)
        if bits == 8:
            u.copy_(raw)
        elif bits == 4:
            u[..., 0::2], u[..., 1::2] = (raw % 16).double(), (raw // 16).double()
        else:
            words = raw.reshape(*raw.shape[:-1], P // 32, 3, 2, 2).long()  # granule, word, half, byte
            halves = words[..., 0] + 256 * words[..., 1]
            for e in range(32):
                side, n_th = e // 16, e % 16
                if n_th < 15:
                    entry = (halves[..., n_th // 5, side] // 8 ** (n_th % 5)) % 8
                else:
                    entry = sum((halves[..., w, side] // 32768) * 2 ** w for w in range(3))
                u.reshape(*u.shape[:-1], P // 32, 32)[..., e] = entry.double()
        value = (u - 2 ** (bits - 1)) * scale[..., None]
        if bits == 3:
            bos = pages[0, :, at[4]:at[5]].reshape(kvh, 2, -1)[:, i]
            four = torch.stack((bos % 16, bos // 16), -1).reshape(kvh, P).double()
            value[0, :, 0] = (four - 8) * scale[0, :, 0, None]
        return value.permute(0, 2, 1, 3).reshape(-1, kvh, P)[:n, :, :hd]

    if case["op"] == "read":
        parts = [[head(b, n, i)[n - (e - s):] for b, (s, e, n) in enumerate(zip(starts, starts[1:], lens))] for i in range(2)]
        return {"k": torch.cat(parts[0]), "v": torch.cat(parts[1])}
    out = torch.zeros(state["tokens"], heads, hd, dtype=torch.float64, device=dev)
    q = state["q"].double().reshape(state["tokens"], heads, hd)
    for b, (s, e, n) in enumerate(zip(starts, starts[1:], lens)):
        K, V = head(b, n, 0), head(b, n, 1)
        for t0 in range(s, e, 512):  # a stretch of new tokens at a time
            t1 = min(e, t0 + 512)
            at = torch.arange(n - (e - t0), n - (e - t1), device=dev)[:, None]
            j = torch.arange(n, device=dev)
            hidden = j > at
            if case["window"]:
                hidden |= (j <= at - case["window"]) & (j >= case["sinks"])
            for h in range(kvh):
                group = slice(h * (heads // kvh), (h + 1) * (heads // kvh))
                s_ = torch.einsum("tgd,nd->gtn", q[t0:t1, group], K[:, h]) / hd ** 0.5
                p = torch.softmax(s_.masked_fill(hidden, -math.inf), -1)
                out[t0:t1, group] = torch.einsum("gtn,nd->tgd", p, V[:, h])
    return {"out": out.reshape(state["tokens"], heads * hd)}
