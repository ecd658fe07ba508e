"""Paged low-bit cache and the attention over it on the GPU against the float64 oracle: codes exact, values to fp32
rounding, attention within a bound made of its roundings (`attention_bound`)."""
import numpy as np
import pytest
import torch

from oracle import paged

pytestmark = pytest.mark.gpu

EPS32 = float(np.float32(1e-5))
HALF_BF16, HALF_F16, HALF_F32 = 2.0 ** -8, 2.0 ** -11, 2.0 ** -24


class Setup:
    """A cache, a batch with a shuffled page table, and the oracle's copy of both."""

    def __init__(self, a48, dev, bits, kvh, hd, page, q_lens, kv_lens, seed=0, spare=2, tail=0, width=None, garbage=False):
        rng = np.random.default_rng(seed)
        counts = [(max(n, 0) + page - 1) // page for n in kv_lens]
        n_pages = sum(counts) + spare
        order = rng.permutation(n_pages)
        self.table = np.full((len(kv_lens), width or max(max(counts), 1)), -1, np.int32)
        at = 0
        for b, c in enumerate(counts):
            c = min(c, self.table.shape[1])
            self.table[b, :c] = order[at:at + c]
            at += c
        self.q_start = np.concatenate([[0], np.cumsum(q_lens)]).astype(np.int32)
        self.kv_len = np.array(kv_lens, np.int32)
        self.n_tokens = int(self.q_start[-1]) + tail
        self.dev, self.a48, self.bits, self.kvh, self.hd, self.page = dev, a48, bits, kvh, hd, page
        self.cache = a48.PagedCache(bits, kvh, hd, page, n_pages, device=dev)
        if garbage:  # what a recycled page may hold: bits that are no numbers
            self.cache.pool.fill_(255)
        self.oracle = paged.Cache(bits, kvh, hd, page, n_pages)
        self.batch = self.view(self.q_start, self.kv_len, self.n_tokens)

    def view(self, q_start, kv_len, n_tokens, max_q=None, max_kv=None):
        q_lens = np.diff(q_start)
        return self.a48.PagedBatch(torch.tensor(q_start, dtype=torch.int32, device=self.dev), torch.tensor(kv_len, dtype=torch.int32, device=self.dev),
                                   torch.tensor(self.table, device=self.dev), n_tokens, max_q or max(1, int(q_lens.max())),
                                   max_kv or max(1, int(np.max(kv_len))))

    def fill(self, rng, spread=1.0, dtype=torch.bfloat16):
        """All positions of every sequence written in one call (keys rotated), on both sides."""
        starts = np.concatenate([[0], np.cumsum(np.maximum(self.kv_len, 0))]).astype(np.int32)
        n = int(starts[-1])
        if n == 0:
            return
        k, v = (torch.tensor(rng.standard_normal((n, self.kvh * self.hd)) * spread, dtype=torch.float32).to(dtype) for _ in range(2))
        self.a48.paged_write(self.cache, self.view(starts, np.maximum(self.kv_len, 0), n), k.to(self.dev), v.to(self.dev))
        self.oracle.write(starts, np.maximum(self.kv_len, 0), self.table, k.double().numpy(), v.double().numpy(), 10000.0, EPS32)


def attention_bound(out, mag, top, hd, vmax):
    """Half a bf16 step of the result; half an fp16 step of every probability (times its value: `mag`); the fp32 scores, whose
    error (a product and a sum per entry, each rounded by 2^-23 at most on the tensor cores, and six more roundings: scales,
    softmax factor, difference, exponential of two units) acts on every probability and on the sum; probabilities that fall
    below fp16's range, 2^-30 of the largest value."""
    score = (hd + 6) * 2.0 ** -23 * top[..., None] + 8 * 2.0 ** -23
    return HALF_BF16 * np.abs(out) + (HALF_F16 + 2 * score) * mag * (1 + HALF_BF16) + 2.0 ** -30 * vmax + 1e-30


def check_attention(s, q, n_heads, window=0, sinks=0, scale=0.0, batch=None, **kw):
    got = s.a48.attention_paged(s.cache, batch or s.batch, q.to(s.dev), scale=scale, window=window, sinks=sinks, **kw)
    out, mag, top = s.oracle.attend(s.q_start, s.kv_len, s.table, q.double().numpy(), n_heads, scale, window, sinks)
    got = got.double().cpu().numpy().reshape(out.shape)
    rows = slice(int(s.q_start[0]), int(s.q_start[-1]))
    vmax = np.abs(s.oracle.scales[1]).max() * 128
    err, tol = np.abs(got - out)[rows], attention_bound(out, mag, top, s.hd, vmax)[rows]
    assert np.isfinite(got[rows]).all()
    worst = float((err / tol).max()) if err.size else 0.0
    assert worst <= 1.0, worst
    assert s.a48.kernel_status()[0] == 0
    return got


# ------------------------------------------------------------------------------------------------ write and read
@pytest.mark.parametrize("bits", [8, 4, 3])
@pytest.mark.parametrize("hd,kvh,heads,page", [(128, 2, 4, 16), (100, 1, 1, 32), (96, 3, 3, 64), (64, 2, 8, 128), (4, 1, 2, 16), (36, 5, 5, 16)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_write_codes_and_read_back(a48, cuda_dev, bits, hd, kvh, heads, page, dtype):
    rng = np.random.default_rng(hd + bits)
    q_lens, kv_lens = [3, 0, 1, 40, 17], [3, 5, 1, 77, 17 + page]
    s = Setup(a48, cuda_dev, bits, kvh, hd, page, q_lens, kv_lens, seed=hd, garbage=True)
    n = s.n_tokens
    k, v, q = (torch.tensor(rng.standard_normal((n, m * hd)) * rng.choice([1.0, 30.0], (1, m * hd)), dtype=torch.float32).to(dtype)
               for m in (kvh, kvh, heads))
    v[2] = 0  # a head of zeros
    before = s.cache.pool.cpu().numpy().copy()
    q_out = a48.paged_write(s.cache, s.batch, k.to(cuda_dev), v.to(cuda_dev), q=q.to(cuda_dev), rope_base=10000.0)
    s.oracle.write(s.q_start, s.kv_len, s.table, k.double().numpy(), v.double().numpy(), 10000.0, EPS32)
    raw = s.cache.pool.cpu().numpy()
    codes, scales, bos = paged.unpack_pool(raw, bits, kvh, hd, page, s.cache.n_pages)
    for _, b, _, pos in paged.tokens(s.q_start, s.kv_len):
        p, slot = paged.place(s.table, b, pos, page, s.cache.n_pages)
        first = bits == 3 and pos == 0
        got = bos[:, p] if first else codes[:, p, :, slot]
        want = s.oracle.bos[:, p] if first else s.oracle.codes[:, p, :, slot]
        assert np.array_equal(got[..., :hd], want)
        assert (got[..., hd:] == 0).all()  # padding is the code of zero
        ref = s.oracle.scales[:, p, :, slot]
        assert np.all(np.abs(scales[:, p, :, slot] - ref) <= HALF_F32 * ref * (1 + 1e-6))
    # slots that no token maps to are as they were (a slot's code rows and scales: compare the decoded views)
    old = paged.unpack_pool(before, bits, kvh, hd, page, s.cache.n_pages)
    touched = np.zeros((s.cache.n_pages, page), bool)
    for _, b, _, pos in paged.tokens(s.q_start, s.kv_len):
        touched[paged.place(s.table, b, pos, page, s.cache.n_pages)] = True
    for a, o in zip((codes, scales), old):
        moved = np.moveaxis(a, 3, 2)[:, ~touched], np.moveaxis(o, 3, 2)[:, ~touched]
        assert np.array_equal(*(np.ascontiguousarray(x).view(np.uint8) for x in moved))
    # the rotated queries: fp32 products (three roundings each) rounded to bf16
    qn = q.double().numpy().reshape(n, heads, hd)
    for row, _, _, pos in paged.tokens(s.q_start, s.kv_len):
        want = paged.rotate(qn[row], pos, 10000.0)
        part = np.abs(np.concatenate([qn[row][..., hd // 2:], qn[row][..., :hd // 2]], -1)) + np.abs(qn[row])
        err = np.abs(q_out[row].double().cpu().numpy().reshape(heads, hd) - want)
        assert (err <= HALF_BF16 * np.abs(want) + 4 * HALF_F32 * part * (1 + HALF_BF16)).all()
    # reading back: fp32 is the scale times the code, one rounding of the scale and one of the product; bf16 one more
    ref = s.oracle.read(s.q_start, s.kv_len, s.table, n)
    for out_dtype, tol in ((torch.float32, 2 * HALF_F32), (torch.bfloat16, HALF_BF16 + 2 * HALF_F32)):
        kv = a48.paged_read(s.cache, s.batch, dtype=out_dtype)
        for got, want in zip(kv, ref):
            assert (np.abs(got.double().cpu().numpy() - want) <= tol * np.abs(want) * (1 + 1e-6)).all()


def test_write_ties_and_far_positions(a48, cuda_dev):
    """Entries on rounding ties (exact in the input type: gamma = L makes the multiplier 1 with eps 0) round to even, and
    the angle of a position past 2^20 is that of float64."""
    hd, bits = 64, 4
    s = Setup(a48, cuda_dev, bits, 1, hd, 128, [2], [2], seed=5)
    x = torch.zeros(2, hd)
    x[0, 0], x[1, 0] = 7.0, -7.0
    x[:, 1:15] = torch.arange(14) - 6.5  # -6.5 .. 6.5
    a48.paged_write(s.cache, s.batch, x.to(cuda_dev), x.to(cuda_dev), rope_base=0.0, eps=0.0)
    k, v = a48.paged_read(s.cache, s.batch, dtype=torch.float32)
    assert torch.equal(k.cpu()[:, 0], torch.round(x)) and torch.equal(v.cpu(), k.cpu())
    n = (1 << 20) + 37  # one page table entry far out; the others have no page
    far = Setup(a48, cuda_dev, 8, 2, hd, 128, [3], [3], seed=6, width=(n + 127) // 128)
    far.kv_len = np.array([n], np.int32)
    far.table[:] = -1
    far.table[0, -1] = 1
    far.batch = far.view(far.q_start, far.kv_len, 3)
    rng = np.random.default_rng(3)
    k, v, q = (torch.tensor(rng.standard_normal((3, 2 * hd)), dtype=torch.float32) for _ in range(3))
    q_out = a48.paged_write(far.cache, far.batch, k.to(cuda_dev), v.to(cuda_dev), q=q.to(cuda_dev))
    far.oracle.write(far.q_start, far.kv_len, far.table, k.numpy(), v.numpy(), 10000.0, EPS32)
    got = a48.paged_read(far.cache, far.batch, dtype=torch.float32)
    ref = far.oracle.read(far.q_start, far.kv_len, far.table, 3)
    for a, b in zip(got, ref):
        assert (np.abs(a.cpu().double().numpy() - b) <= 2 * HALF_F32 * np.abs(b) * (1 + 1e-6)).all()
    want = paged.rotate(q.double().numpy().reshape(3, 2, hd)[2], n - 1, 10000.0).reshape(-1)
    assert np.abs(q_out[2].cpu().double().numpy() - want).max() <= HALF_BF16 * np.abs(want).max() + 1e-6


def test_strided_and_in_place_write(a48, cuda_dev):
    """q, k and v as slices of one projection, the rotated queries written over the queries; tokens outside the plan's
    rows and positions without a page are left alone."""
    rng = np.random.default_rng(8)
    hd, kvh, heads = 100, 1, 2  # slices that start on 8-byte boundaries only
    s = Setup(a48, cuda_dev, 4, kvh, hd, 16, [5, 2], [5, 40], seed=9, tail=3)
    s.table[1, 2] = 10 ** 6  # sequence 1's tokens sit on a page that does not exist
    s.batch = s.view(s.q_start, s.kv_len, s.n_tokens)
    qkv = torch.tensor(rng.standard_normal((s.n_tokens, (heads + 2 * kvh) * hd)), dtype=torch.float32).to(torch.bfloat16)
    x = qkv.to(cuda_dev)
    q, k, v = x.split([heads * hd, kvh * hd, kvh * hd], 1)
    out = a48.paged_write(s.cache, s.batch, k, v, q=q, q_out=q)
    assert out.data_ptr() == x.data_ptr()
    s.oracle.write(s.q_start, s.kv_len, s.table, k.double().cpu().numpy(), v.double().cpu().numpy(), 10000.0, EPS32)
    got = a48.paged_read(s.cache, s.batch, dtype=torch.float32)
    ref = s.oracle.read(s.q_start, s.kv_len, s.table, s.n_tokens)
    for g, r in zip(got, ref):
        assert (np.abs(g.double().cpu().numpy() - r)[:7] <= 2 * HALF_F32 * np.abs(r[:7]) * (1 + 1e-6)).all()
        assert (g[5:7] == 0).all()  # no page: read as zero
    assert torch.equal(x[7:].cpu(), qkv[7:])  # rows behind the last sequence
    qn = qkv[:, :heads * hd].double().numpy().reshape(-1, heads, hd)
    for row, _, _, pos in paged.tokens(s.q_start, s.kv_len):
        want = paged.rotate(qn[row], pos, 10000.0).reshape(-1)
        assert np.abs(out[row].double().cpu().numpy() - want).max() <= HALF_BF16 * np.abs(want).max() + 1e-5


# ------------------------------------------------------------------------------------------------ attention
SHAPES = [(128, 2, 8, 64), (128, 2, 2, 16), (100, 2, 4, 32), (96, 1, 3, 128), (64, 2, 14, 64), (36, 1, 1, 16), (4, 1, 16, 16)]


@pytest.mark.parametrize("bits", [8, 4, 3])
@pytest.mark.parametrize("hd,kvh,heads,page", SHAPES)
@pytest.mark.parametrize("window,sinks", [(0, 0), (50, 4), (1, 0), (17, 40)])
def test_decode(a48, cuda_dev, bits, hd, kvh, heads, page, window, sinks):
    """One new token per sequence at lengths around page ends, from one position on."""
    rng = np.random.default_rng(bits * 1000 + hd)
    kv_lens = [1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 300]
    s = Setup(a48, cuda_dev, bits, kvh, hd, page, [1] * len(kv_lens), kv_lens, seed=hd, garbage=True)
    s.fill(rng)
    q = torch.tensor(rng.standard_normal((s.n_tokens, heads * hd)) * 2, dtype=torch.float32).to(torch.bfloat16)
    check_attention(s, q, heads, window, sinks)


@pytest.mark.parametrize("bits", [8, 4, 3])
@pytest.mark.parametrize("hd,kvh,heads,page", SHAPES)
@pytest.mark.parametrize("window,sinks", [(0, 0), (40, 3)])
def test_chunks(a48, cuda_dev, bits, hd, kvh, heads, page, window, sinks):
    """Ragged chunks in one call: empty sequences, single tokens, whole prompts and chunks behind a cached part."""
    rng = np.random.default_rng(bits * 100 + hd)
    q_lens, kv_lens = [1, 0, 7, 70, 130, 2], [200, 9, 7, 70, 333, 131]
    s = Setup(a48, cuda_dev, bits, kvh, hd, page, q_lens, kv_lens, seed=hd, garbage=True, tail=2)
    s.fill(rng)
    q = torch.tensor(rng.standard_normal((s.n_tokens, heads * hd)) * 2, dtype=torch.float32).to(torch.bfloat16)
    out = torch.full((s.n_tokens, heads * hd), 7.0, dtype=torch.bfloat16, device=cuda_dev)
    check_attention(s, q, heads, window, sinks, out=out)
    assert (out[-2:] == 7).all()  # rows behind the last sequence


@pytest.mark.parametrize("bits,hd,kvh,heads", [(4, 128, 1, 4), (3, 64, 1, 1), (8, 128, 2, 2)])
@pytest.mark.parametrize("q_len,kv_len,window,sinks", [(1, 5000, 0, 0), (1, 5000, 700, 4), (3, 4097, 0, 0), (260, 3000, 0, 0), (300, 3000, 500, 2)])
def test_long_contexts(a48, cuda_dev, bits, hd, kvh, heads, q_len, kv_len, window, sinks):
    """One sequence over thousands of positions: the axis that is split."""
    rng = np.random.default_rng(kv_len + bits)
    s = Setup(a48, cuda_dev, bits, kvh, hd, 64, [q_len], [kv_len], seed=1)
    s.fill(rng)
    q = torch.tensor(rng.standard_normal((q_len, heads * hd)), dtype=torch.float32).to(torch.bfloat16)
    check_attention(s, q, heads, window, sinks)


@pytest.mark.parametrize("q_len", [1, 90])
def test_rows_that_see_nothing(a48, cuda_dev, q_len):
    """More new tokens than positions, positions without pages, lengths past the table: zeros where nothing is seen."""
    rng = np.random.default_rng(4)
    kv_lens = [0, max(1, q_len - 30), 64, 208]  # the last fills its pages
    s = Setup(a48, cuda_dev, 4, 2, 64, 16, [q_len] * 4, kv_lens, seed=2, garbage=True)
    s.fill(rng)
    s.table[2, :] = -1          # none of sequence 2's positions has a page
    s.table[3, 1:3] = [-7, 1 << 30]  # nor do some of sequence 3's
    s.kv_len = np.array([0, kv_lens[1], 64, 208], np.int32)
    s.batch = s.view(s.q_start, s.kv_len, s.n_tokens)
    q = torch.tensor(rng.standard_normal((s.n_tokens, 4 * 64)), dtype=torch.float32).to(torch.bfloat16)
    got = check_attention(s, q, 4)
    assert (got[:q_len] == 0).all() and (got[2 * q_len:3 * q_len] == 0).all()
    if q_len > 1:
        assert (got[q_len:q_len + 29] == 0).all()
    # a length past what the table holds: the positions past it have no page
    s.kv_len = np.array([0, kv_lens[1], 64, 10 ** 9], np.int32)
    s.batch = s.view(s.q_start, s.kv_len, s.n_tokens, max_kv=256)
    check_attention(s, q, 4)


@pytest.mark.parametrize("q_len", [1, 4, 100])
def test_scores_far_apart_and_unlike_scales(a48, cuda_dev, q_len):
    """Scores that leave one position all the weight, keys and values whose scales differ by many octaves, large and small
    queries; and numbers that are no numbers where nothing is seen."""
    rng = np.random.default_rng(6)
    hd, kv = 128, 400
    s = Setup(a48, cuda_dev, 4, 1, hd, 32, [q_len], [kv], seed=3)
    k = rng.standard_normal((kv, hd)) * np.exp2(rng.integers(-6, 7, (kv, 1)))
    v = rng.standard_normal((kv, hd)) * np.exp2(rng.integers(-9, 10, (kv, 1)))
    starts = np.array([0, kv], np.int32)
    kt, vt = (torch.tensor(x, dtype=torch.float32) for x in (k, v))
    a48.paged_write(s.cache, s.view(starts, [kv], kv), kt.to(cuda_dev), vt.to(cuda_dev), rope_base=0.0)
    s.oracle.write(starts, [kv], s.table, kt.double().numpy(), vt.double().numpy(), 0.0, EPS32)
    for size in (1.0, 300.0, 1e-20, 0.0):
        q = torch.tensor(rng.standard_normal((q_len, 2 * hd)) * size, dtype=torch.float32).to(torch.bfloat16)
        check_attention(s, q, 2, scale=0.05)
    # positions that nothing sees (outside the window) hold scales that are infinite or no numbers
    bad = vt.clone()
    bad[:kv - q_len - 64] = float("nan")
    bad[5] = float("inf")
    kb = kt.clone()
    kb[:kv - q_len - 64] = float("inf")
    a48.paged_write(s.cache, s.view(starts, [kv], kv), kb.to(cuda_dev), bad.to(cuda_dev), rope_base=0.0)
    q = torch.tensor(rng.standard_normal((q_len, 2 * hd)), dtype=torch.float32).to(torch.bfloat16)
    check_attention(s, q, 2, window=64, scale=0.05)


@pytest.mark.parametrize("q_len", [1, 33, 200])
def test_strided_rows(a48, cuda_dev, q_len):
    rng = np.random.default_rng(7)
    hd, heads = 100, 4
    s = Setup(a48, cuda_dev, 4, 2, hd, 64, [q_len, q_len], [q_len + 70, q_len + 3], seed=4)
    s.fill(rng)
    q = torch.tensor(rng.standard_normal((s.n_tokens, heads * hd)), dtype=torch.float32).to(torch.bfloat16)
    plain = check_attention(s, q, heads)
    wide = torch.full((s.n_tokens, heads * hd + 108), float("nan"), dtype=torch.bfloat16, device=cuda_dev)
    wide[:, 4:4 + heads * hd] = q.to(cuda_dev)
    dst = torch.full((s.n_tokens, heads * hd + 12), 3.0, dtype=torch.bfloat16, device=cuda_dev)
    a48.attention_paged(s.cache, s.batch, wide[:, 4:4 + heads * hd], out=dst[:, 4:4 + heads * hd])
    assert np.array_equal(dst[:, 4:4 + heads * hd].double().cpu().numpy().reshape(plain.shape), plain)
    assert (dst[:, :4] == 3).all() and (dst[:, 4 + heads * hd:] == 3).all()


def test_results_do_not_depend_on_the_rest_of_the_batch_or_repeat(a48, cuda_dev):
    """The same call twice gives the same bits."""
    rng = np.random.default_rng(11)
    s = Setup(a48, cuda_dev, 4, 2, 128, 64, [1, 200, 1, 5], [3000, 1200, 17, 900], seed=5)
    s.fill(rng)
    q = torch.tensor(rng.standard_normal((s.n_tokens, 8 * 128)), dtype=torch.float32).to(torch.bfloat16).to(cuda_dev)
    first = a48.attention_paged(s.cache, s.batch, q).clone()
    for _ in range(3):
        assert torch.equal(a48.attention_paged(s.cache, s.batch, q), first)


def test_captured_step_replayed_with_other_lengths(a48, cuda_dev):
    """Write and attention captured once; replayed as the sequences grow, with the plan's contents changed in place."""
    rng = np.random.default_rng(12)
    hd, kvh, heads, page, B, top = 64, 2, 4, 16, 3, 120
    s = Setup(a48, cuda_dev, 4, kvh, hd, page, [1] * B, [top] * B, seed=6)
    batch = s.view(s.q_start, [1] * B, B, max_q=1, max_kv=top)
    k, v = (torch.zeros(B, kvh * hd, device=cuda_dev) for _ in range(2))
    q = torch.zeros(B, heads * hd, device=cuda_dev)
    qr = torch.empty(B, heads * hd, dtype=torch.bfloat16, device=cuda_dev)
    out = torch.empty_like(qr)
    ws = torch.empty(max(16, a48.attention_paged_workspace_bytes(s.cache, batch, heads)), dtype=torch.uint8, device=cuda_dev)
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):  # warm up outside the capture
        a48.paged_write(s.cache, batch, k, v, q=q, q_out=qr)
        a48.attention_paged(s.cache, batch, qr, out=out, workspace=ws)
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        a48.paged_write(s.cache, batch, k, v, q=q, q_out=qr)
        a48.attention_paged(s.cache, batch, qr, out=out, workspace=ws)
    s.cache.pool.zero_()
    for step in range(1, top + 1):
        lens = np.array([step, max(1, step - 7), max(1, step // 2)], np.int32)
        kn, vn, qn = (rng.standard_normal((B, m * hd)).astype(np.float32) for m in (kvh, kvh, heads))
        for dst, src in ((k, kn), (v, vn), (q, qn)):
            dst.copy_(torch.tensor(src))
        batch.kv_len.copy_(torch.tensor(lens))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        s.oracle.write(s.q_start, lens, s.table, kn, vn, 10000.0, EPS32)
        if step in (1, 2, 16, 17, 60, 119, 120):
            ref, mag, top_ = s.oracle.attend(s.q_start, lens, s.table, qr.double().cpu().numpy(), heads)
            got = out.double().cpu().numpy().reshape(ref.shape)
            assert (np.abs(got - ref) <= attention_bound(ref, mag, top_, hd, np.abs(s.oracle.scales[1]).max() * 128)).all()


def test_other_stream_and_two_calls_at_once(a48, cuda_dev):
    """Calls on streams of their own, each with its own workspace and output, overlap without touching one another."""
    rng = np.random.default_rng(13)
    s = Setup(a48, cuda_dev, 3, 2, 128, 64, [1, 1, 150], [2500, 700, 1500], seed=7)
    s.fill(rng)
    q = torch.tensor(rng.standard_normal((s.n_tokens, 4 * 128)), dtype=torch.float32).to(torch.bfloat16)
    want = check_attention(s, q, 4)
    x = q.to(cuda_dev)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    outs = [[a48.attention_paged(s.cache, s.batch, x, stream=st) for _ in range(4)] for st in streams]
    torch.cuda.synchronize()
    for o in outs:
        for y in o:
            assert np.array_equal(y.double().cpu().numpy().reshape(want.shape), want)


def test_offsets_past_32_bits(a48, cuda_dev):
    """A pool of more than 4 GB, the sequence on its last pages."""
    hd, kvh, page = 128, 8, 128
    n_pages = (1 << 32) // (kvh * (2 * page * hd + 8 * page)) + 40
    cache = a48.PagedCache(8, kvh, hd, page, n_pages, device=cuda_dev)
    assert cache.nbytes > 1 << 32
    small = paged.Cache(8, kvh, hd, page, 3)
    rng = np.random.default_rng(14)
    kv, q_len = 300, 70
    table_small = np.array([[2, 0, 1]], np.int32)
    table = torch.tensor(n_pages - 3 + table_small, dtype=torch.int32, device=cuda_dev)
    k, v = (torch.tensor(rng.standard_normal((kv, kvh * hd)), dtype=torch.float32) for _ in range(2))
    one = lambda n, t: a48.PagedBatch(torch.tensor([0, t], dtype=torch.int32, device=cuda_dev), torch.tensor([n], dtype=torch.int32, device=cuda_dev), table, t, t, n)  # noqa: E731
    a48.paged_write(cache, one(kv, kv), k.to(cuda_dev), v.to(cuda_dev))
    small.write([0, kv], [kv], table_small, k.numpy(), v.numpy(), 10000.0, EPS32)
    got = a48.paged_read(cache, one(kv, kv), dtype=torch.float32)
    for g, r in zip(got, small.read([0, kv], [kv], table_small, kv)):
        assert (np.abs(g.double().cpu().numpy() - r) <= 2 * HALF_F32 * np.abs(r) * (1 + 1e-6)).all()
    for t in (1, q_len):
        q = torch.tensor(rng.standard_normal((t, 8 * hd)), dtype=torch.float32).to(torch.bfloat16)
        got = a48.attention_paged(cache, one(kv, t), q.to(cuda_dev)).double().cpu().numpy().reshape(t, 8, hd)
        ref, mag, top = small.attend([0, t], [kv], table_small, q.double().numpy(), 8)
        assert (np.abs(got - ref) <= attention_bound(ref, mag, top, hd, np.abs(small.scales[1]).max() * 128)).all()


def test_shared_prefix_and_many_sequences(a48, cuda_dev):
    """Hundreds of sequences (the plan is searched in several steps), all on the same first pages."""
    rng = np.random.default_rng(15)
    hd, kvh, heads, page, B = 32, 1, 2, 16, 300
    s = Setup(a48, cuda_dev, 4, kvh, hd, page, [64], [64], seed=8, spare=B)
    s.fill(rng)
    base = s.table[0].copy()
    free = [p for p in range(s.cache.n_pages) if p not in set(base.tolist())]
    s.table = np.array([list(base[:3]) + [free[b]] for b in range(B)], np.int32)
    q_lens = [b % 3 for b in range(B)]
    s.q_start = np.concatenate([[0], np.cumsum(q_lens)]).astype(np.int32)
    s.kv_len = np.array([48 + max(1, n) + b % 9 for b, n in enumerate(q_lens)], np.int32)
    starts = np.concatenate([[0], np.cumsum(s.kv_len - 48)]).astype(np.int32)
    n = int(starts[-1])
    k, v = (torch.tensor(rng.standard_normal((n, kvh * hd)), dtype=torch.float32) for _ in range(2))
    a48.paged_write(s.cache, s.view(starts, s.kv_len, n), k.to(cuda_dev), v.to(cuda_dev))
    s.oracle.write(starts, s.kv_len, s.table, k.numpy(), v.numpy(), 10000.0, EPS32)
    s.n_tokens = int(s.q_start[-1])
    s.batch = s.view(s.q_start, s.kv_len, s.n_tokens)
    q = torch.tensor(rng.standard_normal((s.n_tokens, heads * hd)), dtype=torch.float32).to(torch.bfloat16)
    check_attention(s, q, heads)


# ------------------------------------------------------------------------------------------------ as they are used
def test_layer_over_the_cache(a48, cuda_dev):
    """q/k/v BitLinears, write, attention, output BitLinear: prompts of unlike lengths, then tokens one at a time by a captured
    graph.  The attention of every step is the oracle's over the rows that the projections gave."""
    rng = np.random.default_rng(21)
    H, heads, kvh, hd, page, B, k_o = 256, 4, 2, 64, 16, 3, 128
    lens = np.array([90, 1, 37])
    steps, eps = 4, 1e-5
    total = lens + steps
    w = {n: a48.pack_ternary(torch.tensor(rng.standard_normal((m, H if n != "o" else heads * hd)), dtype=torch.float32, device=cuda_dev))
         for n, m in (("q", heads * hd), ("k", kvh * hd), ("v", kvh * hd), ("o", H))}
    s = Setup(a48, cuda_dev, 3, kvh, hd, page, [0] * B, total, seed=9)

    def layer(x, batch, bufs=None):
        codes, scale = a48.quant_int4_bf16(x, eps)
        q, k, v = (a48.linear_bf16(w[n], codes, scale) for n in "qkv")
        qr = a48.paged_write(s.cache, batch, k, v, q=q)
        y = a48.attention_paged(s.cache, batch, qr)
        c8, s8 = a48.topk_quant_int8_bf16(y, k_o, eps)
        return k, v, qr, y, a48.linear_bf16(w["o"], c8, s8, kind=a48.ACT_TOPK_INT8)

    def check(q_start, kv_len, parts):
        k, v, qr, y, out = (t.double().cpu().numpy() for t in parts)
        s.oracle.write(q_start, kv_len, s.table, k, v, 10000.0, EPS32)
        ref, mag, top = s.oracle.attend(q_start, kv_len, s.table, qr, heads)
        vmax = np.abs(s.oracle.scales[1]).max() * 128
        assert (np.abs(y.reshape(ref.shape) - ref) <= attention_bound(ref, mag, top, hd, vmax)).all()
        assert np.isfinite(out).all() and (out != 0).any(axis=1).all()

    x = torch.tensor(rng.standard_normal((int(lens.sum()), H)), dtype=torch.float32).to(torch.bfloat16).to(cuda_dev)
    q_start = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
    check(q_start, lens, layer(x, s.view(q_start, lens, int(lens.sum()))))

    q_start = np.arange(B + 1, dtype=np.int32)
    batch = s.view(q_start, lens + 1, B, max_q=1, max_kv=int(total.max()))
    xs = torch.zeros(B, H, dtype=torch.bfloat16, device=cuda_dev)
    pool = s.cache.pool.clone()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        layer(xs, batch)
    stream.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        parts = layer(xs, batch)
    s.cache.pool.copy_(pool)
    for step in range(1, steps + 1):
        xs.copy_(torch.tensor(rng.standard_normal((B, H))))
        batch.kv_len.copy_(torch.tensor(lens + step, dtype=torch.int32))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        check(q_start, lens + step, parts)
        eager = layer(xs, batch)  # (writes the same codes again)
        assert all(torch.equal(a, b) for a, b in zip(parts, eager))
    assert a48.kernel_status()[0] == 0


@pytest.mark.parametrize("bits,hd,window,sinks", [(4, 64, 0, 0), (3, 128, 0, 0), (8, 36, 90, 5)])
def test_more_tiles_of_rows_than_sms(a48, cuda_dev, bits, hd, window, sinks):
    """CTAs of the tile kernel take over rows of others: unlike lengths, sequences with a few rows or none among them."""
    rng = np.random.default_rng(22)
    kvh, heads, page = 8, 32, 32
    q_lens = [300, 1, 700, 0, 33, 64, 257, 5, 129, 480, 17, 90]
    kv_lens = [n + int(rng.integers(0, 300)) for n in q_lens]
    s = Setup(a48, cuda_dev, bits, kvh, hd, page, q_lens, kv_lens, seed=10, tail=3)
    s.fill(rng)
    assert sum((4 * n + 255) // 256 for n in q_lens if n > 8) * kvh > 148
    q = torch.tensor(rng.standard_normal((s.n_tokens, heads * hd)), dtype=torch.float32).to(torch.bfloat16)
    out = torch.full((s.n_tokens, heads * hd), 7.0, dtype=torch.bfloat16, device=cuda_dev)
    first = check_attention(s, q, heads, window, sinks, out=out)
    assert (out[int(s.q_start[-1]):] == 7).all()  # rows behind the last sequence
    for _ in range(3):
        again = a48.attention_paged(s.cache, s.batch, q.to(cuda_dev), window=window, sinks=sinks)
        assert np.array_equal(again.double().cpu().numpy().reshape(first.shape)[:-3], first[:-3])


def test_captured_prompts_replayed_with_other_lengths(a48, cuda_dev):
    rng = np.random.default_rng(23)
    hd, kvh, heads, page, B, top = 64, 4, 16, 64, 4, 600
    s = Setup(a48, cuda_dev, 4, kvh, hd, page, [top] * B, [top] * B, seed=11)
    s.fill(rng)
    n = 1100
    q = torch.tensor(rng.standard_normal((n, heads * hd)), dtype=torch.float32).to(torch.bfloat16)
    x, out = q.to(cuda_dev), torch.zeros(n, heads * hd, dtype=torch.bfloat16, device=cuda_dev)
    batch = s.view(np.array([0] * B + [top], np.int32), [top] * B, n, max_q=top, max_kv=top)
    ws = torch.empty(max(16, a48.attention_paged_workspace_bytes(s.cache, batch, heads)), dtype=torch.uint8, device=cuda_dev)
    a48.attention_paged(s.cache, batch, x, out=out, workspace=ws)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        a48.attention_paged(s.cache, batch, x, out=out, workspace=ws)
    for q_lens, kv_lens in (([600, 500, 0, 0], [600, 500, 0, 9]), ([1, 2, 3, 600], [600, 600, 600, 600]), ([275] * 4, [275, 300, 599, 600]), ([0] * 4, [1] * 4)):
        s.q_start = np.concatenate([[0], np.cumsum(q_lens)]).astype(np.int32)
        s.kv_len = np.array(kv_lens, np.int32)
        batch.q_start.copy_(torch.tensor(s.q_start))
        batch.kv_len.copy_(torch.tensor(s.kv_len))
        out.fill_(7)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        ref, mag, best = s.oracle.attend(s.q_start, s.kv_len, s.table, q.double().numpy(), heads)
        got, end = out.double().cpu().numpy().reshape(ref.shape), int(s.q_start[-1])
        bound = attention_bound(ref, mag, best, hd, np.abs(s.oracle.scales[1]).max() * 128)
        assert (np.abs(got - ref) <= bound)[:end].all() and (got[end:] == 7).all()


def test_bounds_smaller_than_the_batch(a48, cuda_dev):
    """max_q and max_kv size the launch only: tokens within max_q are right, the others right or left alone."""
    rng = np.random.default_rng(24)
    hd, kvh, heads, page = 64, 2, 8, 16
    s = Setup(a48, cuda_dev, 4, kvh, hd, page, [150, 3, 40], [400, 3, 90], seed=12)
    s.fill(rng)
    q = torch.tensor(rng.standard_normal((s.n_tokens, heads * hd)), dtype=torch.float32).to(torch.bfloat16)
    ref, mag, top = s.oracle.attend(s.q_start, s.kv_len, s.table, q.double().numpy(), heads)
    bound = attention_bound(ref, mag, top, hd, np.abs(s.oracle.scales[1]).max() * 128)
    for max_q, max_kv in ((1, 1), (2, 400), (20, 16), (100, 50), (150, 1)):
        out = torch.full((s.n_tokens, heads * hd), 7.0, dtype=torch.bfloat16, device=cuda_dev)
        a48.attention_paged(s.cache, s.view(s.q_start, s.kv_len, s.n_tokens, max_q=max_q, max_kv=max_kv), q.to(cuda_dev), out=out)
        got = out.double().cpu().numpy().reshape(ref.shape)
        right, alone = (np.abs(got - ref) <= bound).all(axis=(1, 2)), (got == 7).all(axis=(1, 2))
        assert (right | alone).all()
        for b in range(3):
            within = int(s.q_start[b]) + min(max_q, int(s.q_start[b + 1] - s.q_start[b]))
            assert right[int(s.q_start[b]):within].all()


@pytest.mark.parametrize("q_lens,kv_lens", [([1, 2], [40, 2]), ([90, 0, 30], [200, 7, 30])])
def test_rows_ahead_of_the_first_sequence(a48, cuda_dev, q_lens, kv_lens):
    """q_start need not begin at 0: the rows ahead of it and behind the last are neither read nor written."""
    rng = np.random.default_rng(25)
    hd, kvh, heads, page, ahead, behind = 32, 2, 4, 16, 5, 4
    s = Setup(a48, cuda_dev, 4, kvh, hd, page, q_lens, kv_lens, seed=13, tail=behind)
    s.fill(rng)
    s.q_start, s.n_tokens = s.q_start + ahead, s.n_tokens + ahead
    s.batch = s.view(s.q_start, s.kv_len, s.n_tokens)
    lo, hi = int(s.q_start[0]), int(s.q_start[-1])
    k, v, q = (torch.tensor(rng.standard_normal((s.n_tokens, m * hd)), dtype=torch.float32) for m in (kvh, kvh, heads))
    for t in (k, v, q):
        t[:lo], t[hi:] = float("nan"), float("nan")
    qr = torch.full((s.n_tokens, heads * hd), 7.0, dtype=torch.bfloat16, device=cuda_dev)
    a48.paged_write(s.cache, s.batch, k.to(cuda_dev), v.to(cuda_dev), q=q.to(cuda_dev), q_out=qr)
    s.oracle.write(s.q_start, s.kv_len, s.table, k.numpy(), v.numpy(), 10000.0, EPS32)
    out = torch.full_like(qr, 7.0)
    check_attention(s, qr.cpu(), heads, out=out)
    ko, vo = (torch.full((s.n_tokens, kvh, hd), 7.0, device=cuda_dev) for _ in range(2))
    a48.paged_read(s.cache, s.batch, dtype=torch.float32, k_out=ko, v_out=vo)
    for t in (qr, out, ko, vo):
        assert (t[:lo] == 7).all() and (t[hi:] == 7).all() and (t[lo:hi] != 7).any()
    for g, r in zip((ko, vo), s.oracle.read(s.q_start, s.kv_len, s.table, s.n_tokens)):
        assert (np.abs(g.double().cpu().numpy() - r) <= 2 * HALF_F32 * np.abs(r) * (1 + 1e-6))[lo:hi].all()


@pytest.mark.parametrize("heads,kvh,hd,q_len,kv", [(300, 1, 32, 3, 70), (300, 1, 32, 1, 40), (40, 8, 64, 2, 300), (514, 2, 4, 2, 33)])
def test_many_heads_to_a_key_head(a48, cuda_dev, heads, kvh, hd, q_len, kv):
    """A token's query heads fill more than a tile, so that tiles begin and end inside a token."""
    rng = np.random.default_rng(26)
    s = Setup(a48, cuda_dev, 8, kvh, hd, 16, [q_len, 1, q_len], [kv, 1, q_len], seed=14)
    s.fill(rng)
    q = torch.tensor(rng.standard_normal((s.n_tokens, heads * hd)), dtype=torch.float32).to(torch.bfloat16)
    check_attention(s, q, heads)


def test_tensors_of_other_devices_are_refused(a48, cuda_dev):
    s = Setup(a48, cuda_dev, 4, 1, 32, 16, [1], [1], seed=15)
    x = torch.zeros(1, 32)
    with pytest.raises(AssertionError):
        a48.paged_write(s.cache, s.batch, x, x)
    with pytest.raises(AssertionError):
        a48.paged_write(s.cache, s.batch, x.to(cuda_dev), x)
    with pytest.raises(AssertionError):
        a48.attention_paged(s.cache, s.batch, x.to(torch.bfloat16))
    with pytest.raises(AssertionError):
        a48.attention_paged(s.cache, s.batch, x.to(cuda_dev, torch.bfloat16), workspace=torch.empty(64, dtype=torch.uint8))


@pytest.mark.parametrize("q_len", [1, 6, 100])
@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
def test_queries_that_are_no_numbers_stay_alone(a48, cuda_dev, q_len, bad):
    """A query head with an infinity or NaN, where its other heads and the next two tokens have the largest entries of all."""
    rng = np.random.default_rng(27)
    hd, kvh, heads = 128, 1, 4
    s = Setup(a48, cuda_dev, 4, kvh, hd, 16, [q_len, 2], [q_len + 60, 33], seed=16)
    s.fill(rng)
    x = rng.standard_normal((s.n_tokens, heads, hd)) * 2.0 ** -6
    x[:3, :, 5] *= 2.0 ** 15
    q = torch.tensor(x.reshape(s.n_tokens, -1), dtype=torch.float32).to(torch.bfloat16)
    ref, mag, top = s.oracle.attend(s.q_start, s.kv_len, s.table, q.double().numpy(), heads)
    q.view(s.n_tokens, heads, hd)[0, 1, 5] = bad
    got = a48.attention_paged(s.cache, s.batch, q.to(cuda_dev)).double().cpu().numpy().reshape(ref.shape)
    right = np.abs(got - ref) <= attention_bound(ref, mag, top, hd, np.abs(s.oracle.scales[1]).max() * 128)
    right[0, 1] = True
    assert right.all()


@pytest.mark.parametrize("bits", [8, 4, 3])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_heads_of_zeros_and_of_tiny_numbers_without_eps(a48, cuda_dev, bits, dtype):
    """eps 0: a head of zeros has no scale to divide by and reads as zeros; the smallest numbers keep their codes."""
    rng = np.random.default_rng(28)
    hd, kvh, n = 32, 2, 7
    s = Setup(a48, cuda_dev, bits, kvh, hd, 16, [n], [n], seed=17)
    k, v = (torch.tensor(rng.standard_normal((n, kvh * hd)), dtype=torch.float32) for _ in range(2))
    k[2], v[1], v[0, :hd] = 0, 0, 0
    k[3], v[3] = k[3] * 1e-30, v[3] * 1e-30
    k, v = k.to(dtype), v.to(dtype)
    a48.paged_write(s.cache, s.batch, k.to(cuda_dev), v.to(cuda_dev), rope_base=0.0, eps=0.0)
    got = [t.double().cpu().numpy() for t in a48.paged_read(s.cache, s.batch, dtype=torch.float32)]
    for g, x in zip(got, (k, v)):
        x = x.double().numpy().reshape(n, kvh, hd)
        gamma = np.abs(x).max(-1, keepdims=True)
        assert (g[x == 0] == 0).all()
        levels = np.where((np.arange(n) == 0) & (bits == 3), 7, 2 ** (bits - 1) - 1)[:, None, None]
        assert (np.abs(g - x) <= 0.5 * gamma / levels * (1 + 1e-5)).all()  # half a step of the code
    q = torch.tensor(rng.standard_normal((n, kvh * hd)), dtype=torch.float32).to(torch.bfloat16)
    assert torch.isfinite(a48.attention_paged(s.cache, s.batch, q.to(cuda_dev)).float()).all()


def weight_tail(n, vmax):
    """What n weights below fp16's normal numbers lose at most: a weight times its value scale and unit is rounded by half a
    subnormal step, 2^-25, and once more, by as much, if it is scaled down by 1/2 or less (so 1.5 2^-25 < 2^-24 in all); the unit
    brings the largest value scale so far to 8 or more and codes are 128 at most, which makes it 2^-27 of the largest value
    (`vmax` = 128 times the largest scale); the sum of the weights is 1/2 at least."""
    return n * 2.0 ** -26 * vmax


@pytest.mark.parametrize("bits", [8, 4, 3])
@pytest.mark.parametrize("kv,tiles", [(128, 1), (512, 4)])
def test_references_that_move_twice_within_a_tile(a48, cuda_dev, bits, kv, tiles):
    """Every tile of 128 positions has a larger score than all before it in its first 64 positions and a larger one still in the
    others: the second move finds the first's weights (and, behind the first tile, its outputs) just stored."""
    rng = np.random.default_rng(29)
    hd, q_len = 64, 128
    s = Setup(a48, cuda_dev, bits, 1, hd, 32, [q_len, q_len], [kv + q_len] * 2, seed=18)
    n = kv + q_len
    direction = np.where(np.arange(hd) % 2, 1.0, -1.0)
    k = 0.02 * rng.standard_normal((2 * n, hd))
    size = 0.0
    for t in range(tiles + 1):
        for at in (128 * t + 5 + t, 128 * t + 70 + t):
            size += 1.0
            k[[at, n + at]] = size * direction
    v = rng.standard_normal((2 * n, hd))
    starts = np.array([0, n, 2 * n], np.int32)
    kt, vt = (torch.tensor(x, dtype=torch.float32) for x in (k, v))
    a48.paged_write(s.cache, s.view(starts, [n, n], 2 * n), kt.to(cuda_dev), vt.to(cuda_dev), rope_base=0.0)
    s.oracle.write(starts, [n, n], s.table, kt.double().numpy(), vt.double().numpy(), 0.0, EPS32)
    # the steps from one to the next are 1.5 .. 12 octaves times a row's factor: the new weights swallow the old ones or not
    q = direction * rng.choice([0.25, 0.5, 1.0, 2.0], (2 * q_len, 2, 1)) + 0.01 * rng.standard_normal((2 * q_len, 2, hd))
    q = torch.tensor(q.reshape(2 * q_len, -1), dtype=torch.float32).to(torch.bfloat16)
    got = a48.attention_paged(s.cache, s.batch, q.to(cuda_dev), scale=0.125)
    out, mag, top = s.oracle.attend(s.q_start, s.kv_len, s.table, q.double().numpy(), 2, 0.125)
    vmax = np.abs(s.oracle.scales[1]).max() * 128
    assert (np.abs(got.double().cpu().numpy().reshape(out.shape) - out) <= attention_bound(out, mag, top, hd, vmax) + weight_tail(n, vmax)).all()
    assert a48.kernel_status()[0] == 0


@pytest.mark.parametrize("captured", [False, True])
def test_plan_queries_and_cache_changed_right_ahead_of_each_mixed_call(a48, cuda_dev, captured):
    """Prompts beside single tokens, step after step without a wait: the kernels of a call see the plan, the queries and the pages
    that kernels just ahead of it wrote, and calls share one workspace in turn."""
    rng = np.random.default_rng(30)
    hd, kvh, heads, page, B, top = 64, 2, 8, 16, 6, 400
    s = Setup(a48, cuda_dev, 4, kvh, hd, page, [0] * B, [top] * B, seed=19)
    plans = [([150, 1, 0, 1, 2, 1], [300, 400, 9, 33, 2, 128]), ([1, 1, 200, 1, 0, 1], [301, 400, 200, 34, 2, 129]),
             ([2, 90, 1, 1, 1, 80], [400, 400, 201, 35, 3, 209]), ([1, 1, 1, 1, 1, 1], [1, 1, 202, 36, 4, 210])]
    n = max(sum(p[0]) for p in plans)
    plan = [torch.tensor(np.concatenate([[0], np.cumsum(p[0]), p[1]]), dtype=torch.int32, device=cuda_dev) for p in plans]
    k, v, q = ([torch.tensor(rng.standard_normal((n, m * hd)), dtype=torch.float32, device=cuda_dev) for _ in plans] for m in (kvh, kvh, heads))
    batch = s.view(np.arange(B + 1, dtype=np.int32), [1] * B, n, max_q=200, max_kv=top)
    now = [torch.zeros(n, m * hd, device=cuda_dev) for m in (kvh, kvh, heads)]
    qr = [torch.zeros(n, heads * hd, dtype=torch.bfloat16, device=cuda_dev) for _ in plans]
    out = [torch.zeros_like(x) for x in qr]
    ws = torch.empty(max(16, a48.attention_paged_workspace_bytes(s.cache, batch, heads)), dtype=torch.uint8, device=cuda_dev)

    def steps():
        for i in range(len(plans)):
            batch.q_start.copy_(plan[i][:B + 1])
            batch.kv_len.copy_(plan[i][B + 1:])
            for dst, src in zip(now, (k[i], v[i], q[i])):
                dst.copy_(src)
            a48.paged_write(s.cache, batch, now[0], now[1], q=now[2], q_out=qr[i])
            a48.attention_paged(s.cache, batch, qr[i], out=out[i], workspace=ws)

    steps()
    torch.cuda.synchronize()
    s.cache.pool.zero_()
    if captured:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            steps()
        s.cache.pool.zero_()
        graph.replay()
    else:
        steps()
    torch.cuda.synchronize()
    for i, (q_lens, kv_lens) in enumerate(plans):
        q_start = np.concatenate([[0], np.cumsum(q_lens)]).astype(np.int32)
        s.oracle.write(q_start, kv_lens, s.table, k[i].double().cpu().numpy(), v[i].double().cpu().numpy(), 10000.0, EPS32)
        ref, mag, best = s.oracle.attend(q_start, kv_lens, s.table, qr[i].double().cpu().numpy(), heads)
        vmax, end = np.abs(s.oracle.scales[1]).max() * 128, int(q_start[-1])
        bound = attention_bound(ref, mag, best, hd, vmax) + weight_tail(top, vmax)
        assert (np.abs(out[i].double().cpu().numpy().reshape(ref.shape) - ref) <= bound)[:end].all()
    assert a48.kernel_status()[0] == 0


@pytest.mark.parametrize("bits", [8, 4, 3])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rope_base,hd", [(0.0, 64), (10000.0, 64), (10000.0, 36), (0.0, 100)])
def test_heads_that_are_no_numbers_are_kept_as_such(a48, cuda_dev, bits, dtype, rope_base, hd):
    """One NaN in a key or value head, and heads of nothing else: no scale is a number where the head is none, the codes and
    scales of all other heads are the oracle's, and attention is NaN exactly for the rows and heads that see them."""
    rng = np.random.default_rng(31)
    kvh, heads, n, page = 3, 6, 150, 16
    s = Setup(a48, cuda_dev, bits, kvh, hd, page, [n], [n], seed=20, garbage=True)
    x = [torch.tensor(rng.standard_normal((n, kvh, hd)), dtype=torch.float32).to(dtype) for _ in range(2)]
    bad = [(0, 0, 1, 3), (0, 17, 0, None), (1, 40, 1, hd - 1), (1, 40, 2, None), (0, 131, 2, hd // 2), (1, 149, 0, 0), (1, 0, 0, 5)]
    sick = np.zeros((2, kvh, n), bool)
    clean = [t.clone() for t in x]
    for which, pos, head, entry in bad:
        x[which][pos, head, slice(None) if entry is None else entry] = float("nan")
        sick[which, head, pos] = True
    a48.paged_write(s.cache, s.batch, *(t.view(n, -1).to(cuda_dev) for t in x), rope_base=rope_base)
    s.oracle.write(s.q_start, s.kv_len, s.table, *(t.view(n, -1).double().numpy() for t in clean), rope_base, EPS32)
    codes, scales, bos = paged.unpack_pool(s.cache.pool.cpu().numpy(), bits, kvh, hd, page, s.cache.n_pages)
    for pos in range(n):
        p, slot = paged.place(s.table, 0, pos, page, s.cache.n_pages)
        first = bits == 3 and pos == 0
        well = ~sick[:, :, pos]
        assert np.array_equal((bos[:, p] if first else codes[:, p, :, slot])[well][:, :hd], (s.oracle.bos[:, p] if first else s.oracle.codes[:, p, :, slot])[well])
        got, ref = scales[:, p, :, slot], s.oracle.scales[:, p, :, slot]
        assert np.isnan(got[~well]).all() and (np.abs(got - ref)[well] <= HALF_F32 * ref[well] * (1 + 1e-6)).all()
    read = [t.cpu().numpy() for t in a48.paged_read(s.cache, s.batch, dtype=torch.float32)]
    for which in range(2):
        assert np.array_equal(np.isnan(read[which]).all(-1), sick[which].T) and np.array_equal(np.isnan(read[which]).any(-1), sick[which].T)
    q = torch.tensor(rng.standard_normal((n, heads * hd)), dtype=torch.float32).to(torch.bfloat16)
    for q_len, window in ((n, 0), (n, 20), (8, 0), (8, 20), (1, 0)):  # tiles, and rows from the last ones on
        q_start = np.array([0, q_len], np.int32)
        got = a48.attention_paged(s.cache, s.view(q_start, s.kv_len, q_len), q[:q_len].to(cuda_dev), window=window)
        got = got.double().cpu().numpy().reshape(q_len, heads, hd)
        ref, mag, top = s.oracle.attend(q_start, s.kv_len, s.table, q[:q_len].double().numpy(), heads, 0.0, window, 0)
        vmax = np.abs(s.oracle.scales[1]).max() * 128
        right = (np.abs(got - ref) <= attention_bound(ref, mag, top, hd, vmax) + weight_tail(n, vmax)).all(-1)
        for i in range(q_len):
            last = n - q_len + i
            sees = sick[:, :, max(0, last + 1 - window) if window else 0:last + 1].any((0, 2)).repeat(heads // kvh)
            assert np.array_equal(np.isnan(got[i]).all(-1), sees) and right[i, ~sees].all(), (q_len, window, i)
    assert a48.kernel_status()[0] == 0


@pytest.mark.parametrize("q_lens,kv_lens", [([1, 1], [700, 33]), ([3, 2], [700, 33]), ([260, 1], [700, 33])])
@pytest.mark.parametrize("window,sinks", [((1 << 31) - 1, 4), ((1 << 31) - 1, (1 << 31) - 1), (1 << 30, 1 << 30), (1, (1 << 31) - 1)])
def test_windows_and_sinks_past_the_context(a48, cuda_dev, q_lens, kv_lens, window, sinks):
    """Windows or sinks that reach over the whole context see what no window does, bit for bit."""
    rng = np.random.default_rng(32)
    hd, kvh, heads = 64, 2, 8
    s = Setup(a48, cuda_dev, 4, kvh, hd, 32, q_lens, kv_lens, seed=21)
    s.fill(rng)
    q = torch.tensor(rng.standard_normal((s.n_tokens, heads * hd)), dtype=torch.float32).to(torch.bfloat16)
    want = check_attention(s, q, heads)
    got = a48.attention_paged(s.cache, s.batch, q.to(cuda_dev), window=window, sinks=sinks)
    assert np.array_equal(got.double().cpu().numpy().reshape(want.shape), want)


@pytest.mark.parametrize("q_lens,kv_lens,kvh,heads,tail,bounds", [
    ([200, 1, 2, 0, 1], [300, 6000, 2500, 5, 1], 1, 4, 0, None),      # parts of decoding sequences beside a prompt
    ([1, 2], [6000, 4001], 2, 8, 700, None),                          # decoding alone, token rows to spare
    ([300, 1], [5000, 5000], 1, 2, 3000, None),                       # parts of both kernels, rows to spare
    ([5, 90, 0, 40, 1], [3000, 2000, 0, 2100, 4000], 1, 4, 0, (2000, 4000)),  # tiles found by search, in parts
    ([40, 40, 3], [2000, 2100, 2200], 1, 2, 5, (33, 3000)),           # sequences longer than max_q says
])
def test_workspace_between_guards(a48, cuda_dev, q_lens, kv_lens, kvh, heads, tail, bounds):
    """A workspace of exactly the bytes asked for, full of what is no number, and the bytes around it left as they were."""
    rng = np.random.default_rng(33)
    hd = 64
    s = Setup(a48, cuda_dev, 4, kvh, hd, 64, q_lens, kv_lens, seed=22, tail=tail)
    s.fill(rng)
    b = s.batch if bounds is None else s.view(s.q_start, s.kv_len, s.n_tokens, max_q=bounds[0], max_kv=bounds[1])
    need = a48.attention_paged_workspace_bytes(s.cache, b, heads)
    assert need > 0
    room = torch.full((need + 8192,), 255, dtype=torch.uint8, device=cuda_dev)
    ws = room[4096:4096 + need]
    q = torch.tensor(rng.standard_normal((s.n_tokens, heads * hd)), dtype=torch.float32).to(torch.bfloat16)
    out = torch.full((s.n_tokens, heads * hd), 7.0, dtype=torch.bfloat16, device=cuda_dev)
    a48.attention_paged(s.cache, b, q.to(cuda_dev), out=out, workspace=ws)
    ref, mag, top = s.oracle.attend(s.q_start, s.kv_len, s.table, q.double().numpy(), heads)
    vmax, end = np.abs(s.oracle.scales[1]).max() * 128, int(s.q_start[-1])
    got = out.double().cpu().numpy().reshape(ref.shape)
    right = (np.abs(got - ref) <= attention_bound(ref, mag, top, hd, vmax) + weight_tail(max(kv_lens), vmax)).all((1, 2))
    if bounds is None or bounds[0] >= max(q_lens):
        assert right[:end].all()
    else:
        for i, n in enumerate(q_lens):
            at = int(s.q_start[i])
            assert right[at:at + min(n, bounds[0])].all()
        assert (right | (got == 7).all((1, 2)))[:end].all()
    assert (got[end:] == 7).all()
    assert (room[:4096] == 255).all() and (room[4096 + need:] == 255).all()
    with pytest.raises(a48.A48Error):
        a48.attention_paged(s.cache, b, q.to(cuda_dev), workspace=ws[:need - 1])
    assert a48.kernel_status()[0] == 0


@pytest.mark.parametrize("bits", [8, 4, 3])
@pytest.mark.parametrize("hd,page", [(64, 16), (128, 64)])
@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
def test_scales_that_are_no_numbers(a48, cuda_dev, bits, hd, page, bad):
    """Key or value scales of single positions made infinite or no numbers in the pool itself: NaN for every row of the head that
    sees one of them, and for no other; the rows kernel (few rows, parts joined in a cluster or by a kernel) and the tile kernel."""
    rng = np.random.default_rng(34)
    kvh, heads, n = 2, 4, 1000
    s = Setup(a48, cuda_dev, bits, kvh, hd, page, [n], [n], seed=23)
    s.fill(rng)
    P = (hd + 31) // 32 * 32
    row = P * bits // 8
    chunk = 2 * page * row + 8 * page + (P if bits == 3 else 0)
    pool = s.cache.pool.view(s.cache.n_pages, kvh, chunk)
    sick = np.zeros((kvh, n), bool)
    for which, pos, head in ((0, 0, 1), (1, 300, 0), (0, 555, 0), (1, 700, 1), (0, 997, 0), (1, 998, 1)):
        p, slot = paged.place(s.table, 0, pos, page, s.cache.n_pages)
        at = 2 * page * row + 4 * page * which + 4 * slot
        pool[p, head, at:at + 4] = torch.tensor([bad], dtype=torch.float32).view(torch.uint8).to(cuda_dev)
        sick[head, pos] = True
    q = torch.tensor(rng.standard_normal((n, heads * hd)), dtype=torch.float32).to(torch.bfloat16)
    for q_len, kv, window, sinks in ((n, n, 0, 0), (300, n, 40, 3), (300, n, 40, 0), (1, n, 0, 0), (1, 997, 200, 0), (4, n, 2, 0), (4, n, 2, 1), (9, 560, 3, 0),
                                     (5, 280, 0, 0)):
        q_start, kv_len = np.array([0, q_len], np.int32), np.array([kv], np.int32)
        got = a48.attention_paged(s.cache, s.view(q_start, kv_len, q_len), q[:q_len].to(cuda_dev), window=window, sinks=sinks)
        got = got.double().cpu().numpy().reshape(q_len, heads, hd)
        ref, mag, top = s.oracle.attend(q_start, kv_len, s.table, q[:q_len].double().numpy(), heads, 0.0, window, sinks)
        vmax = np.abs(s.oracle.scales[1]).max() * 128
        right = (np.abs(got - ref) <= attention_bound(ref, mag, top, hd, vmax) + weight_tail(n, vmax)).all(-1)
        j = np.arange(n)
        for i in range(q_len):
            p = kv - q_len + i
            seen = (j <= p) & ((j > p - window) | (j < sinks) if window else True)
            sees = (sick & seen).any(1).repeat(heads // kvh)
            assert np.array_equal(np.isnan(got[i]).all(-1), sees) and right[i, ~sees].all(), (q_len, kv, window, i)
    assert a48.kernel_status()[0] == 0


def test_one_token_out_of_rows_of_an_odd_length(a48, cuda_dev):
    rng = np.random.default_rng(35)
    hd, kvh, heads = 64, 1, 2
    s = Setup(a48, cuda_dev, 4, kvh, hd, 16, [1], [40], seed=24)
    s.fill(rng)
    width = (heads + 2 * kvh) * hd
    rows = torch.zeros(3, width + 9, device=cuda_dev)  # an odd stride, and row 0 on a 16-byte boundary
    rows[0, :width] = torch.tensor(rng.standard_normal(width), dtype=torch.float32)
    q, k, v = rows[:1, :width].split([heads * hd, kvh * hd, kvh * hd], 1)
    qr = torch.zeros(3, heads * hd + 9, dtype=torch.bfloat16, device=cuda_dev)[:1, :heads * hd]
    assert a48.paged_write(s.cache, s.batch, k, v, q=q, q_out=qr) is qr
    s.oracle.write(s.q_start, s.kv_len, s.table, k.double().cpu().numpy(), v.double().cpu().numpy(), 10000.0, EPS32)
    out = torch.zeros(3, heads * hd + 9, dtype=torch.bfloat16, device=cuda_dev)
    a48.attention_paged(s.cache, s.batch, qr, out=out[:1, :heads * hd])
    want = check_attention(s, qr.cpu(), heads)
    assert np.array_equal(out[:1, :heads * hd].double().cpu().numpy().reshape(want.shape), want)
    assert (out[1:] == 0).all() and (out[0, heads * hd:] == 0).all()


def test_two_host_threads_at_once(a48, cuda_dev):
    """First calls and later ones from threads of their own, each on its stream with a cache of its own and kernels that the
    other launches too."""
    import threading

    rng = np.random.default_rng(36)
    work = []
    for i in range(2):
        s = Setup(a48, cuda_dev, (4, 3)[i], 2, 128, 32, [150, 1, 3], [400, 900, 70], seed=25 + i)
        s.fill(rng)
        q = torch.tensor(rng.standard_normal((s.n_tokens, 8 * 128)), dtype=torch.float32).to(torch.bfloat16)
        work.append((s, q.to(cuda_dev), check_attention(s, q, 8), torch.cuda.Stream(), []))
    torch.cuda.synchronize()
    start = threading.Barrier(2)

    def run(s, q, want, stream, got):
        start.wait()
        with torch.cuda.stream(stream):
            for other in work + work:
                got.append((other[2], a48.attention_paged(other[0].cache, other[0].batch, other[1])))
            stream.synchronize()

    threads = [threading.Thread(target=run, args=w) for w in work]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    for w in work:
        assert len(w[4]) == 4
        for want, y in w[4]:
            assert np.array_equal(y.double().cpu().numpy().reshape(want.shape), want)


@pytest.mark.parametrize("bits", [8, 4, 3])
@pytest.mark.parametrize("hd,kvh,heads,dtype", [(128, 2, 3, torch.bfloat16), (100, 1, 2, torch.float32), (64, 3, 3, torch.float32), (36, 1, 1, torch.bfloat16)])
def test_codes_of_long_prompts_one_by_one(a48, cuda_dev, bits, hd, kvh, heads, dtype):
    """Enough tokens for the form that takes four to a block, a count that four does not divide, sequences that begin and end
    inside a block: every code and scale, and the rotated queries, against float64."""
    rng = np.random.default_rng(37)
    page, q_lens = 32, [1, 601, 0, 2, 593, 90]
    kv_lens = [1, 601, 4, 2, 700, 91]
    s = Setup(a48, cuda_dev, bits, kvh, hd, page, q_lens, kv_lens, seed=27, garbage=True, tail=2)
    n, real = s.n_tokens, int(s.q_start[-1])
    assert n >= 1184 and n % 4
    k, v, q = (torch.tensor(rng.standard_normal((n, m * hd)) * np.exp2(rng.integers(-8, 9, (n, 1))), dtype=torch.float32).to(dtype) for m in (kvh, kvh, heads))
    qr = torch.full((n, heads * hd), 7.0, dtype=torch.bfloat16, device=cuda_dev)
    a48.paged_write(s.cache, s.batch, k.to(cuda_dev), v.to(cuda_dev), q=q.to(cuda_dev), q_out=qr)
    # the definition over all tokens at once, in 64 bits
    where = np.array([(b, pos) for _, b, _, pos in paged.tokens(s.q_start, s.kv_len)])
    pos = where[:, 1]
    angle = pos[:, None] * 10000.0 ** (-2.0 * np.arange(hd // 2) / hd)
    c, sn = np.cos(angle)[:, None], np.sin(angle)[:, None]

    def turned(x):
        lo, hi = x[..., :hd // 2], x[..., hd // 2:]
        return np.concatenate([lo * c - hi * sn, hi * c + lo * sn], -1)

    kn, vn, qn = (t.double().numpy()[:real].reshape(real, -1, hd) for t in (k, v, q))
    codes, scales, bos = paged.unpack_pool(s.cache.pool.cpu().numpy(), bits, kvh, hd, page, s.cache.n_pages)
    at = np.array([paged.place(s.table, b, p, page, s.cache.n_pages) for b, p in where])
    for which, x in enumerate((turned(kn), vn)):
        got = codes[which][at[:, 0], :, at[:, 1]][..., :hd]
        first = pos == 0
        if bits == 3:
            got[first] = bos[which][at[first, 0]][..., :hd]
        for rows, b in ((first, 4 if bits == 3 else bits), (~first, bits)):
            want, scale = paged.quantise(x[rows], b, EPS32)
            assert np.array_equal(got[rows], want)
            held = scales[which][at[rows, 0], :, at[rows, 1]]
            assert (np.abs(held - scale) <= HALF_F32 * scale * (1 + 1e-6)).all()
    want = turned(qn)
    part = np.abs(qn) + np.abs(np.concatenate([qn[..., hd // 2:], qn[..., :hd // 2]], -1))
    out = qr.double().cpu().numpy().reshape(n, heads, hd)
    assert (np.abs(out[:real] - want) <= HALF_BF16 * np.abs(want) + 4 * HALF_F32 * part * (1 + HALF_BF16)).all()
    assert (out[real:] == 7).all()


@pytest.mark.parametrize("q_len,kv_len", [(1, 900), (3, 77), (120, 500)])
def test_a_sequence_among_others(a48, cuda_dev, q_len, kv_len):
    """One sequence alone, beside prompts, beside many single tokens and behind longer bounds: the cut into parts is another each
    time, and each result lies within the bound of the oracle's."""
    rng = np.random.default_rng(38)
    hd, kvh, heads, page = 64, 2, 8, 32
    others = {"alone": ([], []), "prompts": ([300, 90], [300, 1200]), "tokens": ([1] * 40, list(rng.integers(1, 600, 40))), "few": ([2, 5], [33, 64])}
    seen = []
    for name, (q_lens, kv_lens) in others.items():
        s = Setup(a48, cuda_dev, 4, kvh, hd, page, [q_len] + q_lens, [kv_len] + [int(n) for n in kv_lens], seed=28)
        s.fill(np.random.default_rng(39))
        first = a48.PagedBatch(torch.tensor([0, kv_len], dtype=torch.int32, device=cuda_dev), s.batch.kv_len[:1], s.batch.pages[:1], kv_len, kv_len, kv_len)
        x = np.random.default_rng(40)
        k, v = (torch.tensor(x.standard_normal((kv_len, kvh * hd)), dtype=torch.float32) for _ in range(2))
        a48.paged_write(s.cache, first, k.to(cuda_dev), v.to(cuda_dev))
        s.oracle.write([0, kv_len], [kv_len], s.table[:1], k.numpy(), v.numpy(), 10000.0, EPS32)
        q = torch.tensor(np.concatenate([np.random.default_rng(41).standard_normal((q_len, heads * hd)),
                                         rng.standard_normal((sum(q_lens), heads * hd))]), dtype=torch.float32).to(torch.bfloat16)
        for batch in (s.batch, s.view(s.q_start, s.kv_len, s.n_tokens, max_q=700, max_kv=20000)):
            got = a48.attention_paged(s.cache, batch, q.to(cuda_dev)).double().cpu().numpy().reshape(-1, heads, hd)
            ref, mag, top = s.oracle.attend(s.q_start, s.kv_len, s.table, q.double().numpy(), heads)
            vmax = np.abs(s.oracle.scales[1]).max() * 128
            assert (np.abs(got - ref) <= attention_bound(ref, mag, top, hd, vmax) + weight_tail(max(kv_len, 1200), vmax)).all(), name
            seen.append((got[:q_len], ref[:q_len], (attention_bound(ref, mag, top, hd, vmax) + weight_tail(max(kv_len, 1200), vmax))[:q_len]))
    for got, ref, bound in seen[1:]:
        assert np.allclose(ref, seen[0][1], rtol=1e-12, atol=1e-14)  # the same sequence each time
        assert (np.abs(got - seen[0][0]) <= bound + seen[0][2]).all()


@pytest.mark.parametrize("bits,hd,heads,page", [(4, 64, 4, 16), (3, 128, 2, 64), (8, 100, 3, 32)])
def test_beside_the_attention_of_a_contiguous_cache(a48, cuda_dev, bits, hd, heads, page):
    """The keys and values read back from the pages through the framework's attention over a contiguous fp32 cache: the same
    outputs, within the bound of the paged one and the other's fp32 rounding."""
    rng = np.random.default_rng(42)
    B, T, cached = 3, 70, 61
    s = Setup(a48, cuda_dev, bits, heads, hd, page, [T] * B, [T + cached] * B, seed=29)
    s.fill(rng)
    n = T + cached
    every = s.view(np.arange(B + 1, dtype=np.int32) * n, s.kv_len, B * n)
    k, v = (t.view(B, n, heads, hd).transpose(1, 2).contiguous() for t in a48.paged_read(s.cache, every, dtype=torch.float32))
    q = torch.tensor(rng.standard_normal((B * T, heads * hd)), dtype=torch.float32).to(torch.bfloat16)
    want = a48.attention_prefill(q.float().to(cuda_dev), k, v, B, T, pos0=cached).double().cpu().numpy().reshape(B * T, heads, hd)
    got = check_attention(s, q, heads)
    out, mag, top = s.oracle.attend(s.q_start, s.kv_len, s.table, q.double().numpy(), heads)
    vmax = np.abs(s.oracle.scales[1]).max() * 128
    # the other call: 4e-8 |score| relative to the row's largest output, and a rounding of the read value
    other = (4e-8 * top[..., None] + 4 * HALF_F32) * np.abs(out).max(-1, keepdims=True) + 2 * HALF_F32 * (1 + 2 * top[..., None]) * mag
    assert (np.abs(got - want) <= attention_bound(out, mag, top, hd, vmax) + weight_tail(n, vmax) + other).all()


@pytest.mark.parametrize("bits", [8, 4, 3])
@pytest.mark.parametrize("step", [20.0, 24.6, 30.0])
def test_weights_ahead_of_a_far_larger_score(a48, cuda_dev, bits, step):
    """Scores in octaves: 9.5 in the first tile of 128 positions, 14.9 in the first half of the second (their weights do not move
    the reference), 9.5 + `step` behind them.  The last one's value has one entry only, so that the others show in the rest of the
    row: they weigh 2^-9 to 2^-19 of it, which fp16 holds next to it."""
    hd, q_len, n = 64, 128, 384
    s = Setup(a48, cuda_dev, bits, 1, hd, 32, [q_len], [n], seed=30)
    direction = np.where(np.arange(hd) % 2, 1.0, -1.0)
    size, v = np.zeros(n), np.zeros((n, hd))
    size[40], size[128:192], size[200] = 9.5, 14.9, 9.5 + step
    v[40, 0], v[128:192, 1:], v[200, 0] = 1.0, 1.0, 1.0  # (the value scales' unit stays that of the first tile)
    kt, vt = (torch.tensor(x, dtype=torch.float32) for x in (size[:, None] * direction, v))
    a48.paged_write(s.cache, s.view(np.array([0, n], np.int32), [n], n), kt.to(cuda_dev), vt.to(cuda_dev),
                    rope_base=0.0)
    s.oracle.write([0, n], [n], s.table, kt.double().numpy(), vt.double().numpy(), 0.0, EPS32)
    q = torch.tensor(np.tile(direction, (q_len, 2)), dtype=torch.float32).to(torch.bfloat16)
    scale = float(np.float32(np.log(2.0) / hd))
    got = a48.attention_paged(s.cache, s.batch, q.to(cuda_dev), scale=scale).double().cpu().numpy().reshape(q_len, 2, hd)
    out, mag, top = s.oracle.attend(s.q_start, s.kv_len, s.table, q.double().numpy(), 2, scale)
    vmax = np.abs(s.oracle.scales[1]).max() * 2 ** (bits - 1)  # (codes of these bits)
    bound = attention_bound(out, mag, top, hd, vmax) + weight_tail(n, vmax)
    if step < 30:
        assert (np.abs(out[..., 1:]) > 4 * bound[..., 1:]).all()  # (they would be missed)
    assert (np.abs(got - out) <= bound).all()


@pytest.mark.parametrize("q_len", [1, 3, 260])
def test_a_nan_in_one_of_many_parts(a48, cuda_dev, q_len):
    """One sequence whose positions are split into more parts than a cluster joins: a value or key that is no number in one part
    reaches the rows that see it through the join."""
    rng = np.random.default_rng(43)
    hd, kvh, heads, n = 64, 1, 2, 6000
    s = Setup(a48, cuda_dev, 4, kvh, hd, 64, [q_len], [n], seed=31)
    assert a48.attention_paged_workspace_bytes(s.cache, s.batch, heads) > 0
    k, v = (torch.tensor(rng.standard_normal((n, hd)), dtype=torch.float32) for _ in range(2))
    every = s.view(np.array([0, n], np.int32), [n], n)
    q = torch.tensor(rng.standard_normal((q_len, heads * hd)), dtype=torch.float32).to(torch.bfloat16).to(cuda_dev)
    for which, pos in ((0, 2), (1, 3000), (0, n - 1), (1, n - 1)):
        x = [k.clone(), v.clone()]
        x[which][pos, 7] = float("nan")
        a48.paged_write(s.cache, every, x[0].to(cuda_dev), x[1].to(cuda_dev))
        got = torch.isnan(a48.attention_paged(s.cache, s.batch, q))
        first = max(0, pos - (n - q_len))  # the first new token that sees the position
        assert not got[:first].any() and got[first:].all()
