"""Paged low-bit cache without a GPU: the oracle against the definitions it restates, and what the calls refuse."""
import ctypes

import numpy as np
import pytest

from oracle import paged


def test_oracle_quantiser_is_the_head_quantiser(oracle):
    x = np.random.default_rng(0).standard_normal((40, 96)).astype(np.float32)
    for bits in (3, 4, 8):
        q, d = paged.quantise(x, bits, np.float64(np.float32(1e-5)))
        q2, d2 = oracle.quant_heads(x, bits, eps=float(np.float32(1e-5)))
        assert np.array_equal(q, q2) and np.allclose(d, d2, rtol=1e-15, atol=0)


def test_oracle_attention_reduces_to_the_block_s(oracle):
    """One length, every position on a page, no window: the causal attention of the block on the dequantised heads."""
    rng = np.random.default_rng(1)
    B, T, nh, hd, page = 2, 21, 3, 12, 16
    table = np.array([[3, 1], [0, 4]])
    c = paged.Cache(8, nh, hd, page, 5)
    q_start, kv_len = [0, T, 2 * T], [T, T]
    k, v, q = (rng.standard_normal((B * T, nh * hd)) for _ in range(3))
    c.write(q_start, kv_len, table, k, v, rope_base=100.0)
    kv = c.read(q_start, kv_len, table, B * T).reshape(2, B, T, nh, hd).transpose(0, 1, 3, 2, 4)
    out, _, _ = c.attend(q_start, kv_len, table, q, nh)
    ref = oracle.attention_causal(q, kv[0], kv[1], B=B, T=T, n_heads=nh)
    assert np.abs(out.reshape(B * T, -1) - ref).max() < 1e-12
    # the window as its definition, position by position
    win, _, _ = c.attend(q_start, kv_len, table, q, nh, window=5, sinks=2)
    for b in range(B):
        for t in range(T):
            seen = [j for j in range(t + 1) if j > t - 5 or j < 2]
            for h in range(nh):
                s = np.array([kv[0, b, h, j] @ q[b * T + t, h * hd:(h + 1) * hd] for j in seen]) / np.sqrt(hd)
                p = np.exp(s - s.max())
                want = (p / p.sum()) @ kv[1, b, h, seen]
                assert np.abs(win[b * T + t, h] - want).max() < 1e-12


def test_rotation_keeps_lengths_and_angles_are_positions():
    x = np.random.default_rng(2).standard_normal(8)
    assert np.allclose(paged.rotate(x, 0, 10000.0), x)
    far = paged.rotate(x, 1000003, 10000.0)
    assert abs(np.linalg.norm(far) - np.linalg.norm(x)) < 1e-12
    twice = paged.rotate(paged.rotate(x, 5, 7.0), 6, 7.0)
    assert np.abs(twice - paged.rotate(x, 11, 7.0)).max() < 1e-12


def make(a48, bits=4, heads=2, hd=64, page=16, n_pages=4):
    return a48.PagedCacheConfig(bits, heads, hd, page, n_pages)


def batch(a48, **kw):
    d = dict(n_seqs=1, n_tokens=2, max_q=2, max_kv=2, max_pages=1, q_start_dev=4096, kv_len_dev=4096, pages_dev=4096)
    d.update(kw)
    return a48.PagedBatchView(*d.values())


@pytest.mark.parametrize("bits,row", [(8, 128), (4, 64), (3, 48)])
def test_pool_size(a48, bits, row):
    lib = a48.lib()
    for page in (16, 32, 64, 128):
        for hd in (100, 128):
            cfg = make(a48, bits, 3, hd, page, 7)
            assert lib.bitnet_a48_paged_cache_bytes(ctypes.byref(cfg)) == 7 * 3 * (2 * page * row + 8 * page + (128 if bits == 3 else 0))
    big = make(a48, bits, 8, 128, 64, 1 << 20)  # past 32 bits
    assert lib.bitnet_a48_paged_cache_bytes(ctypes.byref(big)) > 1 << 32


@pytest.mark.parametrize("kw", [dict(bits=5), dict(bits=16), dict(heads=0), dict(hd=0), dict(hd=2), dict(hd=132), dict(hd=66),
                                dict(page=8), dict(page=48), dict(page=256), dict(n_pages=0)])
def test_refused_caches(a48, kw):
    cfg = make(a48, **kw)
    assert a48.lib().bitnet_a48_paged_cache_bytes(ctypes.byref(cfg)) == 0


def test_refusals_of_the_calls(a48):
    lib = a48.lib()
    INVALID, SHAPE, ALIGN, LIMIT = 1, 2, 3, 8
    p, null = ctypes.c_void_p(4096), ctypes.c_void_p(0)
    good = make(a48)
    width = 2 * 64

    def write(cfg=good, pool=p, b=None, heads=4, q=p, qs=4 * 64, k=p, ks=width, v=p, vs=width, bf16=1, base=1e4, eps=1e-5, qo=p, qos=4 * 64):
        return lib.bitnet_a48_paged_write(ctypes.byref(cfg), pool, ctypes.byref(b or batch(a48)), heads, q, qs, k, ks, v, vs, bf16, base,
                                          eps, qo, qos, null)

    def read(cfg=good, pool=p, b=None, k=p, v=p):
        return lib.bitnet_a48_paged_read(ctypes.byref(cfg), pool, ctypes.byref(b or batch(a48)), k, v, 1, null)

    def attend(cfg=good, pool=p, b=None, heads=4, q=p, qs=4 * 64, scale=0.0, window=0, sinks=0, out=p, os=4 * 64, ws=p, nbytes=1 << 40):
        return lib.bitnet_a48_attention_paged(ctypes.byref(cfg), pool, ctypes.byref(b or batch(a48)), heads, q, qs, scale, window, sinks,
                                              out, os, ws, nbytes, null)

    for call in (write, read, attend):
        assert call(pool=null) == INVALID
        assert call(pool=ctypes.c_void_p(4104)) == ALIGN
        assert call(cfg=make(a48, bits=2)) == SHAPE
        assert call(b=batch(a48, n_seqs=0)) == SHAPE
        assert call(b=batch(a48, n_seqs=65536)) == LIMIT
        assert call(b=batch(a48, n_tokens=0)) == SHAPE
        assert call(b=batch(a48, max_q=0)) == SHAPE
        assert call(b=batch(a48, max_kv=-1)) == SHAPE
        assert call(b=batch(a48, max_pages=0)) == SHAPE
        for field in ("q_start_dev", "kv_len_dev", "pages_dev"):
            assert call(b=batch(a48, **{field: None})) == INVALID
            assert call(b=batch(a48, **{field: 4098})) == ALIGN
    assert write(k=null) == INVALID and write(v=null) == INVALID
    assert write(q=null) == INVALID and write(qo=null) == INVALID  # both or neither
    assert write(ks=width - 4) == SHAPE and write(vs=width + 2) == SHAPE and write(qs=0) == SHAPE and write(qos=4) == SHAPE
    assert write(k=ctypes.c_void_p(4100)) == ALIGN and write(k=ctypes.c_void_p(4104), bf16=0) == ALIGN
    assert write(heads=0) == SHAPE and write(eps=-1.0) == INVALID and write(base=-2.0) == INVALID and write(base=float("nan")) == INVALID
    assert read(k=null) == INVALID and read(v=ctypes.c_void_p(4104)) == ALIGN
    assert attend(q=null) == INVALID and attend(out=null) == INVALID
    assert attend(heads=3) == SHAPE and attend(heads=0) == SHAPE and attend(heads=65536) == LIMIT
    assert attend(qs=4 * 64 - 4) == SHAPE and attend(os=4 * 64 + 1) == SHAPE
    assert attend(q=ctypes.c_void_p(4100)) == ALIGN and attend(out=ctypes.c_void_p(4098)) == ALIGN and attend(ws=ctypes.c_void_p(8)) == ALIGN
    assert attend(window=-1) == INVALID and attend(sinks=-1) == INVALID and attend(scale=-1.0) == INVALID and attend(scale=float("inf")) == INVALID


def test_limits_and_workspace(a48):
    lib = a48.lib()
    NOMEM, LIMIT = 7, 8
    p, null = ctypes.c_void_p(4096), ctypes.c_void_p(0)
    good = make(a48)

    def attend(b, heads=4, ws=p, nbytes=1 << 40):
        return lib.bitnet_a48_attention_paged(ctypes.byref(good), p, ctypes.byref(b), heads, p, heads * 64, 0.0, 0, 0, p, heads * 64, ws, nbytes, null)

    def need(b, heads=4):
        return lib.bitnet_a48_attention_paged_workspace_bytes(ctypes.byref(good), ctypes.byref(b), heads, 0, 0)

    assert attend(batch(a48, n_tokens=(1 << 30) + 1)) == LIMIT
    assert attend(batch(a48, max_pages=1 << 27)) == LIMIT  # times 16 positions
    assert attend(batch(a48, n_tokens=1 << 30), heads=4) == LIMIT  # rows past 2^31 - 1
    assert lib.bitnet_a48_paged_write(ctypes.byref(good), p, ctypes.byref(batch(a48)), 65536, p, 65536 * 64, p, 128, p, 128, 1, 1e4, 1e-5, p,
                                      65536 * 64, null) == LIMIT
    for b in (batch(a48, max_q=1, max_kv=1 << 20, max_pages=1 << 16), batch(a48, n_tokens=300, max_q=300, max_kv=1 << 16, max_pages=1 << 12)):
        n = need(b)  # one long sequence: parts that are joined through the workspace
        assert n > 0
        assert attend(b, ws=null, nbytes=0) == NOMEM and attend(b, nbytes=n - 1) == NOMEM and attend(b, ws=null, nbytes=n) == NOMEM
    assert need(batch(a48, n_seqs=0)) == 0 and need(batch(a48), heads=3) == 0


def test_binding_refuses(a48):
    with pytest.raises(a48.A48Error):
        a48.PagedCache(5, 2, 64, 16, 4)


@pytest.mark.parametrize("kw,heads", [(dict(n_tokens=300, max_q=300), 4), (dict(max_q=1), 4), (dict(n_seqs=8, n_tokens=32, max_q=4), 2),
                                      (dict(n_seqs=2, n_tokens=4096, max_q=2048), 4)])
@pytest.mark.parametrize("big", [(1 << 30) - 1, 1 << 30, (1 << 31) - 1])
def test_windows_and_sinks_of_any_size(a48, kw, heads, big):
    """A window or sinks as long as the context cut a call up as no window does: the same workspace, however large they are."""
    lib, good = a48.lib(), make(a48, heads=2, n_pages=1 << 12)
    b = batch(a48, **dict(dict(max_kv=1 << 16, max_pages=1 << 12), **kw))
    need = lambda window, sinks: lib.bitnet_a48_attention_paged_workspace_bytes(ctypes.byref(good), ctypes.byref(b), heads, window, sinks)  # noqa: E731
    want = need(0, 0)
    assert want > 0 or kw.get("n_seqs", 1) > 1
    for window, sinks in ((big, 0), (big, 4), (big, big), (1 << 16, big), (1, big), (64, big)):
        assert need(window, sinks) == want, (window, sinks)


@pytest.mark.parametrize("heads,kvh,hd,bits", [(32, 32, 128, 3), (32, 8, 128, 4), (32, 4, 64, 8), (32, 1, 128, 4), (16, 1, 96, 8), (1, 1, 4, 4), (300, 1, 32, 8)])
def test_workspace_holds_only_what_is_split(a48, heads, kvh, hd, bits):
    """Places of partial sums go by the rows that can be split, of which the SMs take 148 tiles of 256 at once and 37 of 16: long
    prompts, many of them, token arrays with room to spare and bounds that are too large add none."""
    lib, cfg = a48.lib(), make(a48, bits, kvh, hd, 64, 1 << 16)
    bound = 520 * (148 * 256 + 37 * 16) + 4 * 256  # 128 sums, exponent and sum of a place; alignment
    sizes = [1, 2, 3, 7, 8, 63, 64, 65, 200, 300, 2048, 16384, 32768, 1 << 20, 1 << 24]
    worst = 0
    for max_q in sizes:
        for n_seqs in (1, 2, 5, 8, 64, 1000, 65535):
            for n_tokens in {max_q, min(max_q * n_seqs, 1 << 24), 1 << 20}:
                for max_kv, window in ((max_q, 0), (1 << 20, 0), (1 << 20, 2048), (1 << 20, 1)):
                    b = batch(a48, n_seqs=n_seqs, n_tokens=n_tokens, max_q=max_q, max_kv=max_kv, max_pages=1 << 14)
                    worst = max(worst, lib.bitnet_a48_attention_paged_workspace_bytes(ctypes.byref(cfg), ctypes.byref(b), heads, window, 4))
    assert 0 < worst <= bound
    prompt = batch(a48, n_tokens=1 << 14, max_q=1 << 14, max_kv=1 << 14, max_pages=1 << 8)
    one = batch(a48, n_tokens=1, max_q=1, max_kv=1 << 14, max_pages=1 << 8)
    need = [lib.bitnet_a48_attention_paged_workspace_bytes(ctypes.byref(cfg), ctypes.byref(b), heads, 0, 0) for b in (prompt, one)]
    if heads > 16:  # the prompt alone fills the SMs: what is left is what one decoding sequence may have
        assert need[0] <= 37 * 16 * 520 + 4 * 256
    if heads // kvh <= 64:  # (more rows than that are the tile kernel's)
        assert need[1] <= 37 * 16 * 520 + 4 * 256


def test_stride_of_a_single_row_does_not_matter(a48):
    """A token's row out of rows of any length: its stride is never used, so none is refused."""
    torch = pytest.importorskip("torch")

    class OnTheHost:
        device_index = -1

    rows = torch.zeros(6, 131)
    assert a48._rows(rows[3:4, 4:132], OnTheHost, 1, 127, torch.float32) == 127
    assert a48._rows(rows[3:4, 4:68], OnTheHost, 1, 64, torch.float32) == 64
    assert a48._rows(rows[2:4, 4:68], OnTheHost, 2, 64, torch.float32) == 131
    with pytest.raises(AssertionError):  # columns apart
        a48._rows(torch.zeros(64, 6).t()[1:2], OnTheHost, 1, 64, torch.float32)
