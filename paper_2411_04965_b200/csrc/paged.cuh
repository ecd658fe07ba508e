// The paged low-bit key/value cache (Section 3's low-bit attention over pages of positions): layout of a page and the
// description of a batch, shared by the kernels that write, read and attend to it.
//
// The pool is [n_pages][n_kv_heads] chunks.  A chunk holds the page_size positions of one page for one head, keys and
// values together, so that a kernel that walks one head of one sequence finds all it needs of a page in one run:
//   key codes [page_size][row] | value codes [page_size][row] | key scales fp32 [page_size] | value scales [page_size]
//   | 3 bits only: the 4-bit codes of the key and the value of position 0 (the bos token), 2 x P / 2 bytes
// with P the head dimension padded to a multiple of 32 and row = P * bits / 8.  page_size is a power of two from 16 to
// 128, so every part starts on a 16-byte boundary.
//
// An entry is the unsigned u = q + L + 1, L = 2^(bits-1) - 1 (padding holds the code of 0).  8 bits: byte i; 4 bits:
// half bytes in order.  3 bits: 32 entries in three words; entries 5j .. 5j+4 sit in bits 0..14 of the low half of word j,
// entry 15 in the three top bits of the low halves, entries 16..31 the same way in the high halves.  The halves of a word
// then unpack together: one mask gives two entries that are 16 bits apart, which is what a pair of fp16 numbers wants.
#pragma once

#include "internal.h"

namespace a48p {

struct Layout {
    int bits, kv_heads, hd, page, page_shift, n_pages;
    int padded, row;                            // P, bytes of a code row
    int v_codes, k_scales, v_scales, bos, chunk;  // byte offsets in a chunk (key codes at 0) and its size
};

// What the kernels need of a batch; lengths live on the device.
struct Batch {
    int n_seqs, n_tokens, max_pages;
    const int32_t* q_start;
    const int32_t* kv_len;
    const int32_t* pages;
};

inline Layout layout_of(const bitnet_a48_paged_cache& c) {
    Layout l;
    l.bits = c.bits;
    l.kv_heads = c.n_kv_heads;
    l.hd = c.head_dim;
    l.page = c.page_size;
    l.page_shift = 0;
    while ((1 << l.page_shift) < c.page_size) ++l.page_shift;
    l.n_pages = c.n_pages;
    l.padded = (c.head_dim + 31) / 32 * 32;
    l.row = l.padded * c.bits / 8;
    l.v_codes = c.page_size * l.row;
    l.k_scales = 2 * l.v_codes;
    l.v_scales = l.k_scales + 4 * c.page_size;
    l.bos = l.v_scales + 4 * c.page_size;
    l.chunk = l.bos + (c.bits == 3 ? l.padded : 0);
    return l;
}

inline Batch batch_of(const bitnet_a48_paged_batch& b) {
    return Batch{b.n_seqs, b.n_tokens, b.max_pages, b.q_start_dev, b.kv_len_dev, b.pages_dev};
}

#ifdef __CUDACC__
// Byte offset of the chunk of (page, head); 64-bit, a pool is as large as memory allows.
__device__ __forceinline__ size_t chunk_at(const Layout& l, int page, int head) {
    return ((size_t)page * l.kv_heads + head) * l.chunk;
}

// The last i in [0, n) with key(i) <= x (key ascending), or -1.  The whole warp searches, 32 keys at a time.
template <typename Key>
__device__ __forceinline__ int last_at_most(int n, long long x, int lane, Key key) {
    int lo = 0;  // the answer is in [lo - 1, lo + n)
    while (n > 0) {
        const int step = (n + 31) / 32;
        const bool below = lane * step < n && key(lo + lane * step) <= x;
        const int hits = __popc(__ballot_sync(0xffffffffu, below));
        if (hits == 0) break;
        const int end = lo + n;
        lo += (hits - 1) * step + 1;  // keys up to lo - 1 are known to be <= x
        n = min(step - 1, end - lo);
    }
    return lo - 1;
}

// The sequence whose new tokens include row `row` of the packed tokens, or -1.
__device__ __forceinline__ int sequence_of(const Batch& b, int row, int lane) {
    const int s = last_at_most(b.n_seqs, row, lane, [&](int i) { return (long long)__ldg(b.q_start + i); });
    return s < 0 || row >= __ldg(b.q_start + s + 1) ? -1 : s;
}

// Page and slot of position `pos` of sequence s; page -1 where the table has none (negative or past the table's or the
// pool's end).
__device__ __forceinline__ int page_of(const Layout& l, const Batch& b, int s, int pos) {
    const int index = pos >> l.page_shift;
    if (pos < 0 || index >= b.max_pages) return -1;
    const int page = __ldg(b.pages + (size_t)s * b.max_pages + index);
    return page >= 0 && page < l.n_pages ? page : -1;
}
#endif

// Token rows of heads: the pointer to four elements, the stride at least the row and a multiple of four elements.
inline bitnet_a48_status check_rows(const void* p, long long stride, long long width, int elem) {
    if (!p) return BITNET_A48_ERR_INVALID_ARG;
    if (stride < width || (stride & 3)) return BITNET_A48_ERR_SHAPE;
    return reinterpret_cast<uintptr_t>(p) & (4 * elem - 1) ? BITNET_A48_ERR_ALIGNMENT : BITNET_A48_OK;
}
// Arguments common to the calls; BITNET_A48_OK or the first thing wrong.
inline bitnet_a48_status check(const bitnet_a48_paged_cache* c, const void* pool, const bitnet_a48_paged_batch* b) {
    if (!c || !pool || !b || !b->q_start_dev || !b->kv_len_dev || !b->pages_dev) return BITNET_A48_ERR_INVALID_ARG;
    if (!bitnet_a48_paged_cache_bytes(c)) return BITNET_A48_ERR_SHAPE;
    if (b->n_seqs <= 0 || b->n_tokens <= 0 || b->max_q <= 0 || b->max_kv <= 0 || b->max_pages <= 0) return BITNET_A48_ERR_SHAPE;
    // rows and positions of a call stay in 32 bits
    if (b->n_seqs > 65535 || b->n_tokens > (1 << 30) || (long long)b->max_pages * c->page_size > (1 << 30)) return BITNET_A48_ERR_LIMIT;
    const uintptr_t plan = reinterpret_cast<uintptr_t>(b->q_start_dev) | reinterpret_cast<uintptr_t>(b->kv_len_dev) |
                           reinterpret_cast<uintptr_t>(b->pages_dev);
    if (!a48_aligned16(pool) || (plan & 3)) return BITNET_A48_ERR_ALIGNMENT;
    return BITNET_A48_OK;
}

}  // namespace a48p
