// Causal attention of new tokens over the paged low-bit cache, with an optional sliding window beside which the first
// tokens of a sequence stay visible.
//
//   out[i] = sum_j softmax_j(scale q[i] . k[j]) v[j]   over j <= p, and with a window w: j > p - w or j < sinks
//
// p the position of token i.  k[j] = sk[j] c[j] and v[j] = sv[j] d[j] with integer codes c, d, so that
//   score = (q . c[j]) sk[j] scale,   out = (sum_j p[j] sv[j] d[j]) / sum_j p[j]:
// both contractions run on the codes, which fp16 holds exactly, and the scales meet the scores and the probabilities in
// fp32.  Query rows are brought into fp16 by a power of two (their bf16 numbers fit its 11 bits), the weights p sv by a
// power of two that follows the largest value scale; what is rounded is the weight, to fp16's 11 bits (bf16's 8 would
// cost as much as the rounding of the output).
//
// The rows of one key/value head (token i, query head of the group) are taken together.  Sequences with few rows
// (decoding, drafted tokens) go to attn_paged_rows_kernel below, those with more to the tile kernel of attn_paged_tc.cu.
#include <climits>

#include "attn_paged.cuh"

namespace {

using a48p::exp2_approx;
using a48p::in_register;
using a48p::Layout;

using a48p::AttnArgs;
using a48p::Span;
using a48p::span_of;

// ---------------------------------------------------------------------------------------------------- few rows
// Measured: one token for each of 64 sequences of up to 8192 positions, 32 heads over 8, 4 bits, 94 us (3.1 TB/s of codes);
// 32 sequences of 1500 to 2048, 32 heads of 100, none shared, 66 us (3.8 TB/s); four drafted tokens of 8 sequences under a
// window of 4096 19 us; one sequence 13 us with its call.  With many sequences the bound is what the SMs do per code (copy, field extraction, fragments), with few the
// chain of page number, codes, products and join.
// A CTA of four warps takes a tile of 8 NT rows of one head and one part of the positions; a warp takes pairs of blocks of 16
// positions out of two stages in shared memory that asynchronous copies fill (a block's codes are one run of a page, so
// are its scales): what hides memory is bytes in flight, and registers hold too few.
//
// The positions are the M side of both contractions (m16n8k16, fp16, fp32 accumulators), the rows the N side: S^T = C Q^T
// and O^T = D^T P^T.  Eight rows are then no padding, and the codes, whose conversion is what a position costs, are
// converted once for all rows.  Entries are dealt to lanes so that every lane converts what it read: lane 4g+t holds
// for S^T the t-th quarter of the key rows of positions g and g + 8 (the order of the entries inside the contraction is
// free: the query fragments are taken in the same order), for O^T the g-th eighth of the value rows of positions 2t, 2t+1,
// 2t+8, 2t+9, whose words are first merged into halves of the same entry of two positions.  S^T's accumulators become
// P^T's operand by one 8x8 transpose each.
//
// The running maximum is one reference per row that moves only when a weight would exceed 2^9 (or a value scale its unit by
// 2^6): nothing is reduced across lanes in the steady state but one vote, and weights stay within fp16.
constexpr int ROW_WARPS = 4, MAX_RANKS = 8;

__device__ __forceinline__ void mma_f16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// the first of a chain: onto `start`, by the column's parity
__device__ __forceinline__ void mma_f16_first(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1,
                                              const float (&start)[2]) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %11, %12, %13};"
        : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(start[0]), "f"(start[1]), "f"(start[0]), "f"(start[1]));
}
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
    return r;
}

// Words of a lane's share of a code row: of the keys a quarter, of the values an eighth (3 bits: the granule it is in).
template <int BITS, int PD>
struct Share {
    static constexpr int K = BITS == 3 ? 3 : PD * BITS / 128, V = BITS == 3 ? 3 : PD * BITS / 256;
};
template <int N>
__device__ __forceinline__ void load_words(const uint8_t* p, uint32_t (&w)[N]) {  // of shared memory
    if constexpr (N % 4 == 0) {
#pragma unroll
        for (int i = 0; i < N / 4; ++i) {
            const uint4 v = reinterpret_cast<const uint4*>(p)[i];
            w[4 * i] = v.x, w[4 * i + 1] = v.y, w[4 * i + 2] = v.z, w[4 * i + 3] = v.w;
        }
    } else if constexpr (N == 2) {
        const uint2 v = *reinterpret_cast<const uint2*>(p);
        w[0] = v.x, w[1] = v.y;
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) w[i] = reinterpret_cast<const unsigned*>(p)[i];
    }
}
__device__ __forceinline__ void copy16(uint32_t dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}

// A block of 16 positions in a stage: key rows, value rows, key scales, value scales.  Value rows are read two apart by
// the lanes of a request (positions 2t): 4- and 8-bit rows lie 16 bytes past a multiple of 64 apart, so that those fall into
// different banks (3-bit rows do so as they are).
template <int BITS, int PD>
struct Block {
    static constexpr int PITCH = BITS == 3 ? 48 : BITS * PD / 8 <= 64 ? 80 : 144;
    static constexpr int K = 0, V = 16 * PD * BITS / 8, SK = V + 16 * PITCH, SV = SK + 64, BYTES = SV + 64;
};
constexpr int STAGES = 2;

// Entry of a key row that is half h of converted word i of quarter t (the order convert_k gives).
template <int BITS, int PD>
__device__ __forceinline__ int k_entry(int t, int i, int h) {
    if (BITS == 3) return 32 * t + 16 * h + i;
    if (BITS == 4) return PD / 4 * t + 8 * (i / 4) + i % 4 + 4 * h;
    return PD / 4 * t + 4 * (i / 2) + i % 2 + 2 * h;
}
// (as raw fields: the query fragments carry 2^-s, the factor of the scores 2^24, and the accumulators start at the offset's
// share, -2^(bits-1) times the sum of the query's entries.  Not so for the values: their sums run over thousands of
// positions, and would grow with the offset where those of signed codes do not.)
template <int BITS, int PD>
__device__ __forceinline__ void convert_k(const uint32_t (&w)[Share<BITS, PD>::K], uint32_t (&out)[PD / 8]) {
    if constexpr (BITS == 3) a48p::raw_triples(w[0], w[1], w[2], out);
    else if constexpr (BITS == 4) {
#pragma unroll
        for (int i = 0; i < PD / 32; ++i) a48p::raw_nibbles(w[i], out + 4 * i);
    } else {
#pragma unroll
        for (int i = 0; i < PD / 16; ++i) a48p::raw_bytes(w[i], out + 2 * i);
    }
}
// The PD / 8 entries of an eighth, in order, of two positions a and b.
template <int BITS, int PD>
__device__ __forceinline__ void convert_v(const uint32_t (&a)[Share<BITS, PD>::V], const uint32_t (&b)[Share<BITS, PD>::V], uint32_t halves,
                                          uint32_t (&out)[PD / 8]) {
    if constexpr (BITS == 3) {
        a48p::triples(__byte_perm(a[0], b[0], halves), __byte_perm(a[1], b[1], halves), __byte_perm(a[2], b[2], halves), out);
    } else if constexpr (BITS == 4) {
#pragma unroll
        for (int i = 0; i < PD / 64; ++i) {
            a48p::nibbles(__byte_perm(a[i], b[i], 0x5410), out + 8 * i);
            a48p::nibbles(__byte_perm(a[i], b[i], 0x7632), out + 8 * i + 4);
        }
    } else {
#pragma unroll
        for (int i = 0; i < PD / 32; ++i) {
            a48p::bytes(__byte_perm(a[i], b[i], 0x5410), out + 4 * i);
            a48p::bytes(__byte_perm(a[i], b[i], 0x7632), out + 4 * i + 2);
        }
    }
}

template <int BITS, int PD, int NT>
struct RowsShared {
    static constexpr int ROWS = 8 * NT;
    union {
        alignas(16) uint8_t ring[ROW_WARPS][STAGES][2][Block<BITS, PD>::BYTES];
        alignas(16) float o[ROW_WARPS][ROWS][PD + 4];  // the warps' sums
    };
    float top[ROW_WARPS], start[ROWS], factor;  // start: of a row's accumulators
    float m[ROW_WARPS][ROWS], l[ROW_WARPS][ROWS];
    int token[ROWS], head[ROWS];
    // what the cluster's CTAs send: pieces of four head dims, with the exponent of their reference and their sum of p
    alignas(16) float4 piece[ROWS * PD / 4 + MAX_RANKS];
    union {
        alignas(16) __half q[ROWS][PD + 8];
        float2 piece_ml[ROWS * PD / 4 + MAX_RANKS];
    };
};

__device__ __forceinline__ void cluster_arrive() {
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
}
__device__ __forceinline__ void cluster_wait() {
    __syncwarp();
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t of_rank(const void* p, int rank) {
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
    return r;
}
__device__ __forceinline__ void st_rank(uint32_t at, float4 v) {
    asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(at), "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w) : "memory");
}
__device__ __forceinline__ void st_rank(uint32_t at, float2 v) {
    asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(at), "f"(v.x), "f"(v.y) : "memory");
}

template <int BITS, int PD, int NT>
__device__ __forceinline__ void attend_rows(const AttnArgs& a, RowsShared<BITS, PD, NT>& sm) {
    constexpr int ROWS = 8 * NT, NK = PD / 8;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int kvh = blockIdx.x % a.l.kv_heads, seq = blockIdx.x / a.l.kv_heads / a.tiles;
    const int r0 = (blockIdx.x / a.l.kv_heads % a.tiles) * ROWS;
    const int start = __ldg(a.b.q_start + seq), q_len = __ldg(a.b.q_start + seq + 1) - start;
    const long long all_rows = (long long)q_len * a.group;
    // (the same for all CTAs of a cluster)
    if (all_rows > a.few_rows || r0 >= all_rows || start < 0 || q_len > a.b.n_tokens - start) return;
    const int rows = min(ROWS, (int)min(all_rows - r0, (long long)ROWS));
    const int pos0 = __ldg(a.b.kv_len + seq) - q_len;
    const int pos_lo = pos0 + r0 / a.group, pos_hi = pos0 + (r0 + rows - 1) / a.group;
    const Span span = span_of<5>(a, pos_lo, pos_hi);
    // positions are dealt out evenly, a pair of blocks for every warp of a part at least
    const int rank = blockIdx.y & (a.ranks - 1), cluster = blockIdx.y / a.ranks, parts = gridDim.y;
    const int per = max(ROW_WARPS, (span.count + parts - 1) / parts);
    const int v_begin = blockIdx.y * per, v_end = min(span.count, v_begin + per);

    // ---- the warp's pairs of blocks v_begin + warp + 4k: pages of the first ones under way
    const int window = in_register(a.window), sinks = in_register(a.sinks);
    const int pairs = max(0, (v_end - v_begin - warp + ROW_WARPS - 1) / ROW_WARPS);
    auto first_of = [&](int k) { return span.block(v_begin + warp + ROW_WARPS * k) << 5; };
    auto page_at = [&](int k, int b) {  // of block b of pair k; the second block has the first's page if that is large enough
        return k < pairs && (b == 0 || a.l.page_shift == 4) ? a48p::page_of(a.l, a.b, seq, first_of(k) + 16 * b) : -1;
    };
    int page[STAGES + 1][2];  // of the pairs in the stages and of the next
#pragma unroll
    for (int k = 0; k <= STAGES; ++k)
#pragma unroll
        for (int b = 0; b < 2; ++b) page[k][b] = page_at(k, b);
    if (threadIdx.x < ROWS) {
        const int in_seq = r0 + min((int)threadIdx.x, rows - 1), i = in_seq / a.group;
        sm.token[threadIdx.x] = start + i;
        sm.head[threadIdx.x] = kvh * a.group + in_seq - i * a.group;
    }
    __syncthreads();

    // What a lane copies of a block: 16-byte pieces lane + 32i of the key rows and of the value rows, and (lanes 0..7) one of
    // the scales.
    using B = Block<BITS, PD>;
    constexpr int PIECES = (PD * BITS / 8 + 31) / 32;
    const int row = a.l.row, pitch = BITS == 3 ? row : B::PITCH;
    uint8_t* ring = &sm.ring[warp][0][0][0];
    const uint32_t ring_at = (uint32_t)__cvta_generic_to_shared(ring);
    uint32_t v_dst[PIECES];
#pragma unroll
    for (int i = 0; i < PIECES; ++i) {
        const int at = 16 * (lane + 32 * i);
        v_dst[i] = B::V + (BITS == 3 ? at : at / row * pitch + at % row);
    }
    const uint8_t* head_chunks = a.pool + (size_t)kvh * a.l.chunk;
    const size_t page_bytes = (size_t)a.l.kv_heads * a.l.chunk;
    const int slots = in_register(a.l.page - 1), v_codes = in_register(a.l.v_codes);
    const int scales = lane < 4 ? a.l.k_scales + 16 * lane : a.l.v_scales + 16 * (lane - 4);
    // pair k into a stage; returns its pages (the same for the warp: addresses are formed once for it)
    auto load = [&](int k, int stage, int (&from)[2]) {
        from[0] = __shfl_sync(0xffffffffu, from[0], 0);
        from[1] = a.l.page_shift == 4 ? __shfl_sync(0xffffffffu, from[1], 0) : from[0];
        const int slot = first_of(k) & slots;
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            if (from[b] < 0) continue;
            const int at = (slot + 16 * b) & slots;
            const uint8_t* chunk = head_chunks + from[b] * page_bytes;
            const uint8_t* codes = chunk + at * row + 16 * lane;
            const uint32_t dst = ring_at + (2 * stage + b) * B::BYTES;
#pragma unroll
            for (int i = 0; i < PIECES; ++i)
                if (lane + 32 * i < row) {
                    copy16(dst + B::K + 16 * (lane + 32 * i), codes + 512 * i);
                    copy16(dst + v_dst[i], codes + (v_codes + 512 * i));
                }
            if (lane < 8) copy16(dst + B::SK + 16 * lane, chunk + scales + 4 * at);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int k = 0; k < STAGES; ++k) load(k, k, page[k]);
    // What it reads.  (A lane whose entries lie past the padded head reads some that exist: they meet zeros of the query, or
    // columns that are not stored.)
    const uint32_t k_first = BITS == 3 ? 12 * t : PD * BITS / 32 * t, v_first = BITS == 3 ? 12 * (g >> 1) : PD * BITS / 64 * g;
    const bool k_there = k_first < row, v_there = v_first < row;
    const uint32_t k_off = B::K + (k_there ? k_first : 0) + g * row, v_off = B::V + (v_there ? v_first : 0) + 2 * t * pitch;
    const uint32_t halves = (g & 1) ? 0x7632u : 0x5410u;

    // ---- the query rows to fp16 by one power of two (the largest entry of the tile to [2^14, 2^15): a row 2^14 below it
    // still has all its bits, one 2^23 below it the upper ten)
    {
        constexpr int PER = ROWS / ROW_WARPS;
        float x[PER][4] = {};
        uint32_t top = 0;
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            const int r = warp + ROW_WARPS * k;
            if (r < rows && 4 * lane < a.l.hd) {
                const uint2 u = __ldg(reinterpret_cast<const uint2*>(a.q + sm.token[r] * a.q_stride + (size_t)sm.head[r] * a.l.hd) + lane);
                x[k][0] = __uint_as_float(u.x << 16), x[k][1] = __uint_as_float(u.x & 0xffff0000u);
                x[k][2] = __uint_as_float(u.y << 16), x[k][3] = __uint_as_float(u.y & 0xffff0000u);
            }
            const float mx = fmaxf(fmaxf(fabsf(x[k][0]), fabsf(x[k][1])), fmaxf(fabsf(x[k][2]), fabsf(x[k][3])));
            if (mx <= 3.4e38f) top = max(top, __float_as_uint(mx));
        }
        top = __reduce_max_sync(0xffffffffu, top);
        if (lane == 0) sm.top[warp] = __uint_as_float(top);
        __syncthreads();
#pragma unroll
        for (int w = 0; w < ROW_WARPS; ++w) top = max(top, __float_as_uint(sm.top[w]));
        const int e = a48p::query_exponent(top);
        const float up0 = a48p::power_of_two(e / 2), up1 = a48p::power_of_two(e - e / 2);
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            const int r = warp + ROW_WARPS * k;
            const __half2 lo = __floats2half2_rn(x[k][0] * up0 * up1, x[k][1] * up0 * up1),
                          hi = __floats2half2_rn(x[k][2] * up0 * up1, x[k][3] * up0 * up1);
            // (of the numbers as they are rounded)
            float sum = __low2float(lo) + __high2float(lo) + __low2float(hi) + __high2float(hi);
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
            if (lane == 0) sm.start[r] = -sum * (float)(1 << (BITS - 1)) * 0x1p-24f;
            if (4 * lane < PD)
                *reinterpret_cast<uint2*>(&sm.q[r][4 * lane]) = make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
        }
        if (threadIdx.x == 0) sm.factor = a.scale * 1.4426950408889634f * a48p::power_of_two(24 - e / 2) * a48p::power_of_two(-(e - e / 2));
    }
    __syncthreads();
    const float factor = sm.factor;  // of an accumulator times its key scale: the score in units of log2 e
    uint32_t qf[NT][NK];
    int lim[NT][2];
    float begin[NT][2];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
        for (int i = 0; i < NK; ++i) {
            const __half2 h = __hmul2(__halves2half2(sm.q[8 * n + g][k_entry<BITS, PD>(t, i, 0)], sm.q[8 * n + g][k_entry<BITS, PD>(t, i, 1)]),
                                      __float2half2_rn(1.f / (1 << a48p::raw_shift<BITS>(i))));
            qf[n][i] = *reinterpret_cast<const uint32_t*>(&h);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            lim[n][i] = pos0 + (r0 + min(8 * n + 2 * t + i, rows - 1)) / a.group;  // the last position the row sees
            begin[n][i] = sm.start[8 * n + 2 * t + i];
        }
    }

    if (a.ranks > 1) cluster_arrive();  // (waited for ahead of the first write to another CTA's shared memory, over the queries)

    float o[NT][PD / 16][4], m[NT][2], l[NT][2];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
        for (int i = 0; i < PD / 16; ++i)
#pragma unroll
            for (int c = 0; c < 4; ++c) o[n][i][c] = 0.f;
        m[n][0] = m[n][1] = -1e30f;
        l[n][0] = l[n][1] = 0.f;
    }
    float v_unit = INFINITY;  // 2^6 over a power of two not below the largest value scale so far; infinite while that is 0

    // The pair of blocks in a stage, at positions from `first` on; from[b] < 0: block b is not there.
    auto take = [&](int stage, int first, const int (&from)[2]) {
        float s[2][NT][4], y[2][NT][4], ks[2][2], f[2][2], w[2][2];
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            const uint8_t* block = ring + (2 * stage + b) * B::BYTES;
            uint32_t k0[Share<BITS, PD>::K], k1[Share<BITS, PD>::K], ka[NK], kb[NK];
            load_words(block + k_off, k0);
            load_words(block + k_off + 8 * row, k1);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const float scale = reinterpret_cast<const float*>(block + B::SK)[g + 8 * i];
                ks[b][i] = fmaf(scale, 0.f, scale) * factor;  // (an infinite scale is none, not a score of -inf that would hide its key)
                f[b][i] = reinterpret_cast<const float*>(block + B::SV)[g + 8 * i];
            }
            convert_k<BITS, PD>(k0, ka);
            convert_k<BITS, PD>(k1, kb);
            if (BITS == 3 && b == 0 && first == 0 && from[0] >= 0) {  // the bos heads: 4-bit codes of their own, in convert_k's order
                const uint8_t* bos = a.pool + a48p::chunk_at(a.l, from[b], kvh) + a.l.bos;
                if (g == 0 && k_there) {
#pragma unroll
                    for (int i = 0; i < NK; ++i) {
                        const int e0 = k_entry<BITS, PD>(t, i, 0), e1 = k_entry<BITS, PD>(t, i, 1);
                        const float unit = (float)(1 << a48p::raw_shift<3>(i)) * 0x1p-24f;  // (codes less 8 on top of an offset of 4)
                        const __half2 h = __floats2half2_rn(((float)((bos[e0 / 2] >> (4 * (e0 & 1))) & 15) - 4.f) * unit,
                                                            ((float)((bos[e1 / 2] >> (4 * (e1 & 1))) & 15) - 4.f) * unit);
                        ka[i] = *reinterpret_cast<const uint32_t*>(&h);
                    }
                }
            }
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                mma_f16_first(s[b][n], ka[0], kb[0], ka[1], kb[1], qf[n][0], qf[n][1], begin[n]);
#pragma unroll
                for (int i = 1; i < NK / 2; ++i) mma_f16(s[b][n], ka[2 * i], kb[2 * i], ka[2 * i + 1], kb[2 * i + 1], qf[n][2 * i], qf[n][2 * i + 1]);
            }
        }
        const bool whole = first + 31 <= pos_lo && (window == 0 || first > pos_hi - window || first + 31 < sinks) && (from[0] | from[1]) >= 0;
        auto seen = [&](int b, int n, int c) {  // by row 2t + c % 2, position g + 8 (c / 2) of the block
            const int j = first + 16 * b + g + 8 * (c >> 1), last = lim[n][c & 1];
            return from[b] >= 0 && j <= last && (window == 0 || j > last - window || j < sinks);
        };
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int c = 0; c < 4; ++c) y[b][n][c] = fmaf(s[b][n][c], ks[b][c >> 1], -m[n][c & 1]);
        if (!whole) {
#pragma unroll
            for (int b = 0; b < 2; ++b) {
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int c = 0; c < 4; ++c) y[b][n][c] = seen(b, n, c) ? y[b][n][c] : -INFINITY;
#pragma unroll
                for (int i = 0; i < 2; ++i) {  // what no row sees does not count
                    const int j = first + 16 * b + g + 8 * i;
                    if (!(from[b] >= 0 && j <= pos_hi && (window == 0 || j > pos_lo - window || j < sinks))) f[b][i] = 0.f;
                }
            }
        }
        float most = -INFINITY;
        bool high = false;
#pragma unroll
        for (int b = 0; b < 2; ++b) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                w[b][i] = f[b][i] * v_unit;
                high |= !(w[b][i] <= 64.f);
            }
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    y[b][n][c] = exp2_approx(y[b][n][c]);
                    most = fmaxf(most, y[b][n][c]);
                }
        }
        if (__any_sync(0xffffffffu, high || most > 512.f)) {  // rarely: move the references up
            bool number[2][2];
            float top = 0.f, ratio = 1.f;
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    number[b][i] = f[b][i] <= 3.4e38f;
                    f[b][i] = number[b][i] ? f[b][i] : 0.f;
                    top = fmaxf(top, f[b][i]);
                }
#pragma unroll
            for (int d = 4; d < 32; d <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
            if (top * v_unit > 64.f) {
                // two octaves of room, so that scales of one size do not come back here; within fp32's exponents
                const float unit = scalbnf(1.f, min(max(5 - (ilogbf(top) + 2), -120), 120));
                ratio = v_unit == INFINITY ? 0.f : unit / v_unit;
                v_unit = unit;
            }
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int i = 0; i < 2; ++i) w[b][i] = f[b][i] > 0.f ? f[b][i] * v_unit : 0.f;
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    float z[2][2], mx = -INFINITY;
#pragma unroll
                    for (int b = 0; b < 2; ++b)
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            z[b][k] = whole || seen(b, n, i + 2 * k) ? s[b][n][i + 2 * k] * ks[b][k] : -INFINITY;
                            if (!number[b][k] && z[b][k] != -INFINITY) z[b][k] = NAN;  // a value that is none, for the rows that see it
                            mx = fmaxf(mx, z[b][k]);
                        }
#pragma unroll
                    for (int d = 4; d < 32; d <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, d));
                    const float m_new = fmaxf(m[n][i], mx), corr = exp2_approx(m[n][i] - m_new);
                    m[n][i] = m_new;
                    l[n][i] *= corr;
#pragma unroll
                    for (int k = 0; k < PD / 16; ++k) o[n][k][i] *= corr * ratio, o[n][k][i + 2] *= corr * ratio;
#pragma unroll
                    for (int b = 0; b < 2; ++b)
#pragma unroll
                        for (int k = 0; k < 2; ++k) y[b][n][i + 2 * k] = exp2_approx(z[b][k] - m_new);
                }
        }
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            const uint8_t* block = ring + (2 * stage + b) * B::BYTES;
            uint32_t pb[NT][2];
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int i = 0; i < 2; ++i) {  // positions g, g + 8
                    l[n][0] += y[b][n][2 * i];
                    l[n][1] += y[b][n][2 * i + 1];
                    const __half2 h = __floats2half2_rn(y[b][n][2 * i] * w[b][i], y[b][n][2 * i + 1] * w[b][i]);
                    pb[n][i] = transpose8(*reinterpret_cast<const uint32_t*>(&h));
                }
            uint32_t v0[4][Share<BITS, PD>::V], va[NK], vb[NK];  // positions (2t, 2t+1) and (2t+8, 2t+9)
#pragma unroll
            for (int i = 0; i < 4; ++i) load_words(block + v_off + ((i & 1) + 8 * (i >> 1)) * pitch, v0[i]);
            convert_v<BITS, PD>(v0[0], v0[1], halves, va);
            convert_v<BITS, PD>(v0[2], v0[3], halves, vb);
            if (BITS == 3 && b == 0 && first == 0 && from[0] >= 0) {
                const uint8_t* bos = a.pool + a48p::chunk_at(a.l, from[b], kvh) + a.l.bos + a.l.padded / 2;
                if (t == 0 && v_there) {
#pragma unroll
                    for (int i = 0; i < NK; ++i) {
                        const int e = NK * g + i;
                        const __half h = __float2half((float)((bos[e / 2] >> (4 * (e & 1))) & 15) - 8.f);
                        va[i] = (va[i] & 0xffff0000u) | __half_as_ushort(h);
                    }
                }
            }
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int k = 0; k < PD / 16; ++k) mma_f16(o[n][k], va[2 * k], va[2 * k + 1], vb[2 * k], vb[2 * k + 1], pb[n][0], pb[n][1]);
        }
    };
#pragma unroll 1
    for (int k = 0; k < pairs; ++k) {
        asm volatile("cp.async.wait_group %0;" ::"n"(STAGES - 1) : "memory");
        __syncwarp();
        take(k & 1, first_of(k), page[0]);
        __syncwarp();  // every lane has read the stage
#pragma unroll
        for (int b = 0; b < 2; ++b) page[0][b] = page[1][b], page[1][b] = page[2][b], page[2][b] = page_at(k + STAGES + 1, b);
        load(k + STAGES, k & 1, page[1]);
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    __syncthreads();  // the ring's memory is the sums' now

    // ---- the warps' sums meet in shared memory
    const float unit = v_unit == INFINITY ? 0.f : 1.f / v_unit;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
#pragma unroll
            for (int d = 4; d < 32; d <<= 1) l[n][i] += __shfl_xor_sync(0xffffffffu, l[n][i], d);
            const int r = 8 * n + 2 * t + i;
            if (g == 0) sm.m[warp][r] = m[n][i], sm.l[warp][r] = l[n][i];
#pragma unroll
            for (int k = 0; k < PD / 16; ++k)
                *reinterpret_cast<float2*>(&sm.o[warp][r][NK * g + 2 * k]) = make_float2(o[n][k][i] * unit, o[n][k][i + 2] * unit);
        }
    }
    __syncthreads();
    auto finish = [&](int r, int c, float top, float sum, const float (&acc)[4]) {
        const int token = sm.token[r], head = sm.head[r];
        if (a.clusters > 1) {
            const a48p::Parts& to = a.row_parts;
            const size_t at = (size_t)(cluster * to.rows + ((long long)seq * a.l.kv_heads + kvh) * to.per_head + r0 + r);
            reinterpret_cast<float4*>(to.o + at * 128)[c / 4] = make_float4(acc[0], acc[1], acc[2], acc[3]);
            if (c == 0) to.ml[at] = make_float2(top, sum);
        } else {
            const float inv = sum != 0.f ? 1.f / sum : 0.f;
            const __nv_bfloat162 lo = __floats2bfloat162_rn(acc[0] * inv, acc[1] * inv), hi = __floats2bfloat162_rn(acc[2] * inv, acc[3] * inv);
            *reinterpret_cast<uint2*>(a.out + token * a.out_stride + (size_t)head * a.l.hd + c) =
                make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
        }
    };
    if (a.ranks > 1) cluster_wait();  // every CTA of the cluster runs: its shared memory may be written
    for (int i = threadIdx.x; i < rows * (PD / 4); i += 32 * ROW_WARPS) {
        const int r = i / (PD / 4), c = 4 * (i % (PD / 4));
        if (c >= a.l.hd) continue;
        float top = sm.m[0][r], sum = 0.f, acc[4] = {};
#pragma unroll
        for (int w = 1; w < ROW_WARPS; ++w) top = fmaxf(top, sm.m[w][r]);
#pragma unroll
        for (int w = 0; w < ROW_WARPS; ++w) {
            const float corr = exp2_approx(sm.m[w][r] - top);
            const float4 z = *reinterpret_cast<const float4*>(&sm.o[w][r][c]);
            sum += corr * sm.l[w][r];
            acc[0] += corr * z.x, acc[1] += corr * z.y, acc[2] += corr * z.z, acc[3] += corr * z.w;
        }
        if (a.ranks == 1) {
            finish(r, c, top, sum, acc);
        } else {  // to the CTA that finishes this piece
            const int to = i & (a.ranks - 1), at = (i & -a.ranks) + rank;
            st_rank(of_rank(&sm.piece[at], to), make_float4(acc[0], acc[1], acc[2], acc[3]));
            st_rank(of_rank(&sm.piece_ml[at], to), make_float2(top, sum));
        }
    }
    if (a.ranks == 1) return;
    // ---- and the CTAs' sums: each has sent every other its part of a share of the pieces (piece i goes to rank i % ranks)
    cluster_arrive();
    cluster_wait();
    for (int i = threadIdx.x * a.ranks + rank; i < rows * (PD / 4); i += 32 * ROW_WARPS * a.ranks) {
        const int r = i / (PD / 4), c = 4 * (i % (PD / 4)), at = i - rank;
        if (c >= a.l.hd) continue;
        float top = -1e30f, sum = 0.f, acc[4] = {};
        for (int k = 0; k < a.ranks; ++k) top = fmaxf(top, sm.piece_ml[at + k].x);
        for (int k = 0; k < a.ranks; ++k) {
            const float2 ml = sm.piece_ml[at + k];
            const float4 z = sm.piece[at + k];
            const float corr = exp2_approx(ml.x - top);
            sum += corr * ml.y;
            acc[0] += corr * z.x, acc[1] += corr * z.y, acc[2] += corr * z.z, acc[3] += corr * z.w;
        }
        finish(r, c, top, sum, acc);
    }
}

// Registers are held to what lets four CTAs of eight rows (two of sixteen) share an SM: loads in flight are what hides
// memory.
template <int BITS, int PD, int NT>
__global__ void __launch_bounds__(32 * ROW_WARPS, NT == 2 ? 2 : BITS == 4 || PD == 64 ? 4 : 3) attn_paged_rows_kernel(const __grid_constant__ AttnArgs a) {
    extern __shared__ __align__(16) uint8_t smem[];
    RowsShared<BITS, PD, NT>& sm = *reinterpret_cast<RowsShared<BITS, PD, NT>*>(smem);
    a48_pdl_prologue();
    attend_rows<BITS, PD, NT>(a, sm);
}

// The parts of a row, in order.  One warp per place of a row, the rows kernel's ahead of the tile kernel's, four head dims per
// lane.
__global__ void __launch_bounds__(256) attn_paged_join_kernel(const __grid_constant__ AttnArgs a) {
    a48_pdl_prologue();
    const int lane = threadIdx.x & 31;
    const long long ahead = a.row_parts.parts > 1 ? a.row_parts.rows : 0, place = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
    const bool many = place >= ahead;  // a row of the tile kernel
    const a48p::Parts& from = many ? a.tile_parts : a.row_parts;
    const long long id = many ? place - ahead : place;
    if (from.parts == 1 || id >= from.rows) return;
    int seq, token, head;
    long long row;
    if (from.per_head > 0) {
        const long long of_head = id / from.per_head;
        row = id - of_head * from.per_head;
        seq = (int)(of_head / a.l.kv_heads);
        head = (int)(of_head % a.l.kv_heads) * a.group + (int)(row % a.group);
        token = __ldg(a.b.q_start + seq) + (int)(row / a.group);
    } else {
        token = (int)(id / a.heads), head = (int)(id % a.heads);
        seq = a48p::sequence_of(a.b, token, lane);
        if (seq < 0) return;
        row = (long long)(token - __ldg(a.b.q_start + seq)) * a.group + head % a.group;
    }
    const int start = __ldg(a.b.q_start + seq), end = __ldg(a.b.q_start + seq + 1);
    const long long all_rows = (long long)(end - start) * a.group;
    if (row >= all_rows || all_rows > a.few_rows != many || start < 0 || end > a.b.n_tokens) return;
    const int splits = from.parts;
    float top = -1e30f;
    for (int i = 0; i < splits; ++i) {
        const float2 ml = __ldg(from.ml + i * from.rows + id);
        if (ml.y > 0.f) top = fmaxf(top, ml.x);
    }
    float sum = 0.f, acc[4] = {};
    for (int i = 0; i < splits; ++i) {
        const float2 ml = __ldg(from.ml + i * from.rows + id);
        if (!(ml.y != 0.f)) continue;  // (a sum that is no number is passed on)
        const float corr = exp2_approx(ml.x - top);
        sum += corr * ml.y;
        if (4 * lane < a.l.hd) {
            const float4 x = __ldg(reinterpret_cast<const float4*>(from.o + (i * from.rows + id) * 128) + lane);
            acc[0] += corr * x.x, acc[1] += corr * x.y, acc[2] += corr * x.z, acc[3] += corr * x.w;
        }
    }
    const float inv = sum > 0.f ? 1.f / sum : 0.f;
    if (4 * lane < a.l.hd) {
        const __nv_bfloat162 lo = __floats2bfloat162_rn(acc[0] * inv, acc[1] * inv), hi = __floats2bfloat162_rn(acc[2] * inv, acc[3] * inv);
        *reinterpret_cast<uint2*>(a.out + token * a.out_stride + (size_t)head * a.l.hd + 4 * lane) =
            make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
    }
}

// ---------------------------------------------------------------------------------------------------- host
constexpr int FEW_ROWS = 64, SMS = 148;
constexpr int kFar = 1 << 30;  // what a window is cut to: position differences stay in 32 bits

// How a call is cut up; from its bounds alone, so that the workspace can be asked for ahead.
struct Plan {
    bool many;  // some sequence may be the tile kernel's
    int nt, few_rows, tiles, ranks, clusters, tc_tiles, tc_splits;
    long long row_rows, row_per_head, tile_rows, tile_per_head;  // places of parts (a48p::Parts)
    size_t row_o, tile_ml, tile_o, bytes;  // workspace: offsets of the parts (the rows kernel's exponents come first), and its size
};

long long up(long long x, long long y) { return (x + y - 1) / y; }
int within(long long x, long long lo, long long hi) { return (int)(x < lo ? lo : x > hi ? hi : x); }

Plan plan_of(const bitnet_a48_paged_cache& c, const bitnet_a48_paged_batch& b, int heads, int window, int sinks) {
    Plan p;
    const long long group = heads / c.n_kv_heads, rows = (long long)b.max_q * group;
    p.many = rows > FEW_ROWS;
    // Rows kernel.  Where some sequences are the tile kernel's, the others are taken to be decoding: one tile of rows.
    const int few = p.many ? (group <= 8 ? 8 : 16) : (int)rows;
    p.nt = few > 8 ? 2 : 1;
    p.tiles = (int)up(few, 8 * p.nt);
    p.few_rows = p.many ? few : INT_MAX;
    long long reach = (long long)b.max_pages * c.page_size;
    if (b.max_kv < reach) reach = b.max_kv;
    // positions a tile of `span` tokens may see
    auto seen = [&](long long span) {
        const long long most = (long long)window + sinks + span;
        return window > 0 && most < reach ? most : reach;
    };
    // Parts of the positions, a power of two, each with a pair of blocks for every warp at least.  As many as fit the SMs at
    // once (a second wave costs its start again: 8 sequences of 4 tokens, 27.8 us with 512 CTAs on 296 places, 18 with 256);
    // two where that would be one, which evens out sequences of unlike lengths (64 of 130 .. 8192 positions: 121 us with
    // one part, 94 with two, 96 with four).  Up to eight join inside a cluster; more only where those leave SMs idle.
    const long long base = (long long)b.n_seqs * c.n_kv_heads * p.tiles, most = up(seen(64), 32 * ROW_WARPS);
    const bool narrow = (c.head_dim + 31) / 32 * 32 <= 64 && c.bits != 3;
    const long long places = (long long)SMS * (p.nt == 2 ? 2 : c.bits == 4 || narrow ? 4 : 3);
    p.ranks = 1;
    while (p.ranks < MAX_RANKS && 2 * p.ranks * base <= places && 2 * p.ranks <= most) p.ranks *= 2;
    if (p.ranks == 1 && base <= places && most >= 2) p.ranks = 2;
    p.clusters = p.ranks < MAX_RANKS ? 1 : within(2 * SMS / (base * MAX_RANKS), 1, most / MAX_RANKS < 16 ? most / MAX_RANKS : 16);
    // Tile kernel, one CTA per SM: split while the tiles do not fill the SMs, into parts of two tiles or more.
    p.tc_tiles = 0, p.tc_splits = 1;
    if (p.many) {
        const long long direct = up(rows, a48p::TILE_ROWS), found = (long long)b.n_tokens * group / a48p::TILE_ROWS;
        if (direct * b.n_seqs <= found + b.n_seqs) p.tc_tiles = (int)direct;
        const long long real = (p.tc_tiles ? direct * b.n_seqs : found + 1) * c.n_kv_heads;
        const long long steps = up(seen(a48p::TILE_ROWS / group + 2 * a48p::TILE_POSITIONS), a48p::TILE_POSITIONS);
        p.tc_splits = within(SMS / real, 1, up(steps, 2) < 64 ? up(steps, 2) : 64);
    }
    // Parts have places by the rows that can have them, so that a long prompt beside them, whose rows are not split, adds none:
    // the rows kernel's are 37 x 16 at most (base * clusters is at most 2 SMS / MAX_RANKS where it leaves parts), the tile kernel's
    // 148 x 256 (its tiles times parts fill the SMs once; by token where tiles are found by search, since n_tokens is what bounds
    // those).
    p.row_per_head = p.tiles * 8LL * p.nt, p.row_rows = (long long)b.n_seqs * c.n_kv_heads * p.row_per_head;
    p.tile_per_head = (long long)p.tc_tiles * a48p::TILE_ROWS;
    p.tile_rows = p.tc_tiles ? (long long)b.n_seqs * c.n_kv_heads * p.tile_per_head : (long long)b.n_tokens * heads;
    const size_t row_places = p.clusters > 1 ? (size_t)p.row_rows * p.clusters : 0, tile_places = p.tc_splits > 1 ? (size_t)p.tile_rows * p.tc_splits : 0;
    auto aligned = [](size_t n) { return (n + 255) / 256 * 256; };
    p.row_o = aligned(row_places * sizeof(float2));
    p.tile_ml = p.row_o + row_places * 128 * sizeof(float);
    p.tile_o = p.tile_ml + aligned(tile_places * sizeof(float2));
    p.bytes = p.tile_o + tile_places * 128 * sizeof(float);
    return p;
}

template <int BITS, int PD, int NT>
cudaError_t launch_rows(const AttnArgs& a, cudaStream_t st) {
    constexpr size_t SMEM = sizeof(RowsShared<BITS, PD, NT>);
    static std::atomic<bool> allowed[64];
    const cudaError_t e = a48_allow_smem(attn_paged_rows_kernel<BITS, PD, NT>, SMEM, allowed);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(a.l.kv_heads * a.b.n_seqs * a.tiles, a.ranks * a.clusters);
    cfg.blockDim = dim3(32 * ROW_WARPS);
    cfg.dynamicSmemBytes = SMEM;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim = {1, (unsigned)a.ranks, 1};
    cfg.attrs = attr;
    cfg.numAttrs = a.ranks > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, attn_paged_rows_kernel<BITS, PD, NT>, a);
}
template <int BITS, int PD>
cudaError_t launch_rows(const AttnArgs& a, int nt, cudaStream_t st) {
    return nt == 1 ? launch_rows<BITS, PD, 1>(a, st) : launch_rows<BITS, PD, 2>(a, st);
}

// (the caches and batches that reach this have been checked)
bitnet_a48_status check_attention(const bitnet_a48_paged_cache* cache, const bitnet_a48_paged_batch* batch, int n_heads, int window, int sinks) {
    if (n_heads <= 0 || n_heads % cache->n_kv_heads != 0) return BITNET_A48_ERR_SHAPE;
    if (n_heads > 65535 || (long long)batch->n_tokens * n_heads > INT_MAX ||
        (long long)cache->n_kv_heads * batch->n_seqs * (FEW_ROWS / 8) > INT_MAX) return BITNET_A48_ERR_LIMIT;
    return window < 0 || sinks < 0 ? BITNET_A48_ERR_INVALID_ARG : BITNET_A48_OK;
}

}  // namespace

extern "C" {

size_t bitnet_a48_attention_paged_workspace_bytes(const bitnet_a48_paged_cache* cache, const bitnet_a48_paged_batch* batch, int n_heads,
                                                  int window, int sinks) {
    if (!batch || !bitnet_a48_paged_cache_bytes(cache) || batch->n_seqs <= 0 || batch->n_tokens <= 0 || batch->max_q <= 0 ||
        batch->max_kv <= 0 || batch->max_pages <= 0 || check_attention(cache, batch, n_heads, window, sinks) != BITNET_A48_OK)
        return 0;
    return plan_of(*cache, *batch, n_heads, window, sinks).bytes;
}

bitnet_a48_status bitnet_a48_attention_paged(const bitnet_a48_paged_cache* cache, const void* pool_dev,
                                             const bitnet_a48_paged_batch* batch, int n_heads, const uint16_t* q_dev,
                                             long long q_stride, float scale, int window, int sinks, uint16_t* out_dev,
                                             long long out_stride, void* workspace_dev, size_t workspace_bytes, void* stream) {
    bitnet_a48_status st = a48p::check(cache, pool_dev, batch);
    if (st != BITNET_A48_OK) return st;
    if ((st = check_attention(cache, batch, n_heads, window, sinks)) != BITNET_A48_OK) return st;
    if (!(scale >= 0.f) || scale > 3e38f) return BITNET_A48_ERR_INVALID_ARG;
    const long long width = (long long)n_heads * cache->head_dim;
    if ((st = a48p::check_rows(q_dev, q_stride, width, 2)) != BITNET_A48_OK) return st;
    if ((st = a48p::check_rows(out_dev, out_stride, width, 2)) != BITNET_A48_OK) return st;
    const Plan p = plan_of(*cache, *batch, n_heads, window, sinks);
    if (!a48_aligned16(workspace_dev)) return BITNET_A48_ERR_ALIGNMENT;
    if (p.bytes && (!workspace_dev || workspace_bytes < p.bytes)) return BITNET_A48_ERR_NOMEM;
    if (!a48_have_device()) return BITNET_A48_ERR_CUDA;
    const cudaStream_t cu = (cudaStream_t)stream;
    AttnArgs a;
    a.l = a48p::layout_of(*cache);
    a.b = a48p::batch_of(*batch);
    a.pool = static_cast<const uint8_t*>(pool_dev);
    a.q = reinterpret_cast<const __nv_bfloat16*>(q_dev);
    a.out = reinterpret_cast<__nv_bfloat16*>(out_dev);
    a.q_stride = q_stride, a.out_stride = out_stride;
    a.heads = n_heads, a.group = n_heads / cache->n_kv_heads;
    a.window = window < kFar ? window : kFar, a.sinks = window > 0 ? sinks : 0;
    a.scale = scale > 0.f ? scale : 1.f / sqrtf((float)cache->head_dim);
    a.few_rows = p.few_rows;
    a.tiles = p.tiles, a.tile_rows = 8 * p.nt, a.ranks = p.ranks, a.clusters = p.clusters;
    a.tc_tiles = p.tc_tiles, a.tc_splits = p.tc_splits;
    char* const ws = static_cast<char*>(workspace_dev);
    a.row_parts = {reinterpret_cast<float*>(ws + p.row_o), reinterpret_cast<float2*>(ws), p.row_rows, p.row_per_head, p.clusters};
    a.tile_parts = {reinterpret_cast<float*>(ws + p.tile_o), reinterpret_cast<float2*>(ws + p.tile_ml), p.tile_rows, p.tile_per_head, p.tc_splits};
    if (p.many && (st = a48p::launch_tiles(a, cu)) != BITNET_A48_OK) return st;
    const bool wide = a.l.padded > 64;
    cudaError_t e;
    if (a.l.bits == 3) e = launch_rows<3, 128>(a, p.nt, cu);
    else if (a.l.bits == 4) e = wide ? launch_rows<4, 128>(a, p.nt, cu) : launch_rows<4, 64>(a, p.nt, cu);
    else e = wide ? launch_rows<8, 128>(a, p.nt, cu) : launch_rows<8, 64>(a, p.nt, cu);
    A48_CUDA_TRY(e);
    if (p.bytes) {
        const long long places = (p.clusters > 1 ? p.row_rows : 0) + (p.tc_splits > 1 ? p.tile_rows : 0);
        A48_CUDA_TRY(a48_launch_pdl(attn_paged_join_kernel, dim3((unsigned)((places + 7) / 8)), dim3(256), 0, cu, a));
    }
    return BITNET_A48_OK;
}

}  // extern "C"
