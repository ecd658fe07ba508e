// Attention over the paged low-bit cache for sequences with many rows (chunks of prompts), on the fifth-generation tensor
// cores.  A CTA takes 256 rows (token, query head of the group) of one key/value head as two tiles of 128, and walks the
// positions they see 128 at a time.
//
// Both contractions run on the codes (attn_paged.cu has the formulas): S = Q C^T with Q brought to fp16 by a power of two
// per row, O += P D with P = 2^(score - reference) times the value scale in fp16, fp32 accumulators in tensor memory.  The
// codes of 128 positions are converted to fp16 once for the 256 rows, into shared memory in the 128-byte swizzle, one row
// per position for keys and values alike: the keys are then a K-major operand and the values an MN-major one, and nothing is
// transposed.  The entries of a row keep the order in which the conversion gives them; the query rows are stored in the
// same order, and the output columns are put right when they are stored.
//
//   warps 0-3, 4-7   one thread per row of tile 0, 1: scores from tensor memory, times key scale and row factor, 2^x, the
//                    weights back over the scores.  One pass: the reference moves only when a score exceeds it by 2^8
//                    (or a value scale its unit by 2^6), then the tile is taken again and O rescaled; in the steady state
//                    no pass for the maximum and no rescaling.  Products and sums are two at a time (f32x2).  One thread
//                    of each tile then issues the MMAs O(t) and, behind it on the pipe, S(t+1): while one tile's weights
//                    are taken, the pipe has the other's two products.  (A warp of its own for the MMAs would be the
//                    thirteenth, and leave every thread 128 registers instead of 168.)
//   warps 8-11       one thread per position: codes and scales from memory (the next position's under way while these are
//                    converted), fp16 entries into a ring of four buffers K(t) V(t) K(t+1) V(t+1).
// Tensor memory: two score tiles (128 columns, P over the first 64) and two output tiles (up to 128 columns).
// Every wait is bounded; one that gives up records itself (bitnet_a48_kernel_status), and every later wait of the CTA then
// falls through, so that the kernel ends by itself.
#include <climits>
#include <type_traits>

#include "attn_paged.cuh"

namespace {

using a48p::AttnArgs;
using a48p::exp2_approx;
using a48p::Span;

constexpr int TQ = 128, TK = a48p::TILE_POSITIONS, RING = 4, SCALES = 4;
constexpr int CONVERT_WARP = 8, THREADS = 32 * 12;
constexpr int TMEM_COLS = 512, COL_S = 0, COL_O = 256;
constexpr unsigned long long kWaitClocks = 4000000000ull;  // ~2 s at 2 GHz

__device__ unsigned int g_status[4];

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void mbar_init(uint32_t bar, uint32_t count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void mbar_arrive(uint32_t bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ bool mbar_try(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(bar), "r"(parity)
        : "memory");
    return ok != 0;
}
__device__ __noinline__ void mbar_wait_slow(uint32_t bar, uint32_t parity, volatile uint32_t* abort_flag, uint32_t id, uint32_t iter) {
    const unsigned long long t0 = clock64();
    uint32_t spins = 0;
    while (!mbar_try(bar, parity)) {
        if ((++spins & 255u) == 0) {
            if (*abort_flag) return;
            if (clock64() - t0 > kWaitClocks) {
                *abort_flag = 1;
                if (atomicCAS(&g_status[0], 0u, (unsigned)BITNET_A48_ERR_TIMEOUT) == 0u) {
                    g_status[1] = id;
                    g_status[2] = blockIdx.x + gridDim.x * blockIdx.y;
                    g_status[3] = iter;
                }
                return;
            }
        }
    }
}
__device__ __forceinline__ void mbar_wait(uint32_t bar, uint32_t parity, volatile uint32_t* abort_flag, uint32_t id, uint32_t iter) {
    if (mbar_try(bar, parity)) return;
    if (*abort_flag) return;
    mbar_wait_slow(bar, parity, abort_flag, id, iter);
}
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_commit(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
// D[tmem] (+)= A[smem] * B[smem], fp16 operands, fp32 accumulators
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a_desc, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate)
        : "memory");
}
// D[tmem] (+)= A[tmem] * B[smem]
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
        ::"r"(d), "r"(a), "l"(b_desc), "r"(idesc), "r"(accumulate)
        : "memory");
}
// Descriptor of an operand whose rows of 128 bytes (64 fp16) lie in the 128-byte swizzle, groups of eight rows 1024 bytes
// apart.  K-major (rows along M or N): 16 elements further along K is 32 bytes.  MN-major (rows along K): 16 rows further
// along K is 2048 bytes, and the next 64 columns are one panel of TK rows further on.
__device__ __forceinline__ uint64_t smem_desc(uint32_t addr) {
    return (uint64_t)((addr & 0x3ffffu) >> 4) | (uint64_t)(TK * 128 >> 4) << 16 | (uint64_t)(1024u >> 4) << 32 | (uint64_t)1 << 46 |
           (uint64_t)2 << 61;
}
// kind::f16 instruction descriptor: fp16 x fp16 -> f32, M x N tile, A K-major, B K-major or MN-major
__host__ __device__ constexpr uint32_t idesc_f16(int m, int n, bool b_mn_major) {
    return (1u << 4) | ((b_mn_major ? 1u : 0u) << 16) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}
__device__ __forceinline__ void tmem_ld32(uint32_t taddr, uint32_t (&r)[32]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
          "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
          "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(taddr)
        : "memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t* r) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};"
        ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]),
          "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]),
          "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]),
          "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
        : "memory");
}
__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// two floats as one operand
typedef unsigned long long f2;
__device__ __forceinline__ f2 pack2(float x, float y) {
    f2 r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(x), "f"(y));
    return r;
}
__device__ __forceinline__ void unpack2(f2 v, float& x, float& y) { asm("mov.b64 {%0, %1}, %2;" : "=f"(x), "=f"(y) : "l"(v)); }
__device__ __forceinline__ f2 mul2(f2 a, f2 b) {
    f2 r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ f2 add2(f2 a, f2 b) {
    f2 r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ f2 fma2(f2 a, f2 b, f2 c) {
    f2 r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}

__device__ __forceinline__ void tile_sync(int half) { asm volatile("bar.sync %0, 128;" ::"r"(2 + half) : "memory"); }
__device__ __forceinline__ void convert_sync() { asm volatile("bar.sync 1, 128;" ::: "memory"); }
__device__ __forceinline__ bool convert_any(bool x) {
    uint32_t r;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %1, 0;\n\t"
        "bar.red.or.pred q, 1, 128, p;\n\t"
        "selp.u32 %0, 1, 0, q;\n\t}"
        : "=r"(r)
        : "r"((uint32_t)x)
        : "memory");
    return r != 0;
}

// Scales of the 128 positions of a tile.
struct TileScales {
    float key[TK], value[TK];  // value scales times `unit`
    uint32_t dead[TK / 32];    // positions without a page
    float unit;                // 2^6 over a power of two not below the largest value scale so far; 0 while all are zero
    float pad[3];
};

// Where entry n of a row sits in a row of converted entries, per 32 entries: 3 bits: pairs (n, n + 16); 4 bits: pairs
// (n, n + 4) of eight; 8 bits: pairs (n, n + 2) of four.
template <int BITS>
__host__ __device__ constexpr int entry_of(int i) {  // the entry at place i
    return BITS == 3 ? (i & ~31) + (i & 31) / 2 + 16 * (i & 1)
                     : BITS == 4 ? (i & ~7) + (i & 7) / 2 + 4 * (i & 1) : (i & ~3) + (i & 3) / 2 + 2 * (i & 1);
}

template <int PD>
struct Cfg {
    static constexpr int BUF = TK * PD * 2;  // one tile of keys, values or query rows
    static constexpr int Q_AT = RING * BUF, CTRL_AT = Q_AT + 2 * BUF, SCALES_AT = CTRL_AT + 256;
    static constexpr int SMEM = SCALES_AT + SCALES * (int)sizeof(TileScales) + 1024 /*alignment slack*/;
    static_assert(SMEM <= 227 * 1024, "shared memory budget");
};

// what a wait that gave up was for
enum { WAIT_FULL = 41, WAIT_EMPTY = 42, WAIT_S = 43, WAIT_O = 45 };

template <int BITS, int PD>
__global__ void __launch_bounds__(THREADS, 1) attn_paged_tc_kernel(const __grid_constant__ AttnArgs a) {
    using C = Cfg<PD>;
    constexpr int PANELS = PD / 64, PANEL = TK * 128;
    constexpr int WORDS = PD * BITS / 32;  // of a code row
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    uint8_t* ctrl = smem + C::CTRL_AT;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(ctrl + 192);
    volatile uint32_t* abort_flag = reinterpret_cast<volatile uint32_t*>(ctrl + 196);
    float* top_part = reinterpret_cast<float*>(ctrl + 208);  // largest value scale per converting warp
    TileScales* scales = reinterpret_cast<TileScales*>(smem + C::SCALES_AT);
    const uint32_t ring = smem_u32(smem), sq = ring + C::Q_AT;
    // barriers: full[4] | empty[4] | s[2] | o[2]
    const uint32_t bar_full = smem_u32(ctrl), bar_empty = bar_full + 32, bar_s = bar_full + 64, bar_o = bar_full + 80;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    a48_pdl_prologue();

    // ---- which rows: the tiles with the most positions first
    const int kvh = blockIdx.x % a.l.kv_heads, at = gridDim.x / a.l.kv_heads - 1 - blockIdx.x / a.l.kv_heads;
    int seq, tile;
    if (a.tc_tiles > 0) {
        seq = at % a.b.n_seqs, tile = at / a.b.n_seqs;
    } else {  // sequence b has the tiles from floor(q_start[b] group / 256) + b on, more than it needs
        auto first_tile = [&](int b) { return (long long)__ldg(a.b.q_start + b) * a.group / a48p::TILE_ROWS + b; };
        seq = a48p::last_at_most(a.b.n_seqs, at, lane, first_tile);
        if (seq < 0) return;
        tile = at - (int)first_tile(seq);
    }
    const int start = __ldg(a.b.q_start + seq), q_len = __ldg(a.b.q_start + seq + 1) - start;
    const long long all_rows = (long long)q_len * a.group, r0 = (long long)tile * a48p::TILE_ROWS;
    if (all_rows <= a.few_rows || r0 >= all_rows || start < 0 || q_len > a.b.n_tokens - start) return;
    const int rows = (int)min((long long)a48p::TILE_ROWS, all_rows - r0);
    const int halves = rows > TQ ? 2 : 1;
    const int pos0 = __ldg(a.b.kv_len + seq) - q_len;
    const int pos_lo = pos0 + (int)(r0 / a.group), pos_hi = pos0 + (int)((r0 + rows - 1) / a.group);
    const Span span = a48p::span_of<7>(a, pos_lo, pos_hi);
    const int v0 = blockIdx.y * a.tc_per_split;
    const int n_tiles = max(0, (blockIdx.y + 1 == gridDim.y ? span.count : min(span.count, v0 + a.tc_per_split)) - v0);

    if (threadIdx.x == 0) {
        for (int i = 0; i < RING; ++i) {
            mbar_init(bar_full + 8 * i, TQ);
            mbar_init(bar_empty + 8 * i, halves);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(bar_s + 8 * i, 1);
            mbar_init(bar_o + 8 * i, 1);
        }
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == CONVERT_WARP) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(TMEM_COLS)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;

    if (warp >= CONVERT_WARP) {
        // ------------------------------------------------------------------------------------------ codes to fp16
        const int r = threadIdx.x - 32 * CONVERT_WARP;
        uint32_t kw[WORDS], vw[WORDS];
        float sk = 0.f, sv = 0.f;
        const uint8_t* chunk = nullptr;
        int pos = 0, slot = 0;
        float unit = 0.f;
        // the position of this thread in tile t, its page and scales
        auto locate = [&](int t) {
            pos = span.block(v0 + t) * TK + r;
            slot = pos & (a.l.page - 1);
            const int page = pos <= pos_hi ? a48p::page_of(a.l, a.b, seq, pos) : -1;
            chunk = page >= 0 ? a.pool + a48p::chunk_at(a.l, page, kvh) : nullptr;
        };
        auto load_row = [&](uint32_t (&w)[WORDS], int part) {
            const uint32_t* src = chunk ? reinterpret_cast<const uint32_t*>(chunk + part * a.l.v_codes + slot * a.l.row) : nullptr;
            constexpr int STEP = BITS;  // words of 32 entries
#pragma unroll
            for (int c = 0; c < WORDS; c += STEP) {
                const bool there = src && 4 * c < a.l.row;
                if constexpr (BITS == 3) {
#pragma unroll
                    for (int i = 0; i < 3; ++i) w[c + i] = there ? __ldg(src + c + i) : 0u;
                } else {
#pragma unroll
                    for (int i = 0; i < STEP; i += 4) {
                        const uint4 x = there ? __ldg(reinterpret_cast<const uint4*>(src + c + i)) : make_uint4(0, 0, 0, 0);
                        w[c + i] = x.x, w[c + i + 1] = x.y, w[c + i + 2] = x.z, w[c + i + 3] = x.w;
                    }
                }
            }
        };
        auto load_scales = [&]() {
            sk = chunk ? __ldg(reinterpret_cast<const float*>(chunk + a.l.k_scales) + slot) : 0.f;
            sv = chunk ? __ldg(reinterpret_cast<const float*>(chunk + a.l.v_scales) + slot) : 0.f;
        };
        // a row of fp16 entries to row r of a buffer, 32 entries (four 16-byte pieces) at a time
        auto store_row = [&](uint8_t* buf, const uint32_t (&w)[WORDS], const uint8_t* bos) {
#pragma unroll
            for (int c = 0; c < PD / 32; ++c) {
                uint32_t h[16];
                if constexpr (BITS == 3) {
                    a48p::triples(w[3 * c], w[3 * c + 1], w[3 * c + 2], h);
                    if (bos) {  // position 0: 4-bit codes of its own
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const int e = 32 * c + i;
                            float x = 0.f, y = 0.f;
                            if (32 * c < a.l.padded) {
                                x = (float)((bos[e / 2] >> (4 * (e & 1))) & 15) - 8.f;
                                y = (float)((bos[e / 2 + 8] >> (4 * (e & 1))) & 15) - 8.f;
                            }
                            const __half2 p = __floats2half2_rn(x, y);
                            h[i] = *reinterpret_cast<const uint32_t*>(&p);
                        }
                    }
                } else if constexpr (BITS == 4) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) a48p::nibbles(w[4 * c + i], h + 4 * i);
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) a48p::bytes(w[8 * c + i], h + 2 * i);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    *reinterpret_cast<uint4*>(buf + c / 2 * PANEL + r * 128 + (((c % 2 * 4 + i) ^ (r & 7)) << 4)) =
                        make_uint4(h[4 * i], h[4 * i + 1], h[4 * i + 2], h[4 * i + 3]);
            }
        };
        auto publish = [&](int n) {
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            mbar_arrive(bar_full + 8 * (n % RING));
        };
        if (n_tiles > 0) {
            locate(0);
            load_row(kw, 0);
            load_row(vw, 1);
            load_scales();
        }
        for (int t = 0; t < n_tiles; ++t) {
            const int kn = 2 * t, vn = 2 * t + 1;
            const bool first = BITS == 3 && pos == 0 && chunk;
            const uint8_t* bos = first ? chunk + a.l.bos : nullptr;
            const bool dead = !chunk && pos <= pos_hi;
            // ---- scales; one counts for the unit if it is finite and some row may see its position
            const bool may = a.window == 0 || pos > pos_lo - a.window || pos < a.sinks;
            const float f = may ? sv : 0.f;
            const bool finite = f <= 3.4e38f;
            if (convert_any(finite && (unit == 0.f ? f > 0.f : f * unit > 64.f))) {
                float top = finite ? f : 0.f;
#pragma unroll
                for (int d = 16; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
                if (lane == 0) top_part[warp - CONVERT_WARP] = top;
                convert_sync();
                top = fmaxf(fmaxf(top_part[0], top_part[1]), fmaxf(top_part[2], top_part[3]));
                // two octaves of room, so that scales of one size do not come back here; within fp32's exponents
                unit = scalbnf(1.f, min(max(5 - (ilogbf(top) + 2), -120), 120));
            }
            // ---- keys.  (The ring is what keeps the scales of four tiles apart: K(t) can be written once the scores of
            // t - 2 are done, and the weights of t - 3 were taken before the scores of t - 2 were issued.)
            if (kn >= RING) mbar_wait(bar_empty + 8 * (kn % RING), (kn / RING & 1) ^ 1, abort_flag, WAIT_EMPTY, kn);
            TileScales& ts = scales[t % SCALES];
            ts.key[r] = sk;
            ts.value[r] = f * unit;
            const uint32_t gone = __ballot_sync(0xffffffffu, dead);
            if (lane == 0) ts.dead[warp - CONVERT_WARP] = gone;
            if (r == 0) ts.unit = unit;
            store_row(smem + kn % RING * C::BUF, kw, bos);
            publish(kn);
            // ---- the next tile's keys under way, then the values of this one
            const uint8_t* v_bos = first ? bos + a.l.padded / 2 : nullptr;
            if (t + 1 < n_tiles) {
                locate(t + 1);
                load_row(kw, 0);
                load_scales();
            }
            if (vn >= RING) mbar_wait(bar_empty + 8 * (vn % RING), (vn / RING & 1) ^ 1, abort_flag, WAIT_EMPTY, vn);
            store_row(smem + vn % RING * C::BUF, vw, v_bos);
            publish(vn);
            if (t + 1 < n_tiles) load_row(vw, 1);
        }
    } else {
        // ------------------------------------------------------------------------------------------ rows
        const int half = warp >> 2, row = (warp & 3) * 32 + lane, r = half * TQ + row;
        const uint32_t lanes = tmem + ((uint32_t)((warp & 3) * 32) << 16);
        const uint32_t s_at = lanes + COL_S + TK * half, o_at = lanes + COL_O + 128 * half;
        const bool mine = r < rows;
        const long long in_seq = r0 + (mine ? r : rows - 1);
        const int token = start + (int)(in_seq / a.group), head = kvh * a.group + (int)(in_seq % a.group);
        const int lim = pos0 + (int)(in_seq / a.group);  // the last position the row sees
        float mul;
        // ---- the query row to fp16 by a power of two, in the order of the converted codes
        {
            uint2 x[PD / 4];
            const uint2* src = reinterpret_cast<const uint2*>(a.q + (size_t)token * a.q_stride + (size_t)head * a.l.hd);
            float mx = 0.f;
#pragma unroll
            for (int i = 0; i < PD / 4; ++i) {
                x[i] = mine && 4 * i < a.l.hd ? __ldg(src + i) : make_uint2(0, 0);
                mx = fmaxf(mx, fmaxf(fmaxf(fabsf(__uint_as_float(x[i].x << 16)), fabsf(__uint_as_float(x[i].x & 0xffff0000u))),
                                     fmaxf(fabsf(__uint_as_float(x[i].y << 16)), fabsf(__uint_as_float(x[i].y & 0xffff0000u)))));
            }
            const int e = mx > 0.f && mx <= 3.4e38f ? 14 - ilogbf(mx) : 0;  // the largest goes to [2^14, 2^15)
            mul = scalbnf(a.scale * 1.4426950408889634f, -e);
            const float up0 = scalbnf(1.f, e / 2), up1 = scalbnf(1.f, e - e / 2);  // (2^e may be past fp32)
            auto value = [&](int n) {
                const uint32_t w = n & 2 ? x[n / 4].y : x[n / 4].x;
                return __uint_as_float(n & 1 ? w & 0xffff0000u : w << 16) * up0 * up1;
            };
            uint8_t* dst = smem + C::Q_AT + half * C::BUF + row * 128;
#pragma unroll
            for (int c = 0; c < PD / 8; ++c) {
                uint32_t h[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const __half2 p = __floats2half2_rn(value(entry_of<BITS>(8 * c + 2 * i)), value(entry_of<BITS>(8 * c + 2 * i + 1)));
                    h[i] = *reinterpret_cast<const uint32_t*>(&p);
                }
                *reinterpret_cast<uint4*>(dst + c / 8 * PANEL + (((c % 8) ^ (row & 7)) << 4)) = make_uint4(h[0], h[1], h[2], h[3]);
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        }
        // ---- MMAs of this tile: by one thread, once all have done their part
        constexpr uint32_t idesc_s = idesc_f16(TQ, TK, false), idesc_o = idesc_f16(TQ, PD, true);
        const uint32_t t_s = tmem + COL_S + TK * half, t_o = tmem + COL_O + 128 * half;
        auto wait_full = [&](int n) {
            mbar_wait(bar_full + 8 * (n % RING), n / RING & 1, abort_flag, WAIT_FULL, n);
            tc_fence_after();
            return ring + n % RING * C::BUF;
        };
        auto issue_s = [&](int t) {
            const uint32_t keys = wait_full(2 * t);
#pragma unroll
            for (int ks = 0; ks < PD / 16; ++ks)
                mma_ss(t_s, smem_desc(sq + half * C::BUF + ks / 4 * PANEL) + 2 * (ks % 4), smem_desc(keys + ks / 4 * PANEL) + 2 * (ks % 4), idesc_s, ks != 0);
            tc_commit(bar_s + 8 * half);
            tc_commit(bar_empty + 8 * (2 * t % RING));
        };
        auto issue_o = [&](int t, bool last) {
            const uint32_t values = wait_full(2 * t + 1);
#pragma unroll
            for (int j = 0; j < TK / 16; ++j) mma_ts(t_o, t_s + 8 * j, smem_desc(values + 2048 * j), idesc_o, (t | j) != 0);
            tc_commit(bar_o + 8 * half);
            // (not on the last tile: nothing waits for it, and the CTA must not end before it has arrived)
            if (!last) tc_commit(bar_empty + 8 * ((2 * t + 1) % RING));
        };
        const bool issuer = (threadIdx.x & (TQ - 1)) == 0;
        float m = -1e30f, unit = 0.f;
        float l = 0.f;
        const int used = half < halves ? n_tiles : 0;
        tile_sync(half);
        if (issuer && used > 0) issue_s(0);
        __syncwarp();
        const int lim_lo = __reduce_min_sync(0xffffffffu, lim), lim_hi = __reduce_max_sync(0xffffffffu, lim);
        for (int t = 0; t < used; ++t) {
            mbar_wait(bar_s + 8 * half, t & 1, abort_flag, WAIT_S, t);
            tc_fence_after();
            const TileScales& ts = scales[t % SCALES];
            const int base = span.block(v0 + t) * TK;
            const uint4 dead = *reinterpret_cast<const uint4*>(ts.dead);
            const bool whole = base + TK - 1 <= lim_lo && (a.window == 0 || base > lim_hi - a.window || base + TK - 1 < a.sinks) &&
                               (dead.x | dead.y | dead.z | dead.w) == 0;
            uint32_t p[TK / 2];  // weights, two to a word
            float mx, sum;
            // weights of the tile for reference m; largest product of accumulator and key scale, sum of 2^(score - m)
            auto pass = [&](auto masked) {
                constexpr bool MASKED = decltype(masked)::value;
                const f2 mul_2 = pack2(mul, mul), m_2 = pack2(-m, -m);
                f2 sum2 = pack2(0.f, 0.f);
                mx = -INFINITY;
                const int to = lim - base, from = a.window > 0 ? lim - a.window + 1 - base : INT_MIN, sunk = a.sinks - base;
#pragma unroll
                for (int c = 0; c < TK / 32; ++c) {
                    uint32_t acc[32];
                    tmem_ld32(s_at + 32 * c, acc);
                    tmem_wait_ld();
                    const uint32_t gone = c == 0 ? dead.x : c == 1 ? dead.y : c == 2 ? dead.z : dead.w;
#pragma unroll
                    for (int i = 0; i < 32; i += 4) {
                        const ulonglong2 ks = *reinterpret_cast<const ulonglong2*>(ts.key + 32 * c + i);
                        const ulonglong2 vs = *reinterpret_cast<const ulonglong2*>(ts.value + 32 * c + i);
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            const int n = i + 2 * k;  // of the 32
                            f2 x = mul2(pack2(__uint_as_float(acc[n]), __uint_as_float(acc[n + 1])), k ? ks.y : ks.x);
                            float x0, x1, y0, y1, w0, w1;
                            unpack2(x, x0, x1);
                            bool seen0 = true, seen1 = true;
                            if (MASKED) {
                                const int j = 32 * c + n;
                                seen0 = j <= to && (j >= from || j < sunk) && !((gone >> n) & 1);
                                seen1 = j + 1 <= to && (j + 1 >= from || j + 1 < sunk) && !((gone >> (n + 1)) & 1);
                                x0 = seen0 ? x0 : -INFINITY;
                                x1 = seen1 ? x1 : -INFINITY;
                                x = pack2(x0, x1);
                            }
                            mx = fmaxf(mx, fmaxf(x0, x1));
                            unpack2(fma2(x, mul_2, m_2), y0, y1);
                            if (MASKED) {  // (a row factor of zero times -inf is no number)
                                y0 = seen0 ? y0 : -INFINITY;
                                y1 = seen1 ? y1 : -INFINITY;
                            }
                            const f2 e = pack2(exp2_approx(y0), exp2_approx(y1));
                            sum2 = add2(sum2, e);
                            unpack2(mul2(e, k ? vs.y : vs.x), w0, w1);
                            if (MASKED) {
                                w0 = seen0 ? w0 : 0.f;
                                w1 = seen1 ? w1 : 0.f;
                            }
                            const __half2 h = __floats2half2_rn(w0, w1);
                            p[(32 * c + n) / 2] = *reinterpret_cast<const uint32_t*>(&h);
                        }
                    }
                }
                float s0, s1;
                unpack2(sum2, s0, s1);
                sum = s0 + s1;
            };
            for (bool settled = false;; settled = true) {
                if (whole) pass(std::false_type{});
                else pass(std::true_type{});
                const float u = ts.unit, score = mx == -INFINITY ? -INFINITY : mx * mul;
                if (settled || !__any_sync(0xffffffffu, score > m + 8.f || u != unit)) break;
                const float m_new = score > m + 8.f ? score : m;
                const float corr = exp2_approx(m - m_new), o_corr = unit == 0.f ? 0.f : corr * (u / unit);
                m = m_new;
                unit = u;
                l *= corr;
                if (t == 0) continue;
                mbar_wait(bar_o + 8 * half, (t - 1) & 1, abort_flag, WAIT_O, t);
                tc_fence_after();
#pragma unroll
                for (int c = 0; c < PD / 32; ++c) {
                    uint32_t acc[32];
                    tmem_ld32(o_at + 32 * c, acc);
                    tmem_wait_ld();
#pragma unroll
                    for (int i = 0; i < 32; ++i) acc[i] = __float_as_uint(__uint_as_float(acc[i]) * o_corr);
                    tmem_st32(o_at + 32 * c, acc);
                }
            }
            l += sum;
            tmem_st32(s_at, p);
            tmem_st32(s_at + 32, p + 32);
            tmem_wait_st();
            tc_fence_before();
            tile_sync(half);
            if (issuer) {
                tc_fence_after();
                issue_o(t, t + 1 == used);
                if (t + 1 < used) issue_s(t + 1);  // behind O(t) on the pipe: P(t) is read before scores go over it
            }
            __syncwarp();
        }
        // ---- out = O / (unit l)
        if (used > 0) {
            mbar_wait(bar_o + 8 * half, (used - 1) & 1, abort_flag, WAIT_O, used);
            tc_fence_after();
        }
        const size_t id = (size_t)token * a.heads + head, part = (size_t)blockIdx.y * a.b.n_tokens * a.heads + id;
        const bool split = a.tc_splits > 1;
        const float inv = unit == 0.f ? 0.f : split ? 1.f / unit : l > 0.f ? 1.f / (unit * l) : 0.f;
        if (split && mine) a.part_ml[part] = make_float2(m, l);
        __nv_bfloat16* out = a.out + (size_t)token * a.out_stride + (size_t)head * a.l.hd;
#pragma unroll
        for (int c = 0; c < PD / 32; ++c) {
            uint32_t acc[32];
            float y[32];
            if (used > 0) {  // (the same for the whole warp)
                tmem_ld32(o_at + 32 * c, acc);
                tmem_wait_ld();
            } else {
#pragma unroll
                for (int i = 0; i < 32; ++i) acc[i] = 0u;
            }
#pragma unroll
            for (int i = 0; i < 32; ++i) y[entry_of<BITS>(i)] = inv == 0.f ? 0.f : __uint_as_float(acc[i]) * inv;
#pragma unroll
            for (int i = 0; i < 32; i += 4) {
                if (!mine || 32 * c + i >= a.l.hd) continue;
                if (split) {
                    reinterpret_cast<float4*>(a.part_o + part * 128)[8 * c + i / 4] = make_float4(y[i], y[i + 1], y[i + 2], y[i + 3]);
                } else {
                    const __nv_bfloat162 lo = __floats2bfloat162_rn(y[i], y[i + 1]), hi = __floats2bfloat162_rn(y[i + 2], y[i + 3]);
                    *reinterpret_cast<uint2*>(out + 32 * c + i) =
                        make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
                }
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == CONVERT_WARP) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(TMEM_COLS) : "memory");
    }
}

template <int BITS, int PD>
cudaError_t launch(const AttnArgs& a, cudaStream_t st) {
    const long long tiles = a.tc_tiles > 0 ? (long long)a.tc_tiles * a.b.n_seqs : (long long)a.b.n_tokens * a.group / a48p::TILE_ROWS + a.b.n_seqs;
    const dim3 grid((unsigned)(tiles * a.l.kv_heads), a.tc_splits);
    const cudaError_t e = cudaFuncSetAttribute(attn_paged_tc_kernel<BITS, PD>, cudaFuncAttributeMaxDynamicSharedMemorySize, Cfg<PD>::SMEM);
    return e != cudaSuccess ? e : a48_launch_pdl(attn_paged_tc_kernel<BITS, PD>, grid, dim3(THREADS), (size_t)Cfg<PD>::SMEM, st, a);
}

}  // namespace

bitnet_a48_status a48p::launch_tiles(const AttnArgs& a, cudaStream_t st) {
    const bool wide = a.l.padded > 64;
    cudaError_t e;
    if (a.l.bits == 3) e = wide ? launch<3, 128>(a, st) : launch<3, 64>(a, st);
    else if (a.l.bits == 4) e = wide ? launch<4, 128>(a, st) : launch<4, 64>(a, st);
    else e = wide ? launch<8, 128>(a, st) : launch<8, 64>(a, st);
    A48_CUDA_TRY(e);
    return BITNET_A48_OK;
}

bitnet_a48_status a48_read_attn_paged_status(unsigned int words_host[4]) {
    A48_CUDA_TRY(cudaMemcpyFromSymbol(words_host, g_status, sizeof(unsigned int) * 4));
    const unsigned int zero[4] = {0, 0, 0, 0};
    A48_CUDA_TRY(cudaMemcpyToSymbol(g_status, zero, sizeof(zero)));
    return BITNET_A48_OK;
}
