// Attention over the paged low-bit cache for sequences with many rows (chunks of prompts), on the fifth-generation tensor
// cores.  A CTA takes 256 rows (token, query head of the group) of one key/value head as two tiles of 128, and walks the
// positions they see 128 at a time.
//
// Both contractions run on the codes (attn_paged.cu has the formulas): S = Q C^T, O += P D with P = 2^(score - reference)
// times the value scale in fp16, fp32 accumulators in tensor memory.  Q is brought to fp16 by one power of two for the
// CTA's rows (a row 2^20 below the largest still has all its bits, one 2^29 below it the upper ten); that power, the factor
// of the scores and log2 e go into the key scales, so that an exponent is one fused multiply-add of an accumulator.  The
// codes of 128 positions are converted to fp16 once for the 256 rows, into shared memory in the 128-byte swizzle, one row
// per position for keys and values alike: the keys are then a K-major operand and the values an MN-major one, and nothing is
// transposed.  The entries of a row keep the order in which the conversion gives them; the query rows are stored in the
// same order, and the output columns are put right when they are stored.
//
//   warps 0-3, 4-7   the rows of tile 0, 1: scores from tensor memory, 2^(score - reference), the weights back over the
//                    scores.  One pass: the reference moves only when the weights of a row (a thread's 16 of 64 columns) sum
//                    to more than 2^9, or a value scale exceeds its unit by 2^6; then the columns' maximum is found, O
//                    rescaled and the columns taken again.  The sum bounds each weight, so there is no maximum to keep in the steady
//                    state: per two entries a multiply-add, two exponentials, a sum, the value scale and the conversion
//                    (f32x2 where there is such a form).  A thread has four rows and a quarter of the columns (the
//                    16x256b form of the loads), so that it reads a quarter of the scales.  One thread of each tile then
//                    issues the MMAs O(t) and, behind it on the pipe, S(t+1): while one tile's weights are taken, the
//                    pipe has the other's two products.  (A warp of its own for the MMAs would be the thirteenth, and
//                    leave every thread 128 registers instead of 168.)
//   warps 8-11       codes to fp16: two lanes per row, 32 entries each, so that both the loads and the swizzled stores are
//                    free of conflicts; the next tile's codes and the page numbers of the one after it under way
//                    meanwhile.  A ring of four buffers, K(t) V(t) K(t+1) V(t+1).
// Tensor memory: two score tiles (128 columns, P over the first 64) and two output tiles (up to 128 columns).
//
// A CTA that is through with its rows cancels one that has not started and takes its rows over, so that the codes and queries
// of the next rows are under way while the last weights are multiplied and outputs stored.  Four prompts of 4096 tokens, 32
// heads of 128, 3 bits: 672 us (818 TFLOP/s of the 4 x 128 operations per score); two chunks of up to 2048 tokens with a
// window of 2048, 181 us.  On the way there, for the prompts: one CTA to each tile of rows 854 us, taking over 821, masks by
// groups of 16 positions and no tiles that the first rows do not see 691, queries converted eight rows at a time 669.
//
// What bounds it: 128 positions take a CTA about 4250 clocks, of which the products of both tiles occupy the tensor pipe for
// 2600.  A tile needs 250 clocks from its scores to the first weights, 2400 for the weights (1400 for the 64 columns taken
// while the other tile takes its last 64, 1000 for the others; the exponentials alone are 1024 clocks of the SFUs) and 1300
// for O and the next S; with no room for a second score tile in tensor memory these follow one another.  Without the
// exponentials the 821 us were 749, without the conversion to fp16 829, without the turns that the tiles take 866.  Tiles of
// 64 positions, with two score tiles each, were slower (1015 us against 917 then): products of 64 columns are bound by
// shared memory.  Rows cost about 13000 clocks of their own, half of which the first tile waits for the second; letting it
// go on ahead, with the converting warps finding the largest query entry, was no faster (687 us).
// Every wait is bounded; one that gives up records itself (bitnet_a48_kernel_status), and every later wait of the CTA then
// falls through, so that the kernel ends by itself.
#include <climits>

#include "attn_paged.cuh"

namespace {

using a48p::AttnArgs;
using a48p::exp2_approx;
using a48p::in_register;
using a48p::power_of_two;
using a48p::query_exponent;
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
                    g_status[2] = blockIdx.x;
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
__device__ __noinline__ void mbar_wait_long(uint32_t bar, uint32_t parity, uint32_t iter) {
    const unsigned long long t0 = clock64();
    while (!mbar_try(bar, parity))
        if (clock64() - t0 > 5 * kWaitClocks) {
            if (atomicCAS(&g_status[0], 0u, (unsigned)BITNET_A48_ERR_TIMEOUT) == 0u) {
                g_status[1] = 46;
                g_status[2] = blockIdx.x;
                g_status[3] = iter;
            }
            return;
        }
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
__device__ __forceinline__ bool elect() {
    uint32_t one;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(one) : : "memory");
    return one != 0;
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
// 16 lanes x 16 columns; thread 4g+t has columns 8i + 2t, 8i + 2t + 1 of lane g in r[4i], r[4i+1], of lane g + 8 in the next two
__device__ __forceinline__ void tmem_ld_16x16(uint32_t taddr, uint32_t* r) {
    asm volatile("tcgen05.ld.sync.aligned.16x256b.x2.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
                 : "r"(taddr)
                 : "memory");
}
__device__ __forceinline__ void tmem_st_16x16(uint32_t taddr, const uint32_t* r) {
    asm volatile("tcgen05.st.sync.aligned.16x256b.x2.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"r"(taddr), "r"(r[0]), "r"(r[1]),
                 "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
                 : "memory");
}
// 16 lanes x 32 columns; thread 4g+t has column 4i + t of lane g in r[2i], of lane g + 8 in r[2i+1]
__device__ __forceinline__ void tmem_st_16x32(uint32_t taddr, const uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.16x128b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
        ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]),
          "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
        : "memory");
}
__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
// the same, for loads into these registers: nothing that reads them is moved ahead of the wait
__device__ __forceinline__ void tmem_wait_ld(uint32_t (&r)[2][8]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(r[0][0]), "+r"(r[0][1]), "+r"(r[0][2]), "+r"(r[0][3]), "+r"(r[0][4]), "+r"(r[0][5]), "+r"(r[0][6]), "+r"(r[0][7]),
                   "+r"(r[1][0]), "+r"(r[1][1]), "+r"(r[1][2]), "+r"(r[1][3]), "+r"(r[1][4]), "+r"(r[1][5]), "+r"(r[1][6]), "+r"(r[1][7])
                 :
                 : "memory");
}
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
// The two tiles take their weights in turn: one waits until the other is through, which then has the tensor pipe working.
__device__ __forceinline__ void turn_wait(int half) { asm volatile("bar.sync %0, 256;" ::"r"(5 + half) : "memory"); }
__device__ __forceinline__ void turn_pass(int half) { asm volatile("bar.arrive %0, 256;" ::"r"(6 - half) : "memory"); }
__device__ __forceinline__ void queries_sync() { asm volatile("bar.sync 4, %0;" ::"n"(THREADS) : "memory"); }
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
    float scale[TK / 2][4];    // of two positions: key scales times the factors of a score, value scales times `unit`
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
    static constexpr int Q_AT = RING * BUF, CTRL_AT = Q_AT + 2 * BUF, ROWS_AT = CTRL_AT + 256,
                         SCALES_AT = ROWS_AT + 2 * TQ * 8, ITEM_AT = SCALES_AT + SCALES * (int)sizeof(TileScales), OUT_AT = ITEM_AT + 2 * 128;
    static constexpr int SMEM = OUT_AT + 2 * TQ * 64 + 1024 /*alignment slack*/;
    static_assert(SMEM <= 227 * 1024, "shared memory budget");
};

// what a wait that gave up was for
enum { WAIT_FULL = 41, WAIT_EMPTY = 42, WAIT_S = 43, WAIT_ANSWER = 44, WAIT_O = 45 };

// What a CTA takes at a time: up to 256 rows of a sequence with one key/value head, and the blocks of positions v0 ..
// v0 + n_tiles - 1 of their span.  The tiles with the most positions come first.
struct Item {
    Span span;
    int rows;     // 0: none there; -1: no more items
    int r0;       // first row (rows of a call are counted in 31 bits)
    int kvh, part, seq, start, pos0, pos_lo, pos_hi, v0, n_tiles;
    int used0, used1;  // tiles of positions that a row of either tile may see: the first may not see the last one
};
__device__ __forceinline__ bool item_of(const AttnArgs& a, int index, int lane, Item& it) {  // false: no rows there
    it.rows = it.n_tiles = 0;
    const int x = index / a.tc_splits, at = gridDim.x / a.tc_splits / a.l.kv_heads - 1 - x / a.l.kv_heads;
    it.part = index % a.tc_splits, it.kvh = x % a.l.kv_heads;
    int tile;
    if (a.tc_tiles > 0) {
        it.seq = at % a.b.n_seqs, tile = at / a.b.n_seqs;
    } else {  // sequence b has the tiles from floor(q_start[b] group / 256) + b on, more than it needs
        auto first_tile = [&](int b) { return (long long)__ldg(a.b.q_start + b) * a.group / a48p::TILE_ROWS + b; };
        it.seq = a48p::last_at_most(a.b.n_seqs, at, lane, first_tile);
        if (it.seq < 0) return false;
        tile = at - (int)first_tile(it.seq);
    }
    it.start = __ldg(a.b.q_start + it.seq);
    const int q_len = __ldg(a.b.q_start + it.seq + 1) - it.start;
    const long long all_rows = (long long)q_len * a.group;
    const long long r0 = (long long)tile * a48p::TILE_ROWS;
    it.r0 = (int)r0;
    if (all_rows <= a.few_rows || r0 >= all_rows || it.start < 0 || q_len > a.b.n_tokens - it.start) return false;
    it.rows = (int)min((long long)a48p::TILE_ROWS, all_rows - r0);
    it.pos0 = __ldg(a.b.kv_len + it.seq) - q_len;
    it.pos_lo = it.pos0 + it.r0 / a.group, it.pos_hi = it.pos0 + (it.r0 + it.rows - 1) / a.group;
    it.span = a48p::span_of<7>(a, it.pos_lo, it.pos_hi);
    const int per = max(2, (it.span.count + a.tc_splits - 1) / a.tc_splits);
    it.v0 = it.part * per;
    it.n_tiles = max(0, min(it.span.count, it.v0 + per) - it.v0);
    const int hi = it.pos0 + (it.r0 + min(it.rows, TQ) - 1) / a.group;  // at most TQ = TK positions below pos_hi
    it.used0 = it.n_tiles > 0 && it.span.block(it.v0 + it.n_tiles - 1) * TK > hi ? it.n_tiles - 1 : it.n_tiles;
    it.used1 = it.rows > TQ ? it.n_tiles : 0;
    return true;
}

template <int BITS, int PD>
__global__ void __launch_bounds__(THREADS, 1) attn_paged_tc_kernel(const __grid_constant__ AttnArgs a) {
    using C = Cfg<PD>;
    constexpr int PANELS = PD / 64, PANEL = TK * 128;
    extern __shared__ uint8_t smem_raw[];
    // (an offset, not an aligned integer: the compiler then knows these as shared-memory addresses)
    uint8_t* smem = smem_raw + (-smem_u32(smem_raw) & 1023u);
    uint8_t* ctrl = smem + C::CTRL_AT;
    uint8_t* canceled = ctrl + 128;  // the answer about a CTA not yet started, 16 bytes
    uint32_t* q_tops = reinterpret_cast<uint32_t*>(ctrl + 160);  // the largest query entry, as bits, of three items
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(ctrl + 192);
    volatile uint32_t* abort_flag = reinterpret_cast<volatile uint32_t*>(ctrl + 196);
    float* top_part = reinterpret_cast<float*>(ctrl + 208);     // largest value scale per converting warp
    float2* row_info = reinterpret_cast<float2*>(smem + C::ROWS_AT);  // last position seen; at the end reference and sum
    Item* items = reinterpret_cast<Item*>(smem + C::ITEM_AT);  // this one and the next, by the parity of their number
    TileScales* scales = reinterpret_cast<TileScales*>(smem + C::SCALES_AT);
    const uint32_t ring = smem_u32(smem), sq = ring + C::Q_AT;
    // barriers: full[4] | empty[4] | s[2] | o[2] | answer | next item
    const uint32_t bar_full = smem_u32(ctrl), bar_empty = bar_full + 32, bar_s = bar_full + 64, bar_o = bar_full + 80,
                   bar_answer = bar_full + 96, bar_next = bar_full + 104;
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;  // (known to be the same in a warp)
    a48_pdl_prologue();

    Item first;
    if (!item_of(a, blockIdx.x, lane, first)) return;
    if (threadIdx.x == 0) {
        for (int i = 0; i < RING; ++i) {
            mbar_init(bar_full + 8 * i, TQ);
            mbar_init(bar_empty + 8 * i, 2);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(bar_s + 8 * i, 1);
            mbar_init(bar_o + 8 * i, 1);
        }
        mbar_init(bar_answer, 1);
        mbar_init(bar_next, 1);
        *abort_flag = 0;
        q_tops[0] = 0;
        items[0] = first;
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

    // Items: the CTA's own, then those of CTAs that have not started, which it cancels and takes over one at a time.  One
    // thread asks while the last tile of positions of an item is converted, and hands the answer on; the others have
    // read the one before by then (every item has a queries_sync of all warps).
    auto ask = [&]() {
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], 16;" ::"r"(bar_answer) : "memory");
        asm volatile("clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 [%0], [%1];" ::"r"(
                         smem_u32(canceled)),
                     "r"(bar_answer)
                     : "memory");
    };
    auto hand_on = [&](int k) {  // what was asked for ahead of item k, by the thread's warp
        uint32_t taken = 0, index = 0;
        if (lane == 0) {
            mbar_wait(bar_answer, (k - 1) & 1, abort_flag, WAIT_ANSWER, k);
            asm volatile(
                "{\n\t.reg .pred p;\n\t.reg .b128 answer;\n\t"
                "ld.shared.b128 answer, [%2];\n\t"
                "clusterlaunchcontrol.query_cancel.is_canceled.pred.b128 p, answer;\n\t"
                "selp.u32 %0, 1, 0, p;\n\tmov.u32 %1, 0;\n\t"
                "@p clusterlaunchcontrol.query_cancel.get_first_ctaid::x.b32.b128 %1, answer;\n\t}"
                : "=r"(taken), "=r"(index)
                : "r"(smem_u32(canceled))
                : "memory");
            if (*abort_flag) taken = 0;
        }
        taken = __shfl_sync(0xffffffffu, taken, 0), index = __shfl_sync(0xffffffffu, index, 0);
        Item got;
        if (taken) item_of(a, (int)index, lane, got);
        else got.rows = -1, got.n_tiles = 0;
        if (lane == 0) {
            items[k & 1] = got;
            mbar_arrive(bar_next);
        }
        __syncwarp();
    };
    // (This one wait must not be given up before that thread has come through its own: five times their limit.)
    Item it = first;
    auto item_after = [&](int k) {
        mbar_wait_long(bar_next, (k - 1) & 1, k);
        it = items[k & 1];
    };
    int n0 = 0;  // tiles of positions of the items before
    if (warp >= CONVERT_WARP) {
        // ------------------------------------------------------------------------------------------ codes to fp16
        const int w = warp - CONVERT_WARP, r = 32 * w + lane;  // r: the position whose scales are this thread's
        const int sub = lane >> 1, odd = lane & 1;
        // Codes: block b (16 positions) of the warp's two, entries 64p + 32 odd .. + 31 of the row at position sub.
        typedef uint32_t Codes[2][PANELS][BITS];
        const int window = in_register(a.window), sinks = in_register(a.sinks), row_bytes = in_register(a.l.row), v_codes = in_register(a.l.v_codes),
                  k_scales = in_register(a.l.k_scales), v_scales = in_register(a.l.v_scales), slots = in_register(a.l.page - 1);
        float sk = 0.f, sv = 0.f, unit = 0.f;
        int page[2] = {-1, -1}, next[2] = {-1, -1};  // pages of the blocks, of this tile and of the next
        int base = 0;                                // first position of the warp in the tile
        const uint8_t* chunk[2] = {nullptr, nullptr};
        int slot[2] = {0, 0};
        auto look_up = [&](int t) {
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const int p = t < it.n_tiles ? it.span.block(it.v0 + t) * TK + 32 * w + 16 * b : INT_MAX;
                next[b] = p <= it.pos_hi ? a48p::page_of(a.l, a.b, it.seq, p) : -1;
            }
        };
        auto locate = [&](int t) {
            base = it.span.block(it.v0 + t) * TK + 32 * w;
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                page[b] = next[b];
                chunk[b] = a.pool + a48p::chunk_at(a.l, max(page[b], 0), it.kvh);
                slot[b] = (base + 16 * b) & slots;
            }
        };
        auto load_codes = [&](Codes& x, int part) {
#pragma unroll
            for (int b = 0; b < 2; ++b)
#pragma unroll
                for (int p = 0; p < PANELS; ++p) {
                    const int at = (2 * p + odd) * 4 * BITS;
                    const bool there = page[b] >= 0 && at < row_bytes;
                    const uint8_t* src = chunk[b] + part * v_codes + (slot[b] + sub) * row_bytes + at;
                    if constexpr (BITS == 3) {
#pragma unroll
                        for (int i = 0; i < 3; ++i) x[b][p][i] = there ? __ldg(reinterpret_cast<const uint32_t*>(src) + i) : 0u;
                    } else {
#pragma unroll
                        for (int i = 0; i < BITS; i += 4) {
                            const uint4 v = there ? __ldg(reinterpret_cast<const uint4*>(src + 4 * i)) : make_uint4(0, 0, 0, 0);
                            x[b][p][i] = v.x, x[b][p][i + 1] = v.y, x[b][p][i + 2] = v.z, x[b][p][i + 3] = v.w;
                        }
                    }
                }
        };
        auto load_scales = [&]() {
            const int b = lane >> 4;
            const bool there = page[b] >= 0;
            const uint8_t* from = b ? chunk[1] : chunk[0];
            const int at = (b ? slot[1] : slot[0]) + (lane & 15);
            sk = there ? __ldg(reinterpret_cast<const float*>(from + k_scales) + at) : 0.f;
            sv = there ? __ldg(reinterpret_cast<const float*>(from + v_scales) + at) : 0.f;
        };
        auto store_codes = [&](uint8_t* buf, const Codes& x, const uint8_t* bos) {
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                const int row = 32 * w + 16 * b + sub;
#pragma unroll
                for (int p = 0; p < PANELS; ++p) {
                    uint32_t h[16];
                    const uint32_t(&c)[BITS] = x[b][p];
                    if constexpr (BITS == 3) {
                        a48p::triples(c[0], c[1], c[2], h);
                        if (bos && row == 0) {  // position 0: 4-bit codes of its own
#pragma unroll
                            for (int i = 0; i < 16; ++i) {
                                const int e = 64 * p + 32 * odd + i;
                                float lo = 0.f, hi = 0.f;
                                if (64 * p + 32 * odd < a.l.padded) {
                                    lo = (float)((bos[e / 2] >> (4 * (e & 1))) & 15) - 8.f;
                                    hi = (float)((bos[e / 2 + 8] >> (4 * (e & 1))) & 15) - 8.f;
                                }
                                const __half2 pair = __floats2half2_rn(lo, hi);
                                h[i] = *reinterpret_cast<const uint32_t*>(&pair);
                            }
                        }
                    } else if constexpr (BITS == 4) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) a48p::nibbles(c[i], h + 4 * i);
                    } else {
#pragma unroll
                        for (int i = 0; i < 8; ++i) a48p::bytes(c[i], h + 2 * i);
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        *reinterpret_cast<uint4*>(buf + p * PANEL + row * 128 + (((4 * odd + i) ^ (row & 7)) << 4)) =
                            make_uint4(h[4 * i], h[4 * i + 1], h[4 * i + 2], h[4 * i + 3]);
                }
            }
        };
        Codes keys, values;
        auto wait_empty = [&](int n) {
            if (n >= RING) mbar_wait(bar_empty + 8 * (n % RING), (n / RING & 1) ^ 1, abort_flag, WAIT_EMPTY, n);
            return smem + n % RING * C::BUF;
        };
        auto publish = [&](int n) {
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            mbar_arrive(bar_full + 8 * (n % RING));
        };
#pragma unroll 1
        for (int k = 0; it.rows >= 0;) {
            if (it.n_tiles > 0) {
                unit = 0.f;
                look_up(0);
                locate(0);
                load_scales();
                load_codes(keys, 0);
                load_codes(values, 1);
                look_up(1);
            } else {
                queries_sync();
                if (threadIdx.x == 32 * CONVERT_WARP) ask();
            }
            float factor = 0.f;
#pragma unroll 1
            for (int t = 0; t < it.n_tiles; ++t) {
                const int pos = base + lane;
                const uint8_t* bos = BITS == 3 && base == 0 && page[0] >= 0 ? chunk[0] + a.l.bos : nullptr;  // position 0's codes
                const bool dead = (lane < 16 ? page[0] : page[1]) < 0 && pos <= it.pos_hi;
                // ---- the codes of the keys.  (The ring is what keeps the scales of four tiles apart: K(t) can be written once
                // the scores of t - 2 are done, and the weights of t - 3 were taken before the scores of t - 2 were issued.)
                const int n = 2 * (n0 + t);
                uint8_t* buf = wait_empty(n);
                store_codes(buf, keys, bos);
                if (t == 0) {
                    queries_sync();
                    const int e = query_exponent(q_tops[k % 3]);
                    factor = a.scale * 1.4426950408889634f * power_of_two(-e / 2) * power_of_two(-(e - e / 2));
                }
                if (t + 1 == it.n_tiles && threadIdx.x == 32 * CONVERT_WARP) ask();
                // ---- their scales; one counts if it is finite and some row may see its position
                const bool may = pos <= it.pos_hi && (window == 0 || pos > it.pos_lo - window || pos < sinks);
                const bool finite = sk <= 3.4e38f && sv <= 3.4e38f;
                // The scores of a row that does not see a position are set to -inf ahead of these factors, so they have to be
                // positive and finite; where the scales are not, the rows that do see the position get no numbers from its key.
                const float key = finite && may ? fminf(fmaxf(sk * factor, 1e-37f), 3e38f) : 1.f, f = finite && may ? sv : 0.f;
                const uint32_t sick = __ballot_sync(0xffffffffu, may && !finite), gone = __ballot_sync(0xffffffffu, dead);
                if (convert_any(unit == 0.f ? f > 0.f : f * unit > 64.f)) {
                    float top = f;
#pragma unroll
                    for (int d = 16; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
                    if (lane == 0) top_part[w] = top;
                    convert_sync();
                    top = fmaxf(fmaxf(top_part[0], top_part[1]), fmaxf(top_part[2], top_part[3]));
                    // two octaves of room, so that scales of one size do not come back here; within fp32's exponents
                    unit = scalbnf(1.f, min(max(5 - (ilogbf(top) + 2), -120), 120));
                }
                TileScales& ts = scales[(n0 + t) % SCALES];
                ts.scale[r >> 1][r & 1] = key;
                ts.scale[r >> 1][2 + (r & 1)] = f * unit;
                if (lane == 0) ts.dead[w] = gone;
                if (r == 0) ts.unit = unit;
                if (sick) {
                    __syncwarp();
                    for (int i = 0; i < PD / 8; ++i)
                        if ((sick >> lane) & 1)
                            *reinterpret_cast<uint4*>(buf + i / 8 * PANEL + r * 128 + i % 8 * 16) =
                                make_uint4(0x7e007e00u, 0x7e007e00u, 0x7e007e00u, 0x7e007e00u);
                }
                publish(n);
                // ---- the next tile's keys under way, then the values of this one
                if (t + 1 < it.n_tiles) {
                    locate(t + 1);
                    load_scales();
                    load_codes(keys, 0);
                }
                store_codes(wait_empty(n + 1), values, bos ? bos + a.l.padded / 2 : nullptr);
                publish(n + 1);
                if (t + 1 < it.n_tiles) {
                    load_codes(values, 1);
                    look_up(t + 2);
                }
            }
            if (w == 0) hand_on(k + 1);
            n0 += it.n_tiles;
            item_after(++k);
        }
        // the CTA must not end before the last arrivals on its barriers
        for (int i = 0; i < RING; ++i) {
            const int uses = (2 * n0 - i + RING - 1) / RING;
            if (uses > 0) mbar_wait(bar_empty + 8 * i, (uses - 1) & 1, abort_flag, WAIT_EMPTY, n0);
        }
    } else {
        // ------------------------------------------------------------------------------------------ rows
        const int half = warp >> 2, row = (warp & 3) * 32 + lane, r = half * TQ + row;
        const uint32_t lanes = tmem + ((uint32_t)((warp & 3) * 32) << 16);
        const uint32_t s_at = lanes + COL_S + TK * half, o_at = lanes + COL_O + 128 * half;
        const int window = in_register(a.window), sinks = in_register(a.sinks);
        const bool split = a.tc_splits > 1;
        // Query rows come through the place of their fp16 form, those of the next item while the last weights of this one are
        // multiplied and its outputs stored.  Queries and outputs move four entries to a lane, whole rows to an instruction
        // (with a row to a thread they were a fifth of the time of a prompt).
        constexpr int UNITS = PD / 4, AT_ONCE = 32 / UNITS;
        const int u = lane % UNITS, sub = lane / UNITS;
        uint8_t* queries = smem + C::Q_AT + half * C::BUF + (warp & 3) * 32 * 128;
        int k = 0, u0 = 0;  // u0: tiles of positions that this tile of rows has taken
        auto place_of = [&](const Item& i, int& token, int& head) {  // of this thread's row; without one, of the item's last
            const uint32_t n = i.r0 + min(r, i.rows - 1);
            token = i.start + (int)(n / (uint32_t)a.group), head = i.kvh * a.group + (int)(n % (uint32_t)a.group);
        };
        // Raw, either half of a row lies where its fp16 form will: a warp's rows are its own.
        auto at_unit = [&](int j, int unit) { return queries + j * 128 + unit / 16 * PANEL + unit % 16 * 8; };
        auto fetch = [&]() {
            if (it.rows <= 0) return;
            int token, head;
            place_of(it, token, head);
            const size_t from = (size_t)token * a.q_stride + (size_t)head * a.l.hd;
#pragma unroll 8
            for (int i = 0; i < UNITS; ++i) {
                const int j = AT_ONCE * i + sub;
                const size_t at = __shfl_sync(0xffffffffu, (unsigned long long)from, j);
                const bool real = r - lane + j < it.rows && 4 * u < a.l.hd;
                asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(smem_u32(at_unit(j, u))), "l"(a.q + (real ? at + 4 * u : 0)),
                             "r"(real ? 8 : 0)
                             : "memory");
            }
        };
        fetch();
#pragma unroll 1
        while (it.rows >= 0) {
            if (threadIdx.x == 0) q_tops[(k + 1) % 3] = 0;  // (read for the last time before the queries_sync of k - 1)
            if (it.rows == 0) {
                queries_sync();
                item_after(++k);
                fetch();
                continue;
            }
            uint32_t* q_top = q_tops + k % 3;
            const int rows = it.rows;
            // ---- the query rows to fp16 by a power of two, in the order of the converted codes
            {
                float mx = 0.f;
                asm volatile("cp.async.wait_all;" ::: "memory");
                __syncwarp();
#pragma unroll 8
                for (int i = 0; i < UNITS; ++i) {
                    const uint2 x = *reinterpret_cast<const uint2*>(at_unit(AT_ONCE * i + sub, u));
                    // (numbers only: an infinity of one row must not hide the others' entries, which would overflow)
#pragma unroll
                    for (int n = 0; n < 4; ++n) {
                        const uint32_t w = n & 2 ? x.y : x.x;
                        const float v = fabsf(__uint_as_float(n & 1 ? w & 0xffff0000u : w << 16));
                        mx = v <= 3.4e38f ? fmaxf(mx, v) : mx;
                    }
                }
                const uint32_t top = __reduce_max_sync(0xffffffffu, __float_as_uint(mx));
                if (lane == 0) atomicMax(q_top, top);
                row_info[r].x = __int_as_float(it.pos0 + (it.r0 + min(r, rows - 1)) / a.group);
                queries_sync();
                const int e = query_exponent(*q_top);
                const float up0 = power_of_two(e / 2), up1 = power_of_two(e - e / 2);  // (2^e may be past fp32)
                auto halves_of = [&](uint32_t w) {
                    const __half2 h = __floats2half2_rn(__uint_as_float(w << 16) * up0 * up1, __uint_as_float(w & 0xffff0000u) * up0 * up1);
                    return *reinterpret_cast<const uint32_t*>(&h);
                };
                // Entries n and n + 16 (n + 4 at 4 bits) side by side: of two lanes that far apart, either gives two entries to the
                // other.  At 8 bits the pairs (n, n + 2) are the lane's own.
                constexpr int APART = BITS == 3 ? 4 : BITS == 4 ? 1 : 0;
                const bool upper = (u & APART) != 0;
                const int place = BITS == 3 ? (4 * u & ~31) + 8 * (u & 3) + (u & 4) : 4 * u;
                uint8_t* dst = queries + place / 64 * PANEL + (place & 4) * 2;
#pragma unroll 1
                for (int i = 0; i < UNITS; i += 8) {  // (eight loads, then eight stores: they cannot be told apart)
                    uint2 x[8];
#pragma unroll
                    for (int n = 0; n < 8; ++n) x[n] = *reinterpret_cast<const uint2*>(at_unit(AT_ONCE * (i + n) + sub, u));
#pragma unroll
                    for (int n = 0; n < 8; ++n) {
                        uint32_t lo = halves_of(x[n].x), hi = halves_of(x[n].y);
                        if constexpr (APART > 0) {
                            const uint32_t got = __shfl_xor_sync(0xffffffffu, upper ? lo : hi, APART);
                            lo = upper ? got : lo, hi = upper ? hi : got;
                        }
                        x[n] = make_uint2(__byte_perm(lo, hi, 0x5410), __byte_perm(lo, hi, 0x7632));
                    }
                    __syncwarp();  // (the rows have been read)
#pragma unroll
                    for (int n = 0; n < 8; ++n) {
                        const int j = AT_ONCE * (i + n) + sub;
                        *reinterpret_cast<uint2*>(dst + j * 128 + (((place / 8 % 8) ^ (j & 7)) << 4)) = x[n];
                    }
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            }
            // ---- MMAs of this tile: by one thread, once all have done their part
            constexpr uint32_t idesc_s = idesc_f16(TQ, TK, false), idesc_o = idesc_f16(TQ, PD, true);
            const uint32_t t_s = tmem + COL_S + TK * half, t_o = tmem + COL_O + 128 * half;
            const int used = half ? it.used1 : it.used0, other = half ? it.used0 : it.used1, both = min(used, other);  // tiles of positions
            auto wait_full = [&](int n) {
                mbar_wait(bar_full + 8 * (n % RING), n / RING & 1, abort_flag, WAIT_FULL, n);
                tc_fence_after();
                return ring + n % RING * C::BUF;
            };
            const uint64_t q_desc = smem_desc(sq + half * C::BUF);
            auto issue_s = [&](int t) {
                const uint64_t k_desc = smem_desc(wait_full(2 * (n0 + t)));
                if (elect()) {
#pragma unroll
                    for (int ks = 0; ks < PD / 16; ++ks) {
                        constexpr int STEP = PANEL / 16;  // of a descriptor's address, per 64 entries
                        mma_ss(t_s, q_desc + ks / 4 * STEP + 2 * (ks % 4), k_desc + ks / 4 * STEP + 2 * (ks % 4), idesc_s, ks != 0);
                    }
                    tc_commit(bar_s + 8 * half);
                    for (int i = t < other; i < 2; ++i) tc_commit(bar_empty + 8 * (2 * (n0 + t) % RING));  // (for the other tile too if it is not used there)
                }
                __syncwarp();
            };
            auto issue_o = [&](int t) {
                const uint64_t v_desc = smem_desc(wait_full(2 * (n0 + t) + 1));
                if (elect()) {
                    mma_ts(t_o, t_s, v_desc, idesc_o, t != 0);
#pragma unroll
                    for (int j = 1; j < TK / 16; ++j) mma_ts(t_o, t_s + 8 * j, v_desc + 2048 / 16 * j, idesc_o, 1);
                    tc_commit(bar_o + 8 * half);
                    for (int i = t < other; i < 2; ++i) tc_commit(bar_empty + 8 * ((2 * (n0 + t) + 1) % RING));
                }
                __syncwarp();
            };
            const bool issuer = (warp & 3) == 0;
            tile_sync(half);  // the query rows are in place
            if (issuer && used > 0) issue_s(0);
            // the four rows of this thread between loads and stores: lanes g, g + 8, g + 16, g + 24 of the warp
            const int g = lane >> 2, c0 = 2 * (lane & 3);
            float m[4], l[4], unit = 0.f;
            int lim[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                lim[i] = __float_as_int(row_info[half * TQ + (warp & 3) * 32 + 8 * i + g].x);
                m[i] = -1e30f, l[i] = 0.f;
            }
            const int lim_lo = __reduce_min_sync(0xffffffffu, min(min(lim[0], lim[1]), min(lim[2], lim[3])));
            const int lim_hi = __reduce_max_sync(0xffffffffu, max(max(lim[0], lim[1]), max(lim[2], lim[3])));
            if (half == 1 && both > 0) turn_pass(1);
            for (int t = 0; t < used; ++t) {
                mbar_wait(bar_s + 8 * half, (u0 + t) & 1, abort_flag, WAIT_S, t);
                tc_fence_after();
                const TileScales& ts = scales[(n0 + t) % SCALES];
                const int base = it.span.block(it.v0 + t) * TK;
                const uint4 dead = *reinterpret_cast<const uint4*>(ts.dead);
                const bool whole = base + TK - 1 <= lim_lo && (window == 0 || base > lim_hi - window || base + TK - 1 < sinks) &&
                                   (dead.x | dead.y | dead.z | dead.w) == 0;
                if (!whole) {  // the scores that a row does not see become -inf
#pragma unroll 1
                    for (int c = 0; c < TK / 16; ++c) {  // (most groups of 16 positions are seen by all of the warp's rows, or by none)
                        const int from = base + 16 * c;
                        const uint32_t gone = ts.dead[c >> 1] >> (16 * (c & 1)) & 0xffff;
                        if (gone == 0 && from + 15 <= lim_lo && (window == 0 || from > lim_hi - window || from + 15 < sinks)) continue;
                        uint32_t acc[2][8];
                        if (gone == 0xffff || from > lim_hi || (window > 0 && from + 15 <= lim_lo - window && from >= sinks)) {
#pragma unroll
                            for (int i = 0; i < 16; ++i) acc[i >> 3][i & 7] = 0xff800000u;
                        } else {
                            tmem_ld_16x16(s_at + 16 * c, acc[0]);
                            tmem_ld_16x16(s_at + (16u << 16) + 16 * c, acc[1]);
                            auto below = [](int n) { return (1u << min(max(n, 0), 16)) - 1; };  // bits of the first n of the 16
                            uint32_t seen[4];
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                const int to = lim[i] - from;
                                uint32_t s = below(to + 1);
                                if (window > 0) s &= ~below(to + 1 - window) | below(sinks - from);
                                seen[i] = (s & ~gone) >> c0;
                            }
                            tmem_wait_ld(acc);
#pragma unroll
                            for (int i = 0; i < 16; ++i)
                                if (!((seen[(i >> 3) * 2 + ((i >> 1) & 1)] >> (8 * ((i >> 2) & 1) + (i & 1))) & 1)) acc[i >> 3][i & 7] = 0xff800000u;
                        }
                        tmem_st_16x16(s_at + 16 * c, acc[0]);
                        tmem_st_16x16(s_at + (16u << 16) + 16 * c, acc[1]);
                    }
                    tmem_wait_st();
                }
                if (t < both) turn_wait(half);
                // ---- 64 columns, then the other 64
#pragma unroll 1
                for (int h = 0; h < 2; ++h) {
                    uint32_t p[2][16];  // weights, two columns to a word
                    float sum[4];
                    for (bool settled = false;; settled = true) {
                        // weights and sums of 2^(score - m), 16 columns at a time, the next 16 under way meanwhile
                        f2 m_2[4], sum_2[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) m_2[i] = pack2(-m[i], -m[i]), sum_2[i] = pack2(0.f, 0.f);
                        uint32_t acc[2][2][8];
                        tmem_ld_16x16(s_at + 64 * h, acc[0][0]);
                        tmem_ld_16x16(s_at + (16u << 16) + 64 * h, acc[0][1]);
                        ulonglong2 scale[8];
#pragma unroll
                        for (int k = 0; k < 8; ++k) scale[k] = *reinterpret_cast<const ulonglong2*>(ts.scale[32 * h + 4 * k + c0 / 2]);
#pragma unroll
                        for (int c = 0; c < 4; ++c) {
                            tmem_wait_ld(acc[c & 1]);
                            if (c < 3) {
                                tmem_ld_16x16(s_at + 64 * h + 16 * (c + 1), acc[(c + 1) & 1][0]);
                                tmem_ld_16x16(s_at + (16u << 16) + 64 * h + 16 * (c + 1), acc[(c + 1) & 1][1]);
                            }
#pragma unroll
                            for (int k = 0; k < 2; ++k) {
#pragma unroll
                                for (int i = 0; i < 4; ++i) {
                                    const uint32_t* from = acc[c & 1][i >> 1] + 4 * k + 2 * (i & 1);
                                    float y0, y1, w0, w1;
                                    unpack2(fma2(pack2(__uint_as_float(from[0]), __uint_as_float(from[1])), scale[2 * c + k].x, m_2[i]), y0, y1);
                                    const f2 e = pack2(exp2_approx(y0), exp2_approx(y1));
                                    sum_2[i] = add2(sum_2[i], e);
                                    unpack2(mul2(e, scale[2 * c + k].y), w0, w1);
                                    const __half2 w = __floats2half2_rn(w0, w1);
                                    p[i >> 1][2 * (2 * c + k) + (i & 1)] = *reinterpret_cast<const uint32_t*>(&w);
                                }
                            }
                        }
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            float s0, s1;
                            unpack2(sum_2[i], s0, s1);
                            sum[i] = s0 + s1;
                        }
                        const float u = ts.unit;
                        const bool high = u != unit || fmaxf(fmaxf(sum[0], sum[1]), fmaxf(sum[2], sum[3])) > 512.f;
                        if (settled || !__any_sync(0xffffffffu, high)) break;
                        // ---- rarely: references to the largest scores of these columns where those are higher (rounded up to
                        // whole numbers: what moves along then moves by powers of two), and with them O, and the first columns'
                        // weights while the second's are taken.  (Weights, and O of an earlier move, may still be on their way
                        // into tensor memory: loads are ordered behind stores by this wait alone.)
                        tmem_wait_st();
                        float corr[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) corr[i] = -INFINITY;
#pragma unroll 1
                        for (int c = 0; c < 4; ++c) {
                            tmem_ld_16x16(s_at + 64 * h + 16 * c, acc[0][0]);
                            tmem_ld_16x16(s_at + (16u << 16) + 64 * h + 16 * c, acc[0][1]);
                            tmem_wait_ld(acc[0]);
#pragma unroll
                            for (int i = 0; i < 16; ++i) {
                                const int row = (i >> 3) * 2 + ((i >> 1) & 1);
                                corr[row] = fmaxf(corr[row], __uint_as_float(acc[0][i >> 3][i & 7]) *
                                                                 ts.scale[32 * h + 8 * c + 4 * ((i >> 2) & 1) + c0 / 2][i & 1]);
                            }
                        }
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            corr[i] = fmaxf(corr[i], __shfl_xor_sync(0xffffffffu, corr[i], 1));
                            corr[i] = fmaxf(corr[i], __shfl_xor_sync(0xffffffffu, corr[i], 2));
                            const float m_new = fmaxf(m[i], ceilf(corr[i]));
                            corr[i] = exp2_approx(m[i] - m_new);
                            m[i] = m_new;
                            l[i] *= corr[i];
                        }
                        if (h > 0) {
#pragma unroll 1
                            for (int c = 0; c < 2; ++c) {  // (16 words are 32 weights)
                                tmem_ld_16x16(s_at + 16 * c, acc[0][0]);
                                tmem_ld_16x16(s_at + (16u << 16) + 16 * c, acc[0][1]);
                                tmem_wait_ld(acc[0]);
#pragma unroll
                                for (int i = 0; i < 16; ++i) {
                                    uint32_t& w = acc[0][i >> 3][i & 7];
                                    // (in fp32: the factor may be below fp16's numbers where a weight of up to 2^15 times it is not)
                                    const float by = corr[(i >> 3) * 2 + ((i >> 1) & 1)];
                                    const float2 x = __half22float2(*reinterpret_cast<const __half2*>(&w));
                                    const __half2 y = __floats2half2_rn(x.x * by, x.y * by);
                                    w = *reinterpret_cast<const uint32_t*>(&y);
                                }
                                tmem_st_16x16(s_at + 16 * c, acc[0][0]);
                                tmem_st_16x16(s_at + (16u << 16) + 16 * c, acc[0][1]);
                            }
                        }
                        const float ratio = unit == 0.f ? 0.f : u / unit;  // (the unit moves between tiles only)
                        unit = u;
                        if (t == 0) continue;
                        mbar_wait(bar_o + 8 * half, (u0 + t - 1) & 1, abort_flag, WAIT_O, t);
                        tc_fence_after();
#pragma unroll 1
                        for (int c = 0; c < PD / 16; ++c) {
                            tmem_ld_16x16(o_at + 16 * c, acc[0][0]);
                            tmem_ld_16x16(o_at + (16u << 16) + 16 * c, acc[0][1]);
                            tmem_wait_ld(acc[0]);
#pragma unroll
                            for (int i = 0; i < 16; ++i)
                                acc[0][i >> 3][i & 7] = __float_as_uint(__uint_as_float(acc[0][i >> 3][i & 7]) * (corr[(i >> 3) * 2 + ((i >> 1) & 1)] * ratio));
                            tmem_st_16x16(o_at + 16 * c, acc[0][0]);
                            tmem_st_16x16(o_at + (16u << 16) + 16 * c, acc[0][1]);
                        }
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i) l[i] += sum[i];
                    tmem_st_16x32(s_at + 32 * h, p[0]);  // (over scores that have been taken)
                    tmem_st_16x32(s_at + (16u << 16) + 32 * h, p[1]);
                    if (h == 0 && t + half < both) turn_pass(half);
                }
                tmem_wait_st();
                tc_fence_before();
                tile_sync(half);
                if (issuer) {
                    tc_fence_after();
                    issue_o(t);
                    if (t + 1 < used) issue_s(t + 1);  // behind O(t) on the pipe: P(t) is read before scores go over it
                }
            }
            // ---- out = O / (unit l), one row per thread again
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                l[i] += __shfl_xor_sync(0xffffffffu, l[i], 1);
                l[i] += __shfl_xor_sync(0xffffffffu, l[i], 2);
                if (c0 == 0) row_info[half * TQ + (warp & 3) * 32 + 8 * i + g] = make_float2(m[i], l[i]);
            }
            __syncwarp();
            const float2 ml = row_info[r];
            const Item done = items[k & 1];  // (again: not kept in registers meanwhile)
            int token, head;
            place_of(done, token, head);
            size_t part = 0;
            if (split) {
                const a48p::Parts& of = a.tile_parts;
                const long long place = of.per_head > 0 ? ((long long)done.seq * a.l.kv_heads + done.kvh) * of.per_head + done.r0 + min(r, done.rows - 1)
                                                        : (long long)token * a.heads + head;
                part = (size_t)(done.part * of.rows + place);
            }
            const float inv = unit == 0.f ? 0.f : split ? 1.f / unit : ml.y != 0.f ? 1.f / ml.y / unit : 0.f;
            if (split && r < done.rows) a.tile_parts.ml[part] = ml;
            const size_t to = split ? part * 128 : (size_t)token * a.out_stride + (size_t)head * a.l.hd;
            n0 += done.n_tiles;
            item_after(++k);
            fetch();
            if (used > 0) {
                mbar_wait(bar_o + 8 * half, (u0 + used - 1) & 1, abort_flag, WAIT_O, used);
                tc_fence_after();
            }
            u0 += used;
            // 64 bytes of each row at a time through shared memory: 16 of its row from a thread, eight of one to each lane to memory
            uint8_t* stage = smem + C::OUT_AT + warp * 32 * 64;
            auto put = [&](int chunk, uint32_t x, uint32_t y, uint32_t z, uint32_t w) {
                *reinterpret_cast<uint4*>(stage + lane * 64 + ((chunk ^ ((lane >> 1) & 3)) << 4)) = make_uint4(x, y, z, w);
            };
            auto store_rows = [&](uint8_t* base, int elem, int width) {  // elem: bytes of an entry; width: bytes of a row that there are
                __syncwarp();
                const int u = lane & 7;
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int j = 4 * i + (lane >> 3);
                    const size_t at = __shfl_sync(0xffffffffu, (unsigned long long)to, j);
                    const uint2 v = *reinterpret_cast<const uint2*>(stage + j * 64 + (((u >> 1) ^ ((j >> 1) & 3)) << 4) + 8 * (u & 1));
                    if (r - lane + j < done.rows && 8 * u < width) *reinterpret_cast<uint2*>(base + at * elem + 8 * u) = v;
                }
                __syncwarp();
            };
#pragma unroll 1
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
                if (split) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const float* v = y + 16 * h + 4 * i;
                            put(i, __float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
                        }
                        store_rows(reinterpret_cast<uint8_t*>(a.tile_parts.o) + 128 * c + 64 * h, 4, a.l.hd * 4 - 128 * c - 64 * h);
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        uint32_t w[4];
#pragma unroll
                        for (int n = 0; n < 4; ++n) {
                            const __nv_bfloat162 v = __floats2bfloat162_rn(y[8 * i + 2 * n], y[8 * i + 2 * n + 1]);
                            w[n] = *reinterpret_cast<const uint32_t*>(&v);
                        }
                        put(i, w[0], w[1], w[2], w[3]);
                    }
                    store_rows(reinterpret_cast<uint8_t*>(a.out) + 64 * c, 2, a.l.hd * 2 - 64 * c);
                }
            }
            tc_fence_before();
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
    const dim3 grid((unsigned)(tiles * a.l.kv_heads * a.tc_splits));
    static std::atomic<bool> allowed[64];
    const cudaError_t e = a48_allow_smem(attn_paged_tc_kernel<BITS, PD>, Cfg<PD>::SMEM, allowed);
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
