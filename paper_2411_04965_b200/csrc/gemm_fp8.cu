// Product of two e4m3 matrices with a scale for each block of 128 channels, on the fifth-generation tensor cores:
//   y[m, n] = sum over blocks b of  xs[b][m] * ws[n / 128][b] * (sum over k in b of x[m, k] * w[n, k]).
//
// The scales change every 128 channels, so the tensor core's accumulator holds one block's products only: each block is a
// fresh accumulation (four MMAs of 32 channels) into one of the buffers in tensor memory, and the epilogue warps multiply it by its
// scale and add it to sums in registers.  Tokens are the rows of the tile (a thread of the epilogue has one token) and
// output features its columns: a column block of 128 shares ws, so a thread's factor for a block is one number, and a
// block costs it one multiply-add per feature.
#include <algorithm>
#include <type_traits>

#include "fp8.cuh"
#include "softmax_sums.cuh"
#include "tc.cuh"

namespace {

using a48f8::ScoreArgs;
using a48f8::ScoreParts;
using a48f8::Sums;

using namespace a48tc;
using a48f8::BLOCK;
using a48f8::LinearArgs;

constexpr int TMEM_COLS = 512;
constexpr int CONTROL_WARPS = 4;  // copies, MMAs, and two that only make up a warpgroup

// SUBS x SUBN: features of a tile, as so many accumulators of SUBN columns, each with a warpgroup of its own that takes it
// out of tensor memory.  PAIR: two CTAs share a tile of 256 tokens; each holds half of the weight rows of an accumulator.
template <int SUBS_, int SUBN_, bool PAIR_>
struct Cfg {
    static constexpr int SUBS = SUBS_, SUBN = SUBN_, BN = SUBS * SUBN;
    static constexpr bool PAIR = PAIR_;
    static constexpr int CTAS = PAIR ? 2 : 1, TM = 128 * CTAS;
    static constexpr int SUB_ROWS = SUBN / CTAS;  // weight rows of an accumulator that a CTA holds
    static constexpr int A_BYTES = 128 * BLOCK, SUB_BYTES = SUB_ROWS * BLOCK, STAGE_BYTES = A_BYTES + SUBS * SUB_BYTES;
    static constexpr int OUT_BYTES = 4096, OUT_BUFS = 2;  // 32 rows of 128 bytes on their way out, two to a warp
    static constexpr int EPI_WARPS = 4 * SUBS, NUM_THREADS = 32 * (CONTROL_WARPS + EPI_WARPS);
    static constexpr int OUT_ALL = EPI_WARPS * OUT_BUFS * OUT_BYTES;
    static constexpr int MAX_STAGES = (225 * 1024 - OUT_ALL) / STAGE_BYTES;
    static constexpr int STAGES = MAX_STAGES < 16 ? MAX_STAGES : 16;
    // Blocks of channels that change hands at once between the MMAs and the epilogue, each in columns of its own: what the
    // hand-over costs (about 300 clocks) is spread over 128 columns whatever the tile.
    static constexpr int GROUP = BLOCK / SUBN, ACC_COLS = GROUP * SUBN;
    static constexpr int ACC_BUFS = TMEM_COLS / ACC_COLS;
    static constexpr int SMEM_BYTES = STAGES * STAGE_BYTES + OUT_ALL + 1024 /*alignment*/ + 512 /*barriers*/;
    // With eight epilogue warps 168 registers a thread at launch are all an SM has; the control warps hand theirs over.
    static constexpr bool MOVE_REGISTERS = SUBS == 2;
    static constexpr int CONTROL_REGISTERS = 40, EPI_REGISTERS = 232;
    static_assert(!MOVE_REGISTERS || 128 * CONTROL_REGISTERS + 256 * EPI_REGISTERS <= 384 * 168, "registers of the launch");
    static_assert(STAGES >= ACC_BUFS / SUBS * GROUP, "a stage comes round no sooner than its products have been read");
    static_assert(SUBN % 32 == 0 && SUBN <= BLOCK, "the columns of an accumulator share a weight scale");
    static_assert(ACC_BUFS % SUBS == 0 && STAGE_BYTES % 1024 == 0, "layout");
    static_assert(SMEM_BYTES <= 227 * 1024, "shared memory");
    static_assert(8 * ((1 + SUBS) * STAGES + ACC_BUFS) <= 480, "barriers");
};

struct Params {
    const float* xs;
    const float* ws;
    void* y;
    long long y_stride;
    int M, N, kb, m_tiles, tiles, x_rows, y_bf16;
    int y_map;           // y is stored by tensor copies
    const void* tokens;  // the rest: products that keep sums of their logits
    int tokens64;
    float c;
    float4* stats;
    float* owns;
};

// Sums of the softmax over a thread's columns (the last ones may not exist), and the logit of its row's token.
template <int COLS>
__device__ __forceinline__ Sums sums_of(const float (&sum)[COLS], int cols, float c2, long long token_at, float* own) {
    Sums s;
    float top = -INFINITY;
#pragma unroll
    for (int c = 0; c < COLS; ++c)
        if (c < cols) top = fmaxf(top, sum[c]);
    s.start(top);
    float sixteen = 0.f;  // together, since one by one small terms are lost beside the largest one's 1
#pragma unroll
    for (int c = 0; c < COLS; ++c) {
        if (c < cols) s.add(sum[c], c2, sixteen);
        if (c % 16 == 15) {
            s.s += sixteen;
            sixteen = 0.f;
        }
    }
    if (token_at >= 0 && token_at < cols) {
#pragma unroll
        for (int c = 0; c < COLS; ++c)
            if (token_at == c) *own = sum[c];
    }
    return s;
}

// 32 rows x COLS columns of a warp to y: through shared memory, 128 bytes of every row at a time (16-byte pieces of row r
// exchanged by r % 8, so that neither side has bank conflicts), and from there by tensor stores, or, where y's rows are not
// 16-byte aligned, a row to an instruction.
template <int COLS, bool BF16>
__device__ __forceinline__ void store_rows(const float (&sum)[COLS], const Params& p, const CUtensorMap* tm_y, uint8_t* out, int m0, int n0, int lane,
                                           uint32_t& stores) {
    constexpr int W = BF16 ? 64 : 32;  // columns in 128 bytes
#pragma unroll
    for (int c0 = 0; c0 < COLS; c0 += W) {
        if (n0 + c0 >= p.N) break;
        uint8_t* buf = out + (stores++ & 1u) * 4096;
        if (p.y_map) {
            if (lane == 0) tma_store_wait_read<1>();
        }
        __syncwarp();
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            uint32_t v[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (BF16) {
                    const int c = c0 + 8 * q + 2 * j;
                    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(v[j]) : "f"(c + 1 < COLS ? sum[(c + 1) % COLS] : 0.f), "f"(c < COLS ? sum[c % COLS] : 0.f));
                } else {
                    v[j] = __float_as_uint(sum[(c0 + 4 * q + j) % COLS]);
                }
            }
            *reinterpret_cast<uint4*>(buf + lane * 128 + ((q ^ (lane & 7)) << 4)) = make_uint4(v[0], v[1], v[2], v[3]);
        }
        if (p.y_map) {
            fence_async_shared();
            __syncwarp();
            if (lane == 0) tma_store_2d(tm_y, n0 + c0, m0, smem_u32(buf));
        } else {
            __syncwarp();
            // eight rows' reads before their stores (4096 tokens, 32001 x 4096: 580 us, row by row 654)
            const int rows = min(32, p.M - m0);
            using T = typename std::conditional<BF16, __nv_bfloat16, float>::type;
            T* y = reinterpret_cast<T*>(p.y) + (size_t)m0 * p.y_stride + n0 + c0 + lane;
#pragma unroll
            for (int r0 = 0; r0 < 32; r0 += 8) {
                if (r0 >= rows) break;
                T v[8][W / 32];
#pragma unroll
                for (int r = 0; r < 8; ++r)
#pragma unroll
                    for (int h = 0; h < W / 32; ++h) {
                        constexpr int PIECE = 16 / sizeof(T);
                        const int i = h * 32 + lane;
                        v[r][h] = reinterpret_cast<const T*>(buf + (r0 + r) * 128)[((i / PIECE) ^ r) * PIECE + i % PIECE];
                    }
#pragma unroll
                for (int r = 0; r < 8; ++r)
#pragma unroll
                    for (int h = 0; h < W / 32; ++h)
                        if (r0 + r < rows && h * 32 < COLS - c0 && n0 + c0 + h * 32 + lane < p.N) y[(size_t)(r0 + r) * p.y_stride + h * 32] = v[r][h];
            }
            __syncwarp();
        }
    }
}

template <class C, bool SCORE>
__global__ void __launch_bounds__(C::NUM_THREADS, 1)
    gemm_fp8_kernel(const __grid_constant__ CUtensorMap tm_x, const __grid_constant__ CUtensorMap tm_w, const __grid_constant__ CUtensorMap tm_y,
                    const Params p) {
    constexpr int STAGES = C::STAGES, ACC_BUFS = C::ACC_BUFS, SUBS = C::SUBS, SUBN = C::SUBN;
    constexpr bool PAIR = C::PAIR;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    uint8_t* out_all = smem + STAGES * C::STAGE_BYTES;
    uint8_t* ctrl = out_all + C::OUT_ALL;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(ctrl + 480);
    volatile uint32_t* abort_flag = reinterpret_cast<volatile uint32_t*>(ctrl + 484);
    // full: a stage's bytes have landed.  done: the MMAs that read it have completed, and with them a block's products (of the last
    // accumulator; the one before has a barrier of its own, so that its warps can start): what both the copies and the epilogue
    // wait for, since a commit costs the thread that issues the MMAs some 300 clocks (with commits of their own for both, a block
    // took a single CTA 0.39 and 0.50 us instead of 0.28 and 0.43).  acc_empty: an accumulator has been read.
    const uint32_t bar_full = smem_u32(ctrl), bar_done = bar_full + 8 * STAGES, bar_acc_empty = bar_done + 8 * SUBS * STAGES;
    const uint32_t smem_base = smem_u32(smem);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = PAIR ? (int)(blockIdx.x & 1u) : 0;
    const int unit = PAIR ? (int)(blockIdx.x >> 1) : (int)blockIdx.x, units = (int)gridDim.x / C::CTAS;

    if (threadIdx.x == 0) {
        asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&tm_x)) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&tm_w)) : "memory");
        for (int s = 0; s < STAGES; ++s) {
            mbar_init(bar_full + 8 * s, 1);
            for (int i = 0; i < SUBS; ++i) mbar_init(bar_done + 8 * (i * STAGES + s), 1);
        }
        for (int b = 0; b < ACC_BUFS; ++b) mbar_init(bar_acc_empty + 8 * b, C::CTAS * 4);  // one arrival to a warp of the accumulator's warpgroup
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    a48_pdl_prologue();  // before tensor memory is taken, which the kernel ahead may still need
    if (warp == 1) tc_alloc<PAIR>(smem_u32(tmem_slot), TMEM_COLS);
    tc_fence_before();
    __syncthreads();
    if (PAIR) cluster_sync_all();
    tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;

    if (warp < CONTROL_WARPS) {
        if (C::MOVE_REGISTERS) registers_down<C::CONTROL_REGISTERS>();
        // One thread each for the copies and the MMAs: a wait of a whole warp costs them a vote, and the pipe a gap.
        if (warp == 0 && elect_one()) {
            // --------------------------------------------------------- tensor copies
            uint32_t it = 0, s = 0, ph = 0;
            bool ok = true;
            const uint32_t full0 = PAIR ? map_to_rank(bar_full, 0) : bar_full;  // the pair's copies all report to rank 0
            for (int tile = unit; tile < p.tiles && ok; tile += units) {
                const int nt = tile / p.m_tiles, mt = tile - nt * p.m_tiles;
                const int m0 = mt * C::TM + rank * 128, n0 = nt * C::BN + rank * C::SUB_ROWS;
                for (int b = 0; b < p.kb; ++b, ++it) {
                    ok = mbar_wait(bar_done + 8 * ((SUBS - 1) * STAGES + s), ph ^ 1, abort_flag, 1, it);
                    if (!ok) break;
                    const uint32_t dst = smem_base + s * C::STAGE_BYTES, bar = full0 + 8 * s;
                    if (rank == 0) mbar_expect_tx(bar_full + 8 * s, (uint32_t)(C::CTAS * (p.x_rows * BLOCK + SUBS * C::SUB_BYTES)));
#pragma unroll
                    for (int i = 0; i < SUBS; ++i) {
                        if (PAIR) tma_load_2d_pair(dst + C::A_BYTES + i * C::SUB_BYTES, &tm_w, b * BLOCK, n0 + i * SUBN, bar);
                        else tma_load_2d(dst + C::A_BYTES + i * C::SUB_BYTES, &tm_w, b * BLOCK, n0 + i * SUBN, bar);
                    }
                    if (PAIR) tma_load_2d_pair(dst, &tm_x, b * BLOCK, m0, bar);
                    else tma_load_2d(dst, &tm_x, b * BLOCK, m0, bar);
                    if (++s == (uint32_t)STAGES) { s = 0; ph ^= 1; }
                }
            }
            if (!ok) {  // let the copies already issued land before the CTA exits
                const unsigned long long t0 = clock64();
                if (rank == 0) {
                    for (uint32_t back = 1; back <= (uint32_t)STAGES && back <= it; ++back) {
                        const uint32_t j = it - back, sj = j % STAGES, pj = (j / STAGES) & 1;
                        while (!mbar_try(bar_full + 8 * sj, pj) && clock64() - t0 < kWaitClocks) {
                        }
                    }
                } else {
                    while (clock64() - t0 < 4000000ull) {
                    }
                }
            }
        } else if (warp == 1 && rank == 0 && elect_one()) {
            // --------------------------------------------------------- MMAs (of a pair: rank 0 for both)
            constexpr uint32_t idesc = idesc_e4m3(C::TM, SUBN);
            uint32_t it = 0, s = 0, ph = 0, a = 0, pa = 0;
            bool ok = true;
            for (int tile = unit; tile < p.tiles && ok; tile += units) {
                for (int b = 0; b < p.kb && ok; ++b, ++it) {
                    const int g = b % C::GROUP;
                    const bool last = g == C::GROUP - 1 || b == p.kb - 1;
                    ok = mbar_wait(bar_full + 8 * s, ph, abort_flag, 3, it);
                    if (!ok) break;
                    const uint64_t a_desc = smem_desc_sw128(smem_base + s * C::STAGE_BYTES);
#pragma unroll
                    for (int i = 0; i < SUBS; ++i) {
                        if (g == 0) ok = mbar_wait(bar_acc_empty + 8 * (a + i), pa ^ 1, abort_flag, 2, it);
                        if (!ok) break;
                        tc_fence_after();
                        const uint64_t b_desc = a_desc + ((C::A_BYTES + i * C::SUB_BYTES) >> 4);
                        const uint32_t to = tmem_base + (a + i) * C::ACC_COLS + g * SUBN;
#pragma unroll
                        for (int j = 0; j < 4; ++j) mma_f8<PAIR>(to, a_desc + 2 * j, b_desc + 2 * j, idesc, j > 0);
                        tc_commit<PAIR>(bar_done + 8 * (i * STAGES + s));
                    }
                    if (!ok) break;
                    if (++s == (uint32_t)STAGES) { s = 0; ph ^= 1; }
                    if (last && (a += SUBS) == (uint32_t)ACC_BUFS) { a = 0; pa ^= 1; }
                }
            }
        }
        __syncwarp();
    } else {
        // ------------------------------------------------------------- scales, sums, stores
        if (C::MOVE_REGISTERS) registers_up<C::EPI_REGISTERS>();
        const int quad = warp & 3, sub = (warp - CONTROL_WARPS) >> 2;
        const uint32_t t_lanes = tmem_base + ((uint32_t)(quad * 32) << 16);
        const uint32_t bar_mine = bar_done + 8 * sub * STAGES;
        const uint32_t acc_empty0 = PAIR ? map_to_rank(bar_acc_empty, 0) : bar_acc_empty;
        uint8_t* out = out_all + (warp - CONTROL_WARPS) * C::OUT_BUFS * C::OUT_BYTES;
        uint32_t it = 0, a = sub, stores = 0;
        uint32_t s = 0, ph = 0;  // stage and phase of the next group's first block
        bool ok = true;
        Sums run;  // SCORE, a single CTA with one tile of tokens: over all tiles of this CTA
        run.start(-INFINITY);
        for (int tile = unit; tile < p.tiles && ok; tile += units) {
            __syncwarp();  // loads from tensor memory want the warp together, wherever the lanes' stores and waits went apart
            const int nt = tile / p.m_tiles, mt = tile - nt * p.m_tiles;
            const int m0 = mt * C::TM + rank * 128 + quad * 32, m = m0 + lane, n0 = nt * C::BN + sub * SUBN;
            const bool live = m0 < p.M && n0 < p.N;  // the same for the whole warp
            const float* xs = p.xs + min(m, p.M - 1);
            const float* ws = p.ws + (size_t)(min(n0, p.N - 1) / BLOCK) * p.kb;
            float sum[SUBN];
#pragma unroll
            for (int c = 0; c < SUBN; ++c) sum[c] = 0.f;
            // Scales are under way two groups ahead, 16 columns while the 16 before them are multiplied, and whether the next
            // group's products are there is asked before this group's last columns are.  (32 at a time are no faster and leave the
            // pairs' form too few registers: what the compiler then spills costs 40%.)
            constexpr int GROUP = C::GROUP, CHUNKS = C::ACC_COLS / 16;
            float x_scale[2][GROUP], w_scale[2][GROUP];
#pragma unroll
            for (int u = 0; u < 2 * GROUP; ++u) {
                x_scale[u / GROUP][u % GROUP] = __ldg(xs + (size_t)min(u, p.kb - 1) * p.M);
                w_scale[u / GROUP][u % GROUP] = __ldg(ws + min(u, p.kb - 1));
            }
            // the group's last block: its stage, by which both the products are announced and the next group is found
            auto move_on = [&](int blocks) {
                s += blocks;
                if (s >= (uint32_t)STAGES) { s -= STAGES; ph ^= 1; }
            };
            move_on(min(GROUP, p.kb) - 1);
            bool there = mbar_test(bar_mine + 8 * s, ph);
            for (int b0 = 0; b0 < p.kb && ok; b0 += 2 * GROUP) {
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const int b = b0 + u * GROUP;
                    if (b >= p.kb) break;
                    if (!__all_sync(0xffffffffu, there)) {
                        ok = __all_sync(0xffffffffu, there || mbar_wait_slow(bar_mine + 8 * s, ph, abort_flag, 4, it));
                        if (!ok) break;
                        __syncwarp();
                    }
                    tc_fence_after();
                    float scale[GROUP];
#pragma unroll
                    for (int g = 0; g < GROUP; ++g) {
                        scale[g] = x_scale[u][g] * w_scale[u][g];
                        const int ahead = min(b + 2 * GROUP + g, p.kb - 1);
                        x_scale[u][g] = __ldg(xs + (size_t)ahead * p.M);
                        w_scale[u][g] = __ldg(ws + ahead);
                    }
                    uint32_t r[2][16];
                    const uint32_t from = t_lanes + a * C::ACC_COLS, done = acc_empty0 + 8 * a;
                    ++it;
                    if ((a += SUBS) >= (uint32_t)ACC_BUFS) a = sub;
                    move_on(b + GROUP < p.kb ? min(GROUP, p.kb - b - GROUP) : 1);
                    tmem_ld16(from, r[0]);
#pragma unroll
                    for (int c = 0; c < CHUNKS; ++c) {
                        constexpr int OF_BLOCK = SUBN / 16;
                        uint32_t(&now)[16] = r[c & 1];
                        float factor = scale[c / OF_BLOCK];
                        tmem_wait(factor);
                        if (c + 1 < CHUNKS) tmem_ld16(from + (c + 1) * 16, r[(c + 1) & 1]);
                        if (c + 1 == CHUNKS) {
                            tc_fence_before();
                            mbar_arrive_if<PAIR>(done, lane == 0);
                            there = b + GROUP < p.kb && mbar_test(bar_mine + 8 * s, ph);
                        }
                        if (GROUP == 1 || b + c / OF_BLOCK < p.kb) {  // (columns of blocks past the last hold those of an earlier group)
#pragma unroll
                            for (int j = 0; j < 16; ++j) {  // (two at a time, fma.rn.f32x2, took longer: the pairs of registers have to be made)
                                float& to = sum[c % OF_BLOCK * 16 + j];
                                to = fmaf(__uint_as_float(now[j]), factor, to);
                            }
                        }
                    }
                }
            }
            if (!ok) break;
            if (SCORE) {
                const bool row = m < p.M;
                Sums mine;
                mine.start(-INFINITY);
                if (live) {
                    long long token = -1;
                    if (row) token = p.tokens64 ? __ldg(reinterpret_cast<const long long*>(p.tokens) + m) : __ldg(reinterpret_cast<const int*>(p.tokens) + m);
                    mine = sums_of<SUBN>(sum, min(SUBN, p.N - n0), p.c, token < 0 ? -1 : token - n0, p.owns + m);
                }
                if (PAIR || p.m_tiles > 1) {
                    if (row) p.stats[(size_t)(nt * SUBS + sub) * p.M + m] = make_float4(mine.r, mine.s, mine.d, 0.f);
                } else {
                    run.join(mine, p.c);
                    if (row && tile + units >= p.tiles) p.stats[(size_t)(unit * SUBS + sub) * p.M + m] = make_float4(run.r, run.s, run.d, 0.f);
                }
            } else if (live) {
                if (p.y_bf16) store_rows<SUBN, true>(sum, p, &tm_y, out, m0, n0, lane, stores);
                else store_rows<SUBN, false>(sum, p, &tm_y, out, m0, n0, lane, stores);
            }
        }
        if (!SCORE && lane == 0) tma_store_wait_all();
    }
    tc_fence_before();
    __syncthreads();
    if (PAIR) cluster_sync_all();  // both CTAs are done with both tensor memories and with each other's barriers
    if (warp == 1) {
        tc_fence_after();
        tc_dealloc<PAIR>(tmem_base, TMEM_COLS);
    }
}

template <class C, bool SCORE>
bitnet_a48_status launch(const LinearArgs& a, const ScoreArgs* score, ScoreParts* parts, cudaStream_t st) {
    static std::atomic<bool> ready[64];
    A48_CUDA_TRY(a48_allow_smem(gemm_fp8_kernel<C, SCORE>, C::SMEM_BYTES, ready));
    if (C::MOVE_REGISTERS) {  // warps that ask for more registers than the launch has would wait for ever
        static std::atomic<int> registers;
        int n = registers.load(std::memory_order_relaxed);
        if (n == 0) {
            cudaFuncAttributes attr;
            A48_CUDA_TRY(cudaFuncGetAttributes(&attr, gemm_fp8_kernel<C, SCORE>));
            registers.store(n = attr.numRegs, std::memory_order_relaxed);
        }
        if (n * C::NUM_THREADS < 128 * C::CONTROL_REGISTERS + 32 * C::EPI_WARPS * C::EPI_REGISTERS) return BITNET_A48_ERR_UNSUPPORTED;
    }
    CUtensorMap tm_x, tm_w, tm_y;
    const int x_rows = std::min((a.M + 7) / 8 * 8, 128);
    if (!make_map(&tm_x, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, a.x, (uint64_t)a.M, (uint64_t)a.K, (uint64_t)a.K, (uint32_t)x_rows) ||
        !make_map(&tm_w, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, a.w, (uint64_t)a.N, (uint64_t)a.K, (uint64_t)a.K, (uint32_t)C::SUB_ROWS))
        return BITNET_A48_ERR_CUDA;
    Params p = {};
    const int size = a.y_bf16 ? 2 : 4;
    p.y_map = !SCORE && a48_aligned16(a.y) && a.y_stride * size % 16 == 0 && (unsigned long long)a.y_stride * size < (1ull << 40);
    tm_y = tm_x;  // not used without y_map
    if (p.y_map && !make_map(&tm_y, a.y_bf16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT32, (uint32_t)size, a.y, (uint64_t)a.M,
                             (uint64_t)a.N, (uint64_t)a.y_stride * size, 32))
        return BITNET_A48_ERR_CUDA;
    p.xs = a.xs;
    p.ws = a.ws;
    p.y = a.y;
    p.y_stride = a.y_stride;
    p.M = a.M;
    p.N = a.N;
    p.kb = a48f8::blocks(a.K);
    p.m_tiles = (a.M + C::TM - 1) / C::TM;
    const long long tiles = (long long)p.m_tiles * ((a.N + C::BN - 1) / C::BN);
    if (tiles > (1ll << 30)) return BITNET_A48_ERR_LIMIT;
    p.tiles = (int)tiles;
    p.x_rows = x_rows;
    p.y_bf16 = a.y_bf16;
    const int slots = a48f8::sm_count() / C::CTAS;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(std::min(p.tiles, slots) * C::CTAS));
    cfg.blockDim = dim3(C::NUM_THREADS);
    cfg.dynamicSmemBytes = C::SMEM_BYTES;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = 2;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = C::PAIR ? 2 : 1;
    if (SCORE) {
        p.tokens = score->tokens;
        p.tokens64 = score->tokens64;
        p.c = score->c;
        p.stats = parts->stats;
        p.owns = parts->owns;
        parts->parts = C::SUBS * (C::PAIR || p.m_tiles > 1 ? (a.N + C::BN - 1) / C::BN : (int)cfg.gridDim.x / C::CTAS);
    }
    A48_CUDA_TRY(cudaLaunchKernelEx(&cfg, gemm_fp8_kernel<C, SCORE>, tm_x, tm_w, tm_y, p));
    return BITNET_A48_OK;
}

template <class C>
bitnet_a48_status launch(const LinearArgs& a, const ScoreArgs* score, ScoreParts* parts, cudaStream_t st) {
    return score ? launch<C, true>(a, score, parts, st) : launch<C, false>(a, score, parts, st);
}

}  // namespace

namespace a48f8 {

int sm_count() {
    static std::atomic<int> n[64];
    int dev = 0;
    cudaGetDevice(&dev);
    int c = n[dev & 63].load(std::memory_order_relaxed);
    if (!c) {
        cudaDeviceGetAttribute(&c, cudaDevAttrMultiProcessorCount, dev);
        n[dev & 63].store(c, std::memory_order_relaxed);
    }
    return c;
}

// Tiles: 128 tokens x 64 or 128 features of one CTA, or 256 x 256 of a pair.  A call takes as long as its rounds of tiles over
// the SMs times what a block of 128 channels costs a tile: 0.28, 0.43 and 0.62 us (measured from 40 x 4096 x 1536 to 1024 x
// 4096 x 4096; the model picked the fastest of the three in 13 of 14 of them, e.g. 64 tokens x 32000 x 3200: 29, 26, 35 us,
// 64 x 4096 x 4096: 12, 16, 24 us, 512 x 32000 x 3200: 103, 83, 80 us).
enum Form { NARROW, WIDE, PAIRED };
// Tokens beyond which only pairs are taken, which bounds the workspace of a score; score_stats counts on it.  Their tiles fill the GPU
// then, but not where features are few: 4096 x 128 x 4096 takes 19 us so (10 by the model), 4096 x 512 20 (13.6), 2048 x 1024 20 (13.4);
// from 2000 features on the two are the same.
constexpr int kMostSingle = 1024;

Form form_of(int M, int N) {
    const long long sms = sm_count(), m1 = (M + 127) / 128, m2 = (M + 255) / 256;
    const long long narrow = (m1 * ((N + 63) / 64) + sms - 1) / sms * 28, wide = (m1 * ((N + 127) / 128) + sms - 1) / sms * 43;
    const long long pair = (m2 * ((N + 255) / 256) + sms / 2 - 1) / (sms / 2) * 62;
    if (M > kMostSingle || (pair <= wide && pair <= narrow)) return PAIRED;
    return wide <= narrow ? WIDE : NARROW;
}

bitnet_a48_status launch_gemm(const LinearArgs& a, const ScoreArgs* score, ScoreParts* parts, cudaStream_t st) {
    switch (form_of(a.M, a.N)) {
        case NARROW: return launch<Cfg<1, 64, false>>(a, score, parts, st);
        case WIDE: return launch<Cfg<1, 128, false>>(a, score, parts, st);
        default: return launch<Cfg<2, 128, true>>(a, score, parts, st);
    }
}

size_t score_stats(int M, int N) {
    const size_t single = (size_t)(N + 63) / 64, pair = 2 * ((size_t)(N + 255) / 256);
    return (size_t)M * (M <= kMostSingle ? std::max(single, pair) : pair);
}

}  // namespace a48f8

bitnet_a48_status a48_read_gemm_fp8_status(unsigned int words_host[4]) {
    A48_CUDA_TRY(cudaMemcpyFromSymbol(words_host, g_status, sizeof(unsigned int) * 4));
    const unsigned int zero[4] = {0, 0, 0, 0};
    A48_CUDA_TRY(cudaMemcpyToSymbol(g_status, zero, sizeof(zero)));
    return BITNET_A48_OK;
}
