// Product of two e4m3 matrices with a scale for each block of 128 channels, on the fifth-generation tensor cores:
//   y[m, n] = sum over blocks b of  xs[b][m] * ws[n / 128][b] * (sum over k in b of x[m, k] * w[n, k]).
//
// The scales change every 128 channels, so the tensor core's accumulator holds one block's products only: each block is a
// fresh accumulation (four MMAs of 32 channels) into one of the buffers in tensor memory, and the epilogue warps multiply it by its
// scale and add it to sums in registers.  Tokens are the rows of the tile (a thread of the epilogue has one token) and
// output features its columns: a column block of 128 shares ws, so a thread's factor for a block is one number, and a
// block costs it one packed multiply-add per two features.
#include <algorithm>

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

// AR: rows of the token tile that a stage has room for (the MMA reads 128; what lies behind belongs to tokens that do not
// exist); BN: features of a tile; PAIR: two CTAs share a tile of 256 tokens, each holds half of the weight rows.
template <int AR_, int BN_, bool PAIR_>
struct Cfg {
    static constexpr int AR = AR_, BN = BN_;
    static constexpr bool PAIR = PAIR_;
    static constexpr int CTAS = PAIR ? 2 : 1, TM = 128 * CTAS;
    static constexpr int BROWS = BN / CTAS;
    static constexpr int A_BYTES = AR * BLOCK, B_BYTES = BROWS * BLOCK, STAGE_BYTES = A_BYTES + B_BYTES;
    static constexpr int SLACK = AR < 128 ? (128 - AR) * BLOCK : 0;
    static constexpr int MAX_STAGES = (220 * 1024 - SLACK) / STAGE_BYTES;
    static constexpr int STAGES = MAX_STAGES < 16 ? MAX_STAGES : 16;
    static constexpr int ACC_BUFS = TMEM_COLS / BN < 8 ? TMEM_COLS / BN : 8;
    static constexpr int EPI_SPLIT = BN >= 64 ? 2 : 1;
    static constexpr int COLS = BN / EPI_SPLIT;  // of one thread
    static constexpr int NUM_THREADS = 32 * (2 + 4 * EPI_SPLIT);
    static constexpr int SMEM_BYTES = STAGES * STAGE_BYTES + SLACK + 1024 /*alignment*/ + 512 /*barriers*/;
    static_assert(COLS % 32 == 0 && COLS <= BLOCK, "a thread's columns share a weight scale");
    static_assert(SMEM_BYTES <= 227 * 1024, "shared memory");
    static_assert(8 * (2 * STAGES + 2 * ACC_BUFS) <= 480, "barriers");
};

struct Params {
    const float* xs;
    const float* ws;
    void* y;
    long long y_stride;
    int M, N, kb, m_tiles, tiles, x_rows, y_bf16, y_vec;
    const void* tokens;  // the rest: products that keep sums of their logits
    int tokens64;
    float c;
    float4* stats;
    float* owns;
};

template <class C, bool SCORE>
__global__ void __launch_bounds__(C::NUM_THREADS, 1)
    gemm_fp8_kernel(const __grid_constant__ CUtensorMap tm_x, const __grid_constant__ CUtensorMap tm_w, const Params p) {
    constexpr int STAGES = C::STAGES, ACC_BUFS = C::ACC_BUFS, BN = C::BN, COLS = C::COLS;
    constexpr bool PAIR = C::PAIR;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    uint8_t* ctrl = smem + STAGES * C::STAGE_BYTES + C::SLACK;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(ctrl + 480);
    volatile uint32_t* abort_flag = reinterpret_cast<volatile uint32_t*>(ctrl + 484);
    const uint32_t bar_full = smem_u32(ctrl), bar_empty = bar_full + 8 * STAGES;
    const uint32_t bar_acc_full = bar_empty + 8 * STAGES, bar_acc_empty = bar_acc_full + 8 * ACC_BUFS;
    const uint32_t smem_base = smem_u32(smem);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = PAIR ? (int)(blockIdx.x & 1u) : 0;
    const int unit = PAIR ? (int)(blockIdx.x >> 1) : (int)blockIdx.x, units = (int)gridDim.x / C::CTAS;

    if (threadIdx.x == 0) {
        asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&tm_x)) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&tm_w)) : "memory");
        for (int s = 0; s < STAGES; ++s) {
            mbar_init(bar_full + 8 * s, 1);
            mbar_init(bar_empty + 8 * s, 1);
        }
        for (int b = 0; b < ACC_BUFS; ++b) {
            mbar_init(bar_acc_full + 8 * b, 1);
            mbar_init(bar_acc_empty + 8 * b, C::CTAS * 4 * C::EPI_SPLIT);  // one arrival per epilogue warp
        }
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) tc_alloc<PAIR>(smem_u32(tmem_slot), TMEM_COLS);
    tc_fence_before();
    __syncthreads();
    if (PAIR) cluster_sync_all();
    tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;

    if (warp == 0) {
        // ------------------------------------------------------------- tensor copies
        uint32_t it = 0, s = 0, ph = 0;
        bool ok = true;
        const uint32_t full0 = PAIR ? map_to_rank(bar_full, 0) : bar_full;  // the pair's copies all report to rank 0
        for (int tile = unit; tile < p.tiles && ok; tile += units) {
            const int nt = tile / p.m_tiles, mt = tile - nt * p.m_tiles;
            const int m0 = mt * C::TM + rank * 128, n0 = nt * BN + rank * C::BROWS;
            for (int b = 0; b < p.kb; ++b, ++it) {
                ok = __all_sync(0xffffffffu, mbar_wait(bar_empty + 8 * s, ph ^ 1, abort_flag, 1, it));
                if (!ok) break;
                if (lane == 0) {
                    const uint32_t dst = smem_base + s * C::STAGE_BYTES;
                    if (rank == 0) mbar_expect_tx(bar_full + 8 * s, (uint32_t)(C::CTAS * (p.x_rows * BLOCK + C::B_BYTES)));
                    if (PAIR) {
                        tma_load_2d_pair(dst, &tm_x, b * BLOCK, m0, full0 + 8 * s);
                        tma_load_2d_pair(dst + C::A_BYTES, &tm_w, b * BLOCK, n0, full0 + 8 * s);
                    } else {
                        tma_load_2d(dst + C::A_BYTES, &tm_w, b * BLOCK, n0, full0 + 8 * s);
                        tma_load_2d(dst, &tm_x, b * BLOCK, m0, full0 + 8 * s);
                    }
                }
                __syncwarp();
                if (++s == (uint32_t)STAGES) { s = 0; ph ^= 1; }
            }
        }
        if (!ok && lane == 0) {  // let the copies already issued land before the CTA exits
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
    } else if (warp == 1) {
        // ------------------------------------------------------------- MMAs (of a pair: rank 0 for both)
        if (rank == 0) {
            constexpr uint32_t idesc = idesc_e4m3(C::TM, BN);
            const bool leader = elect_one();
            uint32_t it = 0, s = 0, ph = 0, a = 0, pa = 0;
            bool ok = true;
            for (int tile = unit; tile < p.tiles && ok; tile += units) {
                for (int b = 0; b < p.kb; ++b, ++it) {
                    ok = __all_sync(0xffffffffu, mbar_wait(bar_acc_empty + 8 * a, pa ^ 1, abort_flag, 2, it));
                    if (!ok) break;
                    ok = __all_sync(0xffffffffu, mbar_wait(bar_full + 8 * s, ph, abort_flag, 3, it));
                    if (!ok) break;
                    tc_fence_after();
                    if (leader) {
                        const uint64_t a_desc = smem_desc_sw128(smem_base + s * C::STAGE_BYTES);
                        const uint64_t b_desc = smem_desc_sw128(smem_base + s * C::STAGE_BYTES + C::A_BYTES);
#pragma unroll
                        for (int j = 0; j < 4; ++j) mma_f8<PAIR>(tmem_base + a * BN, a_desc + 2 * j, b_desc + 2 * j, idesc, j > 0);
                        tc_commit<PAIR>(bar_empty + 8 * s);
                        tc_commit<PAIR>(bar_acc_full + 8 * a);
                    }
                    __syncwarp();
                    if (++s == (uint32_t)STAGES) { s = 0; ph ^= 1; }
                    if (++a == (uint32_t)ACC_BUFS) { a = 0; pa ^= 1; }
                }
            }
        }
    } else {
        // ------------------------------------------------------------- scales, sums, stores
        const int quad = warp & 3, col0 = ((warp - 2) >> 2) * COLS;
        const uint32_t t_lanes = tmem_base + ((uint32_t)(quad * 32) << 16) + col0;
        const uint32_t acc_empty0 = PAIR ? map_to_rank(bar_acc_empty, 0) : bar_acc_empty;
        uint32_t it = 0, a = 0, pa = 0;
        bool ok = true;
        Sums run;  // SCORE with one tile of tokens: over all tiles of this CTA
        run.start(-INFINITY);
        for (int tile = unit; tile < p.tiles && ok; tile += units) {
            const int nt = tile / p.m_tiles, mt = tile - nt * p.m_tiles;
            const int m0 = mt * C::TM + rank * 128 + quad * 32, m = m0 + lane, n0 = nt * BN + col0;
            const bool live = m0 < p.M && n0 < p.N;  // the same for the whole warp
            const float* xs = p.xs + min(m, p.M - 1);
            const float* ws = p.ws + (size_t)(min(n0, p.N - 1) / BLOCK) * p.kb;
            float scale = __ldg(xs) * __ldg(ws);
            f32x2 sum[COLS / 2];
#pragma unroll
            for (int c = 0; c < COLS / 2; ++c) sum[c] = 0;
            for (int b = 0; b < p.kb; ++b, ++it) {
                const int next = min(b + 1, p.kb - 1);
                const float scale_next = __ldg(xs + (size_t)next * p.M) * __ldg(ws + next);
                ok = __all_sync(0xffffffffu, mbar_wait(bar_acc_full + 8 * a, pa, abort_flag, 4, it));
                if (!ok) break;
                tc_fence_after();
                const f32x2 s2 = pack2(scale, scale);
                if (live) {
#pragma unroll
                    for (int c = 0; c < COLS; c += 32) {
                        uint32_t r[32];
                        tmem_ld32(t_lanes + a * BN + c, r);
                        tc_wait_ld();
#pragma unroll
                        for (int j = 0; j < 16; ++j)
                            sum[c / 2 + j] = fma2(pack2(__uint_as_float(r[2 * j]), __uint_as_float(r[2 * j + 1])), s2, sum[c / 2 + j]);
                    }
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) {
                    if (PAIR) mbar_arrive_cluster(acc_empty0 + 8 * a);
                    else mbar_arrive(acc_empty0 + 8 * a);
                }
                scale = scale_next;
                if (++a == (uint32_t)ACC_BUFS) { a = 0; pa ^= 1; }
            }
            if (!ok || m >= p.M) continue;
            const int cols = min(COLS, p.N - n0);
            if (SCORE) {
                Sums mine;
                mine.start(-INFINITY);
                if (live) {
                    float top = -INFINITY;
#pragma unroll
                    for (int c = 0; c < COLS; c += 2) {
                        float lo, hi;
                        unpack2(sum[c / 2], lo, hi);
                        if (c < cols) top = fmaxf(top, lo);
                        if (c + 1 < cols) top = fmaxf(top, hi);
                    }
                    mine.start(top);
                    const long long token = p.tokens64 ? __ldg(reinterpret_cast<const long long*>(p.tokens) + m) : __ldg(reinterpret_cast<const int*>(p.tokens) + m);
                    const long long at = token - n0;
#pragma unroll
                    for (int c = 0; c < COLS; c += 2) {
                        float lo, hi;
                        unpack2(sum[c / 2], lo, hi);
                        if (c < cols) mine.add(lo, p.c);
                        if (c + 1 < cols) mine.add(hi, p.c);
                    }
                    if (at >= 0 && at < cols) {
#pragma unroll
                        for (int c = 0; c < COLS; c += 2) {
                            float lo, hi;
                            unpack2(sum[c / 2], lo, hi);
                            if (at == c) p.owns[m] = lo;
                            if (at == c + 1) p.owns[m] = hi;
                        }
                    }
                }
                if (p.m_tiles > 1) {
                    p.stats[(size_t)(nt * C::EPI_SPLIT + col0 / COLS) * p.M + m] = make_float4(mine.r, mine.s, mine.d, 0.f);
                } else {
                    run.join(mine, p.c);
                    if (tile + units >= p.tiles) p.stats[(size_t)(unit * C::EPI_SPLIT + col0 / COLS) * p.M + m] = make_float4(run.r, run.s, run.d, 0.f);
                }
                continue;
            }
            if (!live) continue;
            if (p.y_bf16) {
                __nv_bfloat16* y = reinterpret_cast<__nv_bfloat16*>(p.y) + (size_t)m * p.y_stride + n0;
                if (p.y_vec && cols == COLS) {
#pragma unroll
                    for (int c = 0; c < COLS; c += 8) {
                        uint32_t v[4];
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            float lo, hi;
                            unpack2(sum[c / 2 + j], lo, hi);
                            asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(v[j]) : "f"(hi), "f"(lo));
                        }
                        *reinterpret_cast<uint4*>(y + c) = make_uint4(v[0], v[1], v[2], v[3]);
                    }
                } else {
#pragma unroll
                    for (int c = 0; c < COLS; c += 2) {
                        float lo, hi;
                        unpack2(sum[c / 2], lo, hi);
                        if (c < cols) y[c] = __float2bfloat16_rn(lo);
                        if (c + 1 < cols) y[c + 1] = __float2bfloat16_rn(hi);
                    }
                }
            } else {
                float* y = reinterpret_cast<float*>(p.y) + (size_t)m * p.y_stride + n0;
                if (p.y_vec && cols == COLS) {
#pragma unroll
                    for (int c = 0; c < COLS; c += 4) {
                        float4 v;
                        unpack2(sum[c / 2], v.x, v.y);
                        unpack2(sum[c / 2 + 1], v.z, v.w);
                        *reinterpret_cast<float4*>(y + c) = v;
                    }
                } else {
#pragma unroll
                    for (int c = 0; c < COLS; c += 2) {
                        float lo, hi;
                        unpack2(sum[c / 2], lo, hi);
                        if (c < cols) y[c] = lo;
                        if (c + 1 < cols) y[c + 1] = hi;
                    }
                }
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (PAIR) cluster_sync_all();  // both CTAs are done with both tensor memories and with each other's barriers
    if (warp == 1) {
        tc_fence_after();
        tc_dealloc<PAIR>(tmem_base, TMEM_COLS);
    }
}

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

template <class C, bool SCORE>
bitnet_a48_status launch(const LinearArgs& a, const ScoreArgs* score, ScoreParts* parts, cudaStream_t st) {
    static std::atomic<bool> ready[64];
    A48_CUDA_TRY(a48_allow_smem(gemm_fp8_kernel<C, SCORE>, C::SMEM_BYTES, ready));
    CUtensorMap tm_x, tm_w;
    const int x_rows = std::min((a.M + 7) / 8 * 8, C::AR);
    if (!make_byte_map(&tm_x, a.x, (uint64_t)a.M, (uint64_t)a.K, (uint64_t)a.K, (uint32_t)x_rows) ||
        !make_byte_map(&tm_w, a.w, (uint64_t)a.N, (uint64_t)a.K, (uint64_t)a.K, (uint32_t)C::BROWS))
        return BITNET_A48_ERR_CUDA;
    Params p = {};
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
    p.y_vec = a48_aligned16(a.y) && a.y_stride % (a.y_bf16 ? 8 : 4) == 0;
    const int slots = sm_count() / C::CTAS;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(std::min(p.tiles, slots) * C::CTAS));
    cfg.blockDim = dim3(C::NUM_THREADS);
    cfg.dynamicSmemBytes = C::SMEM_BYTES;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    if (C::PAIR) {
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = 2;
        attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
    }
    if (SCORE) {
        p.tokens = score->tokens;
        p.tokens64 = score->tokens64;
        p.c = score->c;
        p.stats = parts->stats;
        p.owns = parts->owns;
        parts->parts = C::EPI_SPLIT * (p.m_tiles > 1 ? (a.N + C::BN - 1) / C::BN : (int)cfg.gridDim.x / C::CTAS);
    }
    A48_CUDA_TRY(cudaLaunchKernelEx(&cfg, gemm_fp8_kernel<C, SCORE>, tm_x, tm_w, p));
    return BITNET_A48_OK;
}

template <class C>
bitnet_a48_status launch(const LinearArgs& a, const ScoreArgs* score, ScoreParts* parts, cudaStream_t st) {
    return score ? launch<C, true>(a, score, parts, st) : launch<C, false>(a, score, parts, st);
}

}  // namespace

namespace a48f8 {

bitnet_a48_status launch_gemm(const LinearArgs& a, const ScoreArgs* score, ScoreParts* parts, cudaStream_t st) {
    if (a.M <= 32) return launch<Cfg<32, 32, false>>(a, score, parts, st);
    if (a.M <= 64) return launch<Cfg<64, 64, false>>(a, score, parts, st);
    if (a.M <= 128) return launch<Cfg<128, 128, false>>(a, score, parts, st);
    return launch<Cfg<128, 256, true>>(a, score, parts, st);
}

size_t score_stats(int M, int N) {
    // one tile of tokens: a part to each half of the columns of a CTA, of which there are no more than 512 and no more than
    // tiles of 32; more: one to each 128 columns
    const size_t parts = M <= 128 ? std::min<size_t>(1024, 2 * ((N + 31) / 32)) : 2 * (size_t)((N + 255) / 256);
    return parts * M;
}

}  // namespace a48f8

bitnet_a48_status a48_read_gemm_fp8_status(unsigned int words_host[4]) {
    A48_CUDA_TRY(cudaMemcpyFromSymbol(words_host, g_status, sizeof(unsigned int) * 4));
    const unsigned int zero[4] = {0, 0, 0, 0};
    A48_CUDA_TRY(cudaMemcpyToSymbol(g_status, zero, sizeof(zero)));
    return BITNET_A48_OK;
}
