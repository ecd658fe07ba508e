// The product of gemm_fp8.cu for few tokens, where reading the weight is all that counts.  A warp takes 16 weight rows and
// streams them, 128 channels (2 KB) at a time, through registers: four such blocks are under way while one is multiplied
// (mma.sync m16n8k32; its rate does not matter here, and its operands come straight from loads of 16 bytes).  The order of the
// channels in a block is free, so a lane takes 2 x 16 consecutive bytes of its weight rows and of its token instead of the
// order that the instruction names.  The tokens' codes and scales sit in shared memory for the life of the block of threads.
//
// With fewer groups of 16 rows than there are warps, a group is split over 2 .. 16 warps of a block by its channels; they add
// their sums in shared memory, always in the same order.
#include <algorithm>

#include "fp8.cuh"

namespace {

using a48f8::BLOCK;
using a48f8::LinearArgs;

constexpr int AHEAD = 4;
// Warps of a block: as many as have the registers for their sums.
__host__ __device__ constexpr int warps_of(int nt) { return nt <= 2 ? 16 : 8; }
constexpr int SMEM_MOST = 226 * 1024;

__device__ __forceinline__ void mma_e4m3(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k32.row.col.f32.e4m3.e4m3.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Read once and not by neighbours; the row goes on where these bytes end, so L2 is to take 256 at a time from memory (26.7 us
// for 28.7 without, one token, 32000 x 4096).
__device__ __forceinline__ uint4 load_once(const uint8_t* p) {
    uint4 v;
    asm volatile("ld.global.nc.L1::no_allocate.L2::256B.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}

struct Params {
    const uint8_t* x;
    const float* xs;
    const uint8_t* w;
    const float* ws;
    void* y;
    long long y_stride;
    int M, N, K, kb, y_bf16;
    int split, rounds;  // warps to a group of 16 rows; groups to a warp
    int x_row;          // bytes from token to token in shared memory
};

template <int NT>
__global__ void __launch_bounds__(32 * warps_of(NT), 1) rows_fp8_kernel(const Params p) {
    constexpr int WARPS = warps_of(NT), THREADS = 32 * WARPS;
    extern __shared__ __align__(16) uint8_t smem[];
    const int t = threadIdx.x, warp = t >> 5, lane = t & 31, g = lane >> 2, q = lane & 3;
    float* xs_s = reinterpret_cast<float*>(smem);                                   // [kb][8 NT]
    uint8_t* x_s = smem + (size_t)p.kb * 8 * NT * 4;                                // [8 NT][x_row]
    float* part = reinterpret_cast<float*>(x_s + (size_t)8 * NT * p.x_row);         // [WARPS][8 NT][16], with split > 1
    const int slot = warp / p.split, share = warp - slot * p.split, slots = WARPS / p.split;
    const int groups = (p.N + 15) / 16, mine = (p.kb - share + p.split - 1) / p.split;  // blocks of channels of this warp: share, share + split, ..
    const int total = mine * p.rounds;
    const uint4 zero = make_uint4(0, 0, 0, 0);

    uint4 ring[AHEAD][4];
    int next_round = 0, next_i = 0;
    auto load = [&](uint4(&to)[4]) {
        const int group = (next_round * slots + slot) * (int)gridDim.x + (int)blockIdx.x, b = share + next_i * p.split;
        const bool on = next_round < p.rounds && group < groups;
        const uint8_t* lo = p.w + (size_t)min(group * 16 + g, p.N - 1) * p.K;
        const uint8_t* hi = p.w + (size_t)min(group * 16 + g + 8, p.N - 1) * p.K;
        const int k0 = b * BLOCK + q * 16, k1 = k0 + 64;
        to[0] = on && k0 < p.K ? load_once(lo + k0) : zero;
        to[1] = on && k0 < p.K ? load_once(hi + k0) : zero;
        to[2] = on && k1 < p.K ? load_once(lo + k1) : zero;
        to[3] = on && k1 < p.K ? load_once(hi + k1) : zero;
        if (++next_i == mine) {
            next_i = 0;
            ++next_round;
        }
    };
    a48_pdl_prologue();
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) load(ring[u]);

    // tokens: whole blocks of channels (zeros behind the last one), rows 64 bytes further apart than a multiple of 128 so that
    // the eight lanes of a phase read all banks; rows past the last token hold anything, and so do their columns of the result
    const int vectors = p.kb * (BLOCK / 16);
#pragma unroll 8
    for (int i = t; i < p.M * vectors; i += THREADS) {
        const int m = i / vectors, v = i - m * vectors;
        *reinterpret_cast<uint4*>(x_s + (size_t)m * p.x_row + v * 16) =
            v * 16 < p.K ? __ldg(reinterpret_cast<const uint4*>(p.x + (size_t)m * p.K + v * 16)) : zero;
    }
#pragma unroll 4
    for (int i = t; i < p.kb * 8 * NT; i += THREADS) {
        const int b = i / (8 * NT), m = i - b * (8 * NT);
        xs_s[i] = m < p.M ? __ldg(p.xs + (size_t)b * p.M + m) : 0.f;
    }
    __syncthreads();

    float sum[NT][4];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int j = 0; j < 4; ++j) sum[n][j] = 0.f;
    auto store = [&](int m, int n, float v) {
        if (m < p.M && n < p.N) {
            if (p.y_bf16) reinterpret_cast<__nv_bfloat16*>(p.y)[(size_t)m * p.y_stride + n] = __float2bfloat16_rn(v);
            else reinterpret_cast<float*>(p.y)[(size_t)m * p.y_stride + n] = v;
        }
    };
    int round = 0, i = 0;
    for (int step = 0; step < total; step += AHEAD) {
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            if (step + u >= total) break;
            const int group = (round * slots + slot) * (int)gridDim.x + (int)blockIdx.x, b = share + i * p.split;
            const float w_scale = __ldg(p.ws + (size_t)(min(group * 16, p.N - 1) / BLOCK) * p.kb + b);
            const uint32_t wl[8] = {ring[u][0].x, ring[u][0].y, ring[u][0].z, ring[u][0].w, ring[u][2].x, ring[u][2].y, ring[u][2].z, ring[u][2].w};
            const uint32_t wh[8] = {ring[u][1].x, ring[u][1].y, ring[u][1].z, ring[u][1].w, ring[u][3].x, ring[u][3].y, ring[u][3].z, ring[u][3].w};
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const uint8_t* at = x_s + (size_t)(n * 8 + g) * p.x_row + b * BLOCK + q * 16;
                const uint4 x0 = *reinterpret_cast<const uint4*>(at), x1 = *reinterpret_cast<const uint4*>(at + 64);
                const uint32_t xw[8] = {x0.x, x0.y, x0.z, x0.w, x1.x, x1.y, x1.z, x1.w};
                float d[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int j = 0; j < 4; ++j) mma_e4m3(d, wl[2 * j], wh[2 * j], wl[2 * j + 1], wh[2 * j + 1], xw[2 * j], xw[2 * j + 1]);
                const float2 s = *reinterpret_cast<const float2*>(xs_s + b * 8 * NT + n * 8 + 2 * q);
                sum[n][0] = fmaf(d[0], s.x * w_scale, sum[n][0]);
                sum[n][1] = fmaf(d[1], s.y * w_scale, sum[n][1]);
                sum[n][2] = fmaf(d[2], s.x * w_scale, sum[n][2]);
                sum[n][3] = fmaf(d[3], s.y * w_scale, sum[n][3]);
            }
            load(ring[u]);
            if (++i == mine) {  // this warp's part of the group's 16 rows is done
                i = 0;
                ++round;
                if (p.split == 1) {
                    if (group < groups) {
#pragma unroll
                        for (int n = 0; n < NT; ++n)
#pragma unroll
                            for (int j = 0; j < 4; ++j) store(n * 8 + 2 * q + (j & 1), group * 16 + g + (j >> 1) * 8, sum[n][j]);
                    }
                } else {
#pragma unroll
                    for (int n = 0; n < NT; ++n)
#pragma unroll
                        for (int j = 0; j < 4; ++j) part[((size_t)warp * 8 * NT + n * 8 + 2 * q + (j & 1)) * 16 + g + (j >> 1) * 8] = sum[n][j];
                    __syncthreads();
                    for (int e = t; e < slots * 8 * NT * 16; e += THREADS) {
                        const int row = e & 15, m = (e >> 4) % (8 * NT), of = e / (16 * 8 * NT);
                        float v = 0.f;
                        for (int k = 0; k < p.split; ++k) v += part[((size_t)(of * p.split + k) * 8 * NT + m) * 16 + row];
                        store(m, (((round - 1) * slots + of) * (int)gridDim.x + (int)blockIdx.x) * 16 + row, v);
                    }
                    __syncthreads();
                }
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int j = 0; j < 4; ++j) sum[n][j] = 0.f;
            }
        }
    }
}

size_t smem_bytes(int nt, int K, int split) {
    const size_t kb = a48f8::blocks(K);
    return kb * 8 * nt * 4 + (size_t)8 * nt * (kb * BLOCK + 64) + (split > 1 ? (size_t)warps_of(nt) * 8 * nt * 16 * 4 : 0);
}
int tiles_of(int M) { return M <= 8 ? 1 : M <= 16 ? 2 : 4; }

template <int NT>
bitnet_a48_status launch(const LinearArgs& a, cudaStream_t st) {
    static std::atomic<bool> ready[64];
    A48_CUDA_TRY(a48_allow_smem(rows_fp8_kernel<NT>, SMEM_MOST, ready));
    const int sms = a48f8::sm_count(), kb = a48f8::blocks(a.K), groups = (a.N + 15) / 16;
    // The split that leaves a warp the fewest blocks of channels; a round costs about half a block for the stores, and twice that
    // where sums are joined.
    int split = 1, rounds = 1;
    long long best = -1;
    constexpr int WARPS = warps_of(NT);
    for (int s = 1; s <= WARPS && s <= kb; s *= 2) {
        const int at_once = std::min(groups, sms) * (WARPS / s), r = (groups + at_once - 1) / at_once;
        const long long cost = (long long)r * (2 * ((kb + s - 1) / s) + (s > 1 ? 2 : 1));
        if (best < 0 || cost < best) {
            best = cost;
            split = s;
            rounds = r;
        }
    }
    Params p = {a.x, a.xs, a.w, a.ws, a.y, a.y_stride, a.M, a.N, a.K, kb, a.y_bf16, split, rounds, kb * BLOCK + 64};
    A48_CUDA_TRY(a48_launch_pdl(rows_fp8_kernel<NT>, dim3(std::min(groups, sms)), dim3(32 * WARPS), smem_bytes(NT, a.K, split), st, p));
    return BITNET_A48_OK;
}

}  // namespace

namespace a48f8 {

bool few_supported(int M, int K) { return M <= 32 && smem_bytes(tiles_of(M), K, 2) <= (size_t)SMEM_MOST; }

bitnet_a48_status launch_few(const LinearArgs& a, cudaStream_t st) {
    switch (tiles_of(a.M)) {
        case 1: return launch<1>(a, st);
        case 2: return launch<2>(a, st);
        default: return launch<4>(a, st);
    }
}

}  // namespace a48f8
