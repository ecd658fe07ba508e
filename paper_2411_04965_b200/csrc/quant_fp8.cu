// Rounding to e4m3 with a scale for each block of 128: of token rows (a block is 128 channels of one token, after RMSNorm
// where a gain is given) and of weights (128 x 128 entries).  With v = x * gain (or x) and a = max|v| over the block,
//   code = the e4m3 number nearest to 448 v / a, ties to even;   scale = a / 448 (times 1 / rms of the row).
// The row's size is a factor of the scale alone, so a code does not depend on the rounding of a norm.
//
// Codes are those of exact arithmetic.  t = v * (448 / a) in fp32 is off by less than 2^-21 of itself (2^-22 for the
// quotient, 2^-24 each for the product with the gain, for a and for t); where t (1 - 2^-20) and t (1 + 2^-20) round to the
// same code, so does the exact number.  The others, about one in 2^15, are redone in 64 bits, in which the product and
// 448 v are exact and the quotient has one rounding.
//
// HBM bound: every input is read once, eight entries to a thread, and stays in registers.
#include "fp8.cuh"

namespace {

using a48f8::BLOCK;

constexpr float TOP = 448.f;
constexpr float TINY = 1e-30f, HUGE_ = 1e37f;  // a block outside, where fp32 products or quotients may leave the normal range, is done in 64 bits

__device__ __forceinline__ uint32_t e4m3x2(float lo, float hi) {
    unsigned short r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}
// A 64-bit number as fp32 such that rounding that to fewer bits gives what rounding the number itself would: towards zero,
// and the last bit set where anything was cut off.
__device__ __forceinline__ float odd_float(double t) {
    const float f = __double2float_rz(t);
    return (double)f == t ? f : __uint_as_float(__float_as_uint(f) | 1u);
}

template <bool BF16>
__device__ __forceinline__ void load8(const void* X, size_t at, float (&v)[8]) {
    if (BF16) {
        const uint4 u = __ldg(reinterpret_cast<const uint4*>(reinterpret_cast<const uint16_t*>(X) + at));
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float(w[i] << 16);
            v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        }
    } else {
        const float4* p = reinterpret_cast<const float4*>(reinterpret_cast<const float*>(X) + at);
        const float4 a = __ldg(p), b = __ldg(p + 1);
        v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
    }
}

// Largest |v| as bits: a NaN is above infinity, infinity above every number.
__device__ __forceinline__ uint32_t abs_bits(const float (&v)[8]) {
    uint32_t a = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) a = max(a, __float_as_uint(v[i]) & 0x7fffffffu);
    return a;
}
__device__ __forceinline__ double abs_exact(const float (&x)[8], const float (&g)[8]) {
    double a = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) a = fmax(a, fabs((double)x[i] * (double)g[i]));
    return a;
}
// Codes from fp32 alone; false where an entry lies so near a border that 64 bits have to decide.
__device__ __forceinline__ bool fast_codes(const float (&v)[8], float a, uint2& codes) {
    const float r = __fdividef(TOP, a);  // off by 2 units in the last place
    uint32_t lo[4], hi[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float t0 = v[2 * i] * r, t1 = v[2 * i + 1] * r;
        constexpr float E = 0x1p-20f;
        lo[i] = e4m3x2(fmaf(t0, -E, t0), fmaf(t1, -E, t1));
        hi[i] = e4m3x2(fmaf(t0, E, t0), fmaf(t1, E, t1));
    }
    codes = make_uint2(lo[0] | lo[1] << 16, lo[2] | lo[3] << 16);
    return lo[0] == hi[0] && lo[1] == hi[1] && lo[2] == hi[2] && lo[3] == hi[3];
}
__device__ __forceinline__ uint2 exact_codes(const float (&x)[8], const float (&g)[8], double a) {
    uint32_t w[4] = {0, 0, 0, 0};
    if (a > 0) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            w[i] = e4m3x2(odd_float((double)x[2 * i] * (double)g[2 * i] * 448.0 / a), odd_float((double)x[2 * i + 1] * (double)g[2 * i + 1] * 448.0 / a));
    }
    return make_uint2(w[0] | w[1] << 16, w[2] | w[3] << 16);
}

// One token row to a block of threads; thread t has entries 8 t .. 8 t + 7, and those blockDim * 8 further on.  Sixteen
// neighbouring threads share a block of channels.  NV: how often eight entries to a thread cover the row (0: more than
// registers are kept for; the row is then read a second time).
template <bool BF16, bool NORM, int NV>
__global__ void __launch_bounds__(512) quant_rows_kernel(const void* __restrict__ X, long long stride, const float* __restrict__ gain, float eps, int M,
                                                         int K, uint8_t* __restrict__ codes, float* __restrict__ scale) {
    __shared__ double part[16];
    const int row = blockIdx.x, t = threadIdx.x, span = blockDim.x * 8;
    const size_t base = (size_t)row * stride;
    const int steps = NV ? NV : (K + span - 1) / span;
    float x[NV ? NV : 1][8];
    double size = 1.0;
    if (NORM) {
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < steps; ++i) {
            float(&v)[8] = x[NV ? i : 0];
            const int k = i * span + t * 8;
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = 0.f;
            if (k < K) load8<BF16>(X, base + k, v);
#pragma unroll
            for (int j = 0; j < 8; ++j) sum = fmaf(v[j], v[j], sum);
        }
        double total = sum;
#pragma unroll
        for (int o = 16; o; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
        if ((t & 31) == 0) part[t >> 5] = total;
        __syncthreads();
        total = 0;
        for (int i = 0; i < (int)blockDim.x >> 5; ++i) total += part[i];
        if (!(total > 1e-30 && total < 3e38)) {  // squares outside fp32's range: once more in 64 bits
            double wide = 0;
            for (int k = t * 8; k < K; k += span) {
                float v[8];
                load8<BF16>(X, base + k, v);
#pragma unroll
                for (int j = 0; j < 8; ++j) wide += (double)v[j] * (double)v[j];
            }
#pragma unroll
            for (int o = 16; o; o >>= 1) wide += __shfl_xor_sync(0xffffffffu, wide, o);
            __syncthreads();
            if ((t & 31) == 0) part[t >> 5] = wide;
            __syncthreads();
            total = 0;
            for (int i = 0; i < (int)blockDim.x >> 5; ++i) total += part[i];
        }
        size = rsqrt(total / K + (double)eps);
    }
#pragma unroll
    for (int i = 0; i < steps; ++i) {
        float(&v)[8] = x[NV ? i : 0];
        const int k = i * span + t * 8;
        if (k - t % 16 * 8 >= K) break;  // the same for the sixteen threads of a block of channels
        float g[8], p[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) g[j] = 1.f;
        if (!NORM || !NV) {
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = 0.f;
            if (k < K) load8<BF16>(X, base + k, v);
        }
        if (NORM && k < K) load8<false>(gain, k, g);
#pragma unroll
        for (int j = 0; j < 8; ++j) p[j] = NORM ? v[j] * g[j] : v[j];
        const uint32_t mask = 0xffffu << (t & 16);
        uint32_t bits = abs_bits(p);
#pragma unroll
        for (int o = 8; o; o >>= 1) bits = max(bits, __shfl_xor_sync(mask, bits, o));
        const float a = __uint_as_float(bits);
        const bool bad = bits >= 0x7f800000u;
        uint2 c = make_uint2(0, 0);
        const bool fine = bad || (a >= TINY && a <= HUGE_ && fast_codes(p, a, c));
        if (__any_sync(mask, !fine)) {
            double wide = abs_exact(v, g);
#pragma unroll
            for (int o = 8; o; o >>= 1) wide = fmax(wide, __shfl_xor_sync(mask, wide, o));
            if (!fine) c = exact_codes(v, g, wide);
        }
        if (bad) c = make_uint2(0, 0);
        if (k < K) *reinterpret_cast<uint2*>(codes + (size_t)row * K + k) = c;
        if ((t & 15) == 0)
            scale[(size_t)(k / BLOCK) * M + row] = bad ? __uint_as_float(0x7fc00000u) : NORM ? (float)((double)a / 448.0 * size) : __fdiv_rn(a, TOP);
    }
}

// A block of 128 x 128 weights to 256 threads; a thread has eight rows' eight entries.
template <bool BF16>
__global__ void __launch_bounds__(256) quant_weight_kernel(const void* __restrict__ W, long long stride, int N, int K, int kb, uint8_t* __restrict__ codes,
                                                           float* __restrict__ scale) {
    __shared__ uint32_t part[8];
    const int nb = blockIdx.x / kb, b = blockIdx.x - nb * kb, t = threadIdx.x;
    const int k = b * BLOCK + t % 16 * 8, n0 = nb * BLOCK + t / 16;
    float v[8][8];
    uint32_t bits = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[i][j] = 0.f;
        if (k < K && n0 + 16 * i < N) load8<BF16>(W, (size_t)(n0 + 16 * i) * stride + k, v[i]);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) bits = max(bits, abs_bits(v[i]));
    bits = __reduce_max_sync(0xffffffffu, bits);
    if ((t & 31) == 0) part[t >> 5] = bits;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 8; ++i) bits = max(bits, part[i]);
    const float a = __uint_as_float(bits);
    const bool bad = bits >= 0x7f800000u;
    const float ones[8] = {1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        uint2 c = make_uint2(0, 0);
        if (!bad && !(a >= TINY && a <= HUGE_ && fast_codes(v[i], a, c))) c = exact_codes(v[i], ones, (double)a);
        if (k < K && n0 + 16 * i < N) *reinterpret_cast<uint2*>(codes + (size_t)(n0 + 16 * i) * K + k) = c;
    }
    if (t == 0) scale[blockIdx.x] = bad ? __uint_as_float(0x7fc00000u) : __fdiv_rn(a, TOP);
}

template <bool BF16, bool NORM>
cudaError_t launch_rows(const void* X, long long stride, const float* gain, float eps, int M, int K, uint8_t* codes, float* scale, cudaStream_t st) {
    // threads for eight entries each, at most 256 of them twice or four times: more rows to an SM, more loads under way
    const int eights = (K + 7) / 8, threads = eights <= 256 ? a48_round_up(eights, 32) : 256, nv = (eights + threads - 1) / threads;
    if (nv == 1) quant_rows_kernel<BF16, NORM, 1><<<M, threads, 0, st>>>(X, stride, gain, eps, M, K, codes, scale);
    else if (nv == 2) quant_rows_kernel<BF16, NORM, 2><<<M, threads, 0, st>>>(X, stride, gain, eps, M, K, codes, scale);
    else if (nv <= 4) quant_rows_kernel<BF16, NORM, 4><<<M, threads, 0, st>>>(X, stride, gain, eps, M, K, codes, scale);
    else quant_rows_kernel<BF16, NORM, 0><<<M, threads, 0, st>>>(X, stride, gain, eps, M, K, codes, scale);
    return cudaGetLastError();
}

}  // namespace

namespace a48f8 {

bitnet_a48_status launch_quant_rows(const void* X, int bf16, long long stride, const float* gain, float eps, int M, int K, uint8_t* codes, float* scale,
                                    cudaStream_t st) {
    A48_CUDA_TRY(bf16 ? (gain ? launch_rows<true, true>(X, stride, gain, eps, M, K, codes, scale, st) : launch_rows<true, false>(X, stride, gain, eps, M, K, codes, scale, st))
                      : (gain ? launch_rows<false, true>(X, stride, gain, eps, M, K, codes, scale, st) : launch_rows<false, false>(X, stride, gain, eps, M, K, codes, scale, st)));
    return BITNET_A48_OK;
}

bitnet_a48_status launch_quant_weight(const void* W, int bf16, long long stride, int N, int K, uint8_t* codes, float* scale, cudaStream_t st) {
    const int kb = blocks(K);
    const unsigned grid = (unsigned)(blocks(N) * kb);
    if (bf16) quant_weight_kernel<true><<<grid, 256, 0, st>>>(W, stride, N, K, kb, codes, scale);
    else quant_weight_kernel<false><<<grid, 256, 0, st>>>(W, stride, N, K, kb, codes, scale);
    A48_CUDA_TRY(cudaGetLastError());
    return BITNET_A48_OK;
}

}  // namespace a48f8
