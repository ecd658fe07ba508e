// Rounding to e4m3 with a scale for each block of 128: of token rows (a block is 128 channels of one token, after RMSNorm
// where a gain is given) and of weights (128 x 128 entries).  With v = x * gain (or x) and a = max|v| over the block,
//   code = the e4m3 number nearest to 448 v / a, ties to even;   scale = a / 448 (times 1 / rms of the row).
// The row's size is a factor of the scale alone, so a code does not depend on the rounding of a norm.
//
// Codes are those of exact arithmetic.  v * (448 / a) in fp32 is off by at most 5 * 2^-24 of itself (the product with the gain, a,
// the quotient, the factor and the product, a rounding each); where it rounds to the same code with a factor 3 * 2^-23 smaller and
// 3 * 2^-23 larger, so does the exact number.  For the others, about one in 10^5, 448 v is compared with a times the
// border between the two codes, as sums of a few fp32 numbers each, exactly.  In 64 bits this took registers from the rest: 95 us
// for 16384 rows of 4096 with a gain.  Blocks outside fp32's middle range are brought there by a power of two first.
//
// Every input is read once, eight entries to a thread, and stays in registers.  With a gain instructions bound it (29 an entry, 65% of
// the issue slots with DRAM at 45%), without one memory does nearly (16384 x 4096 fp32 55 us, the bytes alone 51).
#include <cuda_fp16.h>

#include "fp8.cuh"
#include "softmax_sums.cuh"

namespace {

using a48f8::BLOCK;
using a48f8::max_nan;

constexpr float TOP = 448.f;
// Outside, fp32 products (448 times an entry among them), quotients, or what is left of products may leave fp32's range.
constexpr float TINY = 1e-24f, HUGE_ = 5e35f;

__device__ __forceinline__ uint32_t e4m3x2(float lo, float hi) {
    unsigned short r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}
// Eight entries as they are in memory.
template <bool BF16>
struct Raw {
    uint4 u[BF16 ? 1 : 2];
    __device__ __forceinline__ void load(const void* X, size_t at) {
        const uint4* p = reinterpret_cast<const uint4*>(reinterpret_cast<const char*>(X) + at * (BF16 ? 2 : 4));
#pragma unroll
        for (int i = 0; i < (BF16 ? 1 : 2); ++i) u[i] = __ldg(p + i);
    }
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int i = 0; i < (BF16 ? 1 : 2); ++i) u[i] = make_uint4(0, 0, 0, 0);
    }
    __device__ __forceinline__ void widen(float (&v)[8]) const {
        if (BF16) {
            const uint32_t w[4] = {u[0].x, u[0].y, u[0].z, u[0].w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                v[2 * i] = __uint_as_float(w[i] << 16);
                v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
            }
        } else {
            const uint4 a = u[0], b = u[BF16 ? 0 : 1];
            const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(w[i]);
        }
    }
};

__device__ __forceinline__ float abs_max(const float (&v)[8], float a) {
#pragma unroll
    for (int i = 0; i < 8; ++i) a = max_nan(a, fabsf(v[i]));
    return a;
}
// Values of two codes.
__device__ __forceinline__ float2 of_e4m3x2(uint32_t c) {
    uint32_t h;
    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h) : "h"((unsigned short)c));
    return __half22float2(*reinterpret_cast<const __half2*>(&h));
}
__device__ __forceinline__ bool middle_range(float a) { return a >= TINY && a <= HUGE_; }
// The power of two that brings a into the middle range (what is lost of entries far below a huge a is no part of their code).
__device__ __forceinline__ float to_middle(float a) { return a < TINY ? 0x1p100f : a > HUGE_ ? 0x1p-64f : 1.f; }
// up * v * g as two factors that stay in range and lose nothing of what counts: a tiny product may have a huge entry and a subnormal
// gain (or none: 0), so the power goes to the gain where the entry is 1 or more, and to the entry below.
struct Factors {
    float v, g;
};
__device__ __forceinline__ Factors scaled(float v, float g, float up) { return fabsf(v) >= 1.f ? Factors{v, g * up} : Factors{v * up, g}; }
// What fp32 leaves of that product, p.
__device__ __forceinline__ float rest_of(float v, float g, float p, float up) {
    const Factors f = scaled(v, g, up);
    return fmaf(f.v, f.g, -p);
}

// Codes of bf16 numbers v and their largest a, in fp32: 448 v has 11 bits, and a quotient so near a border (5 bits) that it is not
// on it would need 448 v and a times the border, 13 bits at most, to differ by less than they can.  So only quotients on a border
// have to come out exactly, and one step of refinement, q - (q a - 448 v) / a, does that.  (They are frequent: 448 = 7 * 64, and
// one border in eight is a multiple of 7 * 3.)
__device__ __forceinline__ void bf16_codes(const float (&v)[8], float a, uint32_t (&c)[4]) {
    const float s = to_middle(a), n448 = TOP * s, b = a * s, r = __fdividef(1.f, b);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float q[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const float n = v[2 * i + j] * n448, first = n * r;
            q[j] = fmaf(-fmaf(first, b, -n), r, first);  // in this form -0 stays -0
        }
        c[i] = e4m3x2(q[0], q[1]);
    }
}

// Codes from fp32 alone, a in the middle range, with the smaller and the larger factor; false where they differ.
__device__ __forceinline__ bool fast_codes(const float (&v)[8], float a, uint32_t (&lo)[4], uint32_t (&hi)[4]) {
    const float i = __fdividef(1.f, a), first = TOP * i, r = fmaf(fmaf(-first, a, TOP), i, first);  // a step of refinement: 2^-24
    const float less = r * (1.f - 3 * 0x1p-23f), more = r * (1.f + 3 * 0x1p-23f);
    uint32_t differ = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        lo[i] = e4m3x2(v[2 * i] * less, v[2 * i + 1] * less);
        hi[i] = e4m3x2(v[2 * i] * more, v[2 * i + 1] * more);
        differ |= lo[i] ^ hi[i];
    }
    return differ == 0;
}
// Whether 448 |v + rest| lies beyond the border between a code and the next, times (a + a_rest): the next one's code then, or on the
// border the even one's.  For v and a that are so near it, the difference of the products' leading parts is exact in few bits, and so are
// what fp32 leaves of them and the sum.  The smaller products are exact as sums of two numbers each; what adding them loses is kept too
// (Knuth's two-sum), and comes to few bits again.  So the sign is that of exact arithmetic: every number here is a multiple of
// a * 2^-66, which TINY keeps above the smallest.
template <bool RESTS>
__device__ __forceinline__ uint32_t decide(uint32_t code, float v, float rest, float a, float a_rest) {
    const float2 values = of_e4m3x2(code | (code + 1) << 8);
    const float border = 0.5f * (fabsf(values.x) + fabsf(values.y)), t = fabsf(v);
    const float n = t * TOP, m = border * a;
    float over = (n - m) + (fmaf(t, TOP, -n) - fmaf(border, a, -m));
    if (RESTS && (rest != 0.f || a_rest != 0.f)) {
        rest = v < 0.f ? -rest : rest;
        float low = 0.f;
        auto add = [&](float x) {
            const float sum = over + x, of_x = sum - over;
            low += (over - (sum - of_x)) + (x - of_x);
            over = sum;
        };
        const float x = rest * TOP, y = border * a_rest;
        add(x);
        add(-y);
        over += low + (fmaf(rest, TOP, -x) - fmaf(border, a_rest, -y));
    }
    return code + (over > 0.f || (over == 0.f && (code & 1u)));
}
__device__ __forceinline__ float pick(const float (&x)[8], int e) {
    float r = x[0];
#pragma unroll
    for (int j = 1; j < 8; ++j) r = e == j ? x[j] : r;
    return r;
}
// Decides where the codes with the smaller and the larger factor, neighbours then, differ: one entry of a thread at a time, which is
// little code: 8192 x 8640 bf16 with a gain of ones, where entries on a border are frequent, take 102 us (in line for all eight 195, a
// function for each 140).  rest(e, v): what fp32 leaves of entry e, v.
template <bool RESTS, class Rest>
__device__ __forceinline__ void settle(uint32_t (&c)[4], const uint32_t (&hi)[4], const float (&p)[8], float a, float a_rest, Rest rest) {
    uint32_t todo = 0;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const uint32_t d = c[q] ^ hi[q];
        todo |= ((d & 255u) ? 1u << 2 * q : 0u) | ((d >> 8) ? 2u << 2 * q : 0u);
    }
#pragma unroll 1
    for (; todo; todo &= todo - 1) {
        const int e = __ffs(todo) - 1, shift = e & 1 ? 8 : 0;
        const uint32_t pair = e < 4 ? (e < 2 ? c[0] : c[1]) : (e < 6 ? c[2] : c[3]), code = pair >> shift & 255u;
        const float v = pick(p, e);
        const uint32_t up = (decide<RESTS>(code, v, RESTS ? rest(e, v) : 0.f, a, a_rest) - code) << shift;
#pragma unroll
        for (int q = 0; q < 4; ++q) c[q] += e >> 1 == q ? up : 0u;
    }
}

// The codes of a block of a row, eight entries v (and gains g) to each of sixteen threads, and its scale.  With a gain
// that is still to be multiplied by the row's size; a block that was brought up by 2^100 waits for that as it is, with a minus
// sign, for its scale may be a normal number although a / 448 is none.  For whole warps: with masks of sixteen threads every
// exchange costs an instruction more.
template <bool BF16, bool NORM>
__device__ __forceinline__ uint2 block_codes(const float (&v)[8], const float (&g)[8], float& unit) {
    float p[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) p[j] = NORM ? v[j] * g[j] : v[j];
    auto largest = [&]() {
        float a = abs_max(p, 0.f);
#pragma unroll
        for (int o = 8; o; o >>= 1) a = max_nan(a, __shfl_xor_sync(0xffffffffu, a, o));
        return a;
    };
    float a = largest(), up = 1.f;
    const bool bad = !(a < INFINITY);
    uint32_t c[4];
    if (BF16 && !NORM) {
        bf16_codes(p, a, c);
    } else {
        const bool outside = !bad && a > 0.f && !middle_range(a);  // the same for the sixteen threads
        if (__any_sync(0xffffffffu, outside)) {
            up = outside ? to_middle(a) : 1.f;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const Factors f = scaled(v[j], g[j], up);
                p[j] = f.v * f.g;
            }
            a = largest();
        }
        uint32_t hi[4];
        const bool fine = fast_codes(p, a, c, hi) || !(a > 0.f) || bad;
        if (NORM ? __any_sync(0xffffffffu, !fine) : !fine) {
            float a_rest = 0.f;
            bool rests = false;  // none with gains of 1 or of eight bits, where entries on a border are frequent
            if (NORM) {
#pragma unroll
                for (int j = 0; j < 8; ++j) rests |= fmaf(v[j], g[j], -p[j]) != 0.f;  // (not 0 either where p is scaled)
                rests = __any_sync(0xffffffffu, rests);
            }
            if (rests) {
                a_rest = -INFINITY;  // of the largest |x g|
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (fabsf(p[j]) == a) a_rest = fmaxf(a_rest, copysignf(1.f, p[j]) * rest_of(v[j], g[j], p[j], up));
#pragma unroll
                for (int o = 8; o; o >>= 1) a_rest = fmaxf(a_rest, __shfl_xor_sync(0xffffffffu, a_rest, o));
            }
            if (!fine) settle<NORM>(c, hi, p, a, a_rest, [&](int e, float x) { return rests ? rest_of(pick(v, e), pick(g, e), x, up) : 0.f; });
        }
    }
    if (bad) unit = __uint_as_float(0x7fc00000u);
    else if (NORM) unit = up > 1.f ? -a / TOP : up < 1.f ? a / TOP / up : a * (1.f / TOP);
    else unit = up == 1.f ? __fdiv_rn(a, TOP) : a / TOP / up;
    return a > 0.f && !bad ? make_uint2(__byte_perm(c[0], c[1], 0x5410), __byte_perm(c[2], c[3], 0x5410)) : make_uint2(0, 0);
}

// A block's scale from `unit` and the sum of its row's squares; false where squares lie outside of fp32's range.
__device__ __forceinline__ bool row_scale(float unit, float sum, float inv_k, float eps, float& scale) {
    const float mean = fmaf(sum, inv_k, eps);
    const bool zeros = unit == 0.f && sum == 0.f;  // whatever eps is
    scale = zeros ? 0.f : fabsf(unit) * rsqrtf(mean) * (unit < 0.f ? 0x1p-100f : 1.f);  // (what squares below fp32's range lose of it is 2^-149)
    return zeros || !(mean <= 1e-30f || sum >= 3e38f);  // (a sum that is no number stays none)
}
// The scales of a warp's blocks for which that was false, with the squares in 64 bits: once for each of the rows among them, by all of
// the warp's threads.  64 rows of 16384 fp32 with one such row take 15 us, without 10; 147 where each block's thread added them alone.
template <bool BF16>
__device__ __noinline__ void wide_scales(const char* X, long long row_bytes, int row0, int batch, int M, int K, float inv_k, float eps, const float (*part)[16],
                                         const float* units, int units_row, int warps, float* scale) {
    const int lane = threadIdx.x & 31, most = batch * ((K + BLOCK - 1) / BLOCK);
    for (int j0 = threadIdx.x - lane; j0 < most; j0 += blockDim.x) {
        const int j = j0 + lane, b = j / batch, q = j - b * batch, row = row0 + q;
        float unit = 0.f, sum = 0.f, s;
        if (j < most && row < M) {
            for (int i = 0; i < warps; ++i) sum += part[q][i];
            unit = units ? units[q * units_row + b] : scale[(size_t)b * M + row];
        }
        bool odd = !row_scale(unit, sum, inv_k, eps, s) && j < most && row < M;
        for (uint32_t left; (left = __ballot_sync(0xffffffffu, odd));) {
            const int of = __shfl_sync(0xffffffffu, row, __ffs(left) - 1);
            double wide = 0;
            for (int k = lane * 8; k < K; k += 256) {
                Raw<BF16> again;
                float v[8];
                again.load(X + of * row_bytes, k);
                again.widen(v);
#pragma unroll
                for (int i = 0; i < 8; ++i) wide += (double)v[i] * (double)v[i];
            }
#pragma unroll
            for (int o = 16; o; o >>= 1) wide += __shfl_xor_sync(0xffffffffu, wide, o);
            if (odd && row == of) {
                scale[(size_t)b * M + row] = (float)(fabs((double)unit) * (unit < 0.f ? 0x1p-100 : 1.0) * rsqrt(wide / K + (double)eps));
                odd = false;
            }
        }
    }
}

// One token row at a time to a block of threads; thread t has entries 8 t .. 8 t + 7, and those blockDim * 8 further on.  Sixteen
// neighbouring threads share a block of channels.  NV: how often eight entries to a thread cover the row, whose next row is then
// under way while one is worked on (0: more often than registers are kept for).  The codes do not wait for the row's sum of
// squares: only the scales need it, at the end, and those of `batch` rows together, so that warps wait for one another once for
// several rows.  16384 rows of 4096 fp32 with a gain take 74 us, bf16 70 (first the sum, then the codes: 94 us for 88 at the time;
// row by row: 88 for 82).
constexpr int BATCH_MOST = 4;

template <bool BF16, bool NORM, int NV>
__global__ void __launch_bounds__(512, 2) quant_rows_kernel(const void* __restrict__ X, long long stride, const float* __restrict__ gain, float eps, int M,
                                                         int K, int batch, float inv_k, uint8_t* __restrict__ codes, float* __restrict__ scale) {
    __shared__ float part[2][BATCH_MOST][16], units[2][BATCH_MOST][32 * (NV ? NV : 1)];
    constexpr int N = NV ? NV : 1;
    constexpr bool KEEP = NV == 1;
    const int t = threadIdx.x, lane = t & 31, span = blockDim.x * 8, warps = blockDim.x >> 5;
    const int steps = NV ? NV : (K + span - 1) / span;
    const long long row_bytes = stride * (BF16 ? 2 : 4);
    const char* at = reinterpret_cast<const char*>(X) + (long long)blockIdx.x * batch * row_bytes;
    a48_pdl_prologue();
    Raw<BF16> next[N];
    if (NV) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            next[i].clear();
            if (i * span + t * 8 < K) next[i].load(at, i * span + t * 8);
        }
    }
    float gains[KEEP ? N : 1][8];  // of this thread's channels, where they fit
    if (NORM && KEEP) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            Raw<false> raw;
            raw.clear();
            if (i * span + t * 8 < K) raw.load(gain, i * span + t * 8);
            raw.widen(gains[KEEP ? i : 0]);
        }
    }
    int flip = 0;
    for (int row0 = blockIdx.x * batch; row0 < M; row0 += batch * (int)gridDim.x, flip ^= 1) {
#pragma unroll 1
        for (int row = row0; row < min(M, row0 + batch); ++row) {
            const char* here = at;
            const bool ends = row + 1 == row0 + batch, more = (ends ? row0 + batch * (int)gridDim.x : row + 1) < M;
            at += (ends ? (long long)batch * ((int)gridDim.x - 1) + 1 : 1) * row_bytes;
            float sum = 0.f;
#pragma unroll
            for (int i = 0; i < steps; ++i) {
                const int k = i * span + t * 8;
                if (k - lane * 8 >= K) break;  // the same for a warp
                float v[8], g[8];
                if (NV) {
                    next[NV ? i : 0].widen(v);
                    next[NV ? i : 0].clear();
                    if (more && k < K) next[NV ? i : 0].load(at, k);
                } else {
                    next[0].clear();
                    if (k < K) next[0].load(here, k);
                    next[0].widen(v);
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) g[j] = 1.f;
                if (NORM) {
                    if (KEEP) {
#pragma unroll
                        for (int j = 0; j < 8; ++j) g[j] = gains[KEEP ? i : 0][j];
                    } else if (k < K) {
                        Raw<false> raw;
                        raw.load(gain, k);
                        raw.widen(g);
                    }
#pragma unroll
                    for (int j = 0; j < 8; ++j) sum = fmaf(v[j], v[j], sum);
                }
                float unit;
                const uint2 c = block_codes<BF16, NORM>(v, g, unit);
                if (k < K) *reinterpret_cast<uint2*>(codes + (size_t)row * K + k) = c;
                if ((t & 15) == 0 && k < K) {
                    if (NORM && NV) units[flip][row - row0][k / BLOCK] = unit;
                    else scale[(size_t)(k / BLOCK) * M + row] = unit;
                }
            }
            if (NORM) {
#pragma unroll
                for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
                if (lane == 0) part[flip][row - row0][t >> 5] = sum;
            }
        }
        if (!NORM) continue;
        __syncthreads();
        const int blocks = (K + BLOCK - 1) / BLOCK;
        bool odd = false;
        for (int j = t; j < batch * blocks; j += blockDim.x) {
            const int b = j / batch, q = j - b * batch, row = row0 + q;
            if (row >= M) continue;
            float sum = 0.f, s;
            for (int i = 0; i < warps; ++i) sum += part[flip][q][i];
            const float u = NV ? units[flip][q][NV ? b : 0] : scale[(size_t)b * M + row];
            if (row_scale(u, sum, inv_k, eps, s)) scale[(size_t)b * M + row] = s;
            else odd = true;
        }
        if (__any_sync(0xffffffffu, odd))
            wide_scales<BF16>(reinterpret_cast<const char*>(X), row_bytes, row0, batch, M, K, inv_k, eps, part[flip], NV ? units[flip][0] : nullptr,
                              (int)(sizeof units[0][0] / sizeof(float)), warps, scale);
    }
}

// A block of 128 x 128 weights to 512 threads; a thread has eight entries of four rows.
template <bool BF16>
__global__ void __launch_bounds__(512, 3) quant_weight_kernel(const void* __restrict__ W, long long stride, int N, int K,
                                                                         uint8_t* __restrict__ codes, float* __restrict__ scale) {
    __shared__ float part[16];
    const int t = threadIdx.x, k = blockIdx.x * BLOCK + t % 16 * 8, n0 = blockIdx.y * BLOCK + t / 16;
    const int rows = k < K ? (N - n0 + 31) / 32 : 0;  // of this thread, if there were no end to the block
    const char* at = reinterpret_cast<const char*>(W) + ((size_t)n0 * stride + k) * (BF16 ? 2 : 4);
    const size_t step = (size_t)stride * 32 * (BF16 ? 2 : 4);
    a48_pdl_prologue();
    Raw<BF16> raw[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        raw[i].clear();
        if (i < rows) raw[i].load(at + i * step, 0);
    }
    float a = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float v[8];
        raw[i].widen(v);
        a = abs_max(v, a);
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) a = max_nan(a, __shfl_xor_sync(0xffffffffu, a, o));
    if ((t & 31) == 0) part[t >> 5] = a;
    __syncthreads();
    a = part[t & 15];
#pragma unroll
    for (int o = 8; o; o >>= 1) a = max_nan(a, __shfl_xor_sync(0xffffffffu, a, o));
    const bool bad = !(a < INFINITY);
    uint8_t* to = codes + (size_t)n0 * K + k;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float v[8];
        raw[i].widen(v);
        uint32_t c[4];
        if (BF16) {
            bf16_codes(v, a, c);
        } else {
            const float up = to_middle(a), b = a * up;
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] *= up;
            uint32_t hi[4];
            if (!fast_codes(v, b, c, hi)) settle<false>(c, hi, v, b, 0.f, [](int, float) { return 0.f; });
        }
        if (i < rows)
            *reinterpret_cast<uint2*>(to + (size_t)i * 32 * K) =
                a > 0.f && !bad ? make_uint2(__byte_perm(c[0], c[1], 0x5410), __byte_perm(c[2], c[3], 0x5410)) : make_uint2(0, 0);
    }
    if (t == 0) scale[(size_t)blockIdx.y * gridDim.x + blockIdx.x] = bad ? __uint_as_float(0x7fc00000u) : __fdiv_rn(a, TOP);
}

template <bool BF16, bool NORM, int NV>
cudaError_t launch_rows(int threads, const void* X, long long stride, const float* gain, float eps, int M, int K, uint8_t* codes, float* scale, cudaStream_t st) {
    static std::atomic<int> resident[17];  // blocks of 32 .. 512 threads that fit on an SM
    int n = resident[threads / 32].load(std::memory_order_relaxed);
    if (n == 0) {
        const cudaError_t e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, quant_rows_kernel<BF16, NORM, NV>, threads, 0);
        if (e != cudaSuccess) return e;
        resident[threads / 32].store(n, std::memory_order_relaxed);
    }
    // four rows at a time only where that leaves none of the blocks idle: fewer rows end sooner one by one
    const int most = a48f8::sm_count() * n, batch = NORM && NV && M >= BATCH_MOST * most ? BATCH_MOST : 1;
    const int batches = (M - 1) / batch + 1;
    return a48_launch_pdl(quant_rows_kernel<BF16, NORM, NV>, dim3(batches < most ? batches : most), dim3(threads), 0, st, X, stride, gain, eps, M, K, batch, 1.f / (float)K,
                          codes, scale);
}

template <bool BF16, bool NORM>
cudaError_t launch_rows(const void* X, long long stride, const float* gain, float eps, int M, int K, uint8_t* codes, float* scale, cudaStream_t st) {
    // (512 threads for all of more than 4096 channels left many of them without the last of their entries: 8192 x 5120 fp32 with a gain
    // took 91 us for 72, 8192 x 8640 127 for 118, now 110)
    const int eights = (K + 7) / 8, nv = (eights + 511) / 512, threads = nv <= 4 ? a48_round_up((eights + nv - 1) / nv, 32) : 512;
    if (nv == 1) return launch_rows<BF16, NORM, 1>(threads, X, stride, gain, eps, M, K, codes, scale, st);
    if (nv == 2) return launch_rows<BF16, NORM, 2>(threads, X, stride, gain, eps, M, K, codes, scale, st);
    if (nv == 3) return launch_rows<BF16, NORM, 3>(threads, X, stride, gain, eps, M, K, codes, scale, st);
    if (nv == 4) return launch_rows<BF16, NORM, 4>(threads, X, stride, gain, eps, M, K, codes, scale, st);
    return launch_rows<BF16, NORM, 0>(threads, X, stride, gain, eps, M, K, codes, scale, st);
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
    const dim3 grid((unsigned)blocks(K), (unsigned)blocks(N));
    A48_CUDA_TRY(a48_launch_pdl(bf16 ? quant_weight_kernel<true> : quant_weight_kernel<false>, grid, dim3(512), 0, st, W, stride, N, K, codes, scale));
    return BITNET_A48_OK;
}

}  // namespace a48f8
