// Writing the paged low-bit cache (rotation, quantisation and placement of new tokens in one pass) and reading it back.
//
// Both kernels move bytes and little else: the write reads q, k and v once and stores the rotated queries and the codes,
// the read loads codes and scales and stores the values.  What has to be kept off their way is the float64 arithmetic
// that makes the codes exact (angles, rotation of the keys, scale and rounding): the angles are taken once per token and
// block, not per head, and the rotation of the queries, whose result is rounded to bf16, is done in fp32.
#include "paged.cuh"

namespace {

using a48p::Batch;
using a48p::Layout;

constexpr int kWarps = 8;

// base^(-i / half) of the rotation pairs, evaluated on the host
struct Rates {
    double f[64];
};

template <bool BF16>
__device__ __forceinline__ float2 load2(const void* row, int e) {
    if (BF16) {
        const unsigned u = __ldg(reinterpret_cast<const unsigned*>(reinterpret_cast<const uint16_t*>(row) + e));
        return make_float2(__uint_as_float(u << 16), __uint_as_float(u & 0xffff0000u));
    }
    return __ldg(reinterpret_cast<const float2*>(reinterpret_cast<const float*>(row) + e));
}

// One warp quantises one head vector, four entries per lane (zero past the head), with Eq. 3's arithmetic in float64:
// gamma = max|x|, u = RoundClip(L / (gamma + eps) x, -(L+1), L) + L + 1.
__device__ __forceinline__ void quantise(const double (&x)[4], int bits, double eps, int (&u)[4], float& scale) {
    double gamma = fmax(fmax(fabs(x[0]), fabs(x[1])), fmax(fabs(x[2]), fabs(x[3])));
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) gamma = fmax(gamma, __shfl_xor_sync(0xffffffffu, gamma, o));
    const int L = (1 << (bits - 1)) - 1;
    const double s = (double)L / (gamma + eps);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int q = __double2int_rn(s * x[i]);
        u[i] = min(max(q, -(L + 1)), L) + L + 1;
    }
    scale = (float)(gamma / (double)L);
}

// The entries of a row, one byte each in shared memory, packed into words by the lanes that have one.
__device__ __forceinline__ void store_row(uint8_t* __restrict__ dst, const uint8_t* u, int padded, int bits, int lane) {
    unsigned* out = reinterpret_cast<unsigned*>(dst);
    if (bits == 8) {
        if (4 * lane < padded) out[lane] = reinterpret_cast<const unsigned*>(u)[lane];
    } else if (bits == 4) {
        if (8 * lane < padded) {
            const uint2 b = reinterpret_cast<const uint2*>(u)[lane];  // byte i: entry i; fold the pairs of bytes
            const unsigned lo = (b.x | (b.x >> 4)) & 0x00ff00ffu, hi = (b.y | (b.y >> 4)) & 0x00ff00ffu;
            out[lane] = ((lo | (lo >> 8)) & 0xffffu) | ((hi | (hi >> 8)) << 16);
        }
    } else if (lane < 3 * padded / 32) {  // three words per 32 entries
        const int granule = lane / 3, j = lane % 3;
        const uint8_t* g = u + 32 * granule;
        unsigned w = 0;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            unsigned v = 0;
#pragma unroll
            for (int e = 0; e < 5; ++e) v |= (unsigned)g[16 * half + 5 * j + e] << (3 * e);
            v |= ((g[16 * half + 15] >> j) & 1u) << 15;
            w |= v << (16 * half);
        }
        out[lane] = w;
    }
}

struct WriteArgs {
    Layout l;
    Batch b;
    uint8_t* pool;
    const void *q, *k, *v;
    long long q_stride, k_stride, v_stride, out_stride;
    __nv_bfloat16* q_out;
    int q_heads, rotate;
    double eps;
    Rates rates;
};

// grid (token, slice of heads).  A warp takes one query head (rotate, round to bf16) or one key/value head (rotate the
// key, quantise both, store) at a time.  Lane l owns entries 2l, 2l+1 and half + 2l, half + 2l + 1: rotation partners
// meet in one lane.
template <bool BF16>
__global__ void __launch_bounds__(32 * kWarps) paged_write_kernel(const __grid_constant__ WriteArgs a) {
    __shared__ double2 turn[64];  // cos, sin of the token's position
    __shared__ alignas(8) uint8_t codes[kWarps][2][128];
    a48_pdl_prologue();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, token = blockIdx.x;
    const int s = a48p::sequence_of(a.b, token, lane);
    if (s < 0) return;  // behind the last sequence
    const int first = __ldg(a.b.q_start + s), end = __ldg(a.b.q_start + s + 1);
    const int pos = __ldg(a.b.kv_len + s) - (end - first) + (token - first);
    const int half = a.l.hd / 2;
    if (a.rotate) {
        for (int i = threadIdx.x; i < half; i += blockDim.x) {
            double sn, cn;
            sincos((double)pos * a.rates.f[i], &sn, &cn);
            turn[i] = make_double2(cn, sn);
        }
        __syncthreads();
    }
    const int page = a48p::page_of(a.l, a.b, s, pos), slot = pos & (a.l.page - 1);
    const int e = 2 * lane;
    const bool mine = e < half;
    double2 t0 = make_double2(1.0, 0.0), t1 = t0;
    if (a.rotate && mine) t0 = turn[e], t1 = turn[e + 1];
    const int items = a.q_heads + a.l.kv_heads;
    for (int item = blockIdx.y * kWarps + warp; item < items; item += gridDim.y * kWarps) {
        if (item < a.q_heads) {
            const size_t elem = BF16 ? 2 : 4;
            const char* row = static_cast<const char*>(a.q) + ((size_t)token * a.q_stride + (size_t)item * a.l.hd) * elem;
            float2 lo = make_float2(0.f, 0.f), hi = lo;
            if (mine) lo = load2<BF16>(row, e), hi = load2<BF16>(row, half + e);
            __syncwarp();  // q_out may be q: every lane has read before any lane writes
            if (mine) {
                const float c0 = (float)t0.x, s0 = (float)t0.y, c1 = (float)t1.x, s1 = (float)t1.y;
                __nv_bfloat16* out = a.q_out + (size_t)token * a.out_stride + (size_t)item * a.l.hd;
                *reinterpret_cast<__nv_bfloat162*>(out + e) = __floats2bfloat162_rn(lo.x * c0 - hi.x * s0, lo.y * c1 - hi.y * s1);
                *reinterpret_cast<__nv_bfloat162*>(out + half + e) = __floats2bfloat162_rn(hi.x * c0 + lo.x * s0, hi.y * c1 + lo.y * s1);
            }
            continue;
        }
        if (page < 0) continue;  // no page for this position: nothing is stored
        const int head = item - a.q_heads;
        uint8_t* chunk = a.pool + a48p::chunk_at(a.l, page, head);
        const size_t elem = BF16 ? 2 : 4;
        const char* krow = static_cast<const char*>(a.k) + ((size_t)token * a.k_stride + (size_t)head * a.l.hd) * elem;
        const char* vrow = static_cast<const char*>(a.v) + ((size_t)token * a.v_stride + (size_t)head * a.l.hd) * elem;
        float2 f[2][2] = {};
        if (mine) {
            f[0][0] = load2<BF16>(krow, e), f[0][1] = load2<BF16>(krow, half + e);
            f[1][0] = load2<BF16>(vrow, e), f[1][1] = load2<BF16>(vrow, half + e);
        }
        const bool bos = a.l.bits == 3 && pos == 0;  // the bos heads keep 4 bits
        const int bits = bos ? 4 : a.l.bits;
#pragma unroll
        for (int n = 0; n < 2; ++n) {
            const double l0 = f[n][0].x, l1 = f[n][0].y, h0 = f[n][1].x, h1 = f[n][1].y;
            double x[4] = {l0, l1, h0, h1};
            if (n == 0 && a.rotate) {
                x[0] = l0 * t0.x - h0 * t0.y;
                x[1] = l1 * t1.x - h1 * t1.y;
                x[2] = h0 * t0.x + l0 * t0.y;
                x[3] = h1 * t1.x + l1 * t1.y;
            }
            int u[4];
            float scale;
            quantise(x, bits, a.eps, u, scale);
            uint8_t* buf = codes[warp][n];
            if (mine) {
                *reinterpret_cast<uchar2*>(buf + e) = make_uchar2(u[0], u[1]);
                *reinterpret_cast<uchar2*>(buf + half + e) = make_uchar2(u[2], u[3]);
            }
            if (a.l.hd + lane < a.l.padded) buf[a.l.hd + lane] = (uint8_t)(1 << (bits - 1));
            __syncwarp();
            uint8_t* dst = bos ? chunk + a.l.bos + n * (a.l.padded / 2) : chunk + (n == 0 ? 0 : a.l.v_codes) + slot * a.l.row;
            store_row(dst, buf, a.l.padded, bits, lane);
            if (lane == 0) reinterpret_cast<float*>(chunk + (n == 0 ? a.l.k_scales : a.l.v_scales))[slot] = scale;
        }
        __syncwarp();  // the row buffers are free again
    }
}

// One warp per (token, slice of its keys and values), four entries per thread and step: the stores of a warp are one run
// of the output row.  A position without a page reads as zero.
template <bool BF16>
__global__ void __launch_bounds__(32 * kWarps) paged_read_kernel(const Layout l, const Batch b, const uint8_t* __restrict__ pool,
                                                                 void* __restrict__ k_out, void* __restrict__ v_out) {
    a48_pdl_prologue();
    const int lane = threadIdx.x & 31, token = blockIdx.x * kWarps + (threadIdx.x >> 5);
    if (token >= b.n_tokens) return;
    const int s = a48p::sequence_of(b, token, lane);
    if (s < 0) return;
    const int first = __ldg(b.q_start + s), end = __ldg(b.q_start + s + 1);
    const int pos = __ldg(b.kv_len + s) - (end - first) + (token - first);
    const int page = a48p::page_of(l, b, s, pos), slot = pos & (l.page - 1);
    const int quads = l.hd / 4, per_row = l.kv_heads * quads;
    const bool bos = l.bits == 3 && pos == 0;
#pragma unroll 4
    for (int i = blockIdx.y * 32 + lane; i < 2 * per_row; i += gridDim.y * 32) {
        const int which = i >= per_row, at = which ? i - per_row : i;
        const int head = at / quads, e = 4 * (at % quads);
        float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
        if (page >= 0) {
            const uint8_t* chunk = pool + a48p::chunk_at(l, page, head);
            const float scale = __ldg(reinterpret_cast<const float*>(chunk + (which ? l.v_scales : l.k_scales)) + slot);
            x = bos ? a48p::four_entries(chunk + l.bos + which * (l.padded / 2), e, 4)
                    : a48p::four_entries(chunk + (which ? l.v_codes : 0) + slot * l.row, e, l.bits);
            x.x *= scale, x.y *= scale, x.z *= scale, x.w *= scale;
        }
        const size_t o = (size_t)token * per_row + at;
        void* out = which ? v_out : k_out;
        if (BF16) {
            const __nv_bfloat162 lo = __floats2bfloat162_rn(x.x, x.y), hi = __floats2bfloat162_rn(x.z, x.w);
            reinterpret_cast<uint2*>(out)[o] =
                make_uint2(*reinterpret_cast<const unsigned*>(&lo), *reinterpret_cast<const unsigned*>(&hi));
        } else {
            reinterpret_cast<float4*>(out)[o] = x;
        }
    }
}

// Rotation rates for a base and head dimension; the last table of this host thread is kept, decode loops ask for one.
const Rates& rates_of(float base, int half) {
    thread_local Rates r;
    thread_local float last_base = 0.f;
    thread_local int last_half = 0;
    if (base != last_base || half != last_half) {
        for (int i = 0; i < half; ++i) r.f[i] = pow((double)base, -(double)i / (double)half);
        last_base = base;
        last_half = half;
    }
    return r;
}

}  // namespace

extern "C" {

size_t bitnet_a48_paged_cache_bytes(const bitnet_a48_paged_cache* c) {
    if (!c || (c->bits != 8 && c->bits != 4 && c->bits != 3) || c->n_kv_heads <= 0 || c->n_kv_heads > 65535 ||
        c->n_pages <= 0 || c->head_dim <= 0 || c->head_dim > 128 || c->head_dim % 4 != 0)
        return 0;
    if (c->page_size != 16 && c->page_size != 32 && c->page_size != 64 && c->page_size != 128) return 0;
    return (size_t)c->n_pages * c->n_kv_heads * a48p::layout_of(*c).chunk;
}

bitnet_a48_status bitnet_a48_paged_write(const bitnet_a48_paged_cache* cache, void* pool_dev, const bitnet_a48_paged_batch* batch,
                                         int n_heads, const void* q_dev, long long q_stride, const void* k_dev, long long k_stride,
                                         const void* v_dev, long long v_stride, int x_bf16, float rope_base, float eps,
                                         uint16_t* q_out_dev, long long q_out_stride, void* stream) {
    bitnet_a48_status st = a48p::check(cache, pool_dev, batch);
    if (st != BITNET_A48_OK) return st;
    if (!(eps >= 0.f) || !(rope_base >= 0.f) || rope_base > 3e38f) return BITNET_A48_ERR_INVALID_ARG;
    const int elem = x_bf16 ? 2 : 4;
    const long long kv_width = (long long)cache->n_kv_heads * cache->head_dim, q_width = (long long)n_heads * cache->head_dim;
    if ((st = a48p::check_rows(k_dev, k_stride, kv_width, elem)) != BITNET_A48_OK) return st;
    if ((st = a48p::check_rows(v_dev, v_stride, kv_width, elem)) != BITNET_A48_OK) return st;
    if (q_dev || q_out_dev) {
        if (n_heads <= 0 || n_heads > 65535) return BITNET_A48_ERR_SHAPE;
        if ((st = a48p::check_rows(q_dev, q_stride, q_width, elem)) != BITNET_A48_OK) return st;
        if ((st = a48p::check_rows(q_out_dev, q_out_stride, q_width, 2)) != BITNET_A48_OK) return st;
    }
    if (!a48_have_device()) return BITNET_A48_ERR_CUDA;
    WriteArgs a;
    a.l = a48p::layout_of(*cache);
    a.b = a48p::batch_of(*batch);
    a.pool = static_cast<uint8_t*>(pool_dev);
    a.q = q_dev, a.k = k_dev, a.v = v_dev;
    a.q_stride = q_stride, a.k_stride = k_stride, a.v_stride = v_stride, a.out_stride = q_out_stride;
    a.q_out = reinterpret_cast<__nv_bfloat16*>(q_out_dev);
    a.q_heads = q_dev ? n_heads : 0;
    a.rotate = rope_base > 0.f;
    a.eps = (double)eps;
    if (a.rotate) a.rates = rates_of(rope_base, cache->head_dim / 2);
    // Few tokens: their heads are spread over blocks, one head per warp; many: a block keeps its token's angles.
    const int items = a.q_heads + a.l.kv_heads, rounds = (items + kWarps - 1) / kWarps;
    int slices = (2048 + batch->n_tokens - 1) / batch->n_tokens;
    slices = slices < rounds ? slices : rounds;
    const dim3 grid(batch->n_tokens, slices);
    auto kernel = x_bf16 ? paged_write_kernel<true> : paged_write_kernel<false>;
    A48_CUDA_TRY(a48_launch_pdl(kernel, grid, dim3(32 * kWarps), 0, (cudaStream_t)stream, a));
    return BITNET_A48_OK;
}

bitnet_a48_status bitnet_a48_paged_read(const bitnet_a48_paged_cache* cache, const void* pool_dev, const bitnet_a48_paged_batch* batch,
                                        void* k_out_dev, void* v_out_dev, int y_bf16, void* stream) {
    const bitnet_a48_status st = a48p::check(cache, pool_dev, batch);
    if (st != BITNET_A48_OK) return st;
    if (!k_out_dev || !v_out_dev) return BITNET_A48_ERR_INVALID_ARG;
    if (!a48_aligned16(k_out_dev) || !a48_aligned16(v_out_dev)) return BITNET_A48_ERR_ALIGNMENT;
    if (!a48_have_device()) return BITNET_A48_ERR_CUDA;
    const Layout l = a48p::layout_of(*cache);
    const int steps = (2 * l.kv_heads * (l.hd / 4) + 31) / 32;  // of a warp over one token
    int slices = (8192 + batch->n_tokens - 1) / batch->n_tokens;
    slices = slices < steps ? slices : steps;
    const dim3 grid((batch->n_tokens + kWarps - 1) / kWarps, slices);
    auto kernel = y_bf16 ? paged_read_kernel<true> : paged_read_kernel<false>;
    A48_CUDA_TRY(a48_launch_pdl(kernel, grid, dim3(32 * kWarps), 0, (cudaStream_t)stream, l, a48p::batch_of(*batch),
                                static_cast<const uint8_t*>(pool_dev), k_out_dev, v_out_dev));
    return BITNET_A48_OK;
}

}  // extern "C"
