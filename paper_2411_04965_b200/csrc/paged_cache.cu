// Writing the paged low-bit cache (rotation, quantisation and placement of new tokens in one pass) and reading it back.
//
// Both kernels move bytes and little else: the write reads q, k and v once and stores the rotated queries and the codes,
// the read loads codes and scales and stores the values.  What has to be kept off their way is arithmetic: the float64 that
// makes the codes exact (the angles are taken once per token and block, not per head, and entries in fp32 unless they lie
// at a rounding border), and divisions by shapes that are not known when this is compiled.  Measured: 302 MB of bf16 keys
// and values read back from 4-bit pages in 89 us (the GPU zero-fills as much in 80); prompts written from fused q/k/v rows and
// read back in 94 us, of which the floor is 49: there the quantiser's instructions count as well.
#include "paged.cuh"

namespace {

using a48p::Batch;
using a48p::Layout;

constexpr int kWarps = 8, MAX_TOKENS = 4, BATCH = 4, READ_TOKENS = 16;

// base^(-i / half) / pi of the rotation pairs, evaluated on the host: half turns per position
struct Rates {
    double f[64];
};

// W consecutive entries of a row, as they lie in memory
template <bool BF16, int W>
struct Raw {
    static constexpr int N = BF16 ? W / 2 : W;
    uint32_t u[N];
    __device__ void load(const void* row, int e) {
        const uint32_t* p = reinterpret_cast<const uint32_t*>(static_cast<const char*>(row) + e * (BF16 ? 2 : 4));
        if constexpr (N == 4) {
            const uint4 v = __ldg(reinterpret_cast<const uint4*>(p));
            u[0] = v.x, u[1] = v.y, u[2] = v.z, u[3] = v.w;
        } else if constexpr (N == 2) {
            const uint2 v = __ldg(reinterpret_cast<const uint2*>(p));
            u[0] = v.x, u[1] = v.y;
        } else {
            u[0] = __ldg(p);
        }
    }
    __device__ void clear() {
#pragma unroll
        for (int i = 0; i < N; ++i) u[i] = 0;
    }
    __device__ float operator[](int i) const {
        return __uint_as_float(!BF16 ? u[i] : i & 1 ? u[i / 2] & 0xffff0000u : u[i / 2] << 16);
    }
};

// W entries from e on, to a row of bf16 or of codes (the low byte of each word; the rest of it may hold anything)
template <int W>
__device__ __forceinline__ void store_bf16(__nv_bfloat16* row, int e, const float (&x)[W]) {
    uint32_t u[W / 2];
#pragma unroll
    for (int i = 0; i < W / 2; ++i) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
        u[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    if constexpr (W == 4) *reinterpret_cast<uint2*>(row + e) = make_uint2(u[0], u[1]);
    else *reinterpret_cast<uint32_t*>(row + e) = u[0];
}
template <int W>
__device__ __forceinline__ void store_codes(uint8_t* row, int e, int bits, const uint32_t (&u)[W]) {
    uint32_t w = __byte_perm(u[0], u[1], 0x0040);  // entries in bytes 0, 1
    if constexpr (W == 4) w = __byte_perm(w, __byte_perm(u[2], u[3], 0x0040), 0x5410);
    if (bits == 8) {
        if constexpr (W == 4) *reinterpret_cast<uint32_t*>(row + e) = w;
        else *reinterpret_cast<uint16_t*>(row + e) = (uint16_t)w;
    } else {  // fold the pairs of bytes
        w = (w | (w >> 4)) & 0x00ff00ffu;
        if constexpr (W == 4) *reinterpret_cast<uint16_t*>(row + e / 2) = (uint16_t)(w | (w >> 8));
        else row[e / 2] = (uint8_t)w;
    }
}

// The larger of two numbers, NaN if either is none.
__device__ __forceinline__ float max_or_nan(float x, float y) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(x), "f"(y));
    return r;
}

// Word `at` of a 3-bit row from its entries, one byte each.
__device__ __forceinline__ uint32_t word_of_triples(const uint8_t* u, int at) {
    const int j = at % 3;
    const uint8_t* g = u + 32 * (at / 3);
    uint32_t w = 0;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        uint32_t v = 0;
#pragma unroll
        for (int e = 0; e < 5; ++e) v |= (uint32_t)g[16 * half + 5 * j + e] << (3 * e);
        v |= ((g[16 * half + 15] >> j) & 1u) << 15;
        w |= v << (16 * half);
    }
    return w;
}

struct WriteArgs {
    Layout l;
    Batch b;
    uint8_t* pool;
    const void *q, *k, *v;
    long long q_stride, k_stride, v_stride, out_stride;
    __nv_bfloat16* q_out;
    int q_heads, rotate, tokens;  // tokens: of a block
    double eps;
    Rates rates;
};

// grid (tokens / `tokens`, slice of heads).  A block's warps are dealt out to its tokens; a group of G lanes takes one head
// vector at a time, of the queries (rotate, round to bf16), the keys (rotate, quantise) or the values (quantise); lane l of
// it has entries W l .. W l + W - 1 and their rotation partners.
//
// The codes are those of float64 arithmetic without float64 for every entry: rotation and scale are taken in fp32, whose
// errors move an entry's multiple of the step by less than L 2^-19 (of L: the rotation 6 2^-24 of gamma, the scale
// 10 2^-24); only where that multiple lies so near a rounding border (one entry in 4000 at 8 bits, one in 70000 at 4) are
// the lane's entries taken again in float64.  The scale itself comes from gamma in float64: of the lanes whose entries can be
// the largest.
template <bool BF16, int W, int G>
__global__ void __launch_bounds__(32 * kWarps, 4) paged_write_kernel(const __grid_constant__ WriteArgs a) {
    constexpr int PER = 32 / G;  // head vectors that a warp takes at a time
    __shared__ double2 turn_of[MAX_TOKENS][64];  // cos, sin of the tokens' positions
    __shared__ float2 turn_f_of[MAX_TOKENS][64];
    __shared__ int positions[MAX_TOKENS];
    __shared__ alignas(8) uint8_t row_codes[kWarps][32][8];  // for 3-bit rows; a group's lanes have room for its padded row
    a48_pdl_prologue();
    const int lane = threadIdx.x & 31, warps = kWarps / a.tokens, of = (threadIdx.x >> 5) / warps, token = blockIdx.x * a.tokens + of;
    const int s = token < a.b.n_tokens ? a48p::sequence_of(a.b, token, lane) : -1;  // (none behind the last sequence)
    int pos = 0;
    if (s >= 0) {
        const int first = __ldg(a.b.q_start + s), end = __ldg(a.b.q_start + s + 1);
        pos = __ldg(a.b.kv_len + s) - (end - first) + (token - first);
    }
    const int half = a.l.hd / 2, l = lane & (G - 1), e = W * l, row_bytes = a.l.hd * (BF16 ? 2 : 4);
    const bool mine = e < half;
    const int page = s >= 0 ? a48p::page_of(a.l, a.b, s, pos) : -1, slot = pos & (a.l.page - 1);
    const int begin = (blockIdx.y * warps + (threadIdx.x >> 5) % warps) * PER + lane / G, stride = gridDim.y * warps * PER;
    // ---- queries, BATCH of a warp's at a time: the first ones under way while the angles are taken
    const char* q_rows = static_cast<const char*>(a.q) + (size_t)token * a.q_stride * (BF16 ? 2 : 4);
    Raw<BF16, W> q[BATCH][2];
    auto load_queries = [&](int head) {
#pragma unroll
        for (int k = 0; k < BATCH; ++k)
            if (s >= 0 && mine && head + k * stride < a.q_heads) {
                const char* row = q_rows + (size_t)(head + k * stride) * row_bytes;
                q[k][0].load(row, e);
                q[k][1].load(row, half + e);
            }
    };
    load_queries(begin);
    if (a.rotate) {
        if (lane == 0) positions[of] = pos;  // (the same from each of the token's warps)
        __syncthreads();
        for (int i = threadIdx.x; i < 64 * a.tokens; i += blockDim.x) {
            if ((i & 63) >= half) continue;
            double sn, cn;
            sincospi((double)positions[i >> 6] * a.rates.f[i & 63], &sn, &cn);
            turn_of[i >> 6][i & 63] = make_double2(cn, sn);
            turn_f_of[i >> 6][i & 63] = make_float2((float)cn, (float)sn);
        }
        __syncthreads();
    }
    if (s < 0) return;
    const double2* turn = turn_of[of];
    float c[W], sn[W];
#pragma unroll
    for (int i = 0; i < W; ++i) {
        const float2 t = a.rotate && mine ? turn_f_of[of][e + i] : make_float2(1.f, 0.f);
        c[i] = t.x, sn[i] = t.y;
    }
    // (q_out may be q: a lane writes the entries that it has read)
    __nv_bfloat16* out = a.q_out + (size_t)token * a.out_stride;
    for (int head = begin; head < a.q_heads; head += BATCH * stride) {
#pragma unroll
        for (int k = 0; k < BATCH; ++k) {
            if (!mine || head + k * stride >= a.q_heads) continue;
            float x[2][W];
#pragma unroll
            for (int i = 0; i < W; ++i) {
                x[0][i] = q[k][0][i] * c[i] - q[k][1][i] * sn[i];
                x[1][i] = q[k][1][i] * c[i] + q[k][0][i] * sn[i];
            }
            store_bf16<W>(out + (head + k * stride) * a.l.hd, e, x[0]);
            store_bf16<W>(out + (head + k * stride) * a.l.hd, half + e, x[1]);
        }
        load_queries(head + BATCH * stride);
    }
    // ---- keys and values: row r is head r / 2's key or value
    if (page < 0) return;  // no page for this position: nothing is stored
    const char* k_rows = static_cast<const char*>(a.k) + (size_t)token * a.k_stride * (BF16 ? 2 : 4);
    const char* v_rows = static_cast<const char*>(a.v) + (size_t)token * a.v_stride * (BF16 ? 2 : 4);
    uint8_t* chunks = a.pool + a48p::chunk_at(a.l, page, 0);
    const bool bos = a.l.bits == 3 && pos == 0;  // the bos heads keep 4 bits
    const int bits = bos ? 4 : a.l.bits, L = (1 << (bits - 1)) - 1;
    const float eps = (float)a.eps, border = 0.5f - (float)L * 0x1p-19f;
    // x step + magic: the nearest multiple's code (q + L + 1) in the low byte of the sum, ties to even
    const float magic = 12582912.f + (float)(L + 1);
    Raw<BF16, W> next[2];  // of the next row
    auto load_row = [&](int r) {
        next[0].clear(), next[1].clear();
        if (mine && r < 2 * a.l.kv_heads) {
            const char* row = (r & 1 ? v_rows : k_rows) + (size_t)(r >> 1) * row_bytes;
            next[0].load(row, e);
            next[1].load(row, half + e);
        }
    };
    load_row(begin);
    for (int r = begin; r - lane / G < 2 * a.l.kv_heads; r += stride) {  // (the same for the warp)
        const int which = r & 1, head = r >> 1;
        const bool there = mine && head < a.l.kv_heads, turned = a.rotate && !which;
        const Raw<BF16, W> lo = next[0], hi = next[1];
        load_row(r + stride);
        float x[2][W];
        // an entry in float64
        auto exact = [&](int h, int i) {
            if (!turned) return (double)(h ? hi[i] : lo[i]);
            const double2 t = turn[e + i];
            return h == 0 ? (double)lo[i] * t.x - (double)hi[i] * t.y : (double)hi[i] * t.x + (double)lo[i] * t.y;
        };
        // (a maximum that keeps what is no number: a head with a NaN has none for a scale, and reads as none)
        float top = 0.f;
#pragma unroll
        for (int i = 0; i < W; ++i) {
            x[0][i] = turned ? lo[i] * c[i] - hi[i] * sn[i] : lo[i];
            x[1][i] = turned ? hi[i] * c[i] + lo[i] * sn[i] : hi[i];
            top = max_or_nan(top, max_or_nan(fabsf(x[0][i]), fabsf(x[1][i])));
        }
        float gamma_f = top;
#pragma unroll
        for (int o = G / 2; o > 0; o >>= 1) gamma_f = max_or_nan(gamma_f, __shfl_xor_sync(0xffffffffu, gamma_f, o));
        double gamma = turned && gamma_f == gamma_f ? 0.0 : (double)gamma_f;
        if (turned && there && top >= gamma_f * (1.f - 0x1p-20f)) {
#pragma unroll
            for (int i = 0; i < W; ++i) gamma = fmax(gamma, fmax(fabs(exact(0, i)), fabs(exact(1, i))));
        }
#pragma unroll
        for (int o = G / 2; o > 0; o >>= 1) gamma = fmax(gamma, __shfl_xor_sync(0xffffffffu, gamma, o));
        const float step = __fdividef((float)L, gamma_f + eps);
        uint32_t u[2][W];
        float worst = 0.f;
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int i = 0; i < W; ++i) {
                const float sum = fmaf(x[h][i], step, magic);
                worst = fmaxf(worst, fabsf(fmaf(x[h][i], step, magic - sum)));
                u[h][i] = __float_as_uint(sum);
            }
        // (out of the bounds' reach: numbers so small or so large, or none, whose codes above may be more than `bits` wide)
        if (there && (worst > border || !(gamma_f > 0x1p-100f && gamma_f < 0x1p100f))) {
            const double multiple = (double)L / (gamma + a.eps);
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < W; ++i) u[h][i] = (uint32_t)(min(max(__double2int_rn(multiple * exact(h, i)), -(L + 1)), L) + L + 1);
        }
        uint8_t* chunk = chunks + (size_t)min(head, a.l.kv_heads - 1) * a.l.chunk;
        uint8_t* dst = bos ? chunk + a.l.bos + which * (a.l.padded / 2) : chunk + which * a.l.v_codes + slot * a.l.row;
        const uint32_t zero = 1u << (bits - 1);
        const int pad = head < a.l.kv_heads ? a.l.padded - a.l.hd : 0;  // entries past the head hold the code of 0
        if (bits != 3) {
            if (there) {
                store_codes<W>(dst, e, bits, u[0]);
                store_codes<W>(dst, half + e, bits, u[1]);
            }
            uint32_t z[W];
#pragma unroll
            for (int i = 0; i < W; ++i) z[i] = zero;
            for (int i = W * l; i < pad; i += W * G) store_codes<W>(dst, a.l.hd + i, bits, z);
        } else {
            uint8_t* buf = &row_codes[threadIdx.x >> 5][lane & ~(G - 1)][0];
            if (there) {
#pragma unroll
                for (int i = 0; i < W; i += 2) {
                    *reinterpret_cast<uint16_t*>(buf + e + i) = (uint16_t)__byte_perm(u[0][i], u[0][i + 1], 0x0040);
                    *reinterpret_cast<uint16_t*>(buf + half + e + i) = (uint16_t)__byte_perm(u[1][i], u[1][i + 1], 0x0040);
                }
            }
            for (int i = l; i < pad; i += G) buf[a.l.hd + i] = (uint8_t)zero;
            __syncwarp();
            if (head < a.l.kv_heads)
                for (int i = l; i < 3 * a.l.padded / 32; i += G) reinterpret_cast<uint32_t*>(dst)[i] = word_of_triples(buf, i);
            __syncwarp();  // the bytes are free again
        }
        if (l == 0 && head < a.l.kv_heads) {
            const float scale = turned ? (float)(gamma * (1.0 / L)) : __fdiv_rn(gamma_f, (float)L);
            reinterpret_cast<float*>(chunk + (which ? a.l.v_scales : a.l.k_scales))[slot] = scale;
        }
    }
}

template <bool BF16>
cudaError_t launch_write(WriteArgs& a, cudaStream_t st) {
    const int half = a.l.hd / 2, wide = a.l.hd % 8 == 0 ? 4 : 2;
    const int group = wide == 4 ? (half <= 32 ? 8 : 16) : (half <= 32 ? 16 : 32);  // (four lanes at least have room for 32 entries)
    // Few tokens: their heads are spread over blocks; many: a block takes four tokens, whose angles take as long as one's.
    a.tokens = a.b.n_tokens >= 8 * 148 ? MAX_TOKENS : 1;
    const int per = kWarps / a.tokens * (32 / group), most = a.q_heads > 2 * a.l.kv_heads ? a.q_heads : 2 * a.l.kv_heads;
    const int rounds = (most + per - 1) / per, blocks = (a.b.n_tokens + a.tokens - 1) / a.tokens;
    int slices = a.tokens > 1 ? 1 : (8 * 148 + blocks - 1) / blocks;
    slices = slices < rounds ? slices : rounds;
    auto kernel = wide == 4 ? (group == 8 ? paged_write_kernel<BF16, 4, 8> : paged_write_kernel<BF16, 4, 16>)
                            : (group == 16 ? paged_write_kernel<BF16, 2, 16> : paged_write_kernel<BF16, 2, 32>);
    return a48_launch_pdl(kernel, dim3(blocks, slices), dim3(32 * kWarps), 0, st, a);
}

// E entries from e on of a code row, as codes minus their offset.  (An integer below 2^23 or-ed into 2^23's pattern is the
// float 2^23 plus it.)
template <int E>
__device__ __forceinline__ void read_codes(const uint8_t* __restrict__ row, int e, int bits, float (&x)[E]) {
    const float off = 8388608.f + (float)(1 << (bits - 1));
    auto entry = [&](uint32_t field) { return __uint_as_float(0x4b000000u | field) - off; };
    if (bits == 8) {
#pragma unroll
        for (int i = 0; i < E; i += 4) {
            const uint32_t w = __ldg(reinterpret_cast<const uint32_t*>(row + e + i));
#pragma unroll
            for (int j = 0; j < 4; ++j) x[i + j] = __uint_as_float(__byte_perm(w, 0x4b000000u, 0x7440 + j)) - off;  // bytes w[j] 0 0 4b
        }
    } else if (bits == 4) {
        const uint32_t w = E == 8 ? __ldg(reinterpret_cast<const uint32_t*>(row + e / 2)) : __ldg(reinterpret_cast<const unsigned short*>(row + e / 2));
#pragma unroll
        for (int i = 0; i < E; ++i) x[i] = entry((w >> (4 * i)) & 15u);
    } else {
        // entry n of 16 at bits 3n of three halves side by side, 15 bits of each; the last one's bits on top of them
        const unsigned short* h = reinterpret_cast<const unsigned short*>(row + (e >> 5) * 12) + ((e >> 4) & 1);
        const uint32_t a = __ldg(h), b = __ldg(h + 2), c = __ldg(h + 4);
        const uint32_t lo = (a & 0x7fffu) | (b << 15);                                                   // entries 0 .. 9
        const uint32_t hi = (c & 0x7fffu) | ((a >> 15) << 15) | ((b >> 15) << 16) | ((c >> 15) << 17);  // 10 .. 15
        const int n = e & 15;
        const uint32_t v = n < 8 ? lo >> (3 * n) : n == 8 ? ((lo >> 24) & 63u) | (hi << 6) : hi >> 6;
#pragma unroll
        for (int i = 0; i < E; ++i) x[i] = entry((v >> (3 * i)) & 7u);
    }
}

// A block takes READ_TOKENS tokens (and a slice of their heads): where they lie is found once, a token per lane, and then
// every load is independent of every other.  LANES lanes share a head vector, E entries each, so that a store is 16 bytes (8
// where the head dimension does not divide by 8).  Items are (token, head, keys or values); a position without a page reads
// as zero.
template <bool BF16, int E, int BITS, int LANES>
__global__ void __launch_bounds__(32 * kWarps) paged_read_kernel(const Layout l, const Batch b, const uint8_t* __restrict__ pool,
                                                                 void* __restrict__ k_out, void* __restrict__ v_out) {
    constexpr int PER = 32 / LANES;  // head vectors that a warp takes at a time
    __shared__ const uint8_t* chunks_of[READ_TOKENS];  // of the token's page, head 0; none: no page
    __shared__ int pos_of[READ_TOKENS], there[READ_TOKENS];
    a48_pdl_prologue();
    const int lane = threadIdx.x & 31, first_token = blockIdx.x * READ_TOKENS;
    if (threadIdx.x < 32) {
        // the first token's sequence or the one behind which it lies, then on from there
        int s = max(0, a48p::last_at_most(b.n_seqs, first_token, lane, [&](int i) { return (long long)__ldg(b.q_start + i); }));
        const int token = first_token + lane;
        if (lane < READ_TOKENS) {
            int end = __ldg(b.q_start + s + 1);
            while (token >= end && s + 1 < b.n_seqs) end = __ldg(b.q_start + ++s + 1);
            const int first = __ldg(b.q_start + s);
            const bool in = token >= first && token < end && token < b.n_tokens;
            const int pos = __ldg(b.kv_len + s) - (end - first) + (token - first), page = in ? a48p::page_of(l, b, s, pos) : -1;
            chunks_of[lane] = page >= 0 ? pool + a48p::chunk_at(l, page, 0) : nullptr;
            pos_of[lane] = pos;
            there[lane] = in;
        }
    }
    __syncthreads();
    const int e = E * (lane & (LANES - 1)), slots = l.page - 1, chunk_bytes = l.chunk, hd = l.hd, rows = 2 * l.kv_heads;
    if (e >= hd) return;
    // a warp takes a token's rows of its slice, then the next token's
    const int warp = threadIdx.x >> 5, begin = blockIdx.y * PER + lane / LANES;
    for (int t = warp; t < READ_TOKENS; t += kWarps) {
        if (!there[t]) continue;
        const uint8_t* chunks = chunks_of[t];
        const int pos = pos_of[t], slot = pos & slots;
        const bool bos = BITS == 3 && pos == 0, page = chunks != nullptr;
        const int codes[2] = {bos ? l.bos : slot * l.row, bos ? l.bos + l.padded / 2 : l.v_codes + slot * l.row};
        const int scales[2] = {l.k_scales + 4 * slot, l.v_scales + 4 * slot};
        const size_t out_row = (size_t)(first_token + t) * (rows / 2) * hd + e;
#pragma unroll 4
        for (int i = begin; i < rows; i += gridDim.y * PER) {
            const int head = i >> 1, which = i & 1;
            float x[E];
#pragma unroll
            for (int j = 0; j < E; ++j) x[j] = 0.f;
            if (page) {
                const uint8_t* chunk = chunks + (size_t)head * chunk_bytes;
                const float scale = __ldg(reinterpret_cast<const float*>(chunk + (which ? scales[1] : scales[0])));
                const uint8_t* row = chunk + (which ? codes[1] : codes[0]);
                if (BITS == 3 && bos) read_codes<E>(row, e, 4, x);
                else read_codes<E>(row, e, BITS, x);
#pragma unroll
                for (int j = 0; j < E; ++j) x[j] *= scale;
            }
            void* out = which ? v_out : k_out;
            const size_t at = out_row + (size_t)head * hd;
            if constexpr (BF16) {
                uint32_t w[E / 2];
#pragma unroll
                for (int j = 0; j < E / 2; ++j) {
                    const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * j], x[2 * j + 1]);
                    w[j] = *reinterpret_cast<const uint32_t*>(&h);
                }
                if constexpr (E == 8) *reinterpret_cast<uint4*>(static_cast<uint16_t*>(out) + at) = make_uint4(w[0], w[1], w[2], w[3]);
                else *reinterpret_cast<uint2*>(static_cast<uint16_t*>(out) + at) = make_uint2(w[0], w[1]);
            } else {
                *reinterpret_cast<float4*>(static_cast<float*>(out) + at) = make_float4(x[0], x[1], x[2], x[3]);
            }
        }
    }
}

template <bool BF16, int E, int LANES>
cudaError_t launch_read(const Layout& l, const Batch& b, const uint8_t* pool, void* k_out, void* v_out, cudaStream_t st) {
    const int steps = (2 * l.kv_heads + 32 / LANES - 1) / (32 / LANES);  // of a warp over one token
    const int blocks = (b.n_tokens + READ_TOKENS - 1) / READ_TOKENS;
    int slices = (8 * 148 + blocks - 1) / blocks;
    slices = slices < steps ? slices : steps;
    const dim3 grid(blocks, slices);
    auto kernel = l.bits == 8 ? paged_read_kernel<BF16, E, 8, LANES> : l.bits == 4 ? paged_read_kernel<BF16, E, 4, LANES> : paged_read_kernel<BF16, E, 3, LANES>;
    return a48_launch_pdl(kernel, grid, dim3(32 * kWarps), 0, st, l, b, pool, k_out, v_out);
}
template <bool BF16, int E>
cudaError_t launch_read(const Layout& l, const Batch& b, const uint8_t* pool, void* k_out, void* v_out, cudaStream_t st) {
    return l.hd <= 8 * E    ? launch_read<BF16, E, 8>(l, b, pool, k_out, v_out, st)
           : l.hd <= 16 * E ? launch_read<BF16, E, 16>(l, b, pool, k_out, v_out, st)
                            : launch_read<BF16, E, 32>(l, b, pool, k_out, v_out, st);
}

// Rotation rates for a base and head dimension; the last table of this host thread is kept, decode loops ask for one.
const Rates& rates_of(float base, int half) {
    thread_local Rates r;
    thread_local float last_base = 0.f;
    thread_local int last_half = 0;
    if (base != last_base || half != last_half) {
        for (int i = 0; i < half; ++i) r.f[i] = pow((double)base, -(double)i / (double)half) * 0.318309886183790671538;  // 1 / pi
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
        if (n_heads <= 0) return BITNET_A48_ERR_SHAPE;
        if (n_heads > 65535) return BITNET_A48_ERR_LIMIT;
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
    A48_CUDA_TRY(x_bf16 ? launch_write<true>(a, (cudaStream_t)stream) : launch_write<false>(a, (cudaStream_t)stream));
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
    const Batch b = a48p::batch_of(*batch);
    const uint8_t* pool = static_cast<const uint8_t*>(pool_dev);
    const cudaStream_t cu = (cudaStream_t)stream;
    const cudaError_t e = !y_bf16 ? launch_read<false, 4>(l, b, pool, k_out_dev, v_out_dev, cu)
                          : l.hd % 8 == 0 ? launch_read<true, 8>(l, b, pool, k_out_dev, v_out_dev, cu)
                                          : launch_read<true, 4>(l, b, pool, k_out_dev, v_out_dev, cu);
    A48_CUDA_TRY(e);
    return BITNET_A48_OK;
}

}  // extern "C"
