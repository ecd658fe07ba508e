// What is read off rows of logits x: with d = (x - max) / T, the log probability d_t - ln sum e^d of a given token t, its
// place in the order of all tokens, the entropy ln sum e^d - sum e^d d / sum e^d, and the k most likely tokens.
//
// One pass.  A thread's sums are taken against a reference of its own and joined at the end, in base 2: 2^((x - r) c), c = log2 e / T.
// The reference is the largest logit so far, of the thread and of what its warp saw at first (a later one is above that once or twice
// in a row, so moving costs nothing that can be measured).  So the row's largest logit counts as 1 exactly, and where it is all but
// certain its log probability and the entropy keep what little the others leave of them, and their signs.  (A reference that only moved
// for logits far above it gave 4e-6 for -4e-8.)
//
// The largest k.  The first segments that a block of threads visits are kept in registers; the k-th largest of the threads'
// maxima over them bounds the row's k-th largest logit from below, and everything at or above that bound, in these segments
// and in the rest of the row, is noted in a list (about 4 k entries of a row of 32000).  The list is then ranked by (logit,
// lower index first).  Segments are visited in an order that leaps over the row, so that a row that rises or falls with the
// index does not fool the bound.  Where many logits equal the bound (masked tokens, coarse types) only what lies above it is
// noted and equal ones are taken from the front of the row; where the list still overflows, the k-th largest is found digit
// by digit over the whole row.  All of this costs time only: the answer is exact in every case.
#include "fp8.cuh"
#include "softmax_sums.cuh"

namespace {

using a48f8::Sums;

constexpr int MAX_TOP = 64, SPARE = 32;
// Threads to a row: many blocks of 256 to an SM, or 1024 where there are fewer rows than SMs.
constexpr int MANY = 256, FEW = 1024;
constexpr int SAMPLED = 32;  // logits of a thread that the bound is made of, of MANY threads; of FEW, half as many
using a48f8::LN2;

struct Args {
    const void* x;
    const void* tokens;
    float* logprob;
    float* entropy;
    int32_t* rank;
    int32_t* top_ids;
    float* top_logprobs;
    long long stride;
    int V, top, tokens64;
    int noted_most, list_most;     // entries that a thread may note, and that all of them may
    int segments, leap, leap_fewer;  // most segments of a row; how far apart those visited one after the other are, for so many and one fewer
    float c, inv_t;  // log2 e / temperature, 1 / temperature
};

// Unsigned numbers in the order of the floats; -0 counts as 0.
__device__ __forceinline__ uint32_t order_of(float x) {
    const uint32_t b = __float_as_uint(x + 0.f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float of_order(uint32_t u) { return __uint_as_float(u & 0x80000000u ? u & 0x7fffffffu : ~u); }
__device__ __forceinline__ unsigned long long entry_of(float x, int id) { return (unsigned long long)order_of(x) << 32 | (uint32_t)~id; }

template <bool BF16>
struct Row {
    static constexpr int E = BF16 ? 8 : 4;  // logits in 16 bytes
    const void* p;
    __device__ __forceinline__ float at(int i) const {
        return BF16 ? __uint_as_float((uint32_t)__ldg(reinterpret_cast<const uint16_t*>(p) + i) << 16) : __ldg(reinterpret_cast<const float*>(p) + i);
    }
    __device__ __forceinline__ uint4 load(int head, int vec) const {
        return __ldg(reinterpret_cast<const uint4*>(reinterpret_cast<const char*>(p) + (size_t)head * (BF16 ? 2 : 4)) + vec);
    }
    static __device__ __forceinline__ void widen(const uint4& u, float (&v)[E]) {
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
        if (BF16) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                v[2 * i] = __uint_as_float(w[i] << 16);
                v[(2 * i + 1) % E] = __uint_as_float(w[i] & 0xffff0000u);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(w[i]);
        }
    }
};

template <bool BF16, int THREADS>
struct Walk {
    Row<BF16> row;
    Sums sums;
    float fresh;  // terms that are not in sums.s yet: beside a 1 there they would be lost one by one, and together are not
    float c;
    float own, at_or_above;  // a logit counts as ahead of the token's from there on: `own` before the token, the next number behind it
    float least;           // logits at or above it go to the list
    int token, ahead;      // ahead: logits that come before the token's in the order
    uint2* notes;  // this thread's, THREADS apart: the logit's bits and index
    int noted, noted_most;

    __device__ __forceinline__ void fold() {
        sums.s += fresh;
        fresh = 0.f;
    }
    template <int N>
    __device__ __forceinline__ void take(const float (&v)[N], int id) {
        float m = v[0];
#pragma unroll
        for (int j = 1; j < N; ++j) m = fmaxf(m, v[j]);
        if (m > sums.r) {
            fold();
            sums.move(m, c);
        }
#pragma unroll
        for (int j = 0; j < N; ++j) sums.add(v[j], c, fresh);
        const float mark = id < token ? own : at_or_above;
        if (m >= mark) {
#pragma unroll
            for (int j = 0; j < N; ++j) ahead += v[j] >= mark;
        }
        if (m >= least) {
#pragma unroll
            for (int j = 0; j < N; ++j)
                if (v[j] >= least) {  // (a list for all threads, with an atomic for each entry, took 158 us for 4096 x 32000, 20 to a row)
                    if (noted < noted_most) notes[noted * THREADS] = make_uint2(__float_as_uint(v[j]), id + j);
                    ++noted;
                }
        }
    }
};

// For all threads of the block together: how many of them before this one, and in all, have the flag.
template <int WARPS>
__device__ __forceinline__ int flags_before(bool flag, uint32_t* warp_counts, int& total) {
    const uint32_t votes = __ballot_sync(0xffffffffu, flag);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (lane == 0) warp_counts[warp] = __popc(votes);
    __syncthreads();
    int before = 0;
    total = 0;
    for (int w = 0; w < WARPS; ++w) {
        before += w < warp ? warp_counts[w] : 0;
        total += warp_counts[w];
    }
    __syncthreads();
    return before + __popc(votes & ((1u << lane) - 1));
}

template <bool BF16, int THREADS>
__global__ void __launch_bounds__(THREADS, THREADS == MANY ? 4 : 1) logprobs_kernel(const Args a) {
    constexpr int E = Row<BF16>::E, WARPS = THREADS / 32;
    constexpr int SAMPLE = (THREADS == MANY ? SAMPLED : SAMPLED / 2) / E;  // segments (16 bytes to a thread) kept in registers
    extern __shared__ unsigned long long list[];  // [list_most], and the threads' notes; not there where nothing is listed
    uint2* notes = reinterpret_cast<uint2*>(list + a.list_most);
    __shared__ float best[THREADS];
    __shared__ float4 part[WARPS];
    __shared__ uint32_t hist[256], counts[WARPS];
    __shared__ uint32_t count, taken, found[2];
    const int t = threadIdx.x, lane = t & 31, warp = t >> 5;
    const long long r = blockIdx.x;
    Walk<BF16, THREADS> w;
    w.row.p = reinterpret_cast<const char*>(a.x) + (size_t)(r * a.stride) * (BF16 ? 2 : 4);
    a48_pdl_prologue();
    w.c = a.c;
    w.notes = notes + t;
    w.noted = 0;
    w.noted_most = a.noted_most;
    w.ahead = 0;
    w.token = -1;
    w.own = w.at_or_above = w.least = __uint_as_float(0x7fc00000u);  // nothing is above no number
    // whole 16 bytes between the first and last few logits, which threads 0 .. E - 1 and E .. 2 E - 1 take one by one
    const int skew = (int)(reinterpret_cast<uintptr_t>(w.row.p) & 15u) / (BF16 ? 2 : 4), head = min(a.V, skew ? E - skew : 0);
    const int vecs = (a.V - head) / E, tail = head + vecs * E;
    const int segments = (vecs + THREADS - 1) / THREADS;
    const int leap = segments == a.segments ? a.leap : a.leap_fewer;
    uint4 kept[SAMPLE];
    int at = 0;  // segment
#pragma unroll
    for (int i = 0; i < SAMPLE; ++i) {
        const int vec = at * THREADS + t;
        const uint32_t none = BF16 ? 0xff80ff80u : 0xff800000u;  // -inf
        kept[i] = i < segments && vec < vecs ? w.row.load(head, vec) : make_uint4(none, none, none, none);
        at += leap;
        at -= at >= segments ? segments : 0;
    }
    if (a.tokens) {
        const long long token = a.tokens64 ? __ldg(reinterpret_cast<const long long*>(a.tokens) + r) : __ldg(reinterpret_cast<const int*>(a.tokens) + r);
        if (token >= 0 && token < a.V) {
            w.token = (int)token;
            w.own = w.row.at(w.token);
            w.at_or_above = of_order(order_of(w.own) + 1);
        }
    }
    const bool top = a.top > 0;
    const int edge = t < E ? (t < head ? t : -1) : t < 2 * E && tail + t - E < a.V ? tail + t - E : -1;
    float edge_x[1] = {-INFINITY};
    if (edge >= 0) edge_x[0] = w.row.at(edge);

    if (t == 0) count = taken = 0;
    float m = edge_x[0];
#pragma unroll
    for (int i = 0; i < SAMPLE; ++i) {
        float v[E];
        Row<BF16>::widen(kept[i], v);
#pragma unroll
        for (int j = 0; j < E; ++j) m = fmaxf(m, v[j]);
    }
    float first = m;
#pragma unroll
    for (int o = 16; o; o >>= 1) first = fmaxf(first, __shfl_xor_sync(0xffffffffu, first, o));
    w.sums.start(first);
    w.fresh = 0.f;
    bool strict = false;
    float bound = -INFINITY;
    if (top) {
        best[t] = m;
        __syncthreads();
        if (warp == 0) {  // the bound: halving the range of orders that holds the k-th largest of the threads' maxima
            uint32_t key[WARPS], hi = 0, lo = ~0u;
            int reach = 0;  // maxima at or above lo, k or more
#pragma unroll
            for (int i = 0; i < WARPS; ++i) {
                key[i] = order_of(best[i * 32 + lane]);
                const bool none = key[i] == order_of(-INFINITY);
                hi = max(hi, key[i]);
                lo = min(lo, none ? ~0u : key[i]);
                reach += !none;
            }
            hi = __reduce_max_sync(0xffffffffu, hi);
            lo = __reduce_min_sync(0xffffffffu, lo);
            reach = __reduce_add_sync(0xffffffffu, reach);
            if (reach < a.top) lo = hi = order_of(-INFINITY);
            while (lo < hi && reach > a.top + a.top / 4 + 2) {
                const uint32_t mid = lo + (hi - lo + 1) / 2;
                int n = 0;
#pragma unroll
                for (int i = 0; i < WARPS; ++i) n += key[i] >= mid;
                n = __reduce_add_sync(0xffffffffu, n);
                if (n >= a.top) {
                    lo = mid;
                    reach = n;
                } else {
                    hi = mid - 1;
                }
            }
            int same = 0;
#pragma unroll
            for (int i = 0; i < WARPS; ++i) same += key[i] == lo;
            same = __reduce_add_sync(0xffffffffu, same);
            if (lane == 0) {
                found[0] = lo;
                found[1] = lo == order_of(-INFINITY) || same > 32;
            }
        }
        __syncthreads();
        bound = of_order(found[0]);
        strict = found[1] != 0;
        w.least = strict ? of_order(found[0] + 1) : bound;
    }
    int seg = 0;
#pragma unroll
    for (int i = 0; i < SAMPLE; ++i) {
        float v[E];
        Row<BF16>::widen(kept[i], v);
        const int vec = seg * THREADS + t;
        if (i < segments && vec < vecs) w.take(v, head + vec * E);
        seg += leap;
        seg -= seg >= segments ? segments : 0;
    }
    if (edge >= 0) w.take(edge_x, edge);
    w.fold();
    for (int i = SAMPLE; i < segments; i += 4) {
        uint4 u[4];
        int id[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int vec = at * THREADS + t;
            id[q] = i + q < segments && vec < vecs ? vec : -1;
            if (id[q] >= 0) u[q] = w.row.load(head, vec);
            at += leap;
            at -= at >= segments ? segments : 0;
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            if (id[q] < 0) continue;
            float v[E];
            Row<BF16>::widen(u[q], v);
            w.take(v, head + id[q] * E);
        }
        w.fold();
    }
    if (t == 0 && w.token >= head && w.token < tail && (w.token - head) % E != 0)  // in the token's own 16 bytes, equal ones from it on do not count
        for (int i = w.token; i < min(tail, head + (w.token - head) / E * E + E); ++i) w.ahead -= w.row.at(i) == w.own;
    if (w.noted > 0) {  // into one list; more than fit are counted all the same
        const uint32_t to = atomicAdd(&count, w.noted > a.noted_most ? a.list_most + 1 : w.noted);
        for (int i = 0; i < min(w.noted, a.noted_most); ++i) {
            const uint2 e = w.notes[i * THREADS];
            if (to + i < (uint32_t)a.list_most) list[to + i] = entry_of(__uint_as_float(e.x), (int)e.y);
        }
    }
    // ---- joined
    float ref = w.sums.r;
#pragma unroll
    for (int o = 16; o; o >>= 1) ref = fmaxf(ref, __shfl_xor_sync(0xffffffffu, ref, o));
    w.sums.move(ref, a.c);
    float s = w.sums.s, d = w.sums.d;
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        s += __shfl_xor_sync(0xffffffffu, s, o);
        d += __shfl_xor_sync(0xffffffffu, d, o);
    }
    int ahead = __reduce_add_sync(0xffffffffu, w.ahead);
    if (lane == 0) part[warp] = make_float4(ref, s, d, __int_as_float(ahead));
    __syncthreads();
    Sums all;
    all.start(-INFINITY);
    ahead = 0;
    if (lane < WARPS) {
        all = {part[lane % WARPS].x, part[lane % WARPS].y, part[lane % WARPS].z};
        ahead = __float_as_int(part[lane % WARPS].w);
    }
    ahead = __reduce_add_sync(0xffffffffu, ahead);
#pragma unroll
    for (int o = WARPS / 2; o; o >>= 1) {
        const Sums more = {__shfl_xor_sync(0xffffffffu, all.r, o), __shfl_xor_sync(0xffffffffu, all.s, o), __shfl_xor_sync(0xffffffffu, all.d, o)};
        all.join(more, a.c);
    }
    all = {__shfl_sync(0xffffffffu, all.r, 0), __shfl_sync(0xffffffffu, all.s, 0), __shfl_sync(0xffffffffu, all.d, 0)};
    const bool valid = all.valid();
    const float log_s = log2f(all.s), nan = __uint_as_float(0x7fc00000u);
    if (t == 0) {
        if (a.logprob) a.logprob[r] = !valid ? nan : w.token < 0 ? 0.f : all.log_share(w.own, a.inv_t, log_s);
        if (a.entropy) a.entropy[r] = valid ? LN2 * (log_s - all.d / all.s) : nan;
        if (a.rank) a.rank[r] = valid && w.token >= 0 ? ahead : -1;
    }
    if (!top) return;
    int32_t* ids = a.top_ids + r * a.top;
    float* logps = a.top_logprobs + r * a.top;
    if (!valid) {
        if (t < a.top) {
            ids[t] = -1;
            logps[t] = nan;
        }
        return;
    }
    int n = (int)count;
    if (n > a.list_most) {  // the k-th largest of the row, eight bits at a time
        uint32_t prefix = 0;
        int need = a.top;
        for (int shift = 24; shift >= 0; shift -= 8) {
            if (t < 256) hist[t] = 0;
            __syncthreads();
            for (int i = t; i < a.V; i += THREADS) {
                const uint32_t o = order_of(w.row.at(i));
                if (shift == 24 || o >> (shift + 8) == prefix >> (shift + 8)) atomicAdd(&hist[o >> shift & 255u], 1u);
            }
            __syncthreads();
            if (t == 0) {
                int left = need, bin = 255;
                while ((int)hist[bin] < left) left -= (int)hist[bin--];
                found[0] = (uint32_t)bin;
                found[1] = (uint32_t)left;
            }
            __syncthreads();
            prefix |= found[0] << shift;
            need = (int)found[1];
            __syncthreads();
        }
        bound = of_order(prefix);
        strict = true;
        if (t == 0) count = 0;
        __syncthreads();
        for (int i = t; i < a.V; i += THREADS)
            if (w.row.at(i) > bound) list[atomicAdd(&count, 1u)] = entry_of(w.row.at(i), i);  // fewer than asked for
        __syncthreads();
        n = (int)count;
    }
    if (strict && n < a.top) {  // those that equal the bound, from the front of the row
        int have = n;
        for (int i0 = 0; have < a.top && i0 < a.V; i0 += THREADS) {
            const int i = i0 + t;
            const bool is = i < a.V && order_of(w.row.at(i)) == order_of(bound);
            int total;
            const int before = flags_before<WARPS>(is, counts, total);
            if (is && have + before < a.top) list[have + before] = entry_of(bound, i);
            have += total;
        }
        n = min(have, a.top);
        __syncthreads();
    }
    // at most 32 entries beyond those asked for (halving again the range that holds the k-th largest), then their order
    __shared__ unsigned long long shortlist[MAX_TOP + SPARE];
    const unsigned long long* from = list;
    if (n > a.top + SPARE) {
        if (warp == 0) {
            uint32_t lo = ~0u, hi = 0;
            for (int i = lane; i < n; i += 32) {
                lo = min(lo, (uint32_t)(list[i] >> 32));
                hi = max(hi, (uint32_t)(list[i] >> 32));
            }
            lo = __reduce_min_sync(0xffffffffu, lo);
            hi = __reduce_max_sync(0xffffffffu, hi);
            int reach = n;
            while (lo < hi && reach > a.top + SPARE) {
                const uint32_t mid = lo + (hi - lo + 1) / 2;
                int above = 0;
                for (int i = lane; i < n; i += 32) above += (uint32_t)(list[i] >> 32) >= mid;
                above = __reduce_add_sync(0xffffffffu, above);
                if (above >= a.top) {
                    lo = mid;
                    reach = above;
                } else {
                    hi = mid - 1;
                }
            }
            if (lane == 0) {
                found[0] = lo;
                found[1] = (uint32_t)reach;
            }
        }
        __syncthreads();
        if ((int)found[1] <= a.top + SPARE) {  // (more only where that many logits are equal)
            for (int i = t; i < n; i += THREADS)
                if ((uint32_t)(list[i] >> 32) >= found[0]) shortlist[atomicAdd(&taken, 1u)] = list[i];
            n = (int)found[1];
            from = shortlist;
            __syncthreads();
        }
    }
    for (int i = t; i < n; i += THREADS) {
        const unsigned long long mine = from[i];
        int place = 0;
        for (int j = 0; j < n; ++j) place += from[j] > mine;
        if (place < a.top) {
            ids[place] = (int)~(uint32_t)mine;
            logps[place] = all.log_share(of_order((uint32_t)(mine >> 32)), a.inv_t, log_s);
        }
    }
}

constexpr int NOTED_MOST = 16, LIST_MOST = 4096;

template <bool BF16, int THREADS>
bitnet_a48_status launch(const Args& a, int M, cudaStream_t st) {
    static std::atomic<bool> ready[64];
    A48_CUDA_TRY(a48_allow_smem(logprobs_kernel<BF16, THREADS>, (LIST_MOST + (size_t)NOTED_MOST * THREADS) * 8, ready));
    const size_t smem = a.top ? (a.list_most + (size_t)a.noted_most * THREADS) * 8 : 0;
    A48_CUDA_TRY(a48_launch_pdl(logprobs_kernel<BF16, THREADS>, dim3(M), dim3(THREADS), smem, st, a));
    return BITNET_A48_OK;
}

// A step near 0.618 n that shares no divisor with n, so that n steps visit all of 0 .. n - 1.
int leap_over(int n) {
    if (n < 3) return 1;
    int d = (int)(0.6180339887 * n);
    for (;; ++d) {
        int a = n, b = d;
        while (b) {
            const int c = a % b;
            a = b;
            b = c;
        }
        if (a == 1) return d;  // n - 1 at the latest
    }
}

// Joins the sums of the parts of a row's logits: eight rows to a block, 32 threads to a row.
__global__ void __launch_bounds__(256) score_join_kernel(const float4* __restrict__ stats, int parts, int M, int V, const void* tokens,
                                                         int tokens64, float c, float inv_t, const float* __restrict__ owns, float* __restrict__ logprob,
                                                         float* __restrict__ entropy) {
    __shared__ Sums sums[32][8];
    const int t = threadIdx.x, row = t & 7, lane = t >> 3, m = blockIdx.x * 8 + row;
    Sums all;
    all.start(-INFINITY);
    a48_pdl_prologue();
    if (m < M) {
#pragma unroll 4
        for (int i = lane; i < parts; i += 32) {
            const float4 f = __ldg(stats + (size_t)i * M + m);
            all.join({f.x, f.y, f.z}, c);
        }
    }
    sums[lane][row] = all;
    __syncthreads();
    for (int half = 16; half; half >>= 1) {
        if (lane < half) {
            all.join(sums[lane + half][row], c);
            sums[lane][row] = all;
        }
        __syncthreads();
    }
    if (lane || m >= M) return;
    const long long token = tokens64 ? reinterpret_cast<const long long*>(tokens)[m] : reinterpret_cast<const int*>(tokens)[m];
    const float log_s = log2f(all.s), nan = __uint_as_float(0x7fc00000u);
    const bool taken = token >= 0 && token < V;
    logprob[m] = !all.valid() ? nan : taken ? all.log_share(owns[m], inv_t, log_s) : 0.f;
    entropy[m] = all.valid() ? LN2 * (log_s - all.d / all.s) : nan;
}

}  // namespace

namespace a48f8 {

bitnet_a48_status launch_score_join(const ScoreArgs& s, const ScoreParts& w, int M, int V, cudaStream_t st) {
    A48_CUDA_TRY(a48_launch_pdl(score_join_kernel, dim3((M + 7) / 8), dim3(256), 0, st, w.stats, w.parts, M, V, s.tokens, s.tokens64, s.c, s.inv_t, w.owns, s.logprob, s.entropy));
    return BITNET_A48_OK;
}

bitnet_a48_status launch_logprobs(const LogprobArgs& g, cudaStream_t st) {
    Args a = {};
    a.x = g.x;
    a.tokens = g.tokens;
    a.logprob = g.logprob;
    a.entropy = g.entropy;
    a.rank = g.rank;
    a.top_ids = g.top_ids;
    a.top_logprobs = g.top_logprobs;
    a.stride = g.stride;
    a.V = g.V;
    a.top = g.top;
    a.tokens64 = g.tokens64;
    a.c = (float)(1.4426950408889634 / (double)g.temperature);
    a.inv_t = 1.f / g.temperature;
    // fewer rows than SMs: more threads to a row (8 rows of 32000: 6.7 us for 8.9, of 128000: 14.6 us for 27.7)
    const int threads = g.M <= sm_count() && g.V >= 8192 ? FEW : MANY, vecs = g.V / (g.x_bf16 ? 8 : 4);
    a.segments = (vecs + threads - 1) / threads;
    a.leap = leap_over(a.segments);
    a.leap_fewer = leap_over(a.segments - 1);
    // Room for what is noted, which is top times row / sample: twice that, and for a thread 6 + 4 times its share (a row with a thread
    // that has more, or one far beyond these sizes, is only slower).  As little as that, since shared memory is what L1 has not.
    const double listed = (double)g.top * (1.0 + (double)g.V / (threads == MANY ? SAMPLED * MANY : SAMPLED / 2 * FEW));
    a.list_most = (int)(listed > (LIST_MOST - 256) / 2 ? LIST_MOST : 256 + 2 * listed);
    a.noted_most = (int)(4 * listed / threads > NOTED_MOST - 6 ? NOTED_MOST : 6 + 4 * listed / threads);
    if (threads == FEW) return g.x_bf16 ? launch<true, FEW>(a, g.M, st) : launch<false, FEW>(a, g.M, st);
    return g.x_bf16 ? launch<true, MANY>(a, g.M, st) : launch<false, MANY>(a, g.M, st);
}

}  // namespace a48f8
