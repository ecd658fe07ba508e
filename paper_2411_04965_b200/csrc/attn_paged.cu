// Causal attention of new tokens over the paged low-bit cache, with an optional sliding window beside which the first
// tokens of a sequence stay visible.
//
//   out[i] = sum_j softmax_j(scale q[i] . k[j]) v[j]   over j <= p, and with a window w: j > p - w or j < sinks
//
// p the position of token i.  k[j] = sk[j] c[j] with integer codes c, so the score is (q . c[j]) sk[j] scale, and the
// value's scale goes to the probability.
#include "paged.cuh"

namespace {

using a48p::Batch;
using a48p::Layout;

struct AttnArgs {
    Layout l;
    Batch b;
    const uint8_t* pool;
    const __nv_bfloat16* q;
    __nv_bfloat16* out;
    long long q_stride, out_stride;
    int heads, group, window, sinks;
    float scale;
};

// One warp per (token, query head), lane l owning entries 4l .. 4l+3 of the head: any shape, one key at a time.
__global__ void __launch_bounds__(256) attn_paged_simple_kernel(const AttnArgs a) {
    a48_pdl_prologue();
    const int lane = threadIdx.x & 31, token = blockIdx.x, h = blockIdx.y * 8 + (threadIdx.x >> 5);
    if (h >= a.heads) return;
    const int s = a48p::sequence_of(a.b, token, lane);
    if (s < 0) return;
    const int first = __ldg(a.b.q_start + s), end = __ldg(a.b.q_start + s + 1);
    const int pos = __ldg(a.b.kv_len + s) - (end - first) + (token - first);
    const int e = 4 * lane, kvh = h / a.group;
    const bool mine = e < a.l.hd;
    float q[4] = {}, o[4] = {};
    if (mine)
#pragma unroll
        for (int i = 0; i < 4; ++i) q[i] = __bfloat162float(a.q[(size_t)token * a.q_stride + (size_t)h * a.l.hd + e + i]);
    float m = -INFINITY, sum = 0.f;
    const int last = (int)min((long long)pos, ((long long)a.b.max_pages << a.l.page_shift) - 1);  // the table's reach
    const int behind = a.window > 0 ? max(0, pos - a.window + 1) : 0;  // first position inside the window
    for (int j = min(a.sinks, behind) > 0 ? 0 : behind; j <= last; ++j) {
        if (j >= a.sinks && j < behind) j = behind;
        const int page = a48p::page_of(a.l, a.b, s, j);
        if (page < 0) continue;
        const int slot = j & (a.l.page - 1);
        const uint8_t* chunk = a.pool + a48p::chunk_at(a.l, page, kvh);
        const bool bos = a.l.bits == 3 && j == 0;
        float4 k = make_float4(0.f, 0.f, 0.f, 0.f), v = k;
        if (mine) {
            k = bos ? a48p::four_entries(chunk + a.l.bos, e, 4) : a48p::four_entries(chunk + slot * a.l.row, e, a.l.bits);
            v = bos ? a48p::four_entries(chunk + a.l.bos + a.l.padded / 2, e, 4)
                    : a48p::four_entries(chunk + a.l.v_codes + slot * a.l.row, e, a.l.bits);
        }
        float dot = q[0] * k.x + q[1] * k.y + q[2] * k.z + q[3] * k.w;
#pragma unroll
        for (int x = 16; x > 0; x >>= 1) dot += __shfl_xor_sync(0xffffffffu, dot, x);
        const float score = dot * (__ldg(reinterpret_cast<const float*>(chunk + a.l.k_scales) + slot) * a.scale);
        const float m_new = fmaxf(m, score), corr = expf(m - m_new), p = expf(score - m_new);
        const float pv = p * __ldg(reinterpret_cast<const float*>(chunk + a.l.v_scales) + slot);
        m = m_new;
        sum = sum * corr + p;
        o[0] = o[0] * corr + pv * v.x;
        o[1] = o[1] * corr + pv * v.y;
        o[2] = o[2] * corr + pv * v.z;
        o[3] = o[3] * corr + pv * v.w;
    }
    const float inv = sum > 0.f ? 1.f / sum : 0.f;
    if (mine) {
        __nv_bfloat162* out = reinterpret_cast<__nv_bfloat162*>(a.out + (size_t)token * a.out_stride + (size_t)h * a.l.hd + e);
        out[0] = __floats2bfloat162_rn(o[0] * inv, o[1] * inv);
        out[1] = __floats2bfloat162_rn(o[2] * inv, o[3] * inv);
    }
}

}  // namespace

extern "C" {

size_t bitnet_a48_attention_paged_workspace_bytes(const bitnet_a48_paged_cache* cache, const bitnet_a48_paged_batch* batch, int n_heads,
                                                  int window, int sinks) {
    (void)cache, (void)batch, (void)n_heads, (void)window, (void)sinks;
    return 0;
}

bitnet_a48_status bitnet_a48_attention_paged(const bitnet_a48_paged_cache* cache, const void* pool_dev,
                                             const bitnet_a48_paged_batch* batch, int n_heads, const uint16_t* q_dev,
                                             long long q_stride, float scale, int window, int sinks, uint16_t* out_dev,
                                             long long out_stride, void* workspace_dev, size_t workspace_bytes, void* stream) {
    bitnet_a48_status st = a48p::check(cache, pool_dev, batch);
    if (st != BITNET_A48_OK) return st;
    if (n_heads <= 0 || n_heads % cache->n_kv_heads != 0) return BITNET_A48_ERR_SHAPE;
    if (n_heads > 65535) return BITNET_A48_ERR_LIMIT;
    if (window < 0 || sinks < 0 || !(scale >= 0.f) || scale > 3e38f) return BITNET_A48_ERR_INVALID_ARG;
    const long long width = (long long)n_heads * cache->head_dim;
    if ((st = a48p::check_rows(q_dev, q_stride, width, 2)) != BITNET_A48_OK) return st;
    if ((st = a48p::check_rows(out_dev, out_stride, width, 2)) != BITNET_A48_OK) return st;
    const size_t need = bitnet_a48_attention_paged_workspace_bytes(cache, batch, n_heads, window, sinks);
    if (need && (!workspace_dev || workspace_bytes < need)) return BITNET_A48_ERR_NOMEM;
    if (!a48_aligned16(workspace_dev)) return BITNET_A48_ERR_ALIGNMENT;
    if (!a48_have_device()) return BITNET_A48_ERR_CUDA;
    AttnArgs a;
    a.l = a48p::layout_of(*cache);
    a.b = a48p::batch_of(*batch);
    a.pool = static_cast<const uint8_t*>(pool_dev);
    a.q = reinterpret_cast<const __nv_bfloat16*>(q_dev);
    a.out = reinterpret_cast<__nv_bfloat16*>(out_dev);
    a.q_stride = q_stride, a.out_stride = out_stride;
    a.heads = n_heads, a.group = n_heads / cache->n_kv_heads;
    a.window = window, a.sinks = window > 0 ? sinks : 0;
    a.scale = scale > 0.f ? scale : 1.f / sqrtf((float)cache->head_dim);
    const dim3 grid(batch->n_tokens, (n_heads + 7) / 8);
    A48_CUDA_TRY(a48_launch_pdl(attn_paged_simple_kernel, grid, dim3(256), 0, (cudaStream_t)stream, a));
    return BITNET_A48_OK;
}

}  // extern "C"
