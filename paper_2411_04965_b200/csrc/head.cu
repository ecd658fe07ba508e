// extern "C" entry points of the 8-bit head: argument checks, then the launches.
#include <cmath>

#include "fp8.cuh"

namespace {

constexpr int kMaxFeatures = 1 << 20;
constexpr int kMaxTop = 64;
constexpr int kMaxRows = 1 << 30;

// Channels of an e4m3 matrix: tensor copies want rows of a multiple of 16 bytes.
bool channels_ok(int K) { return K > 0 && K <= kMaxFeatures && K % 16 == 0; }
bool features_ok(int N) { return N > 0 && N <= kMaxFeatures; }
// Rows of fp32 or bf16 that are read 16 bytes at a time.
bool rows_ok(const void* p, long long stride, int bf16) { return a48_aligned16(p) && stride % (bf16 ? 8 : 4) == 0; }
size_t up256(size_t n) { return (n + 255) / 256 * 256; }

bool temperature_ok(float t) { return t >= 1e-30f && t <= 1e30f; }

// Parts of the workspace of bitnet_a48_score.  The logits of few tokens are stored after all: they stay in L2, and the kernel that
// streams the weight for few tokens is worth more than what they cost.
struct ScoreSpace {
    size_t codes, scale, stats, owns, end;
    ScoreSpace(int M, int N, int K) {
        const bool few = a48f8::few_supported(M, K);
        codes = 0;
        scale = codes + up256((size_t)M * K);
        stats = scale + up256((size_t)a48f8::blocks(K) * M * 4);
        owns = stats + up256(few ? (size_t)M * logits_stride(N) * 4 : a48f8::score_stats(M, N) * sizeof(float4));
        end = owns + up256(few ? 0 : (size_t)M * 4);
    }
    static long long logits_stride(int N) { return (N + 3) / 4 * 4ll; }
};

bitnet_a48_status check_quant(const void* X, int rows, int K, long long stride, int bf16, const void* codes, const void* scale) {
    if (!X || !codes || !scale) return BITNET_A48_ERR_INVALID_ARG;
    if (rows <= 0 || !channels_ok(K)) return BITNET_A48_ERR_SHAPE;
    if (rows > kMaxRows) return BITNET_A48_ERR_LIMIT;
    if (rows > 1 && stride < K) return BITNET_A48_ERR_SHAPE;
    if (!rows_ok(X, rows > 1 ? stride : K, bf16) || !a48_aligned16(codes) || !a48_aligned16(scale)) return BITNET_A48_ERR_ALIGNMENT;
    return BITNET_A48_OK;
}

}  // namespace

extern "C" {

bitnet_a48_status bitnet_a48_quant_fp8(const void* X_dev, long long x_stride, int x_bf16, int M, int K, const float* gain_dev, float norm_eps,
                                       uint8_t* codes_dev, float* scale_dev, void* stream) {
    const bitnet_a48_status s = check_quant(X_dev, M, K, x_stride, x_bf16, codes_dev, scale_dev);
    if (s != BITNET_A48_OK) return s;
    if (!(norm_eps >= 0.f) || std::isinf(norm_eps)) return BITNET_A48_ERR_INVALID_ARG;
    if (!a48_aligned16(gain_dev)) return BITNET_A48_ERR_ALIGNMENT;
    if (!a48_have_device()) return BITNET_A48_ERR_CUDA;
    return a48f8::launch_quant_rows(X_dev, x_bf16, M > 1 ? x_stride : K, gain_dev, norm_eps, M, K, codes_dev, scale_dev, (cudaStream_t)stream);
}

bitnet_a48_status bitnet_a48_quant_fp8_weight(const void* W_dev, long long w_stride, int w_bf16, int N, int K, uint8_t* codes_dev, float* scale_dev,
                                              void* stream) {
    const bitnet_a48_status s = check_quant(W_dev, N, K, w_stride, w_bf16, codes_dev, scale_dev);
    if (s != BITNET_A48_OK) return s;
    if (!features_ok(N)) return BITNET_A48_ERR_SHAPE;
    if (!a48_have_device()) return BITNET_A48_ERR_CUDA;
    return a48f8::launch_quant_weight(W_dev, w_bf16, N > 1 ? w_stride : K, N, K, codes_dev, scale_dev, (cudaStream_t)stream);
}

bitnet_a48_status bitnet_a48_linear_fp8(const uint8_t* codes_dev, const float* scale_dev, int M, const uint8_t* w_codes_dev, const float* w_scale_dev,
                                        int N, int K, void* Y_dev, long long y_stride, int y_bf16, void* stream) {
    if (!codes_dev || !scale_dev || !w_codes_dev || !w_scale_dev || !Y_dev) return BITNET_A48_ERR_INVALID_ARG;
    if (M <= 0 || !features_ok(N) || !channels_ok(K)) return BITNET_A48_ERR_SHAPE;
    if (M > kMaxRows) return BITNET_A48_ERR_LIMIT;
    if (M > 1 && y_stride < N) return BITNET_A48_ERR_SHAPE;
    if (!a48_aligned16(codes_dev) || !a48_aligned16(scale_dev) || !a48_aligned16(w_codes_dev) || !a48_aligned16(w_scale_dev) ||
        (reinterpret_cast<uintptr_t>(Y_dev) & (y_bf16 ? 1u : 3u)))
        return BITNET_A48_ERR_ALIGNMENT;
    if (!a48_have_device()) return BITNET_A48_ERR_CUDA;
    const a48f8::LinearArgs a = {codes_dev, scale_dev, w_codes_dev, w_scale_dev, M, N, K, Y_dev, M > 1 ? y_stride : (N + 7) / 8 * 8ll, y_bf16};
    return a48f8::few_supported(M, K) ? a48f8::launch_few(a, (cudaStream_t)stream) : a48f8::launch_gemm(a, nullptr, nullptr, (cudaStream_t)stream);
}

bitnet_a48_status bitnet_a48_logprobs(const void* logits_dev, long long stride, int x_bf16, int M, int V, float temperature, const void* tokens_dev,
                                      int tokens_i64, float* logprob_dev, float* entropy_dev, int32_t* rank_dev, int top, int32_t* top_ids_dev,
                                      float* top_logprobs_dev, void* stream) {
    if (!logits_dev || top < 0 || !temperature_ok(temperature)) return BITNET_A48_ERR_INVALID_ARG;
    if ((logprob_dev || rank_dev) && !tokens_dev) return BITNET_A48_ERR_INVALID_ARG;
    if (top > 0 && (!top_ids_dev || !top_logprobs_dev)) return BITNET_A48_ERR_INVALID_ARG;
    if (!logprob_dev && !entropy_dev && !rank_dev && top == 0) return BITNET_A48_ERR_INVALID_ARG;
    if (M <= 0 || V <= 0 || (M > 1 && stride < V) || top > V) return BITNET_A48_ERR_SHAPE;
    if (V > kMaxFeatures || top > kMaxTop || M > kMaxRows) return BITNET_A48_ERR_LIMIT;
    if ((reinterpret_cast<uintptr_t>(logits_dev) & (x_bf16 ? 1u : 3u)) || (reinterpret_cast<uintptr_t>(tokens_dev) & (tokens_i64 ? 7u : 3u)) ||
        (reinterpret_cast<uintptr_t>(logprob_dev) & 3u) || (reinterpret_cast<uintptr_t>(entropy_dev) & 3u) || (reinterpret_cast<uintptr_t>(rank_dev) & 3u) ||
        (reinterpret_cast<uintptr_t>(top_ids_dev) & 3u) || (reinterpret_cast<uintptr_t>(top_logprobs_dev) & 3u))
        return BITNET_A48_ERR_ALIGNMENT;
    if (!a48_have_device()) return BITNET_A48_ERR_CUDA;
    const a48f8::LogprobArgs a = {logits_dev, tokens_dev, logprob_dev, entropy_dev, rank_dev, top_ids_dev, top_logprobs_dev, M > 1 ? stride : V,
                                  M, V, top, x_bf16, tokens_i64, temperature};
    return a48f8::launch_logprobs(a, (cudaStream_t)stream);
}

size_t bitnet_a48_score_workspace_bytes(int M, int N, int K) {
    if (M <= 0 || M > kMaxRows || !features_ok(N) || !channels_ok(K)) return 0;
    return ScoreSpace(M, N, K).end;
}

bitnet_a48_status bitnet_a48_score(const void* X_dev, long long x_stride, int x_bf16, int M, const float* gain_dev, float norm_eps,
                                   const uint8_t* w_codes_dev, const float* w_scale_dev, int N, int K, float temperature, const void* tokens_dev,
                                   int tokens_i64, float* logprob_dev, float* entropy_dev, void* workspace_dev, size_t workspace_bytes, void* stream) {
    if (!w_codes_dev || !w_scale_dev || !tokens_dev || !logprob_dev || !entropy_dev || !workspace_dev || !temperature_ok(temperature))
        return BITNET_A48_ERR_INVALID_ARG;
    if (!features_ok(N)) return BITNET_A48_ERR_SHAPE;
    uint8_t* ws = reinterpret_cast<uint8_t*>(workspace_dev);
    bitnet_a48_status s = check_quant(X_dev, M, K, x_stride, x_bf16, ws, ws);
    if (s != BITNET_A48_OK) return s;
    if (!(norm_eps >= 0.f) || std::isinf(norm_eps)) return BITNET_A48_ERR_INVALID_ARG;
    if (!a48_aligned16(gain_dev) || !a48_aligned16(w_codes_dev) || !a48_aligned16(w_scale_dev) ||
        (reinterpret_cast<uintptr_t>(tokens_dev) & (tokens_i64 ? 7u : 3u)) || (reinterpret_cast<uintptr_t>(logprob_dev) & 3u) ||
        (reinterpret_cast<uintptr_t>(entropy_dev) & 3u))
        return BITNET_A48_ERR_ALIGNMENT;
    const ScoreSpace at(M, N, K);
    if (workspace_bytes < at.end) return BITNET_A48_ERR_NOMEM;
    if (!a48_have_device()) return BITNET_A48_ERR_CUDA;
    float* scale = reinterpret_cast<float*>(ws + at.scale);
    s = a48f8::launch_quant_rows(X_dev, x_bf16, M > 1 ? x_stride : K, gain_dev, norm_eps, M, K, ws + at.codes, scale, (cudaStream_t)stream);
    if (s != BITNET_A48_OK) return s;
    a48f8::LinearArgs a = {ws + at.codes, scale, w_codes_dev, w_scale_dev, M, N, K, nullptr, 0, 0};
    if (a48f8::few_supported(M, K)) {
        a.y = ws + at.stats;
        a.y_stride = ScoreSpace::logits_stride(N);
        s = a48f8::launch_few(a, (cudaStream_t)stream);
        if (s != BITNET_A48_OK) return s;
        const a48f8::LogprobArgs l = {a.y, tokens_dev, logprob_dev, entropy_dev, nullptr, nullptr, nullptr, a.y_stride, M, N, 0, 0, tokens_i64, temperature};
        return a48f8::launch_logprobs(l, (cudaStream_t)stream);
    }
    const a48f8::ScoreArgs score = {tokens_dev, tokens_i64, (float)(1.4426950408889634 / (double)temperature), 1.f / temperature, logprob_dev, entropy_dev};
    a48f8::ScoreParts parts = {reinterpret_cast<float4*>(ws + at.stats), reinterpret_cast<float*>(ws + at.owns), 0};
    s = a48f8::launch_gemm(a, &score, &parts, (cudaStream_t)stream);
    if (s != BITNET_A48_OK) return s;
    return a48f8::launch_score_join(score, parts, M, N, (cudaStream_t)stream);
}

}  // extern "C"
