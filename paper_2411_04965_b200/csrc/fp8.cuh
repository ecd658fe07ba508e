// Declarations of the 8-bit head's translation units.
#pragma once

#include "internal.h"

namespace a48f8 {

constexpr int BLOCK = 128;  // channels (and weight rows) that share a scale

inline int blocks(int n) { return (n + BLOCK - 1) / BLOCK; }

struct LinearArgs {
    const uint8_t* x;   // e4m3 [M][K]
    const float* xs;    // [blocks(K)][M]
    const uint8_t* w;   // e4m3 [N][K]
    const float* ws;    // [blocks(N)][blocks(K)]
    int M, N, K;
    void* y;            // [M] rows of N, y_stride elements apart
    long long y_stride;
    int y_bf16;
};

struct LogprobArgs {
    const void* x;       // [M] rows of V, stride elements apart
    const void* tokens;  // int32 or int64 [M], or NULL
    float* logprob;      // [M] or NULL, like the next two
    float* entropy;
    int32_t* rank;
    int32_t* top_ids;  // [M][top]
    float* top_logprobs;
    long long stride;
    int M, V, top, x_bf16, tokens64;
    float temperature;
};

// What a product keeps of its logits instead of storing them: for each row and each of `parts` sets of columns the sums of
// softmax_sums.cuh, and the logit of the row's token.
struct ScoreArgs {
    const void* tokens;  // int32 or int64 [M]
    int tokens64;
    float c, inv_t;  // log2 e / temperature, 1 / temperature
    float* logprob;
    float* entropy;
};
struct ScoreParts {
    float4* stats;  // [parts][M]
    float* owns;    // [M]
    int parts;      // set by launch_gemm
};
size_t score_stats(int M, int N);  // most float4 that stats may take, whatever the device

// ---- quant_fp8.cu
bitnet_a48_status launch_quant_rows(const void* X, int bf16, long long stride, const float* gain, float eps, int M, int K, uint8_t* codes, float* scale,
                                    cudaStream_t st);
bitnet_a48_status launch_quant_weight(const void* W, int bf16, long long stride, int N, int K, uint8_t* codes, float* scale, cudaStream_t st);

// ---- logprobs.cu
bitnet_a48_status launch_logprobs(const LogprobArgs& a, cudaStream_t st);
bitnet_a48_status launch_score_join(const ScoreArgs& s, const ScoreParts& w, int M, int V, cudaStream_t st);

// ---- rows_fp8.cu
bool few_supported(int M, int K);
bitnet_a48_status launch_few(const LinearArgs& a, cudaStream_t st);

// ---- gemm_fp8.cu
int sm_count();  // of the current device
// score, parts: NULL, or the product keeps these and stores no y.
bitnet_a48_status launch_gemm(const LinearArgs& a, const ScoreArgs* score, ScoreParts* parts, cudaStream_t st);

}  // namespace a48f8
