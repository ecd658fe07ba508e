// Arguments of the kernels of bitnet_a48_attention_paged.
#pragma once

#include "paged_codes.cuh"

namespace a48p {

// Where a kernel leaves the sums of a part of the positions: `parts` times `rows` places, of a row each.  The places are those
// of the rows that the kernel may have, not of the call's tokens: a row of a sequence is place (sequence * kv_heads + head) *
// per_head + row, or (per_head 0) token * heads + head.
struct Parts {
    float* o;    // [part][row][128]: sums of p sv d, relative to 2^m
    float2* ml;  // [part][row]: m, the exponent of the reference, and the sum of p
    long long rows, per_head;
    int parts;  // 1: none is left, the kernel has the whole sums
};

struct AttnArgs {
    Layout l;
    Batch b;
    const uint8_t* pool;
    const __nv_bfloat16* q;
    __nv_bfloat16* out;
    long long q_stride, out_stride;
    int heads, group, window, sinks;
    float scale;
    // sequences with at most this many rows (new tokens x group) are the rows kernel's
    int few_rows;
    // rows kernel: tiles of rows per sequence, rows of a tile, parts of the positions: `ranks` CTAs of a cluster that join
    // their sums, `clusters` of them that leave their sums to the join kernel
    int tiles, tile_rows, ranks, clusters;
    // tile kernel: tiles of 256 rows per sequence (0: found by search), parts of the positions
    int tc_tiles, tc_splits;
    Parts row_parts, tile_parts;
};

// What a tile of rows sees of its sequence: blocks of 2^SHIFT positions, [0, n_sink) and [first, first + count - n_sink).
struct Span {
    int n_sink, first, count;
    __device__ int block(int v) const { return v < n_sink ? v : v - n_sink + first; }
};
template <int SHIFT>
__device__ __forceinline__ Span span_of(const AttnArgs& a, int pos_lo, int pos_hi) {
    constexpr int UP = (1 << SHIFT) - 1;
    const long long reach = (long long)a.b.max_pages << a.l.page_shift;  // positions the table can place
    const int end = (int)min((long long)pos_hi + 1, reach);
    Span s{0, 0, 0};
    if (end <= 0) return s;
    const int behind = a.window > 0 ? max(0, pos_lo - a.window + 1) : 0;
    s.first = behind >> SHIFT;
    s.n_sink = min((min(a.sinks, end) + UP) >> SHIFT, s.first);
    s.count = s.n_sink + max(0, ((end + UP) >> SHIFT) - s.first);
    return s;
}

// attn_paged_tc.cu: sequences with more than few_rows rows, on the fifth-generation tensor cores
bitnet_a48_status launch_tiles(const AttnArgs& a, cudaStream_t st);
constexpr int TILE_ROWS = 256, TILE_POSITIONS = 128;

}  // namespace a48p
