// Host-side declarations shared by the libmxnorm translation units (not part of the public ABI).
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

namespace mxn {

constexpr int kSMs = 148;   // B200
inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

enum { STAT_NONE = 0, STAT_RMS = 1, STAT_MX = 2, STAT_POSTROUND = 3 };
enum { ELEM_E4M3 = 0, ELEM_E2M1 = 1, ELEM_E5M2 = 2 };

struct FwdParams {
    const uint16_t* x;      // bf16 [T, D]
    const uint16_t* gain;   // bf16 [D] or nullptr
    const uint16_t* residual; // bf16 [T, D] or nullptr: added to x before the norm (fused residual add)
    uint16_t* h_out;        // bf16 [T, D]: x + residual, written when residual is given
    uint8_t* codes;         // [T, D] (E4M3) or [T, D/2] (E2M1 pairs)
    uint8_t* scales;        // row-major [T, K] or 128x4-tiled
    float* rms_out;         // [T] or nullptr
    int64_t T;
    int D, K;
    int p;
    float coef, eps, global_scale;
    int round, layout;
    int elem;               // ELEM_E4M3 (one byte per element) or ELEM_E2M1 (two elements per byte)
    // filled by the launcher
    int wpr, npass, rows_per_cta, tiles_per_row;
    int chunks;             // per-lane pieces of a row: K * (lanes per block)
    int pr_table;           // post-round estimator: index of the block size's f^-1 table
    double inv_count;       // 1/K (MXNorm) or 1/D (RMSNorm) when that is a power of two (exact), else 0
};

bool fwd_shape_supported(int64_t D, int B);
cudaError_t launch_fwd(FwdParams P, int B, int stat, bool nvfp4, cudaStream_t stream);
cudaError_t selftest_division(unsigned long long* mismatches_host);
int64_t selftest_dispatch(int64_t max_D, int64_t* first_D, int* first_case);   // host only
int64_t selftest_bwd_plans(int64_t max_D, int64_t* first_D, int* first_case);  // host only
cudaError_t postround_prepare(int B);   // uploads the f^-1 table for block size B to the current device (once)

struct TransposedParams {
    const uint16_t* x;      // bf16 [T, D]
    const float* rms;       // [T] or nullptr (rho = 1)
    uint8_t* codes;         // [D, T]
    uint8_t* scales;        // [D, T/32] row-major or 128x4-tiled (rows = D)
    int64_t T;
    int D;
    float eps;
    int round, layout;
    int elem;               // ELEM_E4M3 or ELEM_E5M2
    int KT, tiles_per_row;  // filled by the launcher
};
cudaError_t launch_cast_transposed(TransposedParams P, cudaStream_t stream);

struct BwdParams {
    const uint16_t* x;      // bf16 [T, D]
    const uint16_t* g;      // bf16 [T, D]
    const uint16_t* gain;   // bf16 [D] or nullptr
    const float* rms;       // [T]
    void* dx;               // bf16 or fp32 [T, D]
    float* dgain;           // [D] or nullptr
    float* partial;         // workspace [P, D] fp32
    int64_t T;
    int D;
    int dx_is_fp32;
    int parts;              // number of partial rows in the workspace (= CTAs of the main kernel)
    int stages, stage_bytes; // shared-memory ring (filled by the launcher)
};

bool bwd_shape_supported(int64_t D);
int bwd_parts(int64_t T, int64_t D);
cudaError_t launch_bwd(BwdParams P, cudaStream_t stream);
// bounded device-side waits that ran out (the backward's bulk-copy ring is the only code that waits)
cudaError_t read_timeouts(unsigned int* out);
cudaError_t reset_timeouts();
cudaError_t selftest_bounded_wait(unsigned int polls, cudaStream_t stream);

// per-head norm with the position rotation; index 0: queries, 1: keys
struct HeadsParams {
    const uint16_t* x[2];       // bf16, token stride x_stride, heads side by side (backward: may be null without a norm)
    const uint16_t* grad[2];    // backward: gradient of the output
    uint16_t* y[2];             // output (backward: gradient of x)
    int64_t x_stride[2], grad_stride[2], y_stride[2];
    int heads[2];
    const uint16_t* gain[2];    // bf16 [dim] or nullptr
    float* dgain[2];            // backward: fp32 [dim] or nullptr
    float* partial;             // backward: workspace [ctas, dim] or nullptr
    const float* cos_sin;       // fp32 [table_rows, rot] or nullptr (no rotation)
    const int32_t* positions;   // [T] or nullptr (row index)
    int64_t T, table_rows;
    int dim, rot, pairs, norm;
    float eps, inv_dim;
    int parts, ctas_q;          // filled by the launchers
};
cudaError_t launch_rope_fwd(HeadsParams P, cudaStream_t stream);
cudaError_t launch_rope_bwd(HeadsParams P, cudaStream_t stream);
int rope_bwd_ctas(int64_t T, int q_heads, int k_heads, int dim);   // rows of the workspace
cudaError_t read_heads_bad(unsigned int* out);
cudaError_t reset_heads_bad();

// append to the paged 8-bit cache; index 0: keys, 1: values
struct KvAppendParams {
    const uint16_t* x[2];       // bf16 [n, heads, dim], token stride x_stride
    int64_t x_stride[2];
    uint8_t* codes[2];          // [num_pages, heads, page, dim]
    uint8_t* scales[2];         // [num_pages, heads, page / block]
    const int32_t* cu;          // [seqs + 1]
    const int32_t* lens;        // [seqs], with the new tokens
    const int32_t* page_table;  // [seqs, max_pages]
    const float* cos_sin;       // [table_rows, rot] or nullptr
    int64_t n, num_pages, max_pages, table_rows;
    int seqs, heads, dim, page, block, page_shift, block_shift, rot, pairs;
    int run;                    // filled by the launcher
};
cudaError_t launch_kv_append(KvAppendParams P, cudaStream_t stream);
cudaError_t read_kv_bad(unsigned int* out);
cudaError_t reset_kv_bad();

// attention over the paged 8-bit cache
struct AttnParams {
    const uint16_t* q;          // bf16 [n, q_heads, dim], token stride q_stride
    uint16_t* out;              // bf16, token stride out_stride
    float* lse;                 // [n, q_heads] or nullptr
    const uint8_t *k_codes, *k_scales, *v_codes, *v_scales;
    const int32_t *cu_q, *lens, *page_table;
    int64_t n, q_stride, out_stride, max_pages;
    int num_pages, seqs, q_heads, kv_heads, group, dim, page, page_shift, block_shift, max_q, max_len, causal, window;
    float scale;
    int sinks;                  // first tokens that stay visible beside the window
    const uint32_t* tree;       // [n, tree_words]: bit i of a row: it sees its sequence's new token i; or nullptr
    int tree_words;
    uint32_t group_mul, group_shift;   // row / group = (row * group_mul) >> (32 + group_shift) for rows below 2^31
    __host__ __device__ int by_group(int row) const
    {
        return group == 1 ? row : (int)((((uint64_t)(uint32_t)row * group_mul) >> 32) >> group_shift);
    }
    // filled by the launcher
    float *part_out, *part_lse;
    int64_t chunk;
    int splits, row_tiles;
    int cluster;                // the CTAs of a row tile's chunks are a cluster
    uint32_t whole_units;       // prompts: CTAs of two row tiles; behind them a unit is two CTAs of one
    int by_length;              // trees: the CTAs share out the keys by the lengths as they are, in up to `splits` chunks
};
struct AttnPlan {
    int64_t chunk, splits, row_tiles, whole_units, ctas;
    int row_warps, row_eights;  // warps that share out the query rows of a CTA; groups of eight rows that a warp holds
    bool prompt;                // many query rows: the tcgen05 kernel
    bool cluster;               // few chunks, joined by the CTAs as a cluster
    bool by_length;
    size_t workspace;
};
// room: bytes of workspace at hand, for trees of many rows, which take more of it where there is more (any other plan asks for what it needs)
AttnPlan plan_attention(int64_t n, int64_t seqs, int64_t max_q, int64_t max_len, int64_t window, int64_t sinks, int q_heads, int kv_heads, int dim, bool tree,
                        size_t room);
cudaError_t launch_attention(AttnParams P, const AttnPlan& plan, void* workspace, cudaStream_t stream);
cudaError_t read_attn_counters(unsigned int* timeouts, unsigned int* bad);
cudaError_t reset_attn_timeouts();
cudaError_t reset_attn_bad();

// summed attention weights of the keys
struct WeightsParams {
    AttnParams a;               // queries, keys, lists, sizes
    const float* lse;           // [n, q_heads]
    const float* earlier;       // [num_pages, kv_heads, page] or nullptr
    float* sums;                // the same
    // filled by the plan
    int many;                   // many rows: the tcgen05 kernel, with
    int tile_heads, tile_tokens, head_parts;   // heads and tokens of a tile of queries, parts of a key head's query heads
    int ranks;                  // CTAs (a cluster) that share out the queries of a tile of 256 keys
};
int64_t plan_weights(WeightsParams& W);   // shares the work out; returns the number of CTAs
cudaError_t launch_weights_many(const WeightsParams& W, int64_t ctas, cudaStream_t stream);
cudaError_t read_weights_many_counters(unsigned int* timeouts, unsigned int* bad);
cudaError_t reset_weights_many_counters(bool timeouts);
cudaError_t launch_weights(const WeightsParams& W, int64_t ctas, cudaStream_t stream);
cudaError_t read_weights_counters(unsigned int* timeouts, unsigned int* bad);
cudaError_t reset_weights_counters(bool timeouts);

// choice of the tokens that stay in the cache
struct SelectParams {
    const float* weights;       // [num_pages, heads, page]
    const int32_t *lens, *page_table;
    int32_t *kept, *new_lens;   // [seqs, heads, keep], [seqs]
    int64_t max_pages;
    int num_pages, seqs, heads, page_shift, max_len, keep, sinks, recent;
};
cudaError_t launch_select(const SelectParams& P, cudaStream_t stream);

// moving listed tokens together
struct CompactParams {
    const int32_t* kept;        // [seqs, kept_heads, max_kept]
    const int32_t *first, *new_lens, *lens;   // first: may be nullptr
    const int32_t *table, *out_table;         // the same one: in place
    uint8_t* codes[2];
    uint8_t* scales[2];
    float* weights;             // or nullptr
    uint32_t* work;             // in place: a ticket, then a flag for each unit
    int64_t max_kept, width, out_width;       // pages a sequence in the two tables
    int64_t units;              // of a sequence and head (filled by the launcher)
    int num_pages, seqs, heads, kept_heads, dim, page_shift, block_shift;
};
int64_t compact_units(int64_t max_kept, int places);
cudaError_t launch_compact(CompactParams P, cudaStream_t stream);
cudaError_t read_keep_counters(unsigned int* timeouts, unsigned int* bad);
cudaError_t reset_keep_counters(bool timeouts);

}  // namespace mxn
