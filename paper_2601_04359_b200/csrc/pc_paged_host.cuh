// Host side shared by the paged cache's entry points and launchers.
#pragma once
#include "pc_paged.cuh"

constexpr int PAGED_FEW_ROWS = 16;           // most packed rows of a block of the few-row kernel
constexpr int PAGED_HOME_ROWS = 1024;        // most rows of a call whose prefix is attended apart
constexpr int PAGED_PLAN_HEAD = 8;         // words of the few-row kernel's plan ahead of the sequences' places
constexpr int PAGED_TC_TILE = 128;           // packed rows of a tile of the tcgen05 kernel

struct pc_paged {
    pc_ctx *ctx;
    float *few_o, *home_o;
    float2 *few_ml, *home_ml;
    size_t home_rows;
    long long *plan;
    // bf16: rotated queries, parts of the tcgen05 kernel and their counters
    void *q_rot;
    uint32_t *tc_sync;
    float *tc_o;
    float2 *tc_ml;
};

struct pc_paged_args {
    pc_ctx *ctx;
    PagedBatch batch;
    const pc_pages *pages;
    const void *q;
    const int32_t *q_pos;
    void *out;
    float *lse;
};

// How the tcgen05 kernel shares out a prefix that all rows of a call see: items (pair of tiles of packed rows, KV head) of `tiles` key tiles and `gap` empty places on a line that `ctas` CTAs share evenly.  An
// item of one CTA is at home in scratch, row by row; of an item of several the first CTA's part lies in that CTA's second place, the others' in their first, a place being two tiles of rows.
constexpr int PAGED_TC_LEAST = 4;            // fewest places of a CTA's run
__device__ __forceinline__ int paged_tc_ctas(long long total, int ctas) { return (int)min((long long)ctas, max(1LL, total / PAGED_TC_LEAST)); }
__device__ __forceinline__ int paged_tc_cta(long long total, int ctas, long long place) { return (int)(((place + 1) * ctas + total - 1) / total) - 1; }      // the CTA that has a place
struct PagedTcLine {
    const float *part_o;
    const float2 *part_ml;
    int tiles, gap, ctas;
};

size_t pc_paged_few_parts(const pc_ctx *ctx);        // rows of the few-row kernel's scratch
// shared: the prefix is attended apart from the sequences' own tokens, here or (tc given) by the tcgen05 kernel before
pc_status pc_launch_paged_few(const pc_paged *w, const pc_paged_args &A, bool shared, const PagedTcLine *tc, cudaStream_t stream);
bool pc_paged_tc_shape(const pc_ctx *ctx);           // whether the tcgen05 kernel takes the context's type
size_t pc_paged_tc_tiles(const pc_ctx *ctx), pc_paged_tc_sync_words(const pc_ctx *ctx);
// every sequence over prefix and own tokens, into the output; or (shared) the prefix alone for all rows, into scratch
pc_status pc_launch_paged_tc(const pc_paged *w, const pc_paged_args &A, bool shared, cudaStream_t stream);
PagedTcLine pc_paged_tc_line(const pc_paged *w, const pc_paged_args &A);
