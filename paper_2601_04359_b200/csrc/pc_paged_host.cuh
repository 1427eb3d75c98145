// Host side shared by the paged cache's entry points and launchers.
#pragma once
#include "pc_paged.cuh"

constexpr int PAGED_FEW_ROWS = 16;           // most packed rows of a block of the few-row kernel
constexpr int PAGED_HOME_ROWS = 1024;        // most rows of a call whose prefix is attended apart
constexpr int PAGED_TC_TILE = 128;           // packed rows of a tile of the tcgen05 kernel

struct pc_paged {
    pc_ctx *ctx;
    float *few_o, *home_o;
    float2 *few_ml, *home_ml;
    size_t home_rows;
    int2 *groups_of;                         // the few-row kernel's items: prefix blocks of home_rows rows, then blocks of max_q rows and one a sequence
    // bf16: rotated queries, units, parts and their counters of the tcgen05 kernel
    void *q_rot;
    int *tc_plan, *tc_tickets;
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

// What the tcgen05 kernel leaves of a shared prefix: its keys in `parts` pieces, for every pair of tiles of packed rows and every KV head; a piece is two tiles of rows of d fp32 values and their (maximum,
// sum)
struct PagedTcParts {
    const float *part_o;
    const float2 *part_ml;
    const int *head;                         // [1] parts, [2] CTAs that are left for the sequences' own tokens
};
// first tile of a packed row's pieces (the next one's is two further), and the row in it
struct PagedTcRow { size_t first; int row, parts; };
__device__ __forceinline__ PagedTcRow paged_tc_row(const PagedTcParts &T, int n_kv, int h, long long packed_row) {
    const size_t pair = (size_t)(packed_row / (2 * PAGED_TC_TILE));
    const int parts = __ldcg(T.head + 1);
    return {((pair * n_kv + h) * parts) * 2 + (size_t)(packed_row / PAGED_TC_TILE & 1), (int)(packed_row % PAGED_TC_TILE), parts};
}

size_t pc_paged_few_parts(const pc_ctx *ctx);        // rows of the few-row kernel's scratch
// shared: the prefix is attended apart from the sequences' own tokens, here or (tc given) by the tcgen05 kernel before
pc_status pc_launch_paged_few(const pc_paged *w, const pc_paged_args &A, bool shared, const PagedTcParts *tc, cudaStream_t stream);
bool pc_paged_tc_shape(const pc_ctx *ctx);           // whether the tcgen05 kernel takes the context's type
size_t pc_paged_tc_slots(const pc_ctx *ctx), pc_paged_tc_plan_bytes(const pc_ctx *ctx);
bool pc_paged_tc_holds(const pc_ctx *ctx, const PagedBatch &B);
int pc_paged_few_block(const pc_paged_args &A, bool prefix_here);          // packed rows of a block of the few-row kernel
// every sequence over prefix and own tokens, into the output; or (shared) the prefix alone for all rows, into scratch (left), beside the few-row kernel with blocks of few_block rows
pc_status pc_launch_paged_tc(const pc_paged *w, const pc_paged_args &A, bool shared, int few_block, PagedTcParts *left, cudaStream_t stream);
