// What the kernels of the 4-bit cache share: the layout of a row and the checks of a segment.
#pragma once
#include <cuda_fp16.h>

#include "pc_common.cuh"

constexpr int Q4_GROUP = 32;                       // channels that share a step and a low
constexpr int Q4_STEP = 16;                        // keys that a warp of the attention kernel takes at a time
constexpr float Q4_MAX = 65504.f;                  // largest value of half precision

// A token's row: key codes [Hkv][d / 2], value codes [Hkv][d / 2], then per head the steps and lows of its key and of its value (d / 4 bytes)
inline size_t q4_row(const pc_layer_desc &D) { return (size_t)D.n_kv_heads * (D.head_dim + D.head_dim / 4); }

inline pc_status q4_check_segment(const pc_q4_segment *s, bool allow_empty) {
    if (!s) return PC_ERR_INVALID_ARG;
    if (s->n_tokens < 0 || s->capacity < s->n_tokens || s->t_shift < 0) return PC_ERR_INVALID_ARG;
    if (s->n_tokens == 0) return allow_empty ? PC_OK : PC_ERR_INVALID_ARG;
    if (!s->rows || !s->pos || !pc_aligned16(s->rows) || !pc_aligned16(s->pos)) return PC_ERR_INVALID_ARG;
    if (reinterpret_cast<uintptr_t>(s->weight) & 3u) return PC_ERR_INVALID_ARG;
    return PC_OK;
}

inline bool pc_overlaps(const void *a, size_t na, const void *b, size_t nb) {
    const char *x = static_cast<const char *>(a), *y = static_cast<const char *>(b);
    return a && b && x < y + nb && y < x + na;
}

// What the tensor-core attention kernel needs of a frame over the cache: rows of up to two segments in fp16 (keys turned back by t_shift only: they stay
// rotated at their positions), queries rotated and scaled in two fp16 parts (q16 rows 0 .. n_q - 1 and, from row lo_row0 on, what they leave)
pc_status pc_q4_launch_front(pc_ctx *ctx, const pc_q4_segment *const *segs, int n_seg, void *const *k16, void *const *v16, const void *q, const int32_t *q_pos,
                             int32_t n_q, void *q16, int lo_row0, cudaStream_t stream);
