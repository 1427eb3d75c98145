// The paged cache: rows appended with their rotation, and the entry points of attention over it.
#include <algorithm>
#include <new>

#include "pc_paged_host.cuh"

namespace {

// A warp per row and up to 8 chunks a lane: a chunk is eight channels (16 bytes, 32 in fp32), whole rotary pairs, and all chunks of a lane lie at the same place
// of a head (256 is a multiple of d), so four table entries serve them.  Keys and values are requested first; what they wait for behind that is where they go: the
// row's sequence (a search by all lanes at once, two looks at most), its length, its page.
constexpr int APPEND_THREADS = 256;

struct AppendParams {
    PagedBatch B;
    const char *k, *v;
    const int32_t *pos;
    char *pool_k, *pool_v;
    int chunks;              // of a row
};

template <bool F32> struct Chunk { uint4 a[F32 ? 2 : 1]; };
template <bool F32> __device__ __forceinline__ Chunk<F32> load_chunk(const char *p) {
    Chunk<F32> c;
#pragma unroll
    for (int i = 0; i < (F32 ? 2 : 1); ++i) c.a[i] = pc_ldg_stream(p + 16 * i);
    return c;
}
template <bool F32> __device__ __forceinline__ void turn_chunk(Chunk<F32> &c, const float2 (&cs)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (F32) {
            uint32_t *w = i < 2 ? &c.a[0].x : &c.a[1].x;
            const int at = (i & 1) * 2;
            const float2 y = pc_rotate(__uint_as_float(w[at]), __uint_as_float(w[at + 1]), cs[i]);
            w[at] = __float_as_uint(y.x);
            w[at + 1] = __float_as_uint(y.y);
        } else {
            uint32_t &w = (&c.a[0].x)[i];
            const float2 y = pc_rotate(pc_bf16_lo(w), pc_bf16_hi(w), cs[i]);
            w = pc_pack_bf16(y.x, y.y);
        }
    }
}
template <bool F32> __device__ __forceinline__ void store_chunk(char *p, const Chunk<F32> &c) {
#pragma unroll
    for (int i = 0; i < (F32 ? 2 : 1); ++i) *reinterpret_cast<uint4 *>(p + 16 * i) = c.a[i];
}

template <bool F32, int CPL /* chunks of a lane at a time */>
__global__ void __launch_bounds__(APPEND_THREADS) k_paged_append(const __grid_constant__ AppendParams P, const pc_rope_dev rope, int d) {
    constexpr int BYTES = F32 ? 32 : 16;
    pc_grid_dep_launch();
    const int lane = threadIdx.x & 31, row = (blockIdx.x * APPEND_THREADS + threadIdx.x) >> 5;
    pc_grid_dep_wait();
    const PagedBatch &B = P.B;
    if (row >= B.n_rows) return;
    const size_t width = (size_t)P.chunks * BYTES;
    const char *k = P.k + row * width, *v = P.v + row * width;
    Chunk<F32> ck[CPL], cv[CPL];
    const auto load = [&](int c0) {
#pragma unroll
        for (int i = 0; i < CPL; ++i) {
            const int c = c0 + i * 32 + lane;
            if (c < P.chunks) {
                ck[i] = load_chunk<F32>(k + (size_t)c * BYTES);
                cv[i] = load_chunk<F32>(v + (size_t)c * BYTES);
            }
        }
    };
    load(0);
    // the row's sequence: the last that begins at or before it
    const int stride = (B.n_seqs + 31) / 32;
    const int at0 = lane * stride;
    int s = __popc(__ballot_sync(0xffffffffu, at0 < B.n_seqs && __ldcg(B.row_start + at0) <= row)) - 1;
    if (s >= 0 && stride > 1) {
        const int at1 = s * stride + lane;
        s = s * stride + __popc(__ballot_sync(0xffffffffu, lane < stride && at1 < B.n_seqs && __ldcg(B.row_start + at1) <= row)) - 1;
    }
    if (s < 0) return;                                     // ahead of the first sequence: nobody's
    const PagedSeq S = paged_seq(B, s);
    if (row - S.r0 >= S.n) return;                         // behind the last
    const int slot = S.len - S.n + (row - S.r0);
    if (slot < 0) {                                        // more rows than tokens
        if (lane == 0) pc_flag(B.status, PC_ERR_INVALID_ARG, PC_WHERE_PAGED_ROWS);
        return;
    }
    const int page = __ldcg(B.table + (size_t)s * B.max_pages + (slot >> B.page_shift));
    if (page < 0 || page >= B.n_pages) {
        if (lane == 0) pc_flag(B.status, PC_ERR_INVALID_ARG, PC_WHERE_PAGED_TABLE);
        return;
    }
    const size_t to = (((size_t)page << B.page_shift) + (slot & ((1 << B.page_shift) - 1))) * width;
    const int4 pos = __ldcg(reinterpret_cast<const int4 *>(P.pos) + row);
    float2 cs[4];
    bool bad = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) cs[i] = pc_rope_cs_clamped(rope, ((lane * 8) % d) / 2 + i, pos.x, pos.y, pos.z, bad);
    if (bad) pc_flag(B.status, PC_ERR_INVALID_ARG, PC_WHERE_PAGED_POS);
    for (int c0 = 0;;) {
#pragma unroll
        for (int i = 0; i < CPL; ++i) {
            const int c = c0 + i * 32 + lane;
            if (c < P.chunks) {
                turn_chunk<F32>(ck[i], cs);
                store_chunk<F32>(P.pool_k + to + (size_t)c * BYTES, ck[i]);
                store_chunk<F32>(P.pool_v + to + (size_t)c * BYTES, cv[i]);
            }
        }
        c0 += CPL * 32;
        if (c0 >= P.chunks) break;
        load(c0);
    }
}

int log2_of(int x) {
    int n = 0;
    while ((1 << n) < x) ++n;
    return n;
}

// Everything that the host can see of pages and batch; fills in what kernels want
pc_status check_batch(const pc_ctx *ctx, const pc_pages *pages, const pc_batch *b, int32_t n_rows, PagedBatch *out) {
    if (!ctx || !pages || !b || !out || n_rows < 0) return PC_ERR_INVALID_ARG;
    const int p = pages->page_tokens;
    if (p != 16 && p != 32 && p != 64 && p != 128) return PC_ERR_UNSUPPORTED;
    if (pages->n_pages <= 0 || !pages->k || !pages->v || !pc_aligned16(pages->k) || !pc_aligned16(pages->v)) return PC_ERR_INVALID_ARG;
    if ((int64_t)pages->n_pages * p > INT32_MAX) return PC_ERR_CAPACITY;
    if (b->n_seqs < 0 || b->max_pages < 0 || b->n_prefix < 0 || b->max_rows < 0) return PC_ERR_INVALID_ARG;
    if (b->n_seqs > PC_MAX_SEQS || n_rows > ctx->desc.max_q) return PC_ERR_CAPACITY;
    if ((int64_t)b->max_pages * p > INT32_MAX || (int64_t)b->max_pages * p + b->n_prefix > INT32_MAX - 4096) return PC_ERR_CAPACITY;
    if (b->n_seqs > 0 && (!b->length || !b->row_start || (b->max_pages > 0 && !b->table))) return PC_ERR_INVALID_ARG;
    if (b->n_prefix > 0 && !b->prefix) return PC_ERR_INVALID_ARG;
    for (const int32_t *t : {b->table, b->length, b->row_start, b->prefix})
        if (reinterpret_cast<uintptr_t>(t) & 3u) return PC_ERR_INVALID_ARG;
    int device = -1;
    if (cudaGetDevice(&device) != cudaSuccess) return PC_ERR_CUDA;
    if (device != ctx->device) return PC_ERR_INVALID_ARG;
    *out = PagedBatch{b->table, b->length, b->row_start, b->prefix, b->n_seqs, b->max_pages, b->n_prefix, pages->n_pages, n_rows, b->max_rows, log2_of(p), 0, ctx->status};
    return PC_OK;
}

}  // namespace

extern "C" pc_status pc_paged_append(pc_ctx *ctx, const pc_pages *pages, const pc_batch *batch, const void *k, const void *v, const int32_t *pos, int32_t n_rows, void *stream_) {
    AppendParams P{};
    const pc_status st = check_batch(ctx, pages, batch, n_rows, &P.B);
    if (st != PC_OK) return st;
    if (n_rows == 0 || batch->n_seqs == 0) return PC_OK;
    if (!k || !v || !pos || !pc_aligned16(k) || !pc_aligned16(v) || !pc_aligned16(pos) || batch->max_pages == 0) return PC_ERR_INVALID_ARG;
    const pc_layer_desc &D = ctx->desc;
    P.k = static_cast<const char *>(k);
    P.v = static_cast<const char *>(v);
    P.pos = pos;
    P.pool_k = static_cast<char *>(pages->k);
    P.pool_v = static_cast<char *>(pages->v);
    P.chunks = D.n_kv_heads * D.head_dim / 8;
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    const dim3 grid((unsigned)(((long long)n_rows * 32 + APPEND_THREADS - 1) / APPEND_THREADS)), block(APPEND_THREADS);
    if (D.dtype == PC_F32) PC_LAUNCH((k_paged_append<true, 2>), grid, block, 0, stream, P, ctx->rope, D.head_dim);
    else PC_LAUNCH((k_paged_append<false, 4>), grid, block, 0, stream, P, ctx->rope, D.head_dim);
    return PC_OK;
}

extern "C" pc_status pc_paged_create(pc_ctx *ctx, pc_paged **out) {
    if (!ctx || !out) return PC_ERR_INVALID_ARG;
    *out = nullptr;
    pc_paged *w = new (std::nothrow) pc_paged();
    if (!w) return PC_ERR_CUDA;
    w->ctx = ctx;
    const pc_layer_desc &D = ctx->desc;
    w->home_rows = (size_t)std::min<int>(D.max_q, PAGED_HOME_ROWS);
    const size_t few = pc_paged_few_parts(ctx), home = 2 * w->home_rows * D.n_q_heads;
    const auto fill = [&]() -> pc_status {
        PC_CUDA_TRY(cudaMalloc(&w->few_o, few * D.head_dim * sizeof(float)));
        PC_CUDA_TRY(cudaMalloc(&w->few_ml, few * sizeof(float2)));
        PC_CUDA_TRY(cudaMalloc(&w->home_o, home * D.head_dim * sizeof(float)));
        PC_CUDA_TRY(cudaMalloc(&w->home_ml, home * sizeof(float2)));
        PC_CUDA_TRY(cudaMalloc(&w->groups_of, ((w->home_rows * ctx->group + 7) / 8 + (size_t)D.max_q * ctx->group / 8 + PC_MAX_SEQS + 1) * sizeof(int2)));
        if (pc_paged_tc_shape(ctx)) {
            const size_t tiles = 2 * pc_paged_tc_slots(ctx);
            PC_CUDA_TRY(cudaMalloc(&w->q_rot, (size_t)D.max_q * D.n_q_heads * D.head_dim * sizeof(__nv_bfloat16)));
            PC_CUDA_TRY(cudaMalloc(&w->tc_plan, pc_paged_tc_plan_bytes(ctx)));
            PC_CUDA_TRY(cudaMalloc(&w->tc_tickets, tiles * 4 * sizeof(int)));
            PC_CUDA_TRY(cudaMalloc(&w->tc_o, tiles * PAGED_TC_TILE * D.head_dim * sizeof(float)));
            PC_CUDA_TRY(cudaMalloc(&w->tc_ml, tiles * PAGED_TC_TILE * sizeof(float2)));
        }
        return PC_OK;
    };
    const pc_status st = fill();
    if (st != PC_OK) {
        pc_paged_destroy(w);
        return st;
    }
    *out = w;
    return PC_OK;
}

extern "C" pc_status pc_paged_destroy(pc_paged *w) {
    if (!w) return PC_ERR_INVALID_ARG;
    cudaFree(w->few_o);
    cudaFree(w->few_ml);
    cudaFree(w->home_o);
    cudaFree(w->home_ml);
    cudaFree(w->groups_of);
    cudaFree(w->q_rot);
    cudaFree(w->tc_plan);
    cudaFree(w->tc_tickets);
    cudaFree(w->tc_o);
    cudaFree(w->tc_ml);
    delete w;
    return PC_OK;
}

extern "C" pc_status pc_paged_attend(pc_paged *w, const pc_pages *pages, const pc_batch *batch, const void *q, const int32_t *q_pos, int32_t n_rows, int32_t causal, void *out,
                                     float *lse, void *stream_) {
    if (!w) return PC_ERR_INVALID_ARG;
    pc_paged_args A{};
    const pc_status st = check_batch(w->ctx, pages, batch, n_rows, &A.batch);
    if (st != PC_OK) return st;
    if (n_rows == 0 || batch->n_seqs == 0) return PC_OK;
    if (!q || !q_pos || !out || !pc_aligned16(q) || !pc_aligned16(q_pos) || !pc_aligned16(out) || (lse && !pc_aligned16(lse))) return PC_ERR_INVALID_ARG;
    A.ctx = w->ctx;
    A.batch.causal = causal != 0;
    A.pages = pages;
    A.q = q;
    A.q_pos = q_pos;
    A.out = out;
    A.lse = lse;
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    if (batch->max_rows == 0) return PC_OK;
    // Rows of a sequence and KV head that fill little of a tile of 128 go to the few-row kernel, which reads as many keys and values for a sixteenth of the rows; a prefix that several such
    // sequences share is attended once for all their rows.
    const long long rows = (long long)batch->max_rows * w->ctx->group;
    const bool tc = pc_paged_tc_shape(w->ctx) && w->ctx->attend_impl != 1;
    if (tc && rows > 64) return pc_launch_paged_tc(w, A, false, 0, nullptr, stream);
    const bool shared = batch->n_prefix > 0 && batch->n_seqs > 1 && (size_t)n_rows <= w->home_rows;
    PagedTcParts left{};
    if (tc && shared && (long long)n_rows * w->ctx->group > PAGED_FEW_ROWS && pc_paged_tc_holds(w->ctx, A.batch)) {
        const pc_status ps = pc_launch_paged_tc(w, A, true, pc_paged_few_block(A, false), &left, stream);
        return ps != PC_OK ? ps : pc_launch_paged_few(w, A, true, &left, stream);
    }
    return pc_launch_paged_few(w, A, shared, nullptr, stream);
}
