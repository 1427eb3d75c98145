// Eviction by accumulated attention weight: of a history's older tokens the ones with the largest weight, behind them the newest tokens.
//
// Two launches.  k_evict_select finds the kept tokens: weights become 32-bit keys whose unsigned order is the weights' (score_key); three
// passes over digits of 11, 11 and 10 bits narrow the range in which the want-th largest key lies (fewer, once at most 32 keys are left), and an ordered sweep
// writes the indices of all larger keys and of the first equal ones.  One CTA for short histories; for longer ones a cluster of CTAs that
// each hold a piece of the history in shared memory and count it; through distributed shared memory each CTA adds up its slice of all counts and gives the sums to
// all, between two barriers of the cluster a pass (and one more where the last few keys are exchanged).  k_evict_move copies the kept rows.
//
// The selection is latency: a launch, a fetch, up to three rounds of count, barrier and scan, and the sweep (675 tokens 5.4 us, 24,192 11.6, 47,376 16.3,
// which are 0.03 us of memory).  Of the 27,000 cycles at 47,376 a round is 7,300: counting 1,600, a barrier 1,300, the exchange of counts 2,300, the scan 1,800.  The move is bound by memory: 6,048 rows of 4,096 bytes, 49.5 MB read and
// written, 9.6 us from cold caches (5.2 TB/s).
#include <algorithm>

#include "pc_q4.cuh"
#include "pc_select.cuh"

namespace {

constexpr int SEL_THREADS = 1024, SEL_WARPS = SEL_THREADS / 32;
constexpr int DIGIT_BINS = 2048;
constexpr int MAX_CLUSTER = 8;                     // sixteen: 47,376 tokens 31.4 -> 30.5 us, 24,000 19.7 -> 20.0, 8,000 14.4 -> 15.4
constexpr int FEW = 32;                            // keys that a warp holds at once, a warp for each of them
constexpr int CACHED = 36 * 1024;                  // keys of a CTA's piece kept in shared memory; the rest is read again

struct SelectParams {
    const float *weight;
    const uint8_t *valid;
    int n_old, want, recent;                       // older tokens, how many of them stay (0 < want < n_old), newest tokens
    int piece;                                     // tokens of a CTA, a multiple of 4
    int32_t *sel_idx;
    int32_t *status;
};

__device__ __forceinline__ uint32_t cluster_rank() { uint32_t r; asm("mov.u32 %0, %cluster_ctarank;" : "=r"(r)); return r; }
__device__ __forceinline__ uint32_t cluster_size() { uint32_t r; asm("mov.u32 %0, %cluster_nctarank;" : "=r"(r)); return r; }
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t remote(uint32_t addr, uint32_t rank) {
    uint32_t there;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(addr), "r"(rank));
    return there;
}
__device__ __forceinline__ int4 remote_load(uint32_t addr, uint32_t rank) {
    int4 v;
    asm volatile("ld.shared::cluster.v4.s32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(remote(addr, rank)) : "memory");
    return v;
}
__device__ __forceinline__ void remote_store(uint32_t addr, uint32_t rank, int4 v) {
    asm volatile("st.shared::cluster.v4.s32 [%0], {%1,%2,%3,%4};" ::"r"(remote(addr, rank)), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
__device__ __forceinline__ void remote_store(uint32_t addr, uint32_t rank, uint32_t v) {
    asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(remote(addr, rank)), "r"(v) : "memory");
}
__device__ __forceinline__ int4 operator+(int4 a, int4 b) { return make_int4(a.x + b.x, a.y + b.y, a.z + b.z, a.w + b.w); }

// Sum of v over the threads before this one, and over all
__device__ __forceinline__ int scan_block(int v, int *warp_sums, int &all) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int inc = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int x = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += x;
    }
    __syncthreads();                               // the sums of the call before have been read
    if (lane == 31) warp_sums[warp] = inc;
    __syncthreads();
    const int w = warp_sums[lane];                 // SEL_WARPS == 32
    all = __reduce_add_sync(0xffffffffu, w);
    return __reduce_add_sync(0xffffffffu, lane < warp ? w : 0) + inc - v;
}

__global__ void __launch_bounds__(SEL_THREADS, 1) k_evict_select(const SelectParams P) {
    extern __shared__ uint32_t keys[];             // [min(piece, CACHED)]
    constexpr int SLICE = DIGIT_BINS / MAX_CLUSTER;                  // bins that a CTA of the cluster adds up for all
    __shared__ __align__(16) int hist[2][DIGIT_BINS], total[DIGIT_BINS], slice[MAX_CLUSTER][SLICE];
    __shared__ int warp_sums[SEL_WARPS];
    __shared__ int found[3];
    __shared__ int4 counts[MAX_CLUSTER];
    __shared__ uint32_t few[MAX_CLUSTER][FEW];     // keys of each CTA that share the digits so far, and how many
    __shared__ int few_n[MAX_CLUSTER];
    static_assert(SEL_WARPS == FEW && DIGIT_BINS == 2 * SEL_THREADS, "a lane reads a warp's total, a thread owns two bins");
    pc_grid_dep_launch();
    const int rank = (int)cluster_rank(), ctas = (int)cluster_size();
    const int first = rank * P.piece, n = max(0, min(P.piece, P.n_old - first));
    for (int b = threadIdx.x; b < 2 * DIGIT_BINS; b += SEL_THREADS) (&hist[0][0])[b] = 0;
    if (threadIdx.x < MAX_CLUSTER) few_n[threadIdx.x] = 0;
    pc_grid_dep_wait();
    const auto key_of = [&](int j) {
        const float w = P.weight[first + j];
        if (P.valid && P.valid[first + j] == 0) return 0u;           // after every other token
        return max(score_key(w), 1u);
    };
    bool nan = false;
#pragma unroll 8
    for (int j = threadIdx.x; j < n; j += SEL_THREADS) {
        const float w = P.weight[first + j];
        const bool masked = P.valid && P.valid[first + j] == 0;
        nan |= w != w && !masked;
        if (j < CACHED) keys[j] = masked ? 0u : max(score_key(w), 1u);
    }
    if (nan) pc_flag(P.status, PC_ERR_INVALID_ARG, PC_WHERE_EVICT_NAN);
    const auto key_at = [&](int j) { return j < CACHED ? keys[j] : key_of(j); };

    // digits from the top: `prefix` holds those of the want-th largest key so far
    uint32_t prefix = 0;
    int want = P.want;
    __syncthreads();
#pragma unroll 1
    for (int pass = 0; pass < 3; ++pass) {
        const int shift = pass == 0 ? 21 : (pass == 1 ? 10 : 0), above = pass == 0 ? 32 : (pass == 1 ? 21 : 10);
        const uint32_t mask = (1u << (above - shift)) - 1u;
        int *h = hist[pass & 1];
        for (int j = threadIdx.x; j < n; j += SEL_THREADS) {
            const uint32_t k = key_at(j);
            if (pass == 0 || ((k ^ prefix) >> above) == 0) atomicAdd(&h[(k >> shift) & mask], 1);
        }
        if (ctas > 1) {
            // Every CTA adds up a slice of the bins and gives it to all: 16 KB through distributed shared memory and a barrier more, where every CTA reading all
            // counts of all takes 64 KB and 5,000 cycles
            cluster_sync();
            const int i = 4 * (threadIdx.x % (SLICE / 4)), other = threadIdx.x / (SLICE / 4);
            if (other < MAX_CLUSTER) *reinterpret_cast<int4 *>(&slice[other][i]) = remote_load(pc_smem_u32(h + rank * SLICE + i), other);
            __syncthreads();
            if (other < MAX_CLUSTER) {
                int4 sum = make_int4(0, 0, 0, 0);
#pragma unroll
                for (int r = 0; r < MAX_CLUSTER; ++r) sum = sum + *reinterpret_cast<const int4 *>(&slice[r][i]);
                remote_store(pc_smem_u32(total + rank * SLICE + i), other, sum);
            }
            cluster_sync();
        } else {
            __syncthreads();
        }
        // thread t owns the bins 2047 - 2 t and 2046 - 2 t: counts from the top bin down
        const int b0 = DIGIT_BINS - 1 - 2 * threadIdx.x;
        const int *sums = ctas > 1 ? total : h;
        const int c0 = sums[b0], c1 = sums[b0 - 1];
        int all;
        const int before = scan_block(c0 + c1, warp_sums, all);
        if (before < want && want <= before + c0 + c1) {
            const bool second = before + c0 < want;
            found[0] = b0 - (second ? 1 : 0);
            found[1] = want - before - (second ? c0 : 0);
            found[2] = second ? c1 : c0;
        }
        // All reads of the first pass's counts by other CTAs ended before that pass's second barrier (its own ahead of a barrier of the CTA): cleared for the third
        if (pass == 1)
            for (int b = threadIdx.x; b < DIGIT_BINS; b += SEL_THREADS) hist[0][b] = 0;
        __syncthreads();
        prefix |= (uint32_t)found[0] << shift;
        want = found[1];
        if (want == found[2]) {                    // all keys of the bin stay, whatever their lower digits: no key is compared further
            prefix -= 1;
            want = 0;
            break;
        }
        if (pass < 2 && found[2] <= FEW) {
            // Few keys left: every CTA gets them all, a lane of each warp holds one, and warp i compares the i-th with all
            for (int j = threadIdx.x; j < n; j += SEL_THREADS) {
                const uint32_t k = key_at(j);
                if (((k ^ prefix) >> shift) == 0) few[rank][atomicAdd(&few_n[rank], 1) % FEW] = k;
            }
            __syncthreads();                       // and `found` has been read
            if (ctas > 1) {
                const int other = threadIdx.x / FEW, i = threadIdx.x % FEW;
                if (other < ctas && other != rank) {
                    if (i < few_n[rank]) remote_store(pc_smem_u32(&few[rank][i]), other, few[rank][i]);
                    if (i == 0) remote_store(pc_smem_u32(&few_n[rank]), other, (uint32_t)few_n[rank]);
                }
                cluster_sync();
            }
            const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
            uint32_t key = 0;
            int all = 0;
            for (int r = 0; r < ctas; ++r) {
                const int here = few_n[r];
                if (lane >= all && lane < all + here) key = few[r][lane - all];
                all += here;
            }
            const uint32_t k = __shfl_sync(0xffffffffu, key, warp);  // a warp's own
            const int larger = __popc(__ballot_sync(0xffffffffu, lane < all && key > k));
            const int as_large = __popc(__ballot_sync(0xffffffffu, lane < all && key >= k));
            if (lane == 0 && warp < all && larger < want && want <= as_large) {
                found[0] = (int)k;                 // warps whose keys are equal write the same
                found[1] = want - larger;
            }
            __syncthreads();
            prefix = (uint32_t)found[0];
            want = found[1];
            break;
        }
    }
    // keys above `prefix` stay, and the first `want` equal to it (`prefix` cannot have been 0 where it was lowered by one: fewer tokens stay than there are)
    const int per = (n + SEL_THREADS - 1) / SEL_THREADS, j0 = min(n, (int)threadIdx.x * per), j1 = min(n, j0 + per);
    int gt = 0, eq = 0;
    for (int j = j0; j < j1; ++j) {
        const uint32_t k = key_at(j);
        gt += k > prefix;
        eq += k == prefix;
    }
    int all_gt, all_eq;
    const int gt0 = scan_block(gt, warp_sums, all_gt), eq0 = scan_block(eq, warp_sums, all_eq);
    int gt_before = gt0, eq_before = eq0;
    if (ctas > 1) {
        if (threadIdx.x < MAX_CLUSTER) remote_store(pc_smem_u32(&counts[rank]), threadIdx.x, make_int4(all_gt, all_eq, 0, 0));
        cluster_sync();
        for (int r = 0; r < rank; ++r) {
            gt_before += counts[r].x;
            eq_before += counts[r].y;
        }
    }
    for (int j = j0; j < j1; ++j) {
        const uint32_t k = key_at(j);
        const bool keep = k > prefix || (k == prefix && eq_before < want);
        if (keep) P.sel_idx[gt_before + min(eq_before, want)] = first + j;
        gt_before += k > prefix;
        eq_before += k == prefix;
    }
    for (int j = rank * SEL_THREADS + threadIdx.x; j < P.recent; j += ctas * SEL_THREADS) P.sel_idx[P.want + j] = P.n_old + j;
}

// Nothing to choose: the tokens from `first` on are kept
__global__ void __launch_bounds__(256) k_evict_tail(int32_t *sel_idx, int first, int n) {
    pc_grid_dep_launch();
    pc_grid_dep_wait();
    const int j = blockIdx.x * 256 + threadIdx.x;
    if (j < n) sel_idx[j] = first + j;
}

struct MoveParams {
    const char *a, *b;                             // rows: K and V, or the 4-bit rows and nothing
    char *to_a, *to_b;
    const int32_t *pos;
    int32_t *to_pos;
    const float *weight;
    float *to_weight;
    const int32_t *sel_idx;
    int n, chunks, delta_t;                        // tokens kept, 16-byte pieces of a row
};

// A warp per kept token
__global__ void __launch_bounds__(256) k_evict_move(const MoveParams P) {
    pc_grid_dep_launch();
    const int r = (int)(blockIdx.x * 8 + (threadIdx.x >> 5)), lane = threadIdx.x & 31;
    pc_grid_dep_wait();
    if (r >= P.n) return;
    const int s = __ldg(P.sel_idx + r);
    const size_t from = (size_t)s * P.chunks * 16, to = (size_t)r * P.chunks * 16;
#pragma unroll 4
    for (int c = lane; c < P.chunks; c += 32) pc_stg_stream(P.to_a + to + c * 16, pc_ldg_stream(P.a + from + c * 16));
    if (P.b)
#pragma unroll 4
        for (int c = lane; c < P.chunks; c += 32) pc_stg_stream(P.to_b + to + c * 16, pc_ldg_stream(P.b + from + c * 16));
    if (lane == 0) {
        int4 p = __ldg(reinterpret_cast<const int4 *>(P.pos) + s);
        p.x -= P.delta_t;
        reinterpret_cast<int4 *>(P.to_pos)[r] = p;
        if (P.to_weight) P.to_weight[r] = __ldg(P.weight + s);
    }
}

pc_status check_params(const pc_evict_params *p) {
    if (!p || p->keep < 0 || p->recent < 0 || p->recent > p->keep) return PC_ERR_INVALID_ARG;
    return PC_OK;
}

pc_status select_and_move(pc_ctx *ctx, const float *weight, const pc_evict_params *p, const uint8_t *valid, int n, int32_t *sel_idx, MoveParams M,
                          cudaStream_t stream) {
    const int kept = std::min(p->keep, n), recent = std::min(p->recent, kept), n_old = n - recent, want = kept - recent;
    if (kept == 0) return PC_OK;
    if (want > 0 && want < n_old) {
        SelectParams S{weight, valid, n_old, want, recent, 0, sel_idx, ctx->status};
        // One CTA / a cluster, us a call (16 bits, a quarter kept): 2,000 tokens 9.0 / 11.4, 4,000 11.0 / 12.4, 6,000 13.1 / 13.1, 8,000 15.4 / 14.4,
        // 24,000 29.9 / 19.9
        const int ctas = n_old > 6144 ? MAX_CLUSTER : 1;
        S.piece = ((n_old + ctas - 1) / ctas + 3) / 4 * 4;
        const size_t smem = (size_t)std::min(S.piece, CACHED) * sizeof(uint32_t);
        static bool attr_set[PC_MAX_DEVICES] = {};
        if (ctx->device < 0 || ctx->device >= PC_MAX_DEVICES) return PC_ERR_UNSUPPORTED;
        if (!attr_set[ctx->device]) {
            PC_CUDA_TRY(cudaFuncSetAttribute(k_evict_select, cudaFuncAttributeMaxDynamicSharedMemorySize, CACHED * (int)sizeof(uint32_t)));
            attr_set[ctx->device] = true;
        }
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3(ctas);
        cfg.blockDim = dim3(SEL_THREADS);
        cfg.dynamicSmemBytes = smem;
        cfg.stream = stream;
        cudaLaunchAttribute attr[2];
        attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[0].val.programmaticStreamSerializationAllowed = 1;
        attr[1].id = cudaLaunchAttributeClusterDimension;
        attr[1].val.clusterDim.x = ctas;
        attr[1].val.clusterDim.y = 1;
        attr[1].val.clusterDim.z = 1;
        cfg.attrs = attr;
        cfg.numAttrs = 2;
        PC_CUDA_TRY(cudaLaunchKernelEx(&cfg, k_evict_select, S));
    } else {
        PC_LAUNCH(k_evict_tail, dim3((kept + 255) / 256), dim3(256), 0, stream, sel_idx, n - kept, kept);
    }
    M.sel_idx = sel_idx;
    M.n = kept;
    M.delta_t = p->delta_t;
    PC_LAUNCH(k_evict_move, dim3((unsigned)(((long long)kept * 32 + 255) / 256)), dim3(256), 0, stream, M);
    return PC_OK;
}

}  // namespace

extern "C" pc_status pc_q4_evict(pc_ctx *ctx, const pc_q4_segment *src, const pc_evict_params *params, const uint8_t *valid, pc_q4_segment *dst,
                                 int32_t *sel_idx, void *stream) {
    if (!ctx || !src || !dst) return PC_ERR_INVALID_ARG;
    pc_status st = q4_check_segment(src, true);
    if (st == PC_OK) st = check_params(params);
    if (st != PC_OK) return st;
    const int64_t shift = (int64_t)src->t_shift + params->delta_t;
    if (shift < 0 || shift > INT32_MAX) return PC_ERR_INVALID_ARG;
    const int n = src->n_tokens, kept = std::min(params->keep, n);
    pc_q4_segment made = *dst;
    made.n_tokens = kept;
    made.t_shift = (int32_t)shift;
    if (kept > dst->capacity) return PC_ERR_CAPACITY;
    st = q4_check_segment(&made, true);
    if (st != PC_OK) return st;
    if (n > 0 && !src->weight) return PC_ERR_INVALID_ARG;
    if (kept > 0) {
        if (!sel_idx || !pc_aligned16(sel_idx)) return PC_ERR_INVALID_ARG;
        const size_t row = q4_row(ctx->desc);
        if (pc_overlaps(src->rows, n * row, dst->rows, kept * row) || pc_overlaps(src->pos, (size_t)n * 16, dst->pos, (size_t)kept * 16) ||
            pc_overlaps(src->weight, (size_t)n * 4, dst->weight, (size_t)kept * 4)) return PC_ERR_INVALID_ARG;
        MoveParams M{};
        M.a = static_cast<const char *>(src->rows);
        M.to_a = static_cast<char *>(dst->rows);
        M.pos = src->pos;
        M.to_pos = dst->pos;
        M.weight = src->weight;
        M.to_weight = dst->weight;
        M.chunks = (int)(row / 16);
        st = select_and_move(ctx, src->weight, params, valid, n, sel_idx, M, static_cast<cudaStream_t>(stream));
        if (st != PC_OK) return st;
    }
    *dst = made;
    return PC_OK;
}

extern "C" pc_status pc_evict(pc_ctx *ctx, const pc_segment *src, const float *weight, const pc_evict_params *params, const uint8_t *valid,
                              pc_segment *dst, float *dst_weight, int32_t *sel_idx, void *stream) {
    if (!ctx || !src || !dst) return PC_ERR_INVALID_ARG;
    pc_status st = pc_check_segment(src, true);
    if (st == PC_OK) st = check_params(params);
    if (st != PC_OK) return st;
    const int n = src->n_tokens, kept = std::min(params->keep, n);
    if (kept > dst->capacity) return PC_ERR_CAPACITY;
    pc_segment made = *dst;
    made.n_tokens = kept;
    st = pc_check_segment(&made, true);
    if (st != PC_OK) return st;
    if ((n > 0 && !weight) || ((reinterpret_cast<uintptr_t>(weight) | reinterpret_cast<uintptr_t>(dst_weight)) & 3u)) return PC_ERR_INVALID_ARG;
    if (kept > 0) {
        if (!sel_idx || !pc_aligned16(sel_idx)) return PC_ERR_INVALID_ARG;
        const size_t row = (size_t)ctx->desc.n_kv_heads * ctx->desc.head_dim * ctx->elem_size;
        const void *from[2] = {src->k, src->v}, *to[2] = {dst->k, dst->v};
        for (const void *f : from)
            for (const void *t : to)
                if (pc_overlaps(f, n * row, t, kept * row)) return PC_ERR_INVALID_ARG;
        if (pc_overlaps(src->pos, (size_t)n * 16, dst->pos, (size_t)kept * 16) || pc_overlaps(weight, (size_t)n * 4, dst_weight, (size_t)kept * 4))
            return PC_ERR_INVALID_ARG;
        MoveParams M{};
        M.a = static_cast<const char *>(src->k);
        M.b = static_cast<const char *>(src->v);
        M.to_a = static_cast<char *>(dst->k);
        M.to_b = static_cast<char *>(dst->v);
        M.pos = src->pos;
        M.to_pos = dst->pos;
        M.weight = weight;
        M.to_weight = dst_weight;
        M.chunks = (int)(row / 16);
        st = select_and_move(ctx, weight, params, valid, n, sel_idx, M, static_cast<cudaStream_t>(stream));
        if (st != PC_OK) return st;
    }
    *dst = made;
    return PC_OK;
}
