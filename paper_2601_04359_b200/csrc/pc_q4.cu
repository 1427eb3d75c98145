// Rows of the 4-bit cache: written from, and read back into, rows of the context's element type.
//
// A token of 8 KV heads x 128 channels is 4,096 bytes in bf16 and 1,280 in four bits, so both directions would be bound by memory if the
// arithmetic (a token's rotation, the ranges of 64 groups and 2,048 codes) stayed out of the way.  A thread owns
// eight channels of a row, so a group of 32 channels is four neighbouring lanes (two shuffles give its range) and the d / 8 lanes of a
// token go through up to HEADS of its heads: the four rotary table entries of a thread's channels are looked up once for all of them,
// and the loads of all heads are in flight together.
// 24,193 tokens, bf16, 131 MB either way, from cold caches: k_q4_store 37 us (3.5 TB/s; instructions issue in 78 % of the cycles, and
// the bf16 form spills: 20 bytes stored and 68 loaded a thread, at the 64 registers that four blocks an SM leave), k_q4_load 27 us
// (4.8 TB/s).  One frame of 1,008 tokens, 5.5 MB: 6.9 and 5.0 us, of which about 4 are the launch.
#include "pc_q4.cuh"

namespace {

constexpr int ROW_THREADS = 256;
constexpr int HEADS = 4;                           // heads of a token that one group of lanes takes

template <bool F32> struct Eight { uint4 a; };
template <> struct Eight<true> { uint4 a, b; };

template <bool F32> __device__ __forceinline__ Eight<F32> load8(const void *base, size_t elem) {
    Eight<F32> e;
    if constexpr (F32) {
        const char *p = static_cast<const char *>(base) + elem * 4;
        e.a = pc_ldg_stream(p);
        e.b = pc_ldg_stream(p + 16);
    } else {
        e.a = pc_ldg_stream(static_cast<const char *>(base) + elem * 2);
    }
    return e;
}
template <bool F32> __device__ __forceinline__ void unpack8(const Eight<F32> &e, float (&x)[8]) {
    const uint32_t w[4] = {e.a.x, e.a.y, e.a.z, e.a.w};
    if constexpr (F32) {
        const uint32_t u[4] = {e.b.x, e.b.y, e.b.z, e.b.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) { x[i] = __uint_as_float(w[i]); x[4 + i] = __uint_as_float(u[i]); }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) { x[2 * i] = pc_bf16_lo(w[i]); x[2 * i + 1] = pc_bf16_hi(w[i]); }
    }
}
// Smallest and largest of three; NaN if one is NaN
__device__ __forceinline__ float min3_nan(float a, float b, float c) { float d; asm("min.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c)); return d; }
__device__ __forceinline__ float max3_nan(float a, float b, float c) { float d; asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c)); return d; }
// Into fp16's range; NaN stays
__device__ __forceinline__ float into_f16(float x) { return min3_nan(max3_nan(x, -Q4_MAX, -Q4_MAX), Q4_MAX, Q4_MAX); }

enum { OUT_BF16 = 0, OUT_F32 = 1, OUT_F16 = 2 };
template <int OUT> __device__ __forceinline__ void store8(void *base, size_t elem, const float (&x)[8]) {
    if constexpr (OUT == OUT_F16) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = pc_pack_f16(into_f16(x[2 * i]), into_f16(x[2 * i + 1]));
        *reinterpret_cast<uint4 *>(static_cast<char *>(base) + elem * 2) = make_uint4(w[0], w[1], w[2], w[3]);
    } else if constexpr (OUT == OUT_F32) {
        uint4 *p = reinterpret_cast<uint4 *>(static_cast<char *>(base) + elem * 4);
        p[0] = make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
        p[1] = make_uint4(__float_as_uint(x[4]), __float_as_uint(x[5]), __float_as_uint(x[6]), __float_as_uint(x[7]));
    } else {
        *reinterpret_cast<uint4 *>(static_cast<char *>(base) + elem * 2) =
            make_uint4(pc_pack_bf16(x[0], x[1]), pc_pack_bf16(x[2], x[3]), pc_pack_bf16(x[4], x[5]), pc_pack_bf16(x[6], x[7]));
    }
}

// Two sums by one instruction
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
    float2 d;
    asm("{\n\t.reg .b64 ra, rb, rd;\n\tmov.b64 ra, {%2, %3};\n\tmov.b64 rb, {%4, %5};\n\tadd.rn.f32x2 rd, ra, rb;\n\tmov.b64 {%0, %1}, rd;\n\t}"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}

// A pair turned by (cos, sin) with every product and sum rounded by itself, so that the codes follow from plain fp32 arithmetic (products and sums of two
// at a time came out fused, with other bits)
__device__ __forceinline__ void turn(float &x0, float &x1, float2 cs) {
    const float a = __fsub_rn(__fmul_rn(x0, cs.x), __fmul_rn(x1, cs.y)), b = __fadd_rn(__fmul_rn(x0, cs.y), __fmul_rn(x1, cs.x));
    x0 = a;
    x1 = b;
}

// Codes, step and low of this thread's eight channels; all four lanes of a group get the same step and low.
// Bound by instructions as much as by memory, so: smallest and largest by threes, NaN kept, so that one look at the two tells whether every value is one
// that fp16 can hold (if not, the warp puts its values right in a branch); (x - low) / step is clamped at zero by the multiplication's saturation, in units of
// 16 steps; it is rounded and turned into an integer by adding 1.5 * 2^19, whose last place is then a sixteenth (rounding and conversion
// instructions run at a quarter of the rate: with them 24,193 tokens took 54 us, so 38); and the codes are put together by multiply-adds on the
// sums' bits, from which what the eight 1.5 * 2^19 add up to is taken at the end.
__device__ __forceinline__ uint32_t quantise8(float (&x)[8], __half &step, __half &low, bool &bad) {
    const auto range = [&](float &lo, float &hi) {
        lo = min3_nan(min3_nan(x[0], x[1], x[2]), min3_nan(x[3], x[4], x[5]), min3_nan(x[6], x[7], x[7]));
        hi = max3_nan(max3_nan(x[0], x[1], x[2]), max3_nan(x[3], x[4], x[5]), max3_nan(x[6], x[7], x[7]));
    };
    float lo, hi;
    range(lo, hi);
    const bool off = !(lo >= -Q4_MAX && hi <= Q4_MAX);
    if (__any_sync(0xffffffffu, off)) {
        bad |= off;
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = x[i] != x[i] ? 0.f : fminf(fmaxf(x[i], -Q4_MAX), Q4_MAX);
        range(lo, hi);
    }
#pragma unroll
    for (int o = 1; o < 4; o <<= 1) {
        lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, o));
        hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, o));
    }
    low = __float2half_rn(lo);
    const float l = __half2float(low);
    step = __float2half_rn(__fmul_rn(__fsub_rn(hi, l), 1.0f / 15.0f));
    const float s = __half2float(step), inv = s > 0.f ? __frcp_rn(s) * 0.0625f : 0.f;
    constexpr uint32_t MAGIC = 0x49400000u;        // 1.5 * 2^19
    uint32_t word = 0;
#pragma unroll
    for (int i = 6; i >= 0; i -= 2) {
        const float2 d = add2(make_float2(x[i], x[i + 1]), make_float2(-l, -l));
        const float2 c = add2(make_float2(fminf(__saturatef(__fmul_rn(d.x, inv)), 0.9375f), fminf(__saturatef(__fmul_rn(d.y, inv)), 0.9375f)),
                              make_float2(__uint_as_float(MAGIC), __uint_as_float(MAGIC)));
        word = (word * 16u + __float_as_uint(c.y)) * 16u + __float_as_uint(c.x);
    }
    return word - MAGIC * 0x11111111u;
}

struct RowsArgs {
    const void *k, *v;          // rows in the element type (store: source; load: destination, written through the non-const copies)
    void *k_out, *v_out;
    const int32_t *pos_in;
    int32_t *pos_out;
    char *q4;                   // row 0 of the 4-bit rows of the call
    float *weight;
    int n, n_kv, slices;        // tokens, KV heads, slices of HEADS heads
    int t_shift;
    int32_t *status;
};

template <int D, bool F32>
__global__ void __launch_bounds__(ROW_THREADS, F32 ? 2 : 4) k_q4_store(RowsArgs A, pc_rope_dev rope) {
    constexpr int LANES = D / 8, NG = D / Q4_GROUP;
    const unsigned unit = (blockIdx.x * ROW_THREADS + threadIdx.x) / LANES;      // unsigned: 2^32 threads are more rows than memory holds
    const int u = threadIdx.x % LANES, token = (int)(unit / A.slices), h0 = (int)(unit % A.slices) * HEADS;
    const bool live = token < A.n;                 // lanes of a warp stay together for the shuffles
    const int heads = live ? min(HEADS, A.n_kv - h0) : 0;
    const int g = u >> 2, t = u & 3;
    pc_grid_dep_wait();
    // Only now may the next launch come: with calls queued up, launches that each let the next one in before their own wait filled the SMs with waiting
    // CTAs, and a frame's 126 shared what was left (store and load of 1,008 tokens in a queue of calls 13.3 us, so 8.4; 24,193 tokens 63.3, so 63.5)
    pc_grid_dep_launch();
    Eight<F32> kr[HEADS], vr[HEADS];
    const size_t at = ((size_t)token * A.n_kv + h0) * D + u * 8;
#pragma unroll
    for (int h = 0; h < HEADS; ++h)
        if (h < heads) {
            kr[h] = load8<F32>(A.k, at + h * D);
            vr[h] = load8<F32>(A.v, at + h * D);
        } else {
            kr[h] = Eight<F32>{};
            vr[h] = Eight<F32>{};
        }
    float2 cs[4] = {};
    bool bad_pos = false, bad = false;
    if (live) {
        const int4 p = __ldg(reinterpret_cast<const int4 *>(A.pos_in) + token);
#pragma unroll
        for (int i = 0; i < 4; ++i) cs[i] = pc_rope_cs_clamped(rope, u * 4 + i, p.x + A.t_shift, p.y, p.z, bad_pos);
        if (h0 == 0 && u == 0) {
            reinterpret_cast<int4 *>(A.pos_out)[token] = p;
            if (A.weight) A.weight[token] = 0.f;
        }
    }
    if (bad_pos) pc_flag(A.status, PC_ERR_INVALID_ARG, PC_WHERE_Q4_POS);
    char *row = A.q4 + (size_t)token * A.n_kv * (D + D / 4);
    char *kc_at = row + h0 * (D / 2), *vc_at = kc_at + A.n_kv * (D / 2), *sl_at = row + A.n_kv * D + h0 * (D / 4);
#pragma unroll
    for (int h = 0; h < HEADS; ++h) {
        float x[8];
        __half ks, kl, vs, vl;
        unpack8<F32>(kr[h], x);
#pragma unroll
        for (int i = 0; i < 4; ++i) turn(x[2 * i], x[2 * i + 1], cs[i]);
        const uint32_t kc = quantise8(x, ks, kl, bad);
        unpack8<F32>(vr[h], x);
        const uint32_t vc = quantise8(x, vs, vl, bad);
        if (h < heads) {
            reinterpret_cast<uint32_t *>(kc_at + h * (D / 2))[t * NG + g] = kc;
            reinterpret_cast<uint32_t *>(vc_at + h * (D / 2))[u] = vc;
            reinterpret_cast<__half *>(sl_at + h * (D / 4))[t * NG + g] = t == 0 ? ks : (t == 1 ? kl : (t == 2 ? vs : vl));
        }
    }
    if (bad) pc_flag(A.status, PC_ERR_INVALID_ARG, PC_WHERE_Q4_RANGE);
}

// FROM_POS: keys turned back from (t + t_shift, h, w) to how they came in; else from t_shift alone (they stay rotated at their positions)
template <int D, int OUT, bool FROM_POS>
__device__ __forceinline__ void load_rows(const RowsArgs &A, const pc_rope_dev &rope, unsigned block) {
    constexpr int LANES = D / 8, NG = D / Q4_GROUP;
    const unsigned unit = (block * ROW_THREADS + threadIdx.x) / LANES;
    const int u = threadIdx.x % LANES, token = (int)(unit / A.slices), h0 = (int)(unit % A.slices) * HEADS;
    const bool live = token < A.n;
    const int heads = live ? min(HEADS, A.n_kv - h0) : 0;
    const int g = u >> 2, t = u & 3;
    const char *row = A.q4 + (size_t)token * A.n_kv * (D + D / 4);
    const char *kc_at = row + h0 * (D / 2), *vc_at = kc_at + A.n_kv * (D / 2), *sl_at = row + A.n_kv * D + h0 * (D / 4);
    uint32_t kc[HEADS], vc[HEADS], kq[HEADS], vq[HEADS];       // codes; step and low of the thread's group
#pragma unroll
    for (int h = 0; h < HEADS; ++h) {
        kc[h] = vc[h] = kq[h] = vq[h] = 0;
        if (h < heads) {
            const uint16_t *sl = reinterpret_cast<const uint16_t *>(sl_at + h * (D / 4));
            kc[h] = reinterpret_cast<const uint32_t *>(kc_at + h * (D / 2))[t * NG + g];
            vc[h] = reinterpret_cast<const uint32_t *>(vc_at + h * (D / 2))[u];
            kq[h] = sl[g] | (uint32_t)sl[NG + g] << 16;
            vq[h] = sl[2 * NG + g] | (uint32_t)sl[3 * NG + g] << 16;
        }
    }
    float2 cs[4] = {};
    bool bad_pos = false;
    const bool turned = FROM_POS || A.t_shift != 0;
    if (live && turned) {
        int4 p = make_int4(0, 0, 0, 0);
        if constexpr (FROM_POS) p = __ldg(reinterpret_cast<const int4 *>(A.pos_in) + token);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            cs[i] = pc_rope_cs_clamped(rope, u * 4 + i, p.x + A.t_shift, p.y, p.z, bad_pos);
            cs[i].y = -cs[i].y;
        }
        if constexpr (FROM_POS)
            if (h0 == 0 && u == 0) reinterpret_cast<int4 *>(A.pos_out)[token] = p;
    }
    if (bad_pos) pc_flag(A.status, PC_ERR_INVALID_ARG, PC_WHERE_Q4_POS);
    const size_t at = ((size_t)token * A.n_kv + h0) * D + u * 8;
    // (a code becomes a number as the last places of 2^23 + code: conversion instructions run at a quarter of the rate)
    const auto value = [](uint32_t word, int i, float step, float low) {
        return __fmaf_rn(step, __uint_as_float(((word >> (4 * i)) & 15u) | 0x4B000000u) - 8388608.f, low);
    };
    const auto half_of = [](uint32_t w) { return __half2float(__ushort_as_half((unsigned short)(w & 0xFFFFu))); };
#pragma unroll
    for (int h = 0; h < HEADS; ++h) {
        if (h < heads) {
            float x[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = value(kc[h], i, half_of(kq[h]), half_of(kq[h] >> 16));
            if (turned) {
#pragma unroll
                for (int i = 0; i < 4; ++i) turn(x[2 * i], x[2 * i + 1], cs[i]);
            }
            store8<OUT>(A.k_out, at + h * D, x);
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] = value(vc[h], i, half_of(vq[h]), half_of(vq[h] >> 16));
            store8<OUT>(A.v_out, at + h * D, x);
        }
    }
}
template <int D, int OUT, bool FROM_POS>
__global__ void __launch_bounds__(ROW_THREADS) k_q4_load(RowsArgs A, pc_rope_dev rope) {
    pc_grid_dep_launch();
    pc_grid_dep_wait();
    load_rows<D, OUT, FROM_POS>(A, rope, blockIdx.x);
}

struct QueryArgs {
    const __nv_bfloat16 *q;
    const int32_t *pos;
    int chunks, chunks_row;     // pieces of eight channels, of a query
    float scale;
    __half *to;
    size_t second;              // where the second parts begin
    int32_t *status;
};
// Queries of 128 channels, rotated, times log2(e) / sqrt(d), in two fp16 parts: eight channels a thread.  Beyond +-65504 after that: held there and
// recorded; infinities and NaN become NaN.
__device__ __forceinline__ void make_queries(const QueryArgs &A, const pc_rope_dev &rope, int block) {
    const int c = block * ROW_THREADS + threadIdx.x;
    if (c >= A.chunks) return;
    float x[8], r[8];
    unpack8<false>(load8<false>(A.q, (size_t)c * 8), x);
    const int4 p = __ldg(reinterpret_cast<const int4 *>(A.pos) + c / A.chunks_row);
    bool bad = false, off = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 y = pc_rotate(x[2 * i], x[2 * i + 1], pc_rope_cs_clamped(rope, c % 16 * 4 + i, p.x, p.y, p.z, bad));
        x[2 * i] = y.x * A.scale;
        x[2 * i + 1] = y.y * A.scale;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        off |= fabsf(x[i]) > Q4_MAX;
        x[i] = into_f16(x[i]) + (x[i] - x[i]);     // + 0, or NaN
    }
    if (bad) pc_flag(A.status, PC_ERR_INVALID_ARG, PC_WHERE_Q4_POS);
    if (off) pc_flag(A.status, PC_ERR_INVALID_ARG, PC_WHERE_Q4_RANGE);
#pragma unroll
    for (int i = 0; i < 8; ++i) r[i] = x[i] - __half2float(__float2half_rn(x[i]));
    store8<OUT_F16>(A.to, (size_t)c * 8, x);
    store8<OUT_F16>(A.to, A.second + (size_t)c * 8, r);
}

// What a frame over the cache needs ahead of the attention kernel, in one launch: both segments in fp16, then the queries in two parts.  9,200 tokens
// of 8 KV heads and 1,008 queries of 24 heads, 68 MB with what is written: 16.5 us, most of it writes that stay in L2 (three launches one behind the other: 22).
struct FrontArgs {
    RowsArgs rows[2];
    QueryArgs queries;
    int blocks[2];              // of the two segments
};
__global__ void __launch_bounds__(ROW_THREADS) k_q4_front(const __grid_constant__ FrontArgs A, pc_rope_dev rope) {
    pc_grid_dep_launch();
    pc_grid_dep_wait();
    const int b = (int)blockIdx.x;
    if (b < A.blocks[0]) load_rows<128, OUT_F16, false>(A.rows[0], rope, b);
    else if (b < A.blocks[0] + A.blocks[1]) load_rows<128, OUT_F16, false>(A.rows[1], rope, b - A.blocks[0]);
    else make_queries(A.queries, rope, b - A.blocks[0] - A.blocks[1]);
}

unsigned row_blocks(const pc_layer_desc &D, int n, int slices) {
    const long long threads = (long long)n * slices * (D.head_dim / 8);
    return (unsigned)((threads + ROW_THREADS - 1) / ROW_THREADS);
}

// kernels of a head dimension and an element type (0 bf16, 1 fp32)
pc_status launch_rows(pc_ctx *ctx, const RowsArgs &A, cudaStream_t stream, void (*d128[2])(RowsArgs, pc_rope_dev), void (*d64[2])(RowsArgs, pc_rope_dev)) {
    const auto kernel = (ctx->desc.head_dim == 128 ? d128 : d64)[ctx->desc.dtype == PC_F32];
    PC_LAUNCH(kernel, dim3(row_blocks(ctx->desc, A.n, A.slices)), dim3(ROW_THREADS), 0, stream, A, ctx->rope);
    return PC_OK;
}

}  // namespace

extern "C" pc_status pc_q4_store(pc_ctx *ctx, const pc_segment *src, pc_q4_segment *dst, int32_t at, void *stream_) {
    if (!ctx || !src || !dst) return PC_ERR_INVALID_ARG;
    pc_status st = pc_check_segment(src, true);
    if (st != PC_OK) return st;
    if (at < 0 || at > dst->n_tokens || dst->n_tokens > dst->capacity || dst->t_shift < 0) return PC_ERR_INVALID_ARG;
    if (src->n_tokens > dst->capacity - at) return PC_ERR_CAPACITY;
    if (src->n_tokens == 0) return PC_OK;
    pc_q4_segment whole = *dst;
    whole.n_tokens = whole.n_tokens > at + src->n_tokens ? whole.n_tokens : at + src->n_tokens;
    st = q4_check_segment(&whole, false);
    if (st != PC_OK) return st;
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    RowsArgs A{};
    A.k = src->k;
    A.v = src->v;
    A.pos_in = src->pos;
    A.pos_out = dst->pos + (size_t)at * 4;
    A.q4 = static_cast<char *>(dst->rows) + (size_t)at * q4_row(ctx->desc);
    A.weight = dst->weight ? dst->weight + at : nullptr;
    A.n = src->n_tokens;
    A.n_kv = ctx->desc.n_kv_heads;
    A.slices = (A.n_kv + HEADS - 1) / HEADS;
    A.t_shift = dst->t_shift;
    A.status = ctx->status;
    void (*d128[2])(RowsArgs, pc_rope_dev) = {k_q4_store<128, false>, k_q4_store<128, true>};
    void (*d64[2])(RowsArgs, pc_rope_dev) = {k_q4_store<64, false>, k_q4_store<64, true>};
    st = launch_rows(ctx, A, stream, d128, d64);
    if (st == PC_OK) *dst = whole;
    return st;
}

extern "C" pc_status pc_q4_load(pc_ctx *ctx, const pc_q4_segment *src, int32_t first, int32_t n, pc_segment *dst, void *stream_) {
    if (!ctx || !src || !dst) return PC_ERR_INVALID_ARG;
    pc_status st = q4_check_segment(src, true);
    if (st != PC_OK) return st;
    if (first < 0 || n < 0 || n > src->n_tokens - first) return PC_ERR_INVALID_ARG;
    if (n > dst->capacity) return PC_ERR_CAPACITY;
    pc_segment filled = *dst;
    filled.n_tokens = n;
    st = pc_check_segment(&filled, true);
    if (st != PC_OK) return st;
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    if (n > 0) {
        RowsArgs A{};
        A.k_out = dst->k;
        A.v_out = dst->v;
        A.pos_in = src->pos + (size_t)first * 4;
        A.pos_out = dst->pos;
        A.q4 = static_cast<char *>(src->rows) + (size_t)first * q4_row(ctx->desc);
        A.n = n;
        A.n_kv = ctx->desc.n_kv_heads;
        A.slices = (A.n_kv + HEADS - 1) / HEADS;
        A.t_shift = src->t_shift;
        A.status = ctx->status;
        void (*d128[2])(RowsArgs, pc_rope_dev) = {k_q4_load<128, OUT_BF16, true>, k_q4_load<128, OUT_F32, true>};
        void (*d64[2])(RowsArgs, pc_rope_dev) = {k_q4_load<64, OUT_BF16, true>, k_q4_load<64, OUT_F32, true>};
        st = launch_rows(ctx, A, stream, d128, d64);
        if (st != PC_OK) return st;
    }
    dst->n_tokens = n;
    return PC_OK;
}

pc_status pc_q4_launch_front(pc_ctx *ctx, const pc_q4_segment *const *segs, int n_seg, void *const *k16, void *const *v16, const void *q, const int32_t *q_pos,
                             int32_t n_q, void *q16, int lo_row0, cudaStream_t stream) {
    const pc_layer_desc &D = ctx->desc;
    FrontArgs F{};
    for (int i = 0; i < n_seg; ++i) {
        RowsArgs &A = F.rows[i];
        A.k_out = k16[i];
        A.v_out = v16[i];
        A.q4 = static_cast<char *>(segs[i]->rows);
        A.n = segs[i]->n_tokens;
        A.n_kv = D.n_kv_heads;
        A.slices = (A.n_kv + HEADS - 1) / HEADS;
        A.t_shift = segs[i]->t_shift;
        A.status = ctx->status;
        F.blocks[i] = (int)row_blocks(D, A.n, A.slices);
    }
    const int per_query = D.n_q_heads * 16;
    F.queries = QueryArgs{static_cast<const __nv_bfloat16 *>(q), q_pos, n_q * per_query, per_query, pc_q_rot_scale(128), static_cast<__half *>(q16),
                          (size_t)lo_row0 * D.n_q_heads * 128, ctx->status};
    const int blocks = F.blocks[0] + F.blocks[1] + (F.queries.chunks + ROW_THREADS - 1) / ROW_THREADS;
    PC_LAUNCH(k_q4_front, dim3(blocks), dim3(ROW_THREADS), 0, stream, F, ctx->rope);
    return PC_OK;
}
