// Attention of few queries over the 4-bit cache, and the weights that tokens receive from it.
//
// Mathematics.  With codes c, steps s and lows l of a key's channel groups g,
//     q . k = sum_g s_g (q_g . c_g) + sum_g l_g sum(q_g),          out = sum_j p_j v_j = sum_g (sum_j (p_j s_jg) c_jg + sum_j p_j l_jg),
// so no value is ever decoded: the codes go to the tensor cores as they are, the step scales a sum over 32 channels (keys) or a
// probability (values), and the lows take one multiply-add instruction per 16 keys each.  A code becomes an fp16 number with one AND: the low four bits
// of a 16-bit half are the subnormal c 2^-24, the next four c 2^-20; the powers of two come off at the end.  Queries are scaled by a power of two
// per row and split into two fp16 parts (22 bits).  Softmax runs in base 2 with the running maximum and sum in fp32.
//
// Shape.  m16n8k16 instructions with 16 keys (channels, for the values) as rows and 8 query rows of one KV head as columns: a warp
// takes one KV head and 8 query rows and goes through the keys 16 at a time; the warps of a CTA cover the KV heads (and several
// blocks of rows, or several parts of the keys), so a CTA reads whole token rows.  TMA brings them, boxes of 32 tokens x 128 bytes with the 128-byte
// swizzle, into a ring of units of two steps that the warps refill in turn.  CTAs split the keys evenly; k_q4_join merges their parts, k_q4_weigh
// turns the logits that the history left into weights.
//
// What bounds it.  A token of 8 KV heads x 128 is 1,280 bytes, so 48,512 tokens are 62 MB, 9.6 us of memory.  Measured with 24 query heads, one token, by
// kernel from cold caches: 21 us (3.0 TB/s) + 5 us of merging, which overlap in a run of calls (23.0 us a call); 13,232 tokens 12.0 + 4.9 us (12.0 a call).  In
// the loop a warp step (16 keys of a head) is some 330 instructions and 13 matrix products of eight cycles each: instructions issue in 55 % of all
// cycles, and of a CTA's 32,000 cycles 22,100 are the loop (18,000 if it only streamed), 6,900 come ahead of it (queries and
// their table entries, one dependent fetch behind the other, under which the ring fills) and 3,100 behind it (parts merged and written).  The form
// whose lo parts are no columns of their own has 8 bytes of spills at 128 registers a thread, that of fp32 contexts 52.
#include <algorithm>
#include <new>

#include "pc_q4.cuh"
#include "pc_tc.cuh"

struct pc_q4 {
    pc_ctx *ctx;
    int max_tokens, parts;
    float *part_o, *part_ml, *lse;     // partial sums, (maximum, sum), and lse of a call (device)
    size_t part_rows;
    float *logits;                     // [history token][rows of a pass]
    size_t logit_floats;
    void *v, *q16;                     // values of the whole cache in fp16, queries in two fp16 parts (PC_Q4_FRAMES)
    size_t v_rows;
};

namespace {

constexpr int ROWS = 8;                // query rows of a warp
constexpr int MAX_WARPS = 16;          // of a CTA: 128 registers a thread
constexpr int MAX_SLOTS = 32;
constexpr int RING_AT = 1024;          // barriers and flags before the ring
constexpr int FACTORS_AT = 512;        // of these, steps' factors of each warp
constexpr int SMEM_MOST = 226 * 1024;  // with 1,024 bytes to align the ring
constexpr int UNIT = 2;                // steps that a warp takes together
constexpr int BOX = 128, BOX_BYTES = UNIT * Q4_STEP * BOX; // a box of the rows: a unit's tokens x 128 bytes
// fp16's range, where probabilities and their products with steps are fp16 numbers (bf16 contexts): probabilities are scaled by 2^8 (the sums with them, so
// that it cancels), and the steps of a value's channel group by a power of two that leaves the largest met so far at up to 2^7, so that products
// stay at up to 2^15.  That largest is at 2^5 at least (or the factor 2^15, its most): a product that is 2^-27 of the largest still has all its bits.
// (Unscaled, products below 2^-25 vanished, always towards the group's low.)  fp32 contexts hold products in bf16 parts, which have the range.
constexpr float P_LOG_F16 = 8.f, P_LOG_F32 = 2.f;
constexpr uint32_t SIGNS = 0x80008000u;
constexpr uint32_t STEPS_LIMIT = 0x14011400u;      // (0x9400 - a factor) is 2^7 / factor, with the sign set: less a step, it keeps the sign unless the step is larger
constexpr uint32_t FACTOR_MOST = 0x78007800u;      // 2^15, twice: the factors before any step has been met
constexpr float NO_MAX = -1e30f;       // of a row that has met no key: finite, so that a masked logit (-infinity) gives probability 0

// Queries as the B operand in shared memory, of a task (KV head, block of 8 rows): words [hi and lo parts 8 NG][sums 2] of 32 lanes, then 8 factors
// Of up to four rows (a single token of grouped heads) the lo parts are columns of their own, 4 to 7, and one pass multiplies both ("folded").
__host__ __device__ constexpr int query_words(int d, bool folded) { return folded ? 4 * (d / Q4_GROUP) + 1 : 8 * (d / Q4_GROUP) + 2; }
__host__ __device__ constexpr int query_bytes(int d, bool folded) { return query_words(d, folded) * 128 + ROWS * 4; }

struct Q4Params {
    int n[2], shift[2];                // tokens of anchors, history; what their keys are shifted by
    const uint8_t *valid;              // of the history, or NULL
    const void *q;
    const int32_t *q_pos;
    int n_q, n_q_heads, n_kv, group, n_rows;      // n_rows = n_q * group: query rows of a KV head
    int heads, blocks, subs;           // of a CTA: KV heads, blocks of 8 query rows, parts of the keys
    uint32_t inv_tasks, inv_heads;     // 65536 / (heads * blocks) + 1, 65536 / heads + 1: a warp's number (below 16) is divided by multiplying
    float inv_group;
    int ctas0;                         // CTAs that take the anchors; the others take the history
    int steps[2], more[2];             // of 16 keys: of a CTA of either kind, and how many of these take one more
    int boxes_k, boxes;                // boxes of a unit: of the key codes (as many for the values), all
    int unit_bytes, slots;             // of the ring, which holds `slots` units
    int whole_rows;                    // 1: a unit comes by one instruction
    int queries_at;                    // behind the ring
    float *part_o, *part_ml;           // [split][KV head * n_rows + row]
    float *logits;                     // [history token][n_kv * n_rows] or NULL
    float scale;                       // log2(e) / sqrt(d)
    int32_t *status;
    uint32_t wait_us;
    uint32_t extra_tx;                 // test hook: bytes the first barrier expects beyond what is sent (0 = off)
};

struct JoinParams {
    const float *part_o, *part_ml;
    int splits, rows, n_rows, group, n_q_heads;
    void *out;
    float *lse, *lse_rows;             // the caller's [query][head] and the workspace's [row], either may be NULL
};

__device__ __forceinline__ uint32_t lds32(uint32_t a) { uint32_t v; asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(a)); return v; }
// N 32-bit words of shared memory (2 or 4; N = 1 for the values of d = 64)
template <int N> __device__ __forceinline__ void lds(uint32_t a, uint32_t (&w)[N]) {
    if constexpr (N == 4) asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(a));
    else if constexpr (N == 2) asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "r"(a));
    else w[0] = lds32(a);
}
__device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_first(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}
__device__ __forceinline__ void mma_bf16(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// Four 8 x 8 matrices of 16-bit values, a row at each lane's address (eight lanes a matrix); TRANS: transposed
template <bool TRANS> __device__ __forceinline__ void load_matrices(uint32_t a, uint32_t (&x)[4]) {
    if constexpr (TRANS) asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3]) : "r"(a));
    else asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3]) : "r"(a));
}
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {         // an 8 x 8 matrix of 16-bit values, two a lane
    uint32_t y;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}
__device__ __forceinline__ uint32_t pack_half(float lo, float hi) {
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&v);
}
__device__ __forceinline__ uint32_t mul_half(uint32_t a, uint32_t b) {
    const __half2 v = __hmul2(*reinterpret_cast<const __half2 *>(&a), *reinterpret_cast<const __half2 *>(&b));
    return *reinterpret_cast<const uint32_t *>(&v);
}
// ON: two codes less 8, exactly (the codes lie `shift` bits up)
template <bool ON> __device__ __forceinline__ uint32_t middle(uint32_t codes, int shift) {
    if constexpr (!ON) return codes;
    const uint32_t eight = 0x00080008u << shift;
    const __half2 v = __hsub2(*reinterpret_cast<const __half2 *>(&codes), *reinterpret_cast<const __half2 *>(&eight));
    return *reinterpret_cast<const uint32_t *>(&v);
}
// Two codes less 8 in bf16: in the last places of 128 + code, less 136
__device__ __forceinline__ uint32_t middle_bf16(uint32_t codes) {
    const uint32_t x = (codes & 0x000F000Fu) | 0x43004300u, y = 0x43084308u;
    const __nv_bfloat162 v = __hsub2(*reinterpret_cast<const __nv_bfloat162 *>(&x), *reinterpret_cast<const __nv_bfloat162 *>(&y));
    return *reinterpret_cast<const uint32_t *>(&v);
}
// Factors for two groups' steps of which the largest are `top`: 2^(e - 15) <= top < 2^(e - 14) gives 2^(20 - e), room for a step twice as large
__device__ __forceinline__ uint32_t factors_for(uint32_t top) {
    return (0x00230023u - __vminu2(__vmaxu2((top >> 10) & 0x001F001Fu, 0x00050005u), 0x001D001Du)) << 10;
}
__device__ __forceinline__ int factor_exponent(uint32_t factors, int upper) { return (int)((factors >> (upper ? 26 : 10)) & 31u); }      // + 15
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((uint32_t)(127 + e) << 23); }
__device__ __forceinline__ float2 halves(uint32_t w) { return __half22float2(*reinterpret_cast<const __half2 *>(&w)); }
__device__ __forceinline__ float exp2_fast(float x) { float y; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }

// Key of a step that is row i (0 .. 7) of the instruction's upper half.  The swizzle moves the 16-byte units of a token's 128 bytes by
// exclusive-or with the token's number; lanes that are served together then read different banks: key codes (16 bytes a lane, rows i and
// i + 1 of an even i together: tokens that differ in bit 2) and value codes (8 bytes a lane, four even or four odd rows together: tokens that
// differ in bits 1 and 2).
__device__ __forceinline__ int key_of_row(int i) { return (0x36147250u >> (4 * i)) & 7; }

// Byte `b` of a section (its first box at `box0`) of token `key` (0 .. 7) in a unit
__device__ __forceinline__ uint32_t place(int box0, int b, int key) {
    return (uint32_t)((box0 + (b >> 7)) * BOX_BYTES + key * BOX + ((((b >> 4) & 7) ^ key) << 4) + (b & 15));
}

__device__ __forceinline__ int4 ldg_int4(const int32_t *p) {
    int4 v;
    asm volatile("ld.global.nc.v4.s32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
    return v;
}
__device__ __forceinline__ float2 ldg_float2(const float2 *p) {
    float2 v;
    asm volatile("ld.global.nc.v2.f32 {%0,%1}, [%2];" : "=f"(v.x), "=f"(v.y) : "l"(p));
    return v;
}

// The queries of a task, rotated at (t + shift, h, w), times log2(e) / sqrt(d), as the B operand of Q K^T in shared memory.  The warps of a task (one for
// each part of the keys) take its rows in turn, D / 32 consecutive channels a lane, two rows at a time; columns without a row are zero.
// behind() is called once the first rows' table entries have been requested: what it fetches would hold up these loads, one behind the other.
template <int D, bool F32, bool FOLD, typename Behind>
__device__ __forceinline__ void take_queries(const Q4Params &P, const pc_rope_dev &rope, char *to, int kv_head, int block, int sub, int shift, Behind behind) {
    constexpr int NG = D / Q4_GROUP, CH = D / 32, WORDS = query_words(D, FOLD), PER = 2;
    const int lane = threadIdx.x & 31;
    const int count = min(P.n_rows - block * ROWS, ROWS);            // none or fewer for a warp that has no head or no rows
    // channel 32 g + 8 t + k of a row: 16-bit half k / 4 of word (2 g + k % 2) * 2 + (k / 2) % 2 of lane 4 row + t.  The code words give
    // channels (k, k + 4) as one register: k even in the low four bits of their bytes, k odd in the high four, 2^4 larger
    const int g = lane * CH / Q4_GROUP, t = lane * CH % Q4_GROUP / 8, k0 = lane * CH % 8;
#pragma unroll 1
    for (int base = sub;; base += PER * P.subs) {
        const bool first = base == sub;
        if (!first && base >= count) break;
        int4 p[PER];
        uint32_t raw[PER][CH];
#pragma unroll
        for (int u = 0; u < PER; ++u) {
            const int r = block * ROWS + base + u * P.subs;
            p[u] = make_int4(0, 0, 0, 0);
            if (base + u * P.subs < count) {
                const int query = (int)(((float)r + 0.5f) * P.inv_group), head = kv_head * P.group + r - query * P.group;
                p[u] = ldg_int4(P.q_pos + (size_t)query * 4);
                const char *src = static_cast<const char *>(P.q) + (((size_t)query * P.n_q_heads + head) * D + lane * CH) * (F32 ? 4 : 2);
                constexpr int N = CH * (F32 ? 4 : 2) / 4;
                if constexpr (N == 4) asm volatile("ld.global.nc.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(raw[u][0]), "=r"(raw[u][1]), "=r"(raw[u][2]), "=r"(raw[u][3]) : "l"(src));
                else if constexpr (N == 2) asm volatile("ld.global.nc.v2.u32 {%0,%1}, [%2];" : "=r"(raw[u][0]), "=r"(raw[u][1]) : "l"(src));
                else asm volatile("ld.global.nc.u32 %0, [%1];" : "=r"(raw[u][0]) : "l"(src));
            }
        }
        if (first) {
            if ((FOLD ? (lane >> 2) & 3 : lane >> 2) >= count) {
                for (int w = sub; w < WORDS; w += P.subs) reinterpret_cast<uint32_t *>(to)[w * 32 + lane] = 0u;
                if ((lane & 3) == 0) reinterpret_cast<float *>(to + WORDS * 128)[lane >> 2] = 0.f;
            }
        }
        float2 cs[PER][CH / 2];
        bool bad = false;
#pragma unroll
        for (int c = 0; c < CH / 2; ++c) {
            const int pair = lane * (CH / 2) + c, a = pair % 3;
            const int most = a == 0 ? rope.max_pos[0] : (a == 1 ? rope.max_pos[1] : rope.max_pos[2]);
            const int off = (a == 0 ? rope.off[0] : (a == 1 ? rope.off[1] : rope.off[2])) + pair / 3;
            const int n = a == 0 ? rope.n_axis[0] : (a == 1 ? rope.n_axis[1] : rope.n_axis[2]);
#pragma unroll
            for (int u = 0; u < PER; ++u) {
                const int at = a == 0 ? p[u].x + shift : (a == 1 ? p[u].y : p[u].z);
                bad |= base + u * P.subs < count && (unsigned)at >= (unsigned)most;
                cs[u][c] = ldg_float2(rope.tab + off + (size_t)min(max(at, 0), most - 1) * n);
            }
        }
        if (first) behind();
        if (bad) pc_flag(P.status, PC_ERR_INVALID_ARG, PC_WHERE_Q4_POS);
#pragma unroll
        for (int u = 0; u < PER; ++u) {
            const int col = base + u * P.subs;
            if (col >= count) break;
            float x[CH], most = 0.f, total = 0.f;
#pragma unroll
            for (int c = 0; c < CH; c += 2) {
                const float x0 = F32 ? __uint_as_float(raw[u][c]) : pc_bf16_lo(raw[u][c / 2]);
                const float x1 = F32 ? __uint_as_float(raw[u][c + 1]) : pc_bf16_hi(raw[u][c / 2]);
                const float2 y = pc_rotate(x0, x1, cs[u][c / 2]);
                x[c] = y.x * P.scale;
                x[c + 1] = y.y * P.scale;
                most = fmaxf(most, fmaxf(fabsf(x[c]), fabsf(x[c + 1])));
            }
            // the row's largest value to 2^6 .. 2^7: eight times a sum over 32 channels stays in fp16's range
            most = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(most)));
            const int e = min(100, max(-121, 6 - ((int)(__float_as_uint(most) >> 23) - 127)));
            const float up = __uint_as_float((uint32_t)(e + 127) << 23);
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                const int k = k0 + c;
                const float v = x[c] * up, y = (c & 1) ? v * 0.0625f : v;             // k0 is even
                total += v;
                const __half hi = __float2half_rn(y);
                const int word = (2 * g + (c & 1)) * 2 + ((k >> 1) & 1);
                __half *at16 = reinterpret_cast<__half *>(to + (word * 32 + col * 4 + t) * 4) + (k >> 2);
                at16[0] = hi;
                at16[FOLD ? 32 : 4 * NG * 64] = __float2half_rn(y - __half2float(hi));
            }
            // sums over the groups, which meet the lows: indices NG .. 2 NG - 1 of the instruction's first eight (the others meet the steps: zero, or,
            // where codes are taken around 8, eight times the sums), a second fp16 part at the same places of the other eight
#pragma unroll
            for (int o = 1; o < Q4_GROUP / CH; o <<= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
            constexpr int SUMS = FOLD ? 4 * NG : 8 * NG, SECOND = FOLD ? 16 : 32;       // the second part: the column's other half, or the next word
            uint32_t *sums = reinterpret_cast<uint32_t *>(to) + SUMS * 32 + col * 4;
            const float next = __shfl_down_sync(0xffffffffu, total, Q4_GROUP / CH);   // of the group behind
            if (lane < 4) {                        // a word of two groups a lane, zero where the steps are
                sums[lane] = 0u;
                sums[SECOND + lane] = 0u;
            }
            __syncwarp();
            if (lane % (2 * Q4_GROUP / CH) == 0) {
                const uint32_t h = pack_half(total, next);
                const float2 back = halves(h);
                sums[NG / 2 + g / 2] = h;
                sums[SECOND + NG / 2 + g / 2] = pack_half(total - back.x, next - back.y);
                if constexpr (F32) {
                    sums[g / 2] = pack_half(8.f * back.x, 8.f * back.y);
                    sums[SECOND + g / 2] = pack_half(8.f * (total - back.x), 8.f * (next - back.y));
                }
            }
            // (what takes the scale off again is an fp32 number up to 2^127: a row beyond 2^109 counts as a power of two smaller)
            if (lane == 0) {
                if (e < -102 && most < INFINITY) pc_flag(P.status, PC_ERR_INVALID_ARG, PC_WHERE_Q4_RANGE);
                reinterpret_cast<float *>(to + WORDS * 128)[col] = __uint_as_float((uint32_t)(min(126, 24 - e) + 127) << 23);
            }
        }
    }
    __syncthreads();
}

template <int D, bool F32, bool FOLD>
__global__ void __launch_bounds__(MAX_WARPS * 32, 1) k_q4_attend(const __grid_constant__ CUtensorMap map0, const __grid_constant__ CUtensorMap map1,
                                                                  const __grid_constant__ Q4Params P, const pc_rope_dev rope) {
    constexpr int NG = D / Q4_GROUP;
    extern __shared__ char smem_raw[];
    pc_grid_dep_launch();
    const uint32_t base = (pc_smem_u32(smem_raw) + 1023u) & ~1023u, ring = base + RING_AT;
    char *smem = smem_raw + (base - pc_smem_u32(smem_raw));
    volatile int *abort_flag = reinterpret_cast<volatile int *>(smem + 12 * MAX_SLOTS);
    const auto full = [&](int s) { return base + 8 * s; };
    const auto left = [&](int s) { return base + 8 * MAX_SLOTS + 4 * s; };        // warps that are done with the unit of a slot
    const int warp = __shfl_sync(0xffffffffu, (int)threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const int tasks = P.heads * P.blocks, n_warps = tasks * P.subs;
    if (threadIdx.x == 0) {
        for (int s = 0; s < P.slots; ++s) {
            pc_mbar_init(full(s), 1);
            *reinterpret_cast<int *>(smem + 8 * MAX_SLOTS + 4 * s) = 0;
        }
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    __syncthreads();
    const int first_head = blockIdx.z * P.heads, first_block = blockIdx.y * P.blocks, n_heads = min(P.heads, P.n_kv - first_head);
    const int sub = (int)(warp * P.inv_tasks >> 16), task = warp - sub * tasks;
    const int head = task - (int)(task * P.inv_heads >> 16) * P.heads, block = first_block + (int)(task * P.inv_heads >> 16);
    const bool works = head < n_heads && block * ROWS < P.n_rows;      // else the ring still goes round
    // This CTA's steps, of one segment.  A unit is two of them; the parts of the keys take the units in turn.
    const bool hist = (int)blockIdx.x >= P.ctas0;
    const int bx = (int)blockIdx.x - (hist ? P.ctas0 : 0), more = hist ? P.more[1] : P.more[0];
    const int n_steps = (hist ? P.steps[1] : P.steps[0]) + (bx < more ? 1 : 0), step0 = bx * (hist ? P.steps[1] : P.steps[0]) + min(bx, more);
    const int n_units = (n_steps + UNIT - 1) / UNIT, n_seg = hist ? P.n[1] : P.n[0];
    pc_grid_dep_wait();

    // A unit into a slot, by one elected lane of a warp: all boxes by one instruction where a CTA takes whole rows of whole boxes, else box by box:
    // of the key codes, of the value codes, of the steps and lows.  (A TMA instruction takes its warp 85 cycles: ten a unit held up the
    // warp whose turn it was, and with it the ring.)
    const bool lead = pc_tc::elect_one();
    const CUtensorMap *map = hist ? &map1 : &map0;
    const auto fetch = [&](int unit, int slot) {
        if (lead) {
            const uint32_t bar = full(slot);
            uint32_t dst = ring + slot * P.unit_bytes;
            const int y = (step0 + unit * UNIT) * Q4_STEP;
            pc_mbar_expect_tx(bar, P.unit_bytes + (unit == 0 ? P.extra_tx : 0u));
            if (P.whole_rows) {
                asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                             ::"r"(dst), "l"(map), "r"(0), "r"(y), "r"(0), "r"(bar) : "memory");
            } else {
                int x = first_head * (D / 2);
#pragma unroll 1
                for (int i = 0; i < P.boxes_k; ++i, x += BOX, dst += BOX_BYTES) {
                    pc_tc::tma_load_2d(dst, map, x, y, bar);
                    pc_tc::tma_load_2d(dst + P.boxes_k * BOX_BYTES, map, x + P.n_kv * (D / 2), y, bar);
                }
                dst += P.boxes_k * BOX_BYTES;
                x = P.n_kv * D + first_head * (D / 4);
#pragma unroll 1
                for (int i = 2 * P.boxes_k; i < P.boxes; ++i, x += BOX, dst += BOX_BYTES) pc_tc::tma_load_2d(dst, map, x, y, bar);
            }
        }
        __syncwarp();
    };
    const int t = lane & 3, row = lane >> 2;
    float O[2 * NG][4], L[4];          // out without the lows, channel 32 g + 4 row + {0, 1} ({2, 3}) of columns 2 t, 2 t + 1; the lows' part of group g in row 8 - NG + g
    float W[F32 ? NG : 1][2];          // fp32 contexts, in the place of L: of the lane's own keys
    float m0 = NO_MAX, m1 = NO_MAX, l0 = 0.f, l1 = 0.f;
    constexpr float P_LOG = F32 ? P_LOG_F32 : P_LOG_F16;
    // Factors of the steps of each group, two to a word as the steps are (O has them too): in shared memory, a warp's own, for want of registers
    const uint32_t factors_at = base + FACTORS_AT + 8 * warp;
    const auto set_factor = [&](int w, uint32_t f) { asm volatile("st.shared.u32 [%0], %1;" ::"r"(factors_at + 4 * w), "r"(f) : "memory"); };
    if constexpr (!F32) {
#pragma unroll
        for (int w = 0; w < NG / 2; ++w) set_factor(w, FACTOR_MOST);
    }
#pragma unroll
    for (int i = 0; i < (F32 ? NG : 1); ++i) W[i][0] = W[i][1] = 0.f;
#pragma unroll
    for (int i = 0; i < 2 * NG; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) O[i][j] = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) L[j] = 0.f;
    // places of the lane's keys in a step: codes, steps and lows of its two keys, and of the four whose values it takes (rows 2 t, 2 t + 1
    // of the instruction; the second half lies 8 tokens on)
    const int k0 = key_of_row(row), kva = key_of_row(2 * t), kvb = key_of_row(2 * t + 1);
    constexpr uint32_t EIGHT = 8 * BOX;
    const int box_s = 2 * P.boxes_k;
    const uint32_t at_k = place(0, head * (D / 2) + t * NG * 4, k0), at_ks = place(box_s, head * (D / 4), k0);
    const uint32_t at_vsa = place(box_s, head * (D / 4) + 4 * NG, kva), at_vsb = place(box_s, head * (D / 4) + 4 * NG, kvb);
    // steps and lows as matrices, eight numbers of a token a row, in the order of an A operand: of the key, tokens as rows (the second half of the
    // instruction's index sees them again); of the value, transposed
    const int km = key_of_row(lane & 7);
    const uint32_t at_mk = place(box_s, head * (D / 4), km) + ((lane >> 3) & 1) * EIGHT;
    // value codes likewise: a group's 16 bytes of a token a row; lanes 0-15 give the rows of the even group of a pair, lanes 16-31 of the odd
    uint32_t at_v[NG / 2];
#pragma unroll
    for (int g = 0; g < NG; g += 2) at_v[g / 2] = place(P.boxes_k, head * (D / 2) + (g + (lane >> 4)) * 16, km) + ((lane >> 3) & 1) * EIGHT;
    const uint32_t at_vk = place(box_s, head * (D / 4) + 4 * NG, k0);              // fp32 contexts: steps and lows of the lane's two values
    const uint32_t at_mv = place(box_s, head * (D / 4) + (NG == 4 ? 16 : 0), km) + (lane >> 4) * EIGHT;
    const int r0 = block * ROWS + 2 * t, R = P.n_kv * P.n_rows;        // folded: lanes of the lo parts (t > 1) have no row
    char *queries = smem + P.queries_at + task * query_bytes(D, FOLD);
    take_queries<D, F32, FOLD>(P, rope, queries, first_head + head, head < n_heads ? block : P.n_rows, sub, hist ? P.shift[1] : P.shift[0], [&] {
        for (int u = warp; u < min(P.slots, n_units); u += n_warps) fetch(u, u);
    });
    uint32_t q_hi[2 * NG][2], q_lo[FOLD ? 1 : 2 * NG][2], q_sum[2];
    const uint32_t my_q = pc_smem_u32(queries) + lane * 4;
#pragma unroll
    for (int i = 0; i < 4 * NG; ++i) {
        q_hi[i / 2][i & 1] = lds32(my_q + i * 128);
        if constexpr (!FOLD) q_lo[i / 2][i & 1] = lds32(my_q + (4 * NG + i) * 128);
    }
    q_sum[0] = lds32(my_q + (FOLD ? 4 : 8) * NG * 128);
    q_sum[1] = FOLD ? 0u : lds32(my_q + (8 * NG + 1) * 128);
    const float *factor = reinterpret_cast<const float *>(queries + query_words(D, FOLD) * 128);
    const float f0 = factor[FOLD ? (2 * t) & 3 : 2 * t], f1 = factor[FOLD ? (2 * t + 1) & 3 : 2 * t + 1];
    const uint8_t *valid = hist ? P.valid : nullptr;
    float *logits = hist ? P.logits : nullptr;
    if (logits) logits += (size_t)(first_head + head) * P.n_rows + r0;
    // Raw logits of a step's keys k0, k0 + 8 against columns 2 t, 2 t + 1: to be multiplied by f0, f1
    const auto logits_of = [&](uint32_t rows, float (&S)[4]) {
        uint32_t wa[NG], wb[NG], sa[NG / 2], sb[NG / 2], la[4];
        lds(rows + at_k, wa);
        lds(rows + at_k + EIGHT, wb);
        lds(rows + at_ks, sa);
        lds(rows + at_ks + EIGHT, sb);
        load_matrices<false>(rows + at_mk, la);
        float E[4], C[NG][4];
        mma_first(E, la[0], la[1], la[2], la[3], q_sum[0], q_sum[1]);
#pragma unroll
        for (int h = 0; h < 2; ++h) {            // channels in the low four bits of the code words' bytes, then in the high four
            const uint32_t mask = h ? 0x00F000F0u : 0x000F000Fu;
#pragma unroll
            for (int g = 0; g < NG; ++g) {
                const uint32_t a0 = middle<F32>(wa[g] & mask, 4 * h), a1 = middle<F32>(wb[g] & mask, 4 * h);
                const uint32_t a2 = middle<F32>((wa[g] >> 8) & mask, 4 * h), a3 = middle<F32>((wb[g] >> 8) & mask, 4 * h);
                if (h == 0) mma_first(C[g], a0, a1, a2, a3, q_hi[2 * g][0], q_hi[2 * g][1]);
                else mma(C[g], a0, a1, a2, a3, q_hi[2 * g + 1][0], q_hi[2 * g + 1][1]);
                if constexpr (!FOLD) mma(C[g], a0, a1, a2, a3, q_lo[2 * g + h][0], q_lo[2 * g + h][1]);
            }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) S[j] = E[j] * (1.f / 16777216.f);
#pragma unroll
        for (int g = 0; g < NG; ++g) {
            const float2 pa = halves(sa[g / 2]), pb = halves(sb[g / 2]);
            const float fa = (g & 1) ? pa.y : pa.x, fb = (g & 1) ? pb.y : pb.x;
            S[0] = fmaf(fa, C[g][0], S[0]);
            S[1] = fmaf(fa, C[g][1], S[1]);
            S[2] = fmaf(fb, C[g][2], S[2]);
            S[3] = fmaf(fb, C[g][3], S[3]);
        }
        if constexpr (FOLD) {                    // both halves of the columns get the sum
#pragma unroll
            for (int j = 0; j < 4; ++j) S[j] += __shfl_xor_sync(0xffffffffu, S[j], 2);
        }
    };
    // Keys of a step that are there and not masked: a bit per row of the instruction
    const auto look_at_mask = [&](int first, float (&S)[4], bool there, const uint8_t (&mask)[2]) {
        const int n = there ? n_seg - first : 0;
        const bool ok0 = k0 < n && mask[0] != 0, ok1 = k0 + 8 < n && mask[1] != 0;
        if (!ok0) S[0] = S[1] = -INFINITY;
        if (!ok1) S[2] = S[3] = -INFINITY;
        // lane 4 i speaks for row i, lane 4 i + 1 for row i + 8
        return __ballot_sync(0xffffffffu, t == 0 ? ok0 : ok1);
    };
    const auto leave_logits = [&](int first, const float (&S)[4]) {
        const int n = n_seg - first;
        float *to = logits + (size_t)(first + k0) * R;
        if (k0 < n) {
            if (r0 < P.n_rows) to[0] = S[0] * f0;
            if (r0 + 1 < P.n_rows) to[1] = S[1] * f1;
        }
        if (k0 + 8 < n) {
            to += (size_t)8 * R;
            if (r0 < P.n_rows) to[0] = S[2] * f0;
            if (r0 + 1 < P.n_rows) to[1] = S[3] * f1;
        }
    };
    // O += P V of a step, p = the probabilities of S's keys and columns
    const auto add_values = [&](uint32_t rows, const float (&p)[4], bool all, uint32_t seen) {
        uint32_t steps[4][NG / 2], codes[NG / 2][4], lows[4];        // codes: a group's four of each key, of two keys a word
#pragma unroll
        for (int j = 0; j < 4; ++j) lds(rows + (j & 1 ? at_vsb : at_vsa) + (j >> 1) * EIGHT, steps[j]);
#pragma unroll
        for (int g = 0; g < NG / 2; ++g) load_matrices<true>(rows + at_v[g], codes[g]);
        if constexpr (!F32) load_matrices<true>(rows + at_mv, lows);
        if (!all) {                              // what lies in the place of a masked key may be anything
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (!((seen >> (4 * (2 * t + (j & 1)) + (j >> 1))) & 1u)) {
                    if constexpr (!F32) {
                        lows[j & 2] &= (j & 1) ? 0x0000FFFFu : 0xFFFF0000u;
                        lows[(j & 2) + 1] = lows[j & 2];
                    }
#pragma unroll
                    for (int w = 0; w < NG / 2; ++w) steps[j][w] = 0u;
                }
        }
        if constexpr (!F32) {
            uint32_t factors[NG / 2];
            lds(factors_at, factors);
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int w = 0; w < NG / 2; ++w) steps[j][w] = mul_half(steps[j][w], factors[w]);
        }
        uint32_t pl[2], ph[2];                   // probabilities as the B operand: column = query row lane / 4
        constexpr float UP = F32 ? 8192.f : 1.f; // the second part of a small probability would be a subnormal number
        ph[0] = pack_half(p[0] * UP, p[1] * UP);
        ph[1] = pack_half(p[2] * UP, p[3] * UP);
        if constexpr (F32) {
            const float2 a = halves(ph[0]), b = halves(ph[1]);
            pl[0] = transpose8(pack_half(p[0] * UP - a.x, p[1] * UP - a.y));
            pl[1] = transpose8(pack_half(p[2] * UP - b.x, p[3] * UP - b.y));
            // Values around their group's middle, v = (low + 8 step) + step (code - 8): sums over codes and sums over lows would each be many times
            // larger than their difference, the output, which an fp32 output shows
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                uint32_t st[NG / 2], lo[NG / 2];
                lds(rows + at_vk + i * EIGHT, st);
                lds(rows + at_vk + i * EIGHT + 2 * NG, lo);
                if (!((seen >> (4 * row + i)) & 1u)) continue;
#pragma unroll
                for (int g = 0; g < NG; ++g) {
                    const float2 s2 = halves(st[g / 2]), l2 = halves(lo[g / 2]);
                    const float mid = fmaf(8.f, (g & 1) ? s2.y : s2.x, (g & 1) ? l2.y : l2.x);
                    W[g][0] = fmaf(p[2 * i], mid, W[g][0]);
                    W[g][1] = fmaf(p[2 * i + 1], mid, W[g][1]);
                }
            }
        }
        ph[0] = transpose8(ph[0]);
        ph[1] = transpose8(ph[1]);
        if constexpr (!F32) mma(L, lows[0], lows[1], lows[2], lows[3], ph[0], ph[1]);
#pragma unroll
        for (int g = 0; g < NG; ++g) {
            const uint32_t pick = (g & 1) ? 0x7632u : 0x5410u;
            const uint32_t ta = codes[g / 2][2 * (g & 1)], tb = codes[g / 2][2 * (g & 1) + 1];
            const uint32_t qa = __byte_perm(steps[0][g / 2], steps[1][g / 2], pick), qb = __byte_perm(steps[2][g / 2], steps[3][g / 2], pick);
            const uint32_t ya = ta >> 8, yb = tb >> 8;
            if constexpr (F32) {
                // probability times step in fp32 from the two parts, then in three bf16 parts, whose range no step leaves
                const float2 sa = halves(qa), sb = halves(qb), xh = halves(ph[0]), yh = halves(ph[1]), xl = halves(pl[0]), yl = halves(pl[1]);
                float e[4] = {(xh.x + xl.x) * (sa.x / UP), (xh.y + xl.y) * (sa.y / UP), (yh.x + yl.x) * (sb.x / UP), (yh.y + yl.y) * (sb.y / UP)};
#pragma unroll
                for (int part = 0; part < 3; ++part) {
                    const uint32_t h0 = pc_pack_bf16(e[0], e[1]), h1 = pc_pack_bf16(e[2], e[3]);
                    mma_bf16(O[2 * g], middle_bf16(ta), middle_bf16(ta >> 4), middle_bf16(tb), middle_bf16(tb >> 4), h0, h1);
                    mma_bf16(O[2 * g + 1], middle_bf16(ya), middle_bf16(ya >> 4), middle_bf16(yb), middle_bf16(yb >> 4), h0, h1);
                    e[0] -= pc_bf16_lo(h0);
                    e[1] -= pc_bf16_hi(h0);
                    e[2] -= pc_bf16_lo(h1);
                    e[3] -= pc_bf16_hi(h1);
                }
            } else {
                const uint32_t a0 = ta & 0x000F000Fu, a1 = ta & 0x00F000F0u, a2 = tb & 0x000F000Fu, a3 = tb & 0x00F000F0u;
                const uint32_t c0 = ya & 0x000F000Fu, c1 = ya & 0x00F000F0u, c2 = yb & 0x000F000Fu, c3 = yb & 0x00F000F0u;
                const uint32_t h0 = mul_half(ph[0], qa), h1 = mul_half(ph[1], qb);
                mma(O[2 * g], a0, a1, a2, a3, h0, h1);
                mma(O[2 * g + 1], c0, c1, c2, c3, h0, h1);
            }
        }
    };
    // The warp's units: every subs-th, in the slots of its part of the keys (sub, sub + subs, ...) in turn.  `slots` is a multiple of `subs`, so
    // the barriers of a slot are only waited on by warps that have seen every phase before (a wait by parity cannot tell a phase from the one
    // two before or behind it).  The last of the warps that share a unit to leave it fetches what follows in its slot.
    const auto wait_for = [&](uint32_t bar, uint32_t parity) {
        return __all_sync(0xffffffffu, pc_mbar_wait(bar, parity, abort_flag, P.status, PC_WHERE_Q4_WAIT, P.wait_us)) != 0;
    };
    int slot = sub;
    uint32_t phase = 0;
#pragma unroll 1
    for (int unit = sub; unit < n_units; unit += P.subs) {
        uint8_t mask[2][2] = {{1, 1}, {1, 1}};       // requested ahead of the wait
        if (valid) {
            const int at = (step0 + unit * UNIT) * Q4_STEP + k0;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (at + 8 * i < n_seg) mask[i / 2][i & 1] = __ldg(valid + at + 8 * i);
        }
        if (!wait_for(full(slot), phase)) break;
        if (works) {
            const uint32_t rows = ring + slot * P.unit_bytes, rows1 = rows + Q4_STEP * BOX;
            // (of one step: the second one's place holds tokens of the next CTA, or zeros; its logits count as masked)
            const bool two = unit * UNIT + 1 < n_steps;
            const int first = (step0 + unit * UNIT) * Q4_STEP;
            // Steps beyond what the factors leave room for: a token a lane (of step `lane / 8 % 2` of the unit, row `lane % 8` of its half `lane / 16`)
            uint32_t top[NG / 2], factors[NG / 2];
            if constexpr (!F32) {
                lds(factors_at, factors);
                lds(rows + at_mv + (NG == 4 ? 0 : 8) + ((lane >> 3) & 1) * (Q4_STEP * BOX), top);
            }
            float S0[4], S1[4];
            logits_of(rows, S0);
            logits_of(rows1, S1);
            uint32_t seen0 = 0xffffffffu, seen1 = 0xffffffffu;
            const bool all = !valid && two && first + UNIT * Q4_STEP <= n_seg;
            if (!all) {
                seen0 = look_at_mask(first, S0, true, mask[0]);
                seen1 = look_at_mask(first + Q4_STEP, S1, two, mask[1]);
            }
            if (logits) {
                leave_logits(first, S0);
                if (two) leave_logits(first + Q4_STEP, S1);
            }
            // ---- softmax: maximum of the keys of each column
            float x0 = fmaxf(fmaxf(S0[0], S0[2]), fmaxf(S1[0], S1[2])), x1 = fmaxf(fmaxf(S0[1], S0[3]), fmaxf(S1[1], S1[3]));
#pragma unroll
            for (int o = 4; o < 32; o <<= 1) {
                x0 = fmaxf(x0, __shfl_xor_sync(0xffffffffu, x0, o));
                x1 = fmaxf(x1, __shfl_xor_sync(0xffffffffu, x1, o));
            }
            x0 = fmaf(x0, f0, -P_LOG);
            x1 = fmaf(x1, f1, -P_LOG);
            uint32_t within = SIGNS;
            if constexpr (!F32) {
                const bool there = ((lane & 8 ? seen1 : seen0) >> (4 * (lane & 7) + (lane >> 4))) & 1u;
#pragma unroll
                for (int w = 0; w < NG / 2; ++w) {
                    top[w] = there ? __vmaxs2(top[w], 0u) : 0u;      // (negative, with codes of 0, where a group's low was rounded up past all its values)
                    within &= STEPS_LIMIT - factors[w] - top[w];
                }
            }
            if (__any_sync(0xffffffffu, x0 > m0 || x1 > m1 || within != SIGNS)) {
                if constexpr (!F32)
                    if (__any_sync(0xffffffffu, within != SIGNS)) {
#pragma unroll
                        for (int w = 0; w < NG / 2; ++w) {
#pragma unroll
                            for (int o = 1; o < 32; o <<= 1) top[w] = __vmaxs2(top[w], __shfl_xor_sync(0xffffffffu, top[w], o));
                            const uint32_t now = __vminu2(factors[w], factors_for(top[w]));
#pragma unroll
                            for (int g = 2 * w; g < 2 * w + 2; ++g) {
                                const float c = power_of_two(factor_exponent(now, g & 1) - factor_exponent(factors[w], g & 1));
#pragma unroll
                                for (int i = 0; i < 4; ++i) { O[2 * g][i] *= c; O[2 * g + 1][i] *= c; }
                            }
                            set_factor(w, now);
                        }
                        __syncwarp();
                    }
                const float n0 = fmaxf(m0, x0), n1 = fmaxf(m1, x1), c0 = exp2_fast(m0 - n0), c1 = exp2_fast(m1 - n1);
                m0 = n0;
                m1 = n1;
                l0 *= c0;
                l1 *= c1;
#pragma unroll
                for (int i = 0; i < 2 * NG; ++i) { O[i][0] *= c0; O[i][1] *= c1; O[i][2] *= c0; O[i][3] *= c1; }
                L[0] *= c0;
                L[1] *= c1;
#pragma unroll
                for (int i = 0; i < (F32 ? NG : 1); ++i) { W[i][0] *= c0; W[i][1] *= c1; }
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                S0[j] = exp2_fast(fmaf(S0[j], j & 1 ? f1 : f0, j & 1 ? -m1 : -m0));
                S1[j] = exp2_fast(fmaf(S1[j], j & 1 ? f1 : f0, j & 1 ? -m1 : -m0));
            }
            l0 += (S0[0] + S0[2]) + (S1[0] + S1[2]);
            l1 += (S0[1] + S0[3]) + (S1[1] + S1[3]);
            add_values(rows, S0, all, seen0);
            add_values(rows1, S1, all, seen1);
        }
        __syncwarp();
        int n = 0;
        if (lane == 0) asm volatile("atom.shared.acq_rel.cta.add.u32 %0, [%1], 1;" : "=r"(n) : "r"(left(slot)) : "memory");
        n = __shfl_sync(0xffffffffu, n, 0);
        if (n == tasks - 1 && unit + P.slots < n_units) {
            if (lane == 0) asm volatile("st.shared.u32 [%0], %1;" ::"r"(left(slot)), "r"(0) : "memory");
            __syncwarp();
            fetch(unit + P.slots, slot);
        }
        slot += P.subs;
        if (slot >= P.slots) {
            slot = sub;
            phase ^= 1u;
        }
    }
    __syncthreads();
    if (*abort_flag) {
        if (threadIdx.x == 0) pc_let_copies_land();
        return;
    }

    // ---- the parts of the keys that the CTA's warps took, merged in shared memory (the ring is done with)
    constexpr int PITCH = D + 4;
    float *parts = reinterpret_cast<float *>(smem + RING_AT);      // [warp][8][PITCH], then [warp][8] maxima, sums
    float *ms = parts + n_warps * ROWS * PITCH, *ls = ms + n_warps * ROWS;
    {
        uint32_t factors[NG / 2];
        if constexpr (!F32) lds(factors_at, factors);
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) {
            l0 += __shfl_xor_sync(0xffffffffu, l0, o);
            l1 += __shfl_xor_sync(0xffffffffu, l1, o);
        }
        if (row == 0) {
            ms[warp * ROWS + 2 * t] = m0;
            ms[warp * ROWS + 2 * t + 1] = m1;
            ls[warp * ROWS + 2 * t] = l0;
            ls[warp * ROWS + 2 * t + 1] = l1;
        }
        float *mine = parts + (warp * ROWS + 2 * t) * PITCH + 4 * row;
#pragma unroll
        for (int g = 0; g < NG; ++g) {
            float w0, w1;
            if constexpr (F32) {
                w0 = W[g][0];
                w1 = W[g][1];
#pragma unroll
                for (int o = 4; o < 32; o <<= 1) {
                    w0 += __shfl_xor_sync(0xffffffffu, w0, o);
                    w1 += __shfl_xor_sync(0xffffffffu, w1, o);
                }
            } else {
                w0 = __shfl_sync(0xffffffffu, L[0], (8 - NG + g) * 4 + t);
                w1 = __shfl_sync(0xffffffffu, L[1], (8 - NG + g) * 4 + t);
            }
            // the codes' powers of two and the steps' factor come off
            const float unit = F32 ? 1.f : power_of_two(15 - factor_exponent(factors[g / 2], g & 1));
            const float A = F32 ? 1.f : 16777216.f * unit, B = F32 ? 1.f : 1048576.f * unit;
            *reinterpret_cast<float4 *>(mine + g * Q4_GROUP) =
                make_float4(fmaf(O[2 * g][0], A, w0), fmaf(O[2 * g][2], B, w0), fmaf(O[2 * g + 1][0], A, w0), fmaf(O[2 * g + 1][2], B, w0));
            *reinterpret_cast<float4 *>(mine + PITCH + g * Q4_GROUP) =
                make_float4(fmaf(O[2 * g][1], A, w1), fmaf(O[2 * g][3], B, w1), fmaf(O[2 * g + 1][1], A, w1), fmaf(O[2 * g + 1][3], B, w1));
        }
    }
    __syncthreads();
    if (!works) return;
    // the warps of a task take its rows in turn
    const int rows_all = P.n_kv * P.n_rows, count = min(P.n_rows - block * ROWS, ROWS), step = P.subs * (32 / (D / 4));
    for (int r = sub * (32 / (D / 4)) + lane / (D / 4); r < count; r += step) {
        const int c = lane % (D / 4);
        float M = NO_MAX, l = 0.f;
        for (int b = 0; b < P.subs; ++b) M = fmaxf(M, ms[(b * tasks + task) * ROWS + r]);
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int b = 0; b < P.subs; ++b) {
            const int at = (b * tasks + task) * ROWS + r;
            const float f = exp2_fast(ms[at] - M);
            const float4 x = *reinterpret_cast<const float4 *>(parts + at * PITCH + 4 * c);
            l = fmaf(f, ls[at], l);
            o.x = fmaf(f, x.x, o.x);
            o.y = fmaf(f, x.y, o.y);
            o.z = fmaf(f, x.z, o.z);
            o.w = fmaf(f, x.w, o.w);
        }
        const size_t to = (size_t)blockIdx.x * rows_all + (size_t)(first_head + head) * P.n_rows + block * ROWS + r;
        reinterpret_cast<float4 *>(P.part_o)[to * (D / 4) + c] = o;
        if (c == 0) reinterpret_cast<float2 *>(P.part_ml)[to] = make_float2(M, l);
    }
}

// Parts of a row merged: a block per row, D / 4 lanes a part.  The parts' sums are fetched before their maxima are compared, eight at a time: it is latency
// (a launch, two fetches, a round through shared memory; 148 parts of 24 rows, 1.9 MB in L2: 5.1 us by itself, 160 rows 6.0).
constexpr int JOIN_THREADS = 512;
template <int D, bool F32> __global__ void __launch_bounds__(JOIN_THREADS) k_q4_join(const JoinParams J) {
    constexpr int LANES = D / 4, SETS = JOIN_THREADS / LANES, BATCH = 8;
    __shared__ float4 sums[SETS][LANES];
    __shared__ float2 mls[SETS];
    pc_grid_dep_launch();
    pc_grid_dep_wait();
    const int row = blockIdx.x, c = threadIdx.x % LANES, set = threadIdx.x / LANES;
    const float2 *ml = reinterpret_cast<const float2 *>(J.part_ml) + row;
    const float4 *po = reinterpret_cast<const float4 *>(J.part_o) + (size_t)row * LANES + c;
    float M = NO_MAX, l = 0.f;
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int s0 = set; s0 < J.splits; s0 += SETS * BATCH) {
        float4 x[BATCH];
        float2 y[BATCH];
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
            const int s = s0 + i * SETS;
            y[i] = make_float2(NO_MAX, 0.f);
            x[i] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (s < J.splits) {
                y[i] = __ldg(ml + (size_t)s * J.rows);
                x[i] = __ldg(po + (size_t)s * J.rows * LANES);
            }
        }
        float top = M;
#pragma unroll
        for (int i = 0; i < BATCH; ++i) top = fmaxf(top, y[i].x);
        const float f0 = exp2_fast(M - top);
        l *= f0;
        sum = make_float4(sum.x * f0, sum.y * f0, sum.z * f0, sum.w * f0);
        M = top;
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
            const float f = exp2_fast(y[i].x - top);
            l = fmaf(f, y[i].y, l);
            sum.x = fmaf(f, x[i].x, sum.x);
            sum.y = fmaf(f, x[i].y, sum.y);
            sum.z = fmaf(f, x[i].z, sum.z);
            sum.w = fmaf(f, x[i].w, sum.w);
        }
    }
    sums[set][c] = sum;
    if (c == 0) mls[set] = make_float2(M, l);
    __syncthreads();
    const int r = row % J.n_rows, h = row / J.n_rows * J.group + r % J.group;
    const size_t to = (size_t)(r / J.group) * J.n_q_heads + h;
    if (threadIdx.x >= LANES) return;
#pragma unroll
    for (int i = 0; i < SETS; ++i) M = fmaxf(M, mls[i].x);
    l = 0.f;
    sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int i = 0; i < SETS; ++i) {
        const float f = exp2_fast(mls[i].x - M);
        const float4 x = sums[i][c];
        l = fmaf(f, mls[i].y, l);
        sum.x = fmaf(f, x.x, sum.x);
        sum.y = fmaf(f, x.y, sum.y);
        sum.z = fmaf(f, x.z, sum.z);
        sum.w = fmaf(f, x.w, sum.w);
    }
    const float inv = l > 0.f ? 1.f / l : (l != l ? l : 0.f);          // no key left: 0; NaN stays
    if constexpr (F32) reinterpret_cast<float4 *>(J.out)[to * LANES + c] = make_float4(sum.x * inv, sum.y * inv, sum.z * inv, sum.w * inv);
    else reinterpret_cast<uint2 *>(J.out)[to * LANES + c] = make_uint2(pc_pack_bf16(sum.x * inv, sum.y * inv), pc_pack_bf16(sum.z * inv, sum.w * inv));
    if (c == 0) {
        const float lse2 = M + log2f(l);                                // base 2; -infinity where no key is left
        if (J.lse_rows) J.lse_rows[row] = lse2;
        if (J.lse) J.lse[to] = lse2 * 0.6931471805599453f;
    }
}

// weight_j <- decay weight_j + gain sum over rows of 2^(logit - lse): LANES lanes a token, which take its rows in turn.  The logits were just written and come
// from L2: 24,192 tokens x 24 rows (2.3 MB) 4.5 us, 4,999 x 160 4.6, launches for the most part.
constexpr int WEIGH_THREADS = 256;
template <int LANES> __global__ void __launch_bounds__(WEIGH_THREADS) k_q4_weigh(const float *__restrict__ logits, const float *__restrict__ lse, int n, int rows,
                                                                                 float decay, float gain, float *__restrict__ weight) {
    pc_grid_dep_launch();
    const int lane = threadIdx.x % LANES, j = (int)(((long long)blockIdx.x * WEIGH_THREADS + threadIdx.x) / LANES);
    pc_grid_dep_wait();
    float sum = 0.f;
    if (j < n)
#pragma unroll 4
        for (int r = lane; r < rows; r += LANES) {
            const float z = __ldg(lse + r);
            sum += z == -INFINITY ? 0.f : exp2_fast(__ldg(logits + (size_t)j * rows + r) - z);
        }
#pragma unroll
    for (int o = 1; o < LANES; o <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (j < n && lane == 0) weight[j] = fmaf(decay, weight[j], gain * sum);
}

__global__ void __launch_bounds__(256) k_accumulate(const float *__restrict__ mass, int n, float decay, float gain, float *__restrict__ weight) {
    pc_grid_dep_launch();
    pc_grid_dep_wait();
    const int j = blockIdx.x * 256 + threadIdx.x;
    if (j < n) weight[j] = fmaf(decay, weight[j], gain * mass[j]);
}

int div_up(int a, int b) { return (a + b - 1) / b; }

// Rows as bytes, boxes of 32 tokens x 128 bytes; what lies outside reads as zero.  whole: as [128-byte piece][token][128] with all pieces of 32 tokens as
// one box.
bool make_row_map(CUtensorMap *m, const void *rows, uint64_t n, uint64_t row_bytes, bool whole) {
    const pc_tc::EncodeTiledFn fn = pc_tc::encode_fn();
    if (!fn) return false;
    const cuuint64_t dims[3] = {whole ? BOX : row_bytes, n, row_bytes / BOX}, strides[2] = {row_bytes, BOX};
    const cuuint32_t box[3] = {BOX, UNIT * Q4_STEP, (cuuint32_t)(row_bytes / BOX)}, estr[3] = {1, 1, 1};
    return fn(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, whole ? 3 : 2, const_cast<void *>(rows), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Queries i0 .. i0 + n_q - 1 through the kernels above
pc_status attend_rows(pc_q4 *w, const pc_q4_cache *cache, const uint8_t *valid, const void *q, const int32_t *q_pos, int n_q, void *out,
                      float *lse, const pc_q4_weigh *weigh, float gain, cudaStream_t stream) {
    pc_ctx *ctx = w->ctx;
    const pc_layer_desc &D = ctx->desc;
    Q4Params P{};
    const pc_q4_segment *segs[2] = {&cache->anchors, &cache->history};
    // KV heads of a CTA (up to eight, shared out evenly) and blocks of query rows: of one, two or four times as few heads that with which the CTAs of
    // a piece of the keys have the fewest warps' places in all, so that few stay empty (five queries of 32 / 8 heads are three blocks: 2 x 16 places
    // with eight heads a CTA, 2 x 12 with four).  Warps left over take further parts of the keys.
    P.n_rows = n_q * ctx->group;
    const int n_blocks = div_up(P.n_rows, ROWS);
    int head_sets = 0, block_groups = 0, places = 0;
    for (int fewer = 1; fewer <= 4; fewer *= 2) {
        const int sets = div_up(D.n_kv_heads, 8) * fewer, heads = div_up(D.n_kv_heads, sets);
        if (sets > D.n_kv_heads) break;
        const int groups = div_up(n_blocks, MAX_WARPS / heads), blocks = div_up(n_blocks, groups);
        if (places && sets * heads * groups * blocks >= places) continue;
        places = sets * heads * groups * blocks;
        head_sets = sets;
        block_groups = groups;
        P.heads = heads;
        P.blocks = blocks;
    }
    CUtensorMap maps[2];
    // one set of heads, and sections of whole boxes (4 or 8 KV heads of 128 channels, 8 of 64)
    P.whole_rows = head_sets == 1 && D.n_kv_heads * D.head_dim / 4 % BOX == 0;
    for (int i = 0; i < 2; ++i) {
        P.n[i] = segs[i]->n_tokens;
        P.shift[i] = segs[i]->t_shift;
        const pc_q4_segment *s = P.n[i] > 0 ? segs[i] : segs[1 - i];          // an empty segment is never asked for
        if (!make_row_map(&maps[i], s->rows, (uint64_t)s->n_tokens, q4_row(D), P.whole_rows)) {
            fprintf(stderr, "packcache: cuTensorMapEncodeTiled failed\n");
            return PC_ERR_CUDA;
        }
    }
    P.valid = valid;
    P.q = q;
    P.q_pos = q_pos;
    P.n_q = n_q;
    P.n_q_heads = D.n_q_heads;
    P.n_kv = D.n_kv_heads;
    P.group = ctx->group;
    P.inv_tasks = 65536u / (P.heads * P.blocks) + 1;
    P.inv_heads = 65536u / P.heads + 1;
    P.inv_group = 1.f / (float)P.group;
    P.boxes_k = div_up(P.heads * D.head_dim / 2, BOX);
    P.boxes = 2 * P.boxes_k + div_up(P.heads * D.head_dim / 4, BOX);
    P.unit_bytes = P.boxes * BOX_BYTES;
    const bool fold = P.n_rows <= 4;
    const int query_area = P.heads * P.blocks * query_bytes(D.head_dim, fold);
    P.slots = std::min(MAX_SLOTS, (SMEM_MOST - 1024 - RING_AT - query_area) / P.unit_bytes);         // three of 40 KB at least
    P.subs = std::min(MAX_WARPS / (P.heads * P.blocks), P.slots / 2);
    P.slots -= P.slots % P.subs;
    P.queries_at = RING_AT + P.slots * P.unit_bytes;
    const int n_warps = P.heads * P.blocks * P.subs, merge_bytes = n_warps * ROWS * (D.head_dim + 4 + 2) * (int)sizeof(float);
    const size_t smem = 1024 + std::max(P.queries_at + query_area, RING_AT + merge_bytes);
    P.scale = pc_q_rot_scale(D.head_dim);
    P.status = ctx->status;
    P.wait_us = ctx->wait_limit_us;
    P.extra_tx = ctx->test_extra_tx;
    P.part_o = w->part_o;
    P.part_ml = w->part_ml;
    P.logits = weigh && P.n[1] > 0 ? w->logits : nullptr;
    // Parts of the keys: with ctas * parts CTAs in up to four waves over the SMs, the count that ends first, a CTA's start and end taken as the time
    // of eight steps.  Anchors and history have CTAs of their own, with the same number of steps, or fewer where they do not divide.
    const int rows = P.n_kv * P.n_rows, ctas = head_sets * block_groups;
    const int s0 = div_up(P.n[0], Q4_STEP), s1 = div_up(P.n[1], Q4_STEP), least = (s0 > 0) + (s1 > 0);
    int splits = 0;
    long long best = -1;
    for (int wave = 1; wave <= 4; ++wave) {
        const int want = std::max(least, std::min<int>(wave * ctx->sm_count / ctas, (int)(w->part_rows / rows)));
        int per = std::max(P.subs, div_up(s0 + s1, want));
        while (div_up(s0, per) + div_up(s1, per) > want) ++per;
        const int n = div_up(s0, per) + div_up(s1, per);
        const long long cost = (long long)div_up(ctas * n, ctx->sm_count) * (div_up(per, P.subs * UNIT) * UNIT + 8);
        if (best >= 0 && cost >= best) continue;
        best = cost;
        splits = n;
        P.ctas0 = div_up(s0, per);
    }
    for (int i = 0; i < 2; ++i) {
        const int n = i ? splits - P.ctas0 : P.ctas0, s = i ? s1 : s0;
        if (n == 0) continue;
        P.steps[i] = s / n;
        P.more[i] = s % n;
    }
    const bool f32 = D.dtype == PC_F32;
    const dim3 grid(splits, block_groups, head_sets), block(n_warps * 32);
    static bool attr_set[PC_MAX_DEVICES] = {};
    if (ctx->device < 0 || ctx->device >= PC_MAX_DEVICES) return PC_ERR_UNSUPPORTED;
    if (!attr_set[ctx->device]) {
        for (const auto kernel : {k_q4_attend<128, false, false>, k_q4_attend<128, false, true>, k_q4_attend<128, true, false>, k_q4_attend<128, true, true>,
                                  k_q4_attend<64, false, false>, k_q4_attend<64, false, true>, k_q4_attend<64, true, false>, k_q4_attend<64, true, true>})
            PC_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM_MOST));
        attr_set[ctx->device] = true;
    }
    const auto kernel = D.head_dim == 128 ? (f32 ? (fold ? k_q4_attend<128, true, true> : k_q4_attend<128, true, false>)
                                                 : (fold ? k_q4_attend<128, false, true> : k_q4_attend<128, false, false>))
                                          : (f32 ? (fold ? k_q4_attend<64, true, true> : k_q4_attend<64, true, false>)
                                                 : (fold ? k_q4_attend<64, false, true> : k_q4_attend<64, false, false>));
    PC_LAUNCH(kernel, grid, block, smem, stream, maps[0], maps[1], P, ctx->rope);
    JoinParams J{w->part_o, w->part_ml, splits, rows, P.n_rows, P.group, P.n_q_heads, out, lse, P.logits ? w->lse : nullptr};
    if (D.head_dim == 128 && f32) PC_LAUNCH((k_q4_join<128, true>), dim3(rows), dim3(JOIN_THREADS), 0, stream, J);
    else if (D.head_dim == 128) PC_LAUNCH((k_q4_join<128, false>), dim3(rows), dim3(JOIN_THREADS), 0, stream, J);
    else if (f32) PC_LAUNCH((k_q4_join<64, true>), dim3(rows), dim3(JOIN_THREADS), 0, stream, J);
    else PC_LAUNCH((k_q4_join<64, false>), dim3(rows), dim3(JOIN_THREADS), 0, stream, J);
    if (P.logits) {
        const auto weigh_with = [&](auto kernel, int lanes) -> pc_status {
            PC_LAUNCH(kernel, dim3((unsigned)(((long long)P.n[1] * lanes + WEIGH_THREADS - 1) / WEIGH_THREADS)), dim3(WEIGH_THREADS), 0, stream,
                      w->logits, w->lse, P.n[1], rows, weigh->decay, gain, cache->history.weight);
            return PC_OK;
        };
        // 8 / 32 lanes, us a whole call over 12,196 keys: 8 rows 14.5 / 15.2, 24 15.8 / 16.5, 48 19.3 / 20.1, 72 25.5 / 26.7, 144 32.6 / 32.6
        return rows <= 96 ? weigh_with(k_q4_weigh<8>, 8) : weigh_with(k_q4_weigh<32>, 32);
    }
    return PC_OK;
}

// The whole cache in fp16, then the tensor-core attention kernel
pc_status attend_frame(pc_q4 *w, const pc_q4_cache *cache, const void *q, const int32_t *q_pos, int n_q, void *out, float *lse, cudaStream_t stream) {
    pc_ctx *ctx = w->ctx;
    const size_t row = (size_t)ctx->desc.n_kv_heads * ctx->desc.head_dim * sizeof(__nv_bfloat16);
    ctx->prepared_n_seg = 0;                       // the rotated-key scratch is about to be overwritten
    ctx->anchor_rot_n = 0;
    ctx->last_n_q = 0;
    const pc_q4_segment *segs[2];
    void *k16[2], *v16[2];
    int seg_n[2], n_seg = 0;
    size_t at = 0;                                 // rows; segments start on tile boundaries
    for (const pc_q4_segment *s : {&cache->anchors, &cache->history}) {
        if (s->n_tokens == 0) continue;
        segs[n_seg] = s;
        k16[n_seg] = static_cast<char *>(ctx->k_rot) + at * row;
        v16[n_seg] = static_cast<char *>(w->v) + at * row;
        seg_n[n_seg++] = s->n_tokens;
        at += (size_t)div_up(s->n_tokens, 128) * 128;
    }
    const int lo_row0 = div_up(n_q, 128) * 128;
    const pc_status st = pc_q4_launch_front(ctx, segs, n_seg, k16, v16, q, q_pos, n_q, w->q16, lo_row0, stream);
    return st != PC_OK ? st : pc_launch_attend_fine(ctx, n_seg, seg_n, ctx->k_rot, v16, w->q16, lo_row0, n_q, out, lse, stream);
}

}  // namespace

extern "C" pc_status pc_q4_create(pc_ctx *ctx, int32_t max_tokens, int32_t parts, pc_q4 **out) {
    if (!ctx || !out) return PC_ERR_INVALID_ARG;
    *out = nullptr;
    if (max_tokens <= 0 || (parts & ~(PC_Q4_FRAMES | PC_Q4_WEIGH))) return PC_ERR_INVALID_ARG;
    pc_q4 *w = new (std::nothrow) pc_q4();
    if (!w) return PC_ERR_CUDA;
    w->ctx = ctx;
    w->max_tokens = max_tokens;
    w->parts = parts;
    const pc_layer_desc &D = ctx->desc;
    // every row of the largest call in two parts (anchors and history), and what two CTAs an SM leave in any split
    w->part_rows = std::max((size_t)2 * D.max_q * D.n_q_heads, (size_t)2 * ctx->sm_count * MAX_WARPS * ROWS);
    const auto fill = [&]() -> pc_status {
        PC_CUDA_TRY(cudaMalloc(&w->part_o, w->part_rows * D.head_dim * sizeof(float)));
        PC_CUDA_TRY(cudaMalloc(&w->part_ml, w->part_rows * 2 * sizeof(float)));
        PC_CUDA_TRY(cudaMalloc(&w->lse, (size_t)D.max_q * D.n_q_heads * sizeof(float)));
        if (parts & PC_Q4_WEIGH) {
            // a call's queries go in passes that fit: one at least, up to 64 MB (half of L2) of logits
            const size_t one = (size_t)max_tokens * D.n_q_heads;
            w->logit_floats = std::max(one, std::min(one * (size_t)D.max_q, (size_t)16 << 20));
            PC_CUDA_TRY(cudaMalloc(&w->logits, w->logit_floats * sizeof(float)));
        }
        if ((parts & PC_Q4_FRAMES) && pc_tensor_core_shape(ctx)) {
            w->v_rows = (size_t)(div_up(max_tokens, 128) + 1) * 128;
            PC_CUDA_TRY(cudaMalloc(&w->v, w->v_rows * D.n_kv_heads * D.head_dim * sizeof(__half)));
            PC_CUDA_TRY(cudaMalloc(&w->q16, ((size_t)div_up(D.max_q, 128) * 128 + D.max_q) * D.n_q_heads * D.head_dim * sizeof(__half)));
        }
        return PC_OK;
    };
    const pc_status st = fill();
    if (st != PC_OK) {
        pc_q4_destroy(w);
        return st;
    }
    *out = w;
    return PC_OK;
}

extern "C" pc_status pc_q4_destroy(pc_q4 *w) {
    if (!w) return PC_ERR_INVALID_ARG;
    cudaFree(w->part_o);
    cudaFree(w->part_ml);
    cudaFree(w->lse);
    cudaFree(w->logits);
    cudaFree(w->v);
    cudaFree(w->q16);
    delete w;
    return PC_OK;
}

extern "C" pc_status pc_q4_attend(pc_q4 *w, const pc_q4_cache *cache, const uint8_t *valid, const void *q, const int32_t *q_pos, int32_t n_q,
                                  void *out, float *lse, const pc_q4_weigh *weigh, void *stream_) {
    if (!w || !cache) return PC_ERR_INVALID_ARG;
    pc_ctx *ctx = w->ctx;
    const pc_layer_desc &D = ctx->desc;
    if (!q || !q_pos || !out || n_q <= 0) return PC_ERR_INVALID_ARG;
    if (!pc_aligned16(q) || !pc_aligned16(q_pos) || !pc_aligned16(out) || (lse && !pc_aligned16(lse))) return PC_ERR_INVALID_ARG;
    if (n_q > D.max_q) return PC_ERR_CAPACITY;
    for (const pc_q4_segment *s : {&cache->anchors, &cache->history}) {
        const pc_status st = q4_check_segment(s, true);
        if (st != PC_OK) return st;
    }
    const int64_t keys = (int64_t)cache->anchors.n_tokens + cache->history.n_tokens;
    if (keys == 0) return PC_ERR_INVALID_ARG;
    if (keys > w->max_tokens) return PC_ERR_CAPACITY;
    if (weigh && (!(w->parts & PC_Q4_WEIGH) || (!cache->history.weight && cache->history.n_tokens > 0))) return PC_ERR_INVALID_ARG;
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    // Many query rows of a KV head: the pass that turns the cache into 16 bits is paid once for all, and the tensor-core kernel's tiles of 128 rows are filled.
    // Frame route / kernels of few queries, us: 24 / 8 heads over 9,200 tokens 72 rows 42 / 40, 96 42 / 47, 126 42 / 59; over 25,328 72 97 / 80, 96 97 / 94,
    // 126 98 / 116; 8 / 8 heads 64 rows 40 / 37 and 96 / 66, 100 39 / 51 and 95 / 100; over 537 tokens 24 rows 16 / 17, 96 17 / 24, 12 15 / 16.
    // (By rows alone: what turning the cache into 16 bits costs grows with its keys and KV heads, so over 25,328 keys the rule is 3 % off at 96 rows.)
    // With a mask or weights frames take the kernels of few queries as well: 1,008 queries over 9,200 tokens 1.55 ms masked, 1.7 weighed, where 0.14 to 0.16 is
    // the frame route's; 48,512 tokens 7.7 and 9.7 against 0.71.
    const size_t tile_rows = (size_t)(div_up(cache->anchors.n_tokens, 128) + div_up(cache->history.n_tokens, 128)) * 128;
    const int many = keys <= 1024 ? 24 : 96;
    if (n_q * ctx->group >= many && !valid && !weigh && w->v && ctx->attend_impl != 1 && tile_rows <= w->v_rows && tile_rows <= ctx->k_rot_rows)
        return attend_frame(w, cache, q, q_pos, n_q, out, lse, stream);
    int pass = n_q;
    if (weigh && cache->history.n_tokens > 0) {
        const size_t fit = w->logit_floats / ((size_t)cache->history.n_tokens * D.n_q_heads);
        const int passes = div_up(n_q, (int)std::min<size_t>(fit, n_q));
        pass = div_up(n_q, passes);
    }
    const size_t row = (size_t)D.n_q_heads * D.head_dim * ctx->elem_size;
    pc_q4_weigh now{};
    if (weigh) now = *weigh;
    for (int i = 0; i < n_q; i += pass) {
        const int n = std::min(pass, n_q - i);
        const pc_status st = attend_rows(w, cache, valid, static_cast<const char *>(q) + i * row, q_pos + (size_t)i * 4, n, static_cast<char *>(out) + i * row,
                                         lse ? lse + (size_t)i * D.n_q_heads : nullptr, weigh ? &now : nullptr,
                                         now.gain / ((float)n_q * D.n_q_heads), stream);
        if (st != PC_OK) return st;
        now.decay = 1.f;                           // the first pass has taken it
    }
    return PC_OK;
}

extern "C" pc_status pc_accumulate(pc_ctx *ctx, const float *mass, int32_t n, float decay, float gain, float *weight, void *stream_) {
    if (!ctx || n < 0 || (n > 0 && (!mass || !weight))) return PC_ERR_INVALID_ARG;
    if ((reinterpret_cast<uintptr_t>(mass) | reinterpret_cast<uintptr_t>(weight)) & 3u) return PC_ERR_INVALID_ARG;
    cudaStream_t stream = static_cast<cudaStream_t>(stream_);
    if (n > 0) PC_LAUNCH(k_accumulate, dim3(div_up(n, 256)), dim3(256), 0, stream, mass, n, decay, gain, weight);
    return PC_OK;
}
