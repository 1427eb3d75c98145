// Attention over a paged cache on tcgen05 tensor cores (bf16): prompts, their pieces and frames, and a prefix that many rows share.
//
// Two launches.  k_paged_front rotates the queries, with log2(e) / sqrt(d) folded in, into rows of KV head x (token, head of the group): rows that share keys and values lie side by side,
// so a tile of 128 rows is full whatever the group's size, and a causal tile of G heads spans 128 / G tokens only.
// k_paged_tc: an item is (sequence, pair of such tiles, KV head); its key tiles lie on one line with those of all other items, which the CTAs (one an SM) share evenly.  Where the line is cut follows from
// lengths that lie on the device: every CTA adds them up for itself.  An item that several CTAs share is added up by the last of them, in the order of the keys.
// A CTA: warp 0 walks the line, tells the others of its units by way of a ring of four in shared memory, and fetches by TMA, a lane a page's box (a tile of 128 keys is 1 to 8 pages), two stages of keys and
// of values; warps 1 and 2 issue S = Q_t K^T of the two query tiles, warp 3 O_t += P_t V; warps 4-7 and 8-11 are the softmax of tile 0 and 1: the score row in registers, running
// maximum and sum in fp32, probabilities as bf16 into tensor memory in two halves, O rescaled only where the maximum grew by more than 2^8.  (The division of labour is that of the frame kernel, k_attend_tc.)
// Rows behind a segment's end: scores are replaced by -infinity whatever they are, and the values' rows are cleared in shared memory, since 0 times what lies
// there may be NaN.
// Tried: queries rotated in this kernel, by four warps more, into three places in turn.  Their chains of shuffles, addresses and products are 1,000 instructions a tile at five to ten cycles, 7 us, where
// a unit of three key tiles takes 4.6: packed prompts 227 us a call instead of 89.
#include <algorithm>

#include "pc_paged_host.cuh"
#include "pc_tc.cuh"

namespace {

using namespace pc_tc;

constexpr int TC_THREADS = 384;
constexpr int REGS_LAUNCH = 65536 / TC_THREADS / 8 * 8, REGS_ISSUE = 72, REGS_SOFTMAX = 216;
static_assert(128 * REGS_ISSUE + 256 * REGS_SOFTMAX <= TC_THREADS * REGS_LAUNCH, "more registers than the block has");
constexpr float GROW = 8.f;
constexpr int PAIR = 2 * TILE;                     // packed rows of an item
constexpr int GAP = 2;                             // what crossing into the next item costs, in key tiles: so many empty places lie behind each item on the line
constexpr int UNITS = 4;                           // units that are told ahead

// What a CTA does of an item, and what its warps need to know of that
struct Unit {
    int r0;                  // the sequence's first row in the batch
    int p0, rows;            // first of the pair's packed rows in the sequence, and how many
    int before, own;         // own tokens before the sequence's rows, and in all
    int j0, nj;              // key tiles: those of the prefix first; nj 0: no more units
    int h;
    int c0, parts, part;     // first CTA of the item, CTAs of it, which of them this is
    int pad;
};
static_assert(sizeof(Unit) == 48, "three 16-byte pieces");

template <int D> struct Map {
    static constexpr int HALVES = D / 64, TILE_B = HALVES * HALF_BYTES;
    static constexpr int Q = 0, K = Q + 2 * TILE_B, V = K + 2 * TILE_B, BAR = V + 2 * TILE_B, FLAGS = BAR + 256, UNIT = FLAGS + 64, ALLOC = UNIT + UNITS * 48 + 1024;
    static constexpr int SEQS = 0, ENDS = PC_MAX_SEQS * 16;       // while the line is made, where the queries will be: a sequence's numbers, the line's place behind it
    static_assert(ALLOC <= 232448 && ENDS + PC_MAX_SEQS * 8 <= 2 * TILE_B, "shared memory");
};
enum { BAR_Q = 0 /* [tile] */, BAR_QFREE = 2 /* [tile] */, BAR_K0 = 4, BAR_KV = 5 /* [stage]: values of a step and keys of the next */, BAR_EMPTY = 7 /* [step & 1] */, BAR_SFULL = 9 /* [tile] */,
       BAR_SFREE = 11 /* [tile] */, BAR_PHALF = 13 /* [tile][half] */, BAR_PVDONE = 17 /* [tile] */, BAR_DONE = 19, BAR_UF = 20 /* [unit & 3]: told */, BAR_UE = 24 /* [unit & 3]: taken by all */, N_BARS = 28 };
static_assert(N_BARS * 8 <= 256, "barriers");
constexpr int UNIT_READERS = 11;                   // warps 1 to 11
constexpr int TM_S = 0, TM_P = TILE, TM_O = 2 * TILE;

struct TcParams {
    PagedBatch B;
    int n_q_heads, n_kv, group;
    int head_rows;           // rows of a KV head among the rotated queries
    int shared;              // the prefix alone, rows of all sequences; what comes out goes to scratch row by row for k_paged_join
    __nv_bfloat16 *out;
    float *lse;
    float *part_o;           // [2 CTAs][tile][128][D]: a CTA's first and last item
    float2 *part_ml;
    float *home_o;           // shared: items of one CTA, [rows][query heads][D]
    float2 *home_ml;
    uint32_t *sync;          // [0] number of the call, [1] CTAs that are done, then [CTA][tile][warp] tickets: number of the call and parts that have come
    uint32_t wait_us, extra_tx;
};
constexpr int SYNC_HEAD = 2;

constexpr int FRONT_THREADS = 256;

struct FrontParams {
    PagedBatch B;
    const char *q;
    const int32_t *q_pos;
    char *q_rot;
    int chunks, group, n_kv, d;
    long long head_rows;
    float scale;
};

__global__ void __launch_bounds__(FRONT_THREADS) k_paged_front(const __grid_constant__ FrontParams P, const __grid_constant__ pc_rope_dev rope) {
    pc_grid_dep_wait();
    pc_grid_dep_launch();              // behind the wait: what came before is complete when the attention kernel starts, which looks at lengths and tables ahead of its own
    // a warp a row of the batch, lane's chunks of eight channels 32 apart: all at one place of a head
    const int lane = threadIdx.x & 31, row = (int)((blockIdx.x * FRONT_THREADS + threadIdx.x) >> 5);
    if (row >= paged_rows(P.B)) return;
    const int4 pos = __ldcg(reinterpret_cast<const int4 *>(P.q_pos) + row);
    const char *q = P.q + (size_t)row * P.chunks * 16;
    constexpr int CPL = 8;
    float2 cs[4];
    bool bad = false;
    for (int c0 = 0; c0 < P.chunks; c0 += CPL * 32) {
        uint4 v[CPL];
#pragma unroll
        for (int i = 0; i < CPL; ++i) {
            const int c = c0 + i * 32 + lane;
            if (c < P.chunks) v[i] = __ldcg(reinterpret_cast<const uint4 *>(q) + c);
        }
        if (c0 == 0) {
#pragma unroll
            for (int u = 0; u < 4; ++u) cs[u] = pc_rope_cs_clamped(rope, ((lane * 8) % P.d) / 2 + u, pos.x, pos.y, pos.z, bad);
        }
#pragma unroll
        for (int i = 0; i < CPL; ++i) {
            const int c = c0 + i * 32 + lane;
            if (c >= P.chunks) break;
            const uint32_t w[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
            uint32_t o[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const float2 y = pc_rotate(pc_bf16_lo(w[u]), pc_bf16_hi(w[u]), cs[u]);
                o[u] = pc_pack_bf16(__fmul_rn(y.x, P.scale), __fmul_rn(y.y, P.scale));
            }
            const int head = c * 8 / P.d, h = head / P.group, g = head - h * P.group;
            const size_t to = ((size_t)h * P.head_rows + (size_t)row * P.group + g) * P.d + c * 8 % P.d;
            *reinterpret_cast<uint4 *>(P.q_rot + to * 2) = make_uint4(o[0], o[1], o[2], o[3]);
        }
    }
    if (bad) pc_flag(P.B.status, PC_ERR_INVALID_ARG, PC_WHERE_PAGED_POS);
}

__device__ __forceinline__ int tiles_of(int keys) { return (keys + TILE - 1) / TILE; }
// Key tiles of a pair: up to the last key that one of its rows sees, one at least
__device__ __forceinline__ int pair_tiles(const TcParams &P, int n, int len, int pair) {
    if (P.shared) return max(1, tiles_of(P.B.n_prefix));
    const int last = (min((pair + 1) * PAIR, n * P.group) - 1) / P.group;
    const int sees = P.B.causal ? min(len, max(0, len - n + last + 1)) : len;
    return max(1, tiles_of(P.B.n_prefix) + tiles_of(sees));
}
__device__ __forceinline__ long long cta_cut(long long total, int ctas, int c) { return total * min(c, ctas) / ctas; }

__device__ __forceinline__ void arrive_if(bool who, uint32_t bar) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %1, 0;\n\t@p mbarrier.arrive.shared::cta.b64 _, [%0];\n\t}" ::"r"(bar), "r"((uint32_t)who) : "memory");
}
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, volatile int *abort_flag, int32_t *status, uint32_t limit_us) {
    if (__builtin_expect(__all_sync(0xffffffffu, pc_mbar_try(bar, parity)), 1)) return true;
    return __all_sync(0xffffffffu, pc_mbar_wait(bar, parity, abort_flag, status, PC_WHERE_PAGED_WAIT, limit_us));
}

template <int D>
__global__ void __launch_bounds__(TC_THREADS, 1)
k_paged_tc(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, const __grid_constant__ TcParams P) {
    using M = Map<D>;
    constexpr uint32_t QK = IDESC_QK, PV = (IDESC_PV & ~(0x3Fu << 17)) | ((D >> 3) << 17);
    pc_grid_dep_launch();
    extern __shared__ uint8_t smem_raw[];
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    uint8_t *gen = smem_raw + (base - smem_u32(smem_raw));
    volatile int *abort_flag = reinterpret_cast<volatile int *>(gen + M::FLAGS);
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(gen + M::FLAGS + 4);
    int4 *told = reinterpret_cast<int4 *>(gen + M::UNIT);
    const uint32_t bar0 = base + M::BAR;
    auto bar = [&](int i) { return bar0 + 8u * i; };
    const int warp = __shfl_sync(0xffffffffu, (int)threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int i = 0; i < N_BARS; ++i) {
            const bool by_warps = (i >= BAR_QFREE && i < BAR_K0) || (i >= BAR_EMPTY && i < BAR_SFULL) || (i >= BAR_SFREE && i < BAR_PVDONE);        // of the four of one tile's softmax
            mbar_init(bar(i), by_warps ? 4 : (i == BAR_DONE ? 3 : (i >= BAR_UE ? UNIT_READERS : 1)));
        }
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 2) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(tmem_slot)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    const PagedBatch &B = P.B;
    const int prefix_tiles = tiles_of(B.n_prefix);

    // ---- the line (of what was there before the rotation began, so ahead of the wait for that): every sequence's places, then where this CTA's run begins
    int4 *seqs = reinterpret_cast<int4 *>(gen + M::SEQS);
    long long *ends = reinterpret_cast<long long *>(gen + M::ENDS);
    const int n_seqs = P.shared ? 1 : B.n_seqs;
    for (int s = threadIdx.x; s < n_seqs; s += TC_THREADS) {
        PagedSeq S = {0, 0, 0};
        if (P.shared) S.n = paged_rows(B); else S = paged_seq(B, s);
        seqs[s] = make_int4(S.r0, S.n, S.len, 0);
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    for (int s = warp; s < n_seqs; s += TC_THREADS / 32) {
        const int4 S = seqs[s];
        const int pairs = (S.y * P.group + PAIR - 1) / PAIR;
        long long v = 0;
        for (int i = lane; i < pairs; i += 32) v += pair_tiles(P, S.y, S.z, i) + GAP;
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
        if (lane == 0) ends[s] = v * P.n_kv;
    }
    __syncthreads();
    // warp 0's walk: sequence, pair, KV head, places of the item that lie behind; places left of the run
    struct { int s, r0, n, len, pair, h, off, tiles, ctas; long long left, item, total; } W{};
    if (warp == 0) {
        const auto scan = [&](long long v) {
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const long long u = __shfl_up_sync(0xffffffffu, v, o);
                if (lane >= o) v += u;
            }
            return v;
        };
        long long total = 0;
        for (int s0 = 0; s0 < n_seqs; s0 += 32) {
            const long long v = scan(s0 + lane < n_seqs ? ends[s0 + lane] : 0) + total;
            if (s0 + lane < n_seqs) ends[s0 + lane] = v;
            total = __shfl_sync(0xffffffffu, v, 31);
        }
        __syncwarp();
        W.total = total;
        W.ctas = paged_tc_ctas(total, gridDim.x);
        const long long g0 = cta_cut(total, W.ctas, blockIdx.x);
        W.left = cta_cut(total, W.ctas, blockIdx.x + 1) - g0;
        if (W.left > 0) {
            for (int s0 = 0;; s0 += 32) {
                const unsigned later = __ballot_sync(0xffffffffu, s0 + lane >= n_seqs || ends[s0 + lane] > g0);
                if (later) {
                    W.s = s0 + __ffs(later) - 1;
                    break;
                }
            }
            const int4 S = seqs[W.s];
            W.r0 = S.x;
            W.n = S.y;
            W.len = S.z;
            long long rest = g0 - (W.s > 0 ? ends[W.s - 1] : 0);
            const int pairs = (W.n * P.group + PAIR - 1) / PAIR;
            for (int i0 = 0;; i0 += 32) {
                const int t = i0 + lane < pairs ? pair_tiles(P, W.n, W.len, i0 + lane) + GAP : 0;
                const long long v = scan((long long)t * P.n_kv);
                const unsigned later = __ballot_sync(0xffffffffu, i0 + lane >= pairs || v > rest);
                if (later) {
                    const int i = __ffs(later) - 1;
                    rest -= __shfl_sync(0xffffffffu, v - (long long)t * P.n_kv, i);
                    W.pair = i0 + i;
                    W.tiles = __shfl_sync(0xffffffffu, t, i) - GAP;
                    break;
                }
                rest -= __shfl_sync(0xffffffffu, v, 31);
            }
            W.h = (int)(rest / (W.tiles + GAP));
            W.off = (int)(rest - (long long)W.h * (W.tiles + GAP));
            W.item = g0 - W.off;
        }
    }
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");          // the scratch is the queries' from here on
    __syncthreads();

    // Steps are counted through all units (gs), units by un.  A warp's look at unit un:
    const auto look = [&](int un, bool &alive) {
        alive = warp_wait(bar(BAR_UF + (un & (UNITS - 1))), (un / UNITS) & 1, abort_flag, B.status, P.wait_us);
        const int4 *u = told + 3 * (un & (UNITS - 1));
        const int4 a = u[0], b = u[1], c = u[2];
        __syncwarp();
        arrive_if(lane == 0 && alive, bar(BAR_UE + (un & (UNITS - 1))));
        return Unit{a.x, a.y, a.z, a.w, b.x, alive ? b.y : 0, alive ? b.z : 0, b.w, c.x, c.y, c.z, c.w};
    };
    if (warp == 0) {
        // ---------------------------------------------------------------- the walk and the TMA producer: all lanes
        reg_dealloc<REGS_ISSUE>();
        bool alive = true;
        int un = 0;
        // The next unit is told to the others, and its first tile is this warp's next
        int j = 0, j_end = 0, uh = 0, us = 0, uown = 0, uq = 0, urows = 0;
        const auto next_unit = [&]() {
            Unit U{};
            while (W.left > 0) {
                const int all = W.tiles + GAP, take = (int)min((long long)(all - W.off), W.left);
                U.j0 = W.off;
                U.nj = min(W.tiles, W.off + take) - W.off;
                if (U.nj > 0) {
                    U.r0 = W.r0;
                    U.p0 = W.pair * PAIR;
                    U.rows = min(PAIR, W.n * P.group - U.p0);
                    U.before = W.len - W.n;
                    U.own = W.len;
                    U.h = W.h;
                    U.c0 = blockIdx.x;
                    U.parts = 1;
                    if (W.off > 0 || U.nj < W.tiles) {
                        U.c0 = paged_tc_cta(W.total, W.ctas, W.item);
                        U.parts = paged_tc_cta(W.total, W.ctas, W.item + W.tiles - 1) - U.c0 + 1;
                    }
                    U.part = blockIdx.x - U.c0;
                    us = W.s;
                }
                W.left -= take;
                W.off += take;
                if (W.off == all) {                           // the next item
                    W.off = 0;
                    W.item += all;
                    if (++W.h == P.n_kv) {
                        W.h = 0;
                        ++W.pair;
                        if (W.pair * PAIR >= W.n * P.group) {
                            W.pair = 0;
                            while (W.left > 0 && ++W.s < B.n_seqs) {
                                const PagedSeq S = paged_seq(B, W.s);
                                W.r0 = S.r0;
                                W.n = S.n;
                                W.len = S.len;
                                if (W.n > 0) break;
                            }
                            if (W.s >= B.n_seqs) W.left = 0;
                        }
                        W.tiles = pair_tiles(P, W.n, W.len, W.pair);
                    }
                }
                if (U.nj > 0) break;
                U.nj = 0;
            }
            if (un >= UNITS) alive = alive && warp_wait(bar(BAR_UE + (un & (UNITS - 1))), (un / UNITS - 1) & 1, abort_flag, B.status, P.wait_us);
            if (lane == 0 && alive) {
                int4 *u = told + 3 * (un & (UNITS - 1));
                u[0] = make_int4(U.r0, U.p0, U.rows, U.before);
                u[1] = make_int4(U.own, U.j0, U.nj, U.h);
                u[2] = make_int4(U.c0, U.parts, U.part, 0);
                mbar_arrive(bar(BAR_UF + (un & (UNITS - 1))));
            }
            ++un;
            j = U.j0;
            j_end = U.j0 + U.nj;
            uh = U.h;
            uown = U.own;
            uq = U.h * P.head_rows + U.r0 * P.group + U.p0;
            urows = U.rows;
            return U.nj > 0;
        };
        // Tiles in the order of the steps.  A lane has a page of the tile: lane 8 half + page of the keys' boxes, 16 + 8 half + page of the values', which are at the same place.
        struct TileRef { int y, n, h, q, rows; };             // row of the lane's page, keys (-1: no tile), KV head; of a unit's first tile: the pair's first query row, its rows
        const int page_rows = 1 << B.page_shift, pg = lane & 7, half = (lane >> 3) & 1;
        bool more = true;
        const auto next = [&]() -> TileRef {
            const bool first = j == j_end;
            if (first) more = more && next_unit();
            if (!more) return {0, -1, 0, 0, 0};
            const int in = j - prefix_tiles;
            const int n = min(TILE, in < 0 ? B.n_prefix - j * TILE : max(0, uown - in * TILE));
            int y = 0;
            if (pg * page_rows < n) {
                const int t = (in < 0 ? j : in) * TILE + pg * page_rows;
                const int32_t *table = in < 0 ? B.prefix : B.table + (size_t)us * B.max_pages;
                y = paged_page(B, table + (t >> B.page_shift)) << B.page_shift;
            }
            ++j;
            return {y, n, uh, uq, first ? urows : 0};
        };
        const auto bytes = [&](int n) { return (uint32_t)(((n + page_rows - 1) >> B.page_shift) << B.page_shift) * 128u * M::HALVES; };
        const auto load = [&](const CUtensorMap *map, uint32_t to, const TileRef &T, uint32_t b) {
            if (half < M::HALVES && pg * page_rows < T.n) tma_load_2d(to + half * HALF_BYTES + pg * page_rows * 128, map, T.h * D + half * 64, T.y, b);
        };
        TileRef A = next(), C = next();
        if (A.n >= 0) {
            if (lane == 0) mbar_expect_tx(bar(BAR_K0), bytes(A.n) + P.extra_tx);
            __syncwarp();
            if (lane < 16) load(&map_k, base + M::K, A, bar(BAR_K0));
        }
        pc_grid_dep_wait();                                   // the rotated queries are there
        int queries = 0;                                      // units whose queries have been fetched
        for (int gs = 0; alive && A.n >= 0; ++gs) {
            if (A.rows) {                                     // a new unit: once the last products with the old queries have been read
                for (int t = 0; t < 2 && alive; ++t) {
                    if (queries > 0) alive = warp_wait(bar(BAR_QFREE + t), (queries - 1) & 1, abort_flag, B.status, P.wait_us);
                    if (!alive) break;
                    if (lane == 0) mbar_expect_tx(bar(BAR_Q + t), M::TILE_B);
                    __syncwarp();
                    if (lane < M::HALVES) tma_load_2d(base + M::Q + t * M::TILE_B + lane * HALF_BYTES, &map_q, lane * 64, A.q + (t * TILE < A.rows ? t : 0) * TILE, bar(BAR_Q + t));     // a pair of one tile: the same one twice
                }
                ++queries;
            }
            const TileRef E = next();                         // its page is on the way while this step's copies are issued
            // PV(step - 2) and QK(step - 1) have read what lies where V(step) and K(step + 1) go
            if (gs > 0 && alive) alive = warp_wait(bar(BAR_EMPTY + ((gs - 1) & 1)), ((gs - 1) >> 1) & 1, abort_flag, B.status, P.wait_us);
            if (!alive) break;
            const int st = gs & 1;
            if (lane == 0) mbar_expect_tx(bar(BAR_KV + st), bytes(A.n) + (C.n >= 0 ? bytes(C.n) : 0u));
            __syncwarp();
            if (lane >= 16) load(&map_v, base + M::V + st * M::TILE_B, A, bar(BAR_KV + st));
            else if (C.n >= 0) load(&map_k, base + M::K + (st ^ 1) * M::TILE_B, C, bar(BAR_KV + st));
            A = C;
            C = E;
        }
    } else if (warp < 4) {
        // ---------------------------------------------------------------- warps 1 and 2: S = Q_t K^T; warp 3: O += P V.  All lanes wait, one issues.
        reg_dealloc<REGS_ISSUE>();
        const bool lead = elect_one();
        const uint32_t tm = __shfl_sync(0xffffffffu, tmem, 0);
        auto wait = [&](int b, int parity) {
            const bool ok = warp_wait(bar(b), parity, abort_flag, B.status, P.wait_us);
            tc_fence_after();
            return ok;
        };
        bool alive = true;
        int gs = 0;
        for (int un = 0;; ++un) {
            const Unit U = look(un, alive);
            if (U.nj == 0) break;
            if (warp < 3) {
                const int t = warp - 1;
                const uint64_t dq0 = desc_kmajor(base + M::Q + t * M::TILE_B), dk0 = desc_kmajor(base + M::K);
                alive = wait(BAR_Q + t, un & 1);
#pragma unroll 1
                for (int i = 0; i < U.nj && alive; ++i, ++gs) {
                    // the other tile's scores have left the columns (tile 1's first step: so tile 0 has seen the first keys)
                    alive = gs > 0 ? wait(BAR_KV + ((gs - 1) & 1), ((gs - 1) >> 1) & 1) : (t > 0 || wait(BAR_K0, 0));
                    if (alive && gs + t > 0) alive = wait(BAR_SFREE + (t ^ 1), (gs + t + 1) & 1);
                    if (!alive) break;
                    uint64_t dq = dq0, dk = dk0 + (gs & 1) * (M::TILE_B >> 4);
#pragma unroll 1
                    for (int half = 0; half < M::HALVES; ++half) {
#pragma unroll
                        for (int k4 = 0; k4 < 4; ++k4)
                            if (lead) mma_ss(tm + TM_S, dq + k4 * 2, dk + k4 * 2, QK, (half > 0 || k4 > 0));
                        dq += HALF_BYTES >> 4;
                        dk += HALF_BYTES >> 4;
                    }
                    if (lead) tc_commit(bar(BAR_SFULL + t));
                }
            } else {
                const uint64_t dv0 = desc_mnmajor(base + M::V);
#pragma unroll 1
                for (int i = 0; i < U.nj && alive; ++i, ++gs) {
                    const int st = gs & 1, in = U.j0 + i - prefix_tiles;
                    alive = wait(BAR_KV + st, (gs >> 1) & 1);
                    if (!alive) break;
                    const int n = in < 0 ? B.n_prefix - (U.j0 + i) * TILE : max(0, U.own - in * TILE);
                    if (n < TILE) {                               // values behind the segment's end are whatever the pool holds there
                        for (int hf = 0; hf < M::HALVES; ++hf)
                            for (int c = n * 8 + lane; c < TILE * 8; c += 32) sts128(base + M::V + st * M::TILE_B + hf * HALF_BYTES + c * 16, 0u, 0u, 0u, 0u);
                        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                        __syncwarp();
                    }
#pragma unroll 1
                    for (int t = 0; t < 2 && alive; ++t) {
                        uint64_t dv = dv0 + st * (M::TILE_B >> 4);
                        uint32_t pa = tm + TM_P + t * (TILE / 2);
                        const uint32_t oa = tm + TM_O + t * TILE;
#pragma unroll 1
                        for (int hf = 0; hf < 2; ++hf) {
                            alive = wait(BAR_PHALF + 2 * t + hf, gs & 1);
                            if (!alive) break;
#pragma unroll
                            for (int k4 = 0; k4 < 4; ++k4)
                                if (lead) mma_ts(oa, pa + k4 * 8, dv + k4 * (2048 >> 4), PV, (i > 0 || hf > 0 || k4 > 0));
                            dv += 8192 >> 4;
                            pa += 32;
                        }
                        if (alive && lead) tc_commit(bar(BAR_PVDONE + t));
                    }
                }
            }
            if (!alive) break;
        }
        // nothing of ours still runs on the tensor core when its memory is freed
        if (lead) tc_commit(bar(BAR_DONE));
        __syncwarp();
        pc_mbar_drain(bar(BAR_DONE), 0, B.status, PC_WHERE_PAGED_WAIT);
    } else {
        // ---------------------------------------------------------------- softmax, correction, output
        reg_alloc<REGS_SOFTMAX>();
        const int t = (warp - 4) >> 2, quad = warp & 3, r = quad * 32 + lane;
        const uint32_t lane_addr = (uint32_t)(quad * 32) << 16;
        const uint32_t s_addr = tmem + lane_addr + TM_S, p_addr = tmem + lane_addr + TM_P + t * (TILE / 2), o_addr = tmem + lane_addr + TM_O + t * TILE;
        const bool lead = elect_one();
        bool alive = true;
        int un = 0, j = 0, lim;
        Unit U = look(0, alive);
        // own tokens that this thread's row sees (one behind the last row sees what the last one sees; its output is dropped)
        const auto limit = [&]() { return B.causal ? min(U.own, U.before + (U.p0 + min(t * TILE + r, U.rows - 1)) / P.group + 1) : U.own; };
        lim = limit();
        float m_used = -INFINITY, l = 0.f;
        for (int gs = 0; alive && (U.nj > 0 || gs > 0); ++gs) {
            const bool flush = j == U.nj;
            const Unit V = U;                                 // the unit to flush
            const float m_e = m_used, l_e = l;
            bool end = false;
            if (flush) {
                U = look(++un, alive);
                if (!alive) break;
                end = U.nj == 0;
                lim = limit();
                j = 0;
                m_used = -INFINITY;
                l = 0.f;
            }
            if (!end) {
                alive = warp_wait(bar(BAR_SFULL + t), gs & 1, abort_flag, B.status, P.wait_us);
                if (!alive) break;
                tc_fence_after();
                uint32_t sv[128];
                tmem_ld32(s_addr, sv);
                tmem_ld32(s_addr + 32, sv + 32);
                tmem_ld32(s_addr + 64, sv + 64);
                tmem_ld32(s_addr + 96, sv + 96);
                tmem_wait_ld();
                tc_fence_before();
                __syncwarp();
                arrive_if(lead, bar(BAR_SFREE + t));
                if (j + 1 == U.nj) arrive_if(lead, bar(BAR_QFREE + t));                     // that was the unit's last product with this tile's queries
                const bool pv_done = gs == 0 || pc_mbar_test(bar(BAR_PVDONE + t), (gs - 1) & 1);
                const int jt = U.j0 + j;
                const int seen = jt < prefix_tiles ? B.n_prefix - jt * TILE : lim - (jt - prefix_tiles) * TILE;
                if (__any_sync(0xffffffffu, seen < TILE)) {
#pragma unroll
                    for (int i = 0; i < TILE; ++i) sv[i] = i < seen ? sv[i] : 0xFF800000u;
                }
                float mx0 = -INFINITY, mx1 = -INFINITY, mx2 = -INFINITY, mx3 = -INFINITY;
#pragma unroll
                for (int i = 0; i < TILE; i += 4) {
                    mx0 = fmaxf(mx0, __uint_as_float(sv[i]));
                    mx1 = fmaxf(mx1, __uint_as_float(sv[i + 1]));
                    mx2 = fmaxf(mx2, __uint_as_float(sv[i + 2]));
                    mx3 = fmaxf(mx3, __uint_as_float(sv[i + 3]));
                }
                const float mx = fmaxf(fmaxf(mx0, mx1), fmaxf(mx2, mx3));
                const bool grow = mx > m_used + GROW;
                if (__builtin_expect(!__all_sync(0xffffffffu, pv_done), 0)) {
                    alive = warp_wait(bar(BAR_PVDONE + t), (gs - 1) & 1, abort_flag, B.status, P.wait_us);
                    if (!alive) break;
                }
                tc_fence_after();
                if (t == 1) arrive_if(lead, bar(BAR_EMPTY + (gs & 1)));
                if (__builtin_expect(__any_sync(0xffffffffu, grow), 0)) {
                    const float m_new = fmaxf(m_used, mx);
                    const float corr = m_new == -INFINITY ? 1.f : fast_exp2(m_used - m_new);
                    l *= corr;
                    if (j > 0) {
                        uint32_t v[32];
#pragma unroll 1
                        for (int c = 0; c < D / 32; ++c) {
                            tmem_ld32(o_addr + c * 32, v);
                            tmem_wait_ld();
#pragma unroll
                            for (int i = 0; i < 32; ++i) v[i] = __float_as_uint(__uint_as_float(v[i]) * corr);
                            tmem_st32(o_addr + c * 32, v);
                        }
                    }
                    m_used = m_new;
                }
                const float neg = m_used == -INFINITY ? 0.f : -m_used;
                const float2 neg_m = make_float2(neg, neg);
                float2 la = make_float2(0.f, 0.f), lb = make_float2(0.f, 0.f);
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    uint32_t pk[16];
#pragma unroll
                    for (int i = 0; i < 16; i += 2) {
                        float2 x = add2(make_float2(__uint_as_float(sv[c * 32 + 2 * i]), __uint_as_float(sv[c * 32 + 2 * i + 1])), neg_m);
                        float2 y = add2(make_float2(__uint_as_float(sv[c * 32 + 2 * i + 2]), __uint_as_float(sv[c * 32 + 2 * i + 3])), neg_m);
                        x.x = fast_exp2(x.x); x.y = fast_exp2(x.y);
                        y.x = fast_exp2(y.x); y.y = fast_exp2(y.y);
                        la = add2(la, x);
                        lb = add2(lb, y);
                        pk[i] = pc_pack_bf16(x.x, x.y);
                        pk[i + 1] = pc_pack_bf16(y.x, y.y);
                    }
                    asm volatile("" : "+f"(la.x), "+f"(la.y), "+f"(lb.x), "+f"(lb.y));
                    tmem_st16(p_addr + c * 16, pk);
                    if (c & 1) {
                        tmem_wait_st();
                        tc_fence_before();
                        __syncwarp();
                        arrive_if(lead && !flush, bar(BAR_PHALF + 2 * t + (c >> 1)));
                    }
                }
                l += (la.x + la.y) + (lb.x + lb.y);
            } else {
                alive = warp_wait(bar(BAR_PVDONE + t), (gs - 1) & 1, abort_flag, B.status, P.wait_us);
                if (!alive) break;
                tc_fence_after();
            }
            if (__builtin_expect(flush, 0)) {
                const int h = V.h, at = t * TILE + r, p = V.p0 + at, i = p / P.group;
                const bool there = at < V.rows;
                const size_t row = (size_t)(V.r0 + i) * P.n_q_heads + h * P.group + (p - i * P.group);
                __nv_bfloat16 *orow = P.out + row * D;
                // Places of a CTA in scratch: its last item's (the first part of it), its first item's.  Parts of an item that is added up here lie as 16-byte unit (c, row) at c * 128 + row: a warp's
                // stores and loads are 512 bytes in a row.
                const auto slot_of = [&](int part) { return (size_t)(2 * (V.c0 + part) + (part == 0)) * 2 + t; };
                // The parts in the order of the keys, so the same bits whoever adds them up; this CTA's own from tensor memory (own = its number) or from scratch like the others (own = -1)
                const auto add_up = [&](int own) {
                    const auto ml_of = [&](int q) { return q == own ? make_float2(m_e, l_e) : __ldcg(P.part_ml + slot_of(q) * TILE + r); };
                    float m = -INFINITY, sum = 0.f;
                    for (int q = 0; q < V.parts; ++q) m = fmaxf(m, ml_of(q).x);
                    const auto weight = [&](float x) { return m == -INFINITY ? 1.f : fast_exp2(x - m); };
                    for (int q = 0; q < V.parts; ++q) {
                        const float2 ml = ml_of(q);
                        sum = fmaf(ml.y, weight(ml.x), sum);
                    }
                    const float inv = sum > 0.f ? 1.f / sum : (sum != sum ? sum : 0.f);
#pragma unroll 1
                    for (int c0 = 0; c0 < D; c0 += 64) {
                        float a[64];
#pragma unroll
                        for (int c = 0; c < 64; ++c) a[c] = 0.f;
#pragma unroll 1
                        for (int q = 0; q < V.parts; ++q) {
                            const float f = weight(ml_of(q).x);
                            if (q == own) {
                                uint32_t y[64];
                                tmem_ld32(o_addr + c0, y);
                                tmem_ld32(o_addr + c0 + 32, y + 32);
                                tmem_wait_ld();
#pragma unroll
                                for (int c = 0; c < 64; ++c) a[c] = fmaf(__uint_as_float(y[c]), f, a[c]);
                            } else {
                                const float4 *po = reinterpret_cast<const float4 *>(P.part_o) + slot_of(q) * (TILE * D / 4) + r + c0 / 4 * TILE;
                                float4 x[16];
#pragma unroll
                                for (int c = 0; c < 16; ++c) x[c] = __ldcg(po + c * TILE);
#pragma unroll
                                for (int c = 0; c < 16; ++c) {
                                    a[4 * c] = fmaf(x[c].x, f, a[4 * c]);
                                    a[4 * c + 1] = fmaf(x[c].y, f, a[4 * c + 1]);
                                    a[4 * c + 2] = fmaf(x[c].z, f, a[4 * c + 2]);
                                    a[4 * c + 3] = fmaf(x[c].w, f, a[4 * c + 3]);
                                }
                            }
                        }
                        if (there)
#pragma unroll
                            for (int c = 0; c < 64; c += 8)
                                *reinterpret_cast<uint4 *>(orow + c0 + c) = make_uint4(pc_pack_bf16(a[c] * inv, a[c + 1] * inv), pc_pack_bf16(a[c + 2] * inv, a[c + 3] * inv),
                                                                                       pc_pack_bf16(a[c + 4] * inv, a[c + 5] * inv), pc_pack_bf16(a[c + 6] * inv, a[c + 7] * inv));
                    }
                    if (there && P.lse) P.lse[row] = (m + log2f(sum)) * 0.6931471805599453f;
                };
                uint32_t *ticket = P.sync + SYNC_HEAD + (V.c0 * 2 + t) * 4 + quad;       // every warp for its own 32 rows
                const uint32_t call = __ldcg(P.sync) << 12;
                const bool split = !P.shared && V.parts > 1;
                bool added = false;
                if (end && split) {                           // the run's last item, whose other parts are mostly there by now: they are added to what lies in tensor memory
                    uint32_t seen;
                    asm volatile("ld.acquire.gpu.u32 %0, [%1];" : "=r"(seen) : "l"(ticket) : "memory");
                    added = __all_sync(0xffffffffu, seen == call + V.parts - 1);
                    if (added) {
                        add_up(V.part);
                        if (lane == 0) *ticket = 0;
                    }
                }
                if (!added) {
                    uint32_t v[D];
#pragma unroll
                    for (int c = 0; c < D / 32; ++c) tmem_ld32(o_addr + c * 32, v + c * 32);
                    tmem_wait_ld();
                    if (!end) {
                        tc_fence_before();
                        __syncwarp();
                        arrive_if(lead, bar(BAR_PHALF + 2 * t));
                        arrive_if(lead, bar(BAR_PHALF + 2 * t + 1));
                    }
                    if (P.shared) {
                        const size_t slot = slot_of(V.part) * TILE + r;
                        float *to = V.parts == 1 ? P.home_o + row * D : P.part_o + slot * D;
                        if (there) {
#pragma unroll
                            for (int c = 0; c < D / 4; ++c) *reinterpret_cast<uint4 *>(to + c * 4) = make_uint4(v[4 * c], v[4 * c + 1], v[4 * c + 2], v[4 * c + 3]);
                            *(V.parts == 1 ? P.home_ml + row : P.part_ml + slot) = make_float2(m_e, l_e);
                        }
                    } else if (!split) {
                        const float inv = l_e > 0.f ? 1.f / l_e : (l_e != l_e ? l_e : 0.f);
                        if (there) {
#pragma unroll
                            for (int c = 0; c < D / 8; ++c) {
                                uint4 w;
                                w.x = pc_pack_bf16(__uint_as_float(v[8 * c + 0]) * inv, __uint_as_float(v[8 * c + 1]) * inv);
                                w.y = pc_pack_bf16(__uint_as_float(v[8 * c + 2]) * inv, __uint_as_float(v[8 * c + 3]) * inv);
                                w.z = pc_pack_bf16(__uint_as_float(v[8 * c + 4]) * inv, __uint_as_float(v[8 * c + 5]) * inv);
                                w.w = pc_pack_bf16(__uint_as_float(v[8 * c + 6]) * inv, __uint_as_float(v[8 * c + 7]) * inv);
                                *reinterpret_cast<uint4 *>(orow + c * 8) = w;
                            }
                            if (P.lse) P.lse[row] = (m_e + log2f(l_e)) * 0.6931471805599453f;
                        }
                    } else {
                        uint4 *po = reinterpret_cast<uint4 *>(P.part_o) + slot_of(V.part) * (TILE * D / 4) + r;
#pragma unroll
                        for (int c = 0; c < D / 4; ++c) po[c * TILE] = make_uint4(v[4 * c], v[4 * c + 1], v[4 * c + 2], v[4 * c + 3]);
                        P.part_ml[slot_of(V.part) * TILE + r] = make_float2(m_e, l_e);
                        __threadfence();
                        __syncwarp();
                        // A ticket is worth what this call has put there: one that a call before has left (a wait of it ran out) counts from nothing.
                        uint32_t come = 0;
                        if (lane == 0) {
                            uint32_t seen = __ldcg(ticket);
                            for (;;) {
                                const uint32_t want = (seen & ~4095u) == call ? seen + 1 : call + 1, was = atomicCAS(ticket, seen, want);
                                if (was == seen) {
                                    come = want & 4095u;
                                    break;
                                }
                                seen = was;
                            }
                        }
                        come = __shfl_sync(0xffffffffu, come, 0);
                        if (come == (uint32_t)V.parts) {      // the last to come
                            __threadfence();
                            add_up(-1);
                            if (lane == 0) *ticket = 0;
                        }
                    }
                }
            }
            if (end) break;
            ++j;
        }
    }
    __syncwarp();
    if (*abort_flag) pc_let_copies_land();
    tc_fence_before();
    __syncthreads();
    if (threadIdx.x == 0 && atomicAdd(P.sync + 1, 1u) == gridDim.x - 1) {        // the last CTA of the call: the next one has another number
        P.sync[1] = 0;
        P.sync[0] = (__ldcg(P.sync) + 1) & 0xFFFFFu;
    }
    if (warp == 2) {
        tc_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
    }
}

template <int D> pc_status launch_tc(const pc_ctx *ctx, const CUtensorMap &mq, const CUtensorMap &mk, const CUtensorMap &mv, const TcParams &P, cudaStream_t stream) {
    static bool ready[PC_MAX_DEVICES] = {};
    if (ctx->device < 0 || ctx->device >= PC_MAX_DEVICES) return PC_ERR_UNSUPPORTED;
    if (!ready[ctx->device]) {
        PC_CUDA_TRY(cudaFuncSetAttribute(k_paged_tc<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, Map<D>::ALLOC));
        cudaFuncAttributes a;
        PC_CUDA_TRY(cudaFuncGetAttributes(&a, k_paged_tc<D>));
        if (a.numRegs < REGS_LAUNCH) {                     // setmaxnreg would wait for registers that the block does not have
            fprintf(stderr, "packcache: k_paged_tc has %d registers a thread, %d are shared out\n", a.numRegs, REGS_LAUNCH);
            return PC_ERR_UNSUPPORTED;
        }
        ready[ctx->device] = true;
    }
    PC_LAUNCH(k_paged_tc<D>, dim3(ctx->sm_count), dim3(TC_THREADS), Map<D>::ALLOC, stream, mq, mk, mv, P);
    return PC_OK;
}

}  // namespace

bool pc_paged_tc_shape(const pc_ctx *ctx) { return ctx->desc.dtype == PC_BF16; }
size_t pc_paged_tc_tiles(const pc_ctx *ctx) { return (size_t)4 * ctx->sm_count; }
size_t pc_paged_tc_sync_words(const pc_ctx *ctx) { return SYNC_HEAD + (size_t)8 * ctx->sm_count; }

pc_status pc_launch_paged_tc(const pc_paged *w, const pc_paged_args &A, bool shared, cudaStream_t stream) {
    const pc_ctx *ctx = A.ctx;
    const pc_layer_desc &D = ctx->desc;
    const long long head_rows = (long long)A.batch.n_rows * ctx->group;
    if (head_rows * D.n_kv_heads > INT32_MAX) return PC_ERR_CAPACITY;
    // keys and values as [page x token][KV head x channel], boxes of a page by 64 channels; queries as [KV head x row][channel], boxes of 128 rows
    CUtensorMap mq, mk, mv;
    const uint64_t rows = (uint64_t)A.batch.n_pages << A.batch.page_shift, cols = (uint64_t)D.n_kv_heads * D.head_dim;
    if (!make_map(&mq, w->q_rot, (uint64_t)head_rows * D.n_kv_heads, D.head_dim) || !make_map(&mk, A.pages->k, rows, cols, 1u << A.batch.page_shift) ||
        !make_map(&mv, A.pages->v, rows, cols, 1u << A.batch.page_shift)) {
        fprintf(stderr, "packcache: cuTensorMapEncodeTiled failed\n");
        return PC_ERR_CUDA;
    }
    const FrontParams F{A.batch, static_cast<const char *>(A.q), A.q_pos, static_cast<char *>(w->q_rot), D.n_q_heads * D.head_dim / 8, ctx->group, D.n_kv_heads, D.head_dim, head_rows,
                        pc_q_rot_scale(D.head_dim)};
    PC_LAUNCH(k_paged_front, dim3((unsigned)(((long long)A.batch.n_rows * 32 + FRONT_THREADS - 1) / FRONT_THREADS)), dim3(FRONT_THREADS), 0, stream, F, ctx->rope);
    TcParams P{};
    P.B = A.batch;
    P.head_rows = (int)head_rows;
    P.n_q_heads = D.n_q_heads;
    P.n_kv = D.n_kv_heads;
    P.group = ctx->group;
    P.shared = shared;
    P.out = static_cast<__nv_bfloat16 *>(A.out);
    P.lse = A.lse;
    P.part_o = w->tc_o;
    P.part_ml = w->tc_ml;
    P.home_o = w->home_o + w->home_rows * D.n_q_heads * D.head_dim;          // (the second half: the few-row kernel has the first one for the sequences' own tokens)
    P.home_ml = w->home_ml + w->home_rows * D.n_q_heads;
    P.sync = w->tc_sync;
    P.wait_us = ctx->wait_limit_us;
    P.extra_tx = ctx->test_extra_tx;
    return D.head_dim == 128 ? launch_tc<128>(ctx, mq, mk, mv, P, stream) : launch_tc<64>(ctx, mq, mk, mv, P, stream);
}

PagedTcLine pc_paged_tc_line(const pc_paged *w, const pc_paged_args &A) {
    return PagedTcLine{w->tc_o, w->tc_ml, std::max(1, (A.batch.n_prefix + TILE - 1) / TILE), GAP, A.ctx->sm_count};
}
