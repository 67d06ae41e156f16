// Gradient of attention for blocks of bf16 queries, head size 128, on the 5th-generation tensor cores (formulas in
// attend_backward.cu): tcgen05.mma with TMEM accumulators, operands staged by TMA.
//
// Two kinds of units, both 128 rows tall (rows = TMEM lanes), stream the other side's rows in tiles of 64:
//   key unit    (sequence, 128 keys of one segment, head): stationary K, V; streams Q, dO.
//       S = K Q^T, T = V dO^T (rows keys, columns queries);  dV += P^T dO,  dK += dS^T Q
//   query unit  (sequence, 128 queries, head, chunk of the key list): stationary Q, dO; streams K, V.
//       S = Q K^T, T = dO V^T (rows queries, columns keys);  dQ += dS K
// In both, S and T are products of two K-major shared-memory tiles, P and dS go back to TMEM as bf16 pairs over the S and T
// they came from and are the A operands of the accumulating products, whose B operand is the streamed tile as it lies in
// shared memory (MN-major).  So one code path serves both and nothing is transposed.  S and T are computed twice (seven
// matrix products instead of the five of a pass that also scatters dQ): in exchange every gradient row has one owner that
// sums it in a fixed order in TMEM, without atomics and without fp32 partials of dQ per key tile (at 512 queries and 16,384
// keys of 40 heads those would be 1.3 GB).
// P and dS are rounded to bf16 as matrix operands (2^-8 of each weight at most); sums are fp32.
//
// One persistent block per SM draws units from a counter, query units first (they are the longer ones).  Roles, each
// waiting only for what it consumes:
//   producer (warp 10)  draws units, brings the stationary pair (two buffers: the next unit's loads overlap this one's end)
//       and the streamed tiles (three stages) with plain TMA tensor copies, 128-byte swizzle
//   issuer of S, T (warp 8)   into one of two score buffers of TMEM, up to two tiles ahead of the weights
//   issuer of the accumulating products (warp 9)
//   weights (warps 0-7; two threads per row, 32 columns each)  P and dS from S, T and the statistics; at a unit's end the
//       accumulators out of TMEM
// TMEM columns: [0,128) dK or dQ, [128,256) dV, then per score buffer 64 of S and 64 of T.
// Every wait is bounded; a role whose wait runs out reports it and leaves, and so do the others in turn.
#include "dodo_internal.cuh"
#include "sm100_ptx.cuh"

namespace {

using namespace sm100;

constexpr int DH = 128;
constexpr int BM = 128;                 // rows of a unit
constexpr int BN = 64;                  // rows of a streamed tile
constexpr int kWeightThreads = 256;
constexpr int kThreads = kWeightThreads + 96;
constexpr int kStages = 3;
constexpr int kSlots = 4;               // units announced ahead
constexpr int kXHalf = BM * 128;        // 64 features of a stationary tile
constexpr int kXTile = 2 * kXHalf;
constexpr int kYHalf = BN * 128;
constexpr int kYTile = 2 * kYHalf;
constexpr int kStatBytes = BN * 8;
constexpr int kOffX = 0;                                   // [buffer][X1, X2]
constexpr int kOffY = kOffX + 2 * 2 * kXTile;              // [stage][Y1, Y2]
constexpr int kOffStat = kOffY + kStages * 2 * kYTile;     // [stage][64 x -lse, 64 x -D]
constexpr int kSmemBytes = kOffStat + kStages * kStatBytes;
constexpr uint32_t kTmemCols = 512;
constexpr uint32_t kColAcc2 = 128, kColScore = 256;        // + buffer * 128; T at + 64

struct BackwardMaps { CUtensorMap Q, dO, cK, cV, lK, lV; };   // boxes of 64 elements x 64 rows, 128-byte swizzle

__device__ __forceinline__ float ex2_approx(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint64_t* bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 ::"r"(dst), "l"(src), "r"(bytes), "r"(smem_u32(bar)) : "memory");
}
// a wait by a whole warp: all lanes see the same outcome
__device__ __forceinline__ bool warp_wait(uint64_t* bar, uint32_t parity) { return __all_sync(0xffffffffu, mbar_wait(bar, parity)) != 0; }

struct Unit {
    bool keys;          // key unit
    int i, h;           // sequence of the group, head
    bool cached;        // key unit: segment
    int first, rows;    // stationary rows: first of the segment / of the queries, how many are live
    int row0;           // ... and where in its array
    int t0, n;          // streamed tiles [t0, t0 + n)
    int nt_c, l_vis;    // query unit: cache tiles of the whole list, visible local rows
    int chunk, qt;
};

__device__ __forceinline__ Unit unit_of(const BackwardGroup& g, int H, int id) {
    Unit u;
    u.keys = id >= g.q_blocks;
    const int at = u.keys ? id - g.q_blocks : id;
    int b = 0;
    for (int i = 1; i < g.nseq; ++i) b += (u.keys ? g.seq[i].kv0 : g.seq[i].q0) <= at ? 1 : 0;
    const BackwardSeq& sq = g.seq[b];
    u.i = b;
    int r = at - (u.keys ? sq.kv0 : sq.q0);
    if (u.keys) {
        u.h = r % H;
        int tile = r / H;
        const int nt = (sq.c_len + BM - 1) / BM;
        u.cached = tile < nt;
        if (!u.cached) tile -= nt;
        u.first = tile * BM;
        u.rows = min(BM, (u.cached ? sq.c_len : sq.l_len) - u.first);
        u.row0 = (u.cached ? sq.c_row0 : sq.l_row0) + u.first;
        u.t0 = u.cached ? 0 : max(0, sq.l_pos0 + u.first - sq.q_pos0) / BN;    // queries ahead of a local tile's first key see none of it
        u.n = max(0, (sq.tq + BN - 1) / BN - u.t0);
        u.nt_c = u.l_vis = u.chunk = u.qt = 0;
    } else {
        u.chunk = r % sq.nchunk; r /= sq.nchunk;
        u.h = r % H;
        u.qt = r / H;
        u.cached = false;
        u.first = u.qt * BM;
        u.rows = min(BM, sq.tq - u.first);
        u.row0 = sq.q_row0 + u.first;
        u.l_vis = max(0, min(sq.l_len, sq.q_pos0 + u.first + u.rows - sq.l_pos0));
        u.nt_c = (sq.c_len + BN - 1) / BN;
        const int nt = u.nt_c + (u.l_vis + BN - 1) / BN;
        u.t0 = min(nt, u.chunk * sq.ctiles);
        u.n = min(nt, u.t0 + sq.ctiles) - u.t0;
    }
    return u;
}

struct Tile { bool cached; int first, rows, row0; };   // streamed tile: rows of a segment, or of the queries
__device__ __forceinline__ Tile tile_of(const BackwardSeq& sq, const Unit& u, int t) {
    Tile s;
    if (u.keys) {
        s.cached = false; s.first = t * BN; s.rows = min(BN, sq.tq - s.first); s.row0 = sq.q_row0 + s.first;
    } else if (t < u.nt_c) {
        s.cached = true; s.first = t * BN; s.rows = min(BN, sq.c_len - s.first); s.row0 = sq.c_row0 + s.first;
    } else {
        s.cached = false; s.first = (t - u.nt_c) * BN; s.rows = min(BN, u.l_vis - s.first); s.row0 = sq.l_row0 + s.first;
    }
    return s;
}

// 16 bytes of bf16 with every NaN and infinity replaced by 0
__device__ __forceinline__ uint32_t finite2(uint32_t v) {
    if ((v & 0x7f80u) == 0x7f80u) v &= 0xffff0000u;
    if ((v & 0x7f800000u) == 0x7f800000u) v &= 0xffffu;
    return v;
}

__global__ void __launch_bounds__(kThreads, 1)
backward_dense_kernel(const __grid_constant__ BackwardMaps maps, const __grid_constant__ BackwardGroup g, const BackwardArrays a, int H,
                      float scale, int* __restrict__ next_unit, int* __restrict__ dev_status) {
    extern __shared__ unsigned char smem_raw[];
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    unsigned char* const base_ptr = smem_raw + (base - smem_u32(smem_raw));
    __shared__ __align__(8) uint64_t bar_x[2], bar_xfree[2], bar_y[kStages], bar_yfree[kStages], bar_s[2], bar_p[2], bar_a[2], bar_epi,
        bar_u[kSlots], bar_ufree[kSlots], bar_w;
    __shared__ uint32_t tmem_slot;
    __shared__ int s_unit[kSlots];
    __shared__ int s_flag;

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int total = g.q_blocks + g.kv_blocks;
    if (tid == 0) {
        for (int i = 0; i < 2; ++i) {
            mbar_init(&bar_x[i], 1); mbar_init(&bar_xfree[i], 1); mbar_init(&bar_s[i], 1); mbar_init(&bar_a[i], 1);
            mbar_init(&bar_p[i], kWeightThreads / 32);
        }
        for (int i = 0; i < kStages; ++i) { mbar_init(&bar_y[i], 1); mbar_init(&bar_yfree[i], 1); }
        for (int i = 0; i < kSlots; ++i) { mbar_init(&bar_u[i], 1); mbar_init(&bar_ufree[i], 2 + kWeightThreads / 32); }
        mbar_init(&bar_epi, kWeightThreads / 32);
        mbar_init(&bar_w, kWeightThreads / 32);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 0) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_slot)), "r"(kTmemCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_slot;
    // (launched in plain stream order: everything before this kernel on the stream has completed)

    // the unit announced as number k, or -1 past the last (and when the announcement does not come)
    auto unit_number = [&](int k) {
        if (!mbar_wait(&bar_u[k % kSlots], static_cast<uint32_t>(k / kSlots) & 1u)) return -2;
        return *reinterpret_cast<volatile int*>(&s_unit[k % kSlots]);
    };

    bool ok = true;
    if (warp == 10) {
        // ================================= producer =================================
        if (lane == 0) {
            int m = 0, x = 0;       // streamed tiles and units with tiles so far
            for (int k = 0; ok; ++k) {
                const int slot = k % kSlots;
                if (k >= kSlots && !mbar_wait(&bar_ufree[slot], static_cast<uint32_t>(k / kSlots - 1) & 1u)) { ok = false; break; }
                const int drawn = atomicAdd(next_unit, 1);
                if (drawn == total + static_cast<int>(gridDim.x) - 1) *next_unit = 0;   // every block draws one past the end: the last puts the counter back
                const int id = drawn < total ? drawn : -1;
                *reinterpret_cast<volatile int*>(&s_unit[slot]) = id;
                mbar_arrive(&bar_u[slot]);
                if (id < 0) break;
                const Unit u = unit_of(g, H, id);
                if (u.n == 0) continue;
                const BackwardSeq& sq = g.seq[u.i];
                const int xb = x & 1, col = u.h * DH;
                if (x >= 2 && !mbar_wait(&bar_xfree[xb], static_cast<uint32_t>(x / 2 - 1) & 1u)) { ok = false; break; }
                const CUtensorMap* x1 = !u.keys ? &maps.Q : u.cached ? &maps.cK : &maps.lK;
                const CUtensorMap* x2 = !u.keys ? &maps.dO : u.cached ? &maps.cV : &maps.lV;
                mbar_expect_tx(&bar_x[xb], 2 * kXTile);
                for (int part = 0; part < 4; ++part) {      // (64 features, 64 rows) at a time
                    const uint32_t dst = base + kOffX + xb * 2 * kXTile + (part >> 1) * kXHalf + (part & 1) * (64 * 128);
                    tma_load_2d(dst, x1, col + (part >> 1) * 64, u.row0 + (part & 1) * 64, &bar_x[xb]);
                    tma_load_2d(dst + kXTile, x2, col + (part >> 1) * 64, u.row0 + (part & 1) * 64, &bar_x[xb]);
                }
                ++x;
                for (int j = 0; j < u.n; ++j, ++m) {
                    const int st = m % kStages;
                    if (m >= kStages && !mbar_wait(&bar_yfree[st], static_cast<uint32_t>(m / kStages - 1) & 1u)) { ok = false; break; }
                    const Tile t = tile_of(sq, u, u.t0 + j);
                    const CUtensorMap* y1 = u.keys ? &maps.Q : t.cached ? &maps.cK : &maps.lK;
                    const CUtensorMap* y2 = u.keys ? &maps.dO : t.cached ? &maps.cV : &maps.lV;
                    const uint32_t dst = base + kOffY + st * 2 * kYTile;
                    mbar_expect_tx(&bar_y[st], 2 * kYTile + (u.keys ? kStatBytes : 0));
                    tma_load_2d(dst, y1, col, t.row0, &bar_y[st]);
                    tma_load_2d(dst + kYHalf, y1, col + 64, t.row0, &bar_y[st]);
                    tma_load_2d(dst + kYTile, y2, col, t.row0, &bar_y[st]);
                    tma_load_2d(dst + kYTile + kYHalf, y2, col + 64, t.row0, &bar_y[st]);
                    if (u.keys)
                        bulk_load(base + kOffStat + st * kStatBytes, a.stats + (static_cast<size_t>(u.h) * g.stat_rows + sq.stat0 + t.first) * 2,
                                  kStatBytes, &bar_y[st]);
                }
            }
            if (!ok) {       // leave no copy in flight behind
                for (int i = max(0, m - kStages); i < m; ++i) mbar_wait(&bar_y[i % kStages], static_cast<uint32_t>(i / kStages) & 1u);
                for (int i = max(0, x - 2); i < x; ++i) mbar_wait(&bar_x[i & 1], static_cast<uint32_t>(i / 2) & 1u);
            }
        }
    } else if (warp == 8) {
        // ================================= S = X1 Y1^T, T = X2 Y2^T =================================
        if (lane == 0) {
            int m = 0, x = 0;
            for (int k = 0; ok; ++k) {
                const int id = unit_number(k);
                if (id < 0) { ok = id == -1; break; }
                const Unit u = unit_of(g, H, id);
                mbar_arrive(&bar_ufree[k % kSlots]);
                if (u.n == 0) continue;
                const int xb = x & 1;
                if (!mbar_wait(&bar_x[xb], static_cast<uint32_t>(x / 2) & 1u)) { ok = false; break; }
                const uint64_t a1 = desc_kmajor(base + kOffX + xb * 2 * kXTile), a2 = desc_kmajor(base + kOffX + xb * 2 * kXTile + kXTile);
                const uint32_t idesc = idesc_bf16(BN, false);
                for (int j = 0; j < u.n; ++j, ++m) {
                    const int b = m & 1, st = m % kStages;
                    if (m >= 2 && !mbar_wait(&bar_a[b], static_cast<uint32_t>((m - 2) >> 1) & 1u)) { ok = false; break; }   // P, dS of two tiles ago consumed
                    if (!mbar_wait(&bar_y[st], static_cast<uint32_t>(m / kStages) & 1u)) { ok = false; break; }
                    tc_fence_after();
                    const uint64_t b1 = desc_kmajor(base + kOffY + st * 2 * kYTile), b2 = desc_kmajor(base + kOffY + st * 2 * kYTile + kYTile);
                    const uint32_t d = tmem + kColScore + b * 128;
#pragma unroll
                    for (int i = 0; i < DH / 16; ++i)
                        mma_bf16(d, a1 + static_cast<uint64_t>(((i / 4) * kXHalf + (i % 4) * 32) >> 4),
                                 b1 + static_cast<uint64_t>(((i / 4) * kYHalf + (i % 4) * 32) >> 4), idesc, i > 0);
#pragma unroll
                    for (int i = 0; i < DH / 16; ++i)
                        mma_bf16(d + 64, a2 + static_cast<uint64_t>(((i / 4) * kXHalf + (i % 4) * 32) >> 4),
                                 b2 + static_cast<uint64_t>(((i / 4) * kYHalf + (i % 4) * 32) >> 4), idesc, i > 0);
                    mma_commit(&bar_s[b]);
                }
                if (ok) mma_commit(&bar_xfree[xb]);
                ++x;
            }
        }
    } else if (warp == 9) {
        // ================================= acc1 += dS Y1, acc2 += P Y2 =================================
        if (lane == 0) {
            int m = 0, x = 0;
            for (int k = 0; ok; ++k) {
                const int id = unit_number(k);
                if (id < 0) { ok = id == -1; break; }
                const Unit u = unit_of(g, H, id);
                mbar_arrive(&bar_ufree[k % kSlots]);
                if (u.n == 0) continue;
                if (x >= 1 && !mbar_wait(&bar_epi, static_cast<uint32_t>(x - 1) & 1u)) { ok = false; break; }   // the last unit's accumulators are out
                const uint32_t idesc = idesc_bf16(DH, true);
                for (int j = 0; j < u.n; ++j, ++m) {
                    const int b = m & 1, st = m % kStages;
                    if (!mbar_wait(&bar_p[b], static_cast<uint32_t>(m >> 1) & 1u)) { ok = false; break; }
                    if (!mbar_wait(&bar_y[st], static_cast<uint32_t>(m / kStages) & 1u)) { ok = false; break; }
                    tc_fence_after();
                    const uint64_t y1 = desc_mnmajor(base + kOffY + st * 2 * kYTile, kYHalf), y2 = desc_mnmajor(base + kOffY + st * 2 * kYTile + kYTile, kYHalf);
                    const uint32_t p = tmem + kColScore + b * 128;
                    // (16 rows of Y = 8 columns of pairs; a row's two threads keep to their own half of the S and T columns)
                    if (u.keys) {
#pragma unroll
                        for (int i = 0; i < BN / 16; ++i)
                            mma_bf16_ts(tmem + kColAcc2, p + (i / 2) * 32 + (i % 2) * 8, y2 + static_cast<uint64_t>((i * 2048) >> 4), idesc, j > 0 || i > 0);
                    }
#pragma unroll
                    for (int i = 0; i < BN / 16; ++i)
                        mma_bf16_ts(tmem, p + 64 + (i / 2) * 32 + (i % 2) * 8, y1 + static_cast<uint64_t>((i * 2048) >> 4), idesc, j > 0 || i > 0);
                    mma_commit(&bar_a[b]);
                    mma_commit(&bar_yfree[st]);
                }
                ++x;
            }
        }
    } else {
        // ================================= weights =================================
        const int row = tid & (BM - 1), half = tid >> 7;
        const uint32_t lane_sel = static_cast<uint32_t>((warp & 3) * 32) << 16;
        const float scale2 = scale * 1.4426950408889634f;
        const float2 c2 = make_float2(scale2, scale2);
        int m = 0;
        uint32_t turn = 0;
        // the eight warps meet (a barrier with a bounded wait: a warp that has left must not hold the others)
        auto meet = [&]() {
            __syncwarp();
            if (lane == 0) mbar_arrive(&bar_w);
            if (!warp_wait(&bar_w, turn & 1u)) ok = false;
            ++turn;
        };
        for (int k = 0; ok; ++k) {
            const int id = __shfl_sync(0xffffffffu, unit_number(k), 0);
            if (id < 0) { ok = id == -1; break; }
            const Unit u = unit_of(g, H, id);
            if (lane == 0) mbar_arrive(&bar_ufree[k % kSlots]);
            const BackwardSeq& sq = g.seq[u.i];
            const bool live = row < u.rows;
            float2 score2 = make_float2(0.f, 0.f);

            // a thread's own row: position, and (query unit) statistics; dead rows compute what nobody reads
            int my_pos;
            float nlse = 0.f, ndelta = 0.f;
            if (u.keys) {
                my_pos = !live ? -(1 << 30) : u.cached ? __ldg(a.cache_pos + u.row0 + row) : sq.l_pos0 + u.first + row;
            } else {
                my_pos = live ? sq.q_pos0 + u.first + row : 0x7fffffff;
                const int e = sq.stat0 + u.first + row;
                if (live) {
                    const float* s = a.stats + (static_cast<size_t>(u.h) * g.stat_rows + (e & ~63)) * 2 + (e & 63);
                    nlse = __ldg(s);
                    ndelta = __ldg(s + 64);
                }
            }
            // key unit: a tile needs the position test if its first query lies behind some key of this warp's rows; query
            // unit: if some key of the tile lies behind some query of the warp's rows
            const int edge = u.keys ? __reduce_max_sync(0xffffffffu, my_pos) : __reduce_min_sync(0xffffffffu, my_pos);
            // query unit: positions of a tile's columns, one a lane for the thread's half, fetched a tile ahead
            auto column_pos = [&](int t) {
                const Tile s = tile_of(sq, u, t);
                const int c = half * 32 + lane;
                if (c >= s.rows) return 0x7fffffff;
                return s.cached ? __ldg(a.cache_pos + s.row0 + c) : sq.l_pos0 + s.first + c;
            };
            int next_pos = !u.keys && u.n > 0 ? column_pos(u.t0) : 0;

            for (int j = 0; j < u.n && ok; ++j, ++m) {
                const int b = m & 1, st = m % kStages;
                const Tile t = tile_of(sq, u, u.t0 + j);
                const int cpos = next_pos;
                if (!u.keys && j + 1 < u.n) next_pos = column_pos(u.t0 + j + 1);
                if (!warp_wait(&bar_s[b], static_cast<uint32_t>(m >> 1) & 1u)) { ok = false; break; }
                tc_fence_after();
                const uint32_t ts = tmem + kColScore + b * 128 + half * 32 + lane_sel;
                uint32_t sv[32], tv[32];
                tmem_ld32(ts, sv);
                tmem_ld32(ts + 64, tv);
                uint32_t pp[16], pd[16];
                if (u.keys) {
                    if (!warp_wait(&bar_y[st], static_cast<uint32_t>(m / kStages) & 1u)) { ok = false; break; }   // the statistics came with the tile
                    const float4* nl = reinterpret_cast<const float4*>(base_ptr + kOffStat + st * kStatBytes) + half * 8;
                    const float4* nd = nl + 16;
                    const int q0 = sq.q_pos0 + t.first;
                    const bool test = edge > q0 || t.rows < BN;
                    const int c_lo = my_pos - q0 - half * 32, c_hi = t.rows - half * 32;
#pragma unroll
                    for (int c = 0; c < 8; ++c) {
                        const float4 l4 = nl[c], d4 = nd[c];
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const int i = 4 * c + 2 * e;
                            const float2 x = __ffma2_rn(make_float2(__uint_as_float(sv[i]), __uint_as_float(sv[i + 1])), c2,
                                                        e == 0 ? make_float2(l4.x, l4.y) : make_float2(l4.z, l4.w));
                            float2 p = make_float2(ex2_approx(x.x), ex2_approx(x.y));
                            float2 d = __fmul2_rn(p, __fadd2_rn(make_float2(__uint_as_float(tv[i]), __uint_as_float(tv[i + 1])),
                                                               e == 0 ? make_float2(d4.x, d4.y) : make_float2(d4.z, d4.w)));
                            if (test) {
                                if (i < c_lo || i >= c_hi) p.x = d.x = 0.f;
                                if (i + 1 < c_lo || i + 1 >= c_hi) p.y = d.y = 0.f;
                            }
                            score2 = __fadd2_rn(score2, d);
                            pp[i / 2] = pack_bf16(p.x, p.y);
                            pd[i / 2] = pack_bf16(d.x, d.y);
                        }
                    }
                    tmem_st16(ts, pp);
                    if (t.rows < BN) {   // rows behind the sequence's queries must not reach the products
                        unsigned char* y = base_ptr + kOffY + st * 2 * kYTile;
                        for (int i = tid; i < (BN - t.rows) * 32; i += kWeightThreads) {     // 32 x 16 bytes per row of the pair
                            const int r = t.rows + i / 32, piece = i % 32;
                            *reinterpret_cast<uint4*>(y + (piece >> 4) * kYTile + ((piece >> 3) & 1) * kYHalf + r * 128 + (piece & 7) * 16) = make_uint4(0, 0, 0, 0);
                        }
                        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    }
                } else {
                    const int far = __reduce_max_sync(0xffffffffu, cpos);
                    const bool test = far > edge;
                    const float2 l2 = make_float2(nlse, nlse), d2 = make_float2(ndelta, ndelta);
#pragma unroll
                    for (int i = 0; i < 32; i += 2) {
                        const float2 x = __ffma2_rn(make_float2(__uint_as_float(sv[i]), __uint_as_float(sv[i + 1])), c2, l2);
                        const float2 p = make_float2(ex2_approx(x.x), ex2_approx(x.y));
                        float2 d = __fmul2_rn(p, __fadd2_rn(make_float2(__uint_as_float(tv[i]), __uint_as_float(tv[i + 1])), d2));
                        if (test) {
                            if (__shfl_sync(0xffffffffu, cpos, i) > my_pos) d.x = 0.f;
                            if (__shfl_sync(0xffffffffu, cpos, i + 1) > my_pos) d.y = 0.f;
                        }
                        pd[i / 2] = pack_bf16(d.x, d.y);
                    }
                    // Keys that some query of the tile does not see, and rows behind the segment: dS is 0 there, but 0 times
                    // what the row holds need not be.  Rows behind the segment are zeroed, NaN and infinities of the others
                    // replaced by 0 (a query that sees such a key has a NaN in dS).  Each warp takes 8 rows of its half.
                    if (far > sq.q_pos0 + u.first) {
                        const int r = half * 32 + (warp & 3) * 8 + (lane >> 2), part = lane & 3;
                        uint4* y = reinterpret_cast<uint4*>(base_ptr + kOffY + st * 2 * kYTile + (part >> 1) * kYHalf + r * 128 + (part & 1) * 64);
                        // (the copies' writes are visible to threads that have seen their barrier)
                        if (!warp_wait(&bar_y[st], static_cast<uint32_t>(m / kStages) & 1u)) { ok = false; break; }
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            uint4 v = y[e];
                            y[e] = r >= t.rows ? make_uint4(0, 0, 0, 0) : make_uint4(finite2(v.x), finite2(v.y), finite2(v.z), finite2(v.w));
                        }
                        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    }
                }
                tmem_st16(ts + 64, pd);
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&bar_p[b]);
            }
            if (!ok) break;

            // ---- the unit's accumulators --------------------------------------------------------------------------
            if (u.n > 0) {
                if (!warp_wait(&bar_a[(m - 1) & 1], static_cast<uint32_t>((m - 1) >> 1) & 1u)) { ok = false; break; }
                tc_fence_after();
            }
            const size_t at = (static_cast<size_t>(u.row0 + row) * H + u.h) * DH + half * 64;
            auto take = [&](uint32_t col, uint32_t* v) {      // 32 columns of the thread's row; zeros where nothing was summed
                if (u.n > 0) {
                    tmem_ld32(tmem + col + lane_sel, v);
                } else {
#pragma unroll
                    for (int e = 0; e < 32; ++e) v[e] = 0u;
                }
            };
            auto write_rows = [&](uint32_t col, void* dst, float f) {
#pragma unroll 1
                for (int c = 0; c < 2; ++c) {
                    uint32_t v[32];
                    take(col + half * 64 + c * 32, v);
                    if (live) {
                        uint4* o = reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(dst) + at + c * 32);
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            o[e] = make_uint4(pack_bf16(__uint_as_float(v[8 * e]) * f, __uint_as_float(v[8 * e + 1]) * f),
                                              pack_bf16(__uint_as_float(v[8 * e + 2]) * f, __uint_as_float(v[8 * e + 3]) * f),
                                              pack_bf16(__uint_as_float(v[8 * e + 4]) * f, __uint_as_float(v[8 * e + 5]) * f),
                                              pack_bf16(__uint_as_float(v[8 * e + 6]) * f, __uint_as_float(v[8 * e + 7]) * f));
                    }
                }
            };
            const bool cut = !u.keys && sq.nchunk > 1;
            const int unit0 = u.keys ? 0 : sq.part0 + (u.qt * H + u.h) * sq.nchunk;
            if (cut) {       // [feature][row], so that a warp's lanes write consecutive floats
                float* dst = a.dq_part + static_cast<size_t>(unit0 + u.chunk) * (BM * DH) + (half * 64) * BM + row;
#pragma unroll 1
                for (int c = 0; c < 2; ++c) {
                    uint32_t v[32];
                    take(half * 64 + c * 32, v);
#pragma unroll
                    for (int e = 0; e < 32; ++e) dst[(c * 32 + e) * BM] = __uint_as_float(v[e]);
                }
            } else {
                write_rows(0, u.keys ? (u.cached ? a.dcK : a.dlK) : a.dQ, scale);
                if (u.keys) write_rows(kColAcc2, u.cached ? a.dcV : a.dlV, 1.f);
            }
            if (u.n > 0) {
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&bar_epi);
            }
            // ---- what several units share: the heads' score gradients, the chunks' dQ; the last to arrive adds up -----
            const bool scores = u.keys && u.cached && a.dscore != nullptr;
            if (scores || cut) {
                if (scores && live) a.score_part[(static_cast<size_t>(u.h) * 2 + half) * a.score_rows + u.row0 + row] = score2.x + score2.y;
                __threadfence();
                meet();
                if (ok && tid == 0) {
                    int* counter = scores ? a.tickets + sq.stick0 + u.first / BM : a.tickets + sq.qtick0 + u.qt * H + u.h;
                    const int want = scores ? H : sq.nchunk;
                    const int t = atomicAdd(counter, 1);
                    s_flag = t == want - 1;
                    if (t == want - 1) *counter = 0;
                }
                if (ok) meet();
                if (!ok) break;
                if (s_flag) {
                    __threadfence();
                    if (scores) {
                        if (half == 0 && live) {
                            float s = 0.f;
                            for (int h = 0; h < 2 * H; ++h) s += __ldcg(a.score_part + static_cast<size_t>(h) * a.score_rows + u.row0 + row);
                            a.dscore[u.row0 + row] = s;
                        }
                    } else {
#pragma unroll 1
                        for (int c = 0; c < 2; ++c) {
                            float o[32];
#pragma unroll
                            for (int e = 0; e < 32; ++e) o[e] = 0.f;
                            for (int n = 0; n < sq.nchunk; ++n) {
                                const float* src = a.dq_part + static_cast<size_t>(unit0 + n) * (BM * DH) + (half * 64 + c * 32) * BM + row;
#pragma unroll
                                for (int e = 0; e < 32; ++e) o[e] += __ldcg(src + e * BM);
                            }
                            if (live) {
                                uint4* dst = reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(a.dQ) + at + c * 32);
#pragma unroll
                                for (int e = 0; e < 4; ++e)
                                    dst[e] = make_uint4(pack_bf16(o[8 * e] * scale, o[8 * e + 1] * scale), pack_bf16(o[8 * e + 2] * scale, o[8 * e + 3] * scale),
                                                        pack_bf16(o[8 * e + 4] * scale, o[8 * e + 5] * scale), pack_bf16(o[8 * e + 6] * scale, o[8 * e + 7] * scale));
                            }
                        }
                    }
                }
                meet();     // s_flag is free again
            }
        }
    }
    if (!ok) atomicOr(dev_status, DODO_DEV_WAIT_TIMEOUT);
    tc_fence_before();
    __syncthreads();
    if (warp == 0)
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
}

}  // namespace

BackwardTiles dodo_backward_dense_tiles() { return {BM, BM, BN}; }

int dodo_launch_backward_dense(dodo_ctx* ctx, int H, float sm_scale, const BackwardGroup& g, const BackwardArrays& a, int q_rows, int cache_rows,
                               int loc_rows, int* next_unit, cudaStream_t st) {
    const int total = g.q_blocks + g.kv_blocks;
    if (total == 0) return DODO_OK;
    BackwardMaps maps;
    memset(&maps, 0, sizeof maps);
    struct { CUtensorMap* map; const void* base; int rows; } todo[6] = {{&maps.Q, a.Q, q_rows}, {&maps.dO, a.dO, q_rows}, {&maps.cK, a.cK, cache_rows},
                                                                        {&maps.cV, a.cV, cache_rows}, {&maps.lK, a.lK, loc_rows}, {&maps.lV, a.lV, loc_rows}};
    for (auto& t : todo) {
        if (t.rows == 0) continue;
        const int rc = dodo_encode_bf16_rows(ctx, t.map, t.base, H * DH, t.rows, BN);
        if (rc != DODO_OK) return rc;
    }
    const size_t smem = static_cast<size_t>(kSmemBytes) + 1024;
    if (!ctx->backward_attr_set[4]) {
        const cudaError_t e = cudaFuncSetAttribute(backward_dense_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem));
        if (e != cudaSuccess) return dodo_check_cuda(ctx, e, "attend gradient shared-memory attribute");
        ctx->backward_attr_set[4] = true;
    }
    const int grid = total < ctx->num_sms ? total : ctx->num_sms;
    backward_dense_kernel<<<grid, kThreads, smem, st>>>(maps, g, a, H, sm_scale, next_unit, ctx->dev_status);
    return dodo_check_cuda(ctx, cudaGetLastError(), "attend gradient launch");
}
