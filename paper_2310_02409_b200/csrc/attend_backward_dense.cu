// Gradient of attention for blocks of bf16 queries, head size 64 or 128, on the 5th-generation tensor cores (formulas in
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
//   producer (a warp)  draws units and brings the stationary pairs and the streamed tiles with plain TMA tensor copies, 128-byte
//       swizzle, into seven 32 KB slots: a stationary pair takes two, a tile one.  Slots go back as tiles are consumed, so up
//       to five tiles are on their way (a load takes about 2000 cycles, a tile's whole stay about 6000).
//   issuer of S, then T (a warp)  into a score buffer of TMEM, up to two tiles ahead of the weights
//   weights (8 warps; two threads per row, 32 columns each)  P from S while T is still computed, then dS.  (16 warps spend
//       as long on a tile, be it 16 columns a thread or two tiles at a time: what a warp does per tile besides counts.)
//   issuer of the accumulating products (a warp)  P dO as soon as P is published, dS Q (dS K) behind it
//   a unit's end (4 warps; a thread per row)  moves the accumulators through the slots of the unit's own stationary pair, from
//       where another warp stores them with tensor copies (64 rows at a time; rows of a box that reaches behind the segment are
//       stored directly).  Row by row from registers a warp's store touches 32 lines, 5000 cycles a unit, and done by the
//       weights' warps the end of a unit stood in the way of the next one's tiles.
// What sets the tile period is a score buffer's round (S, P, T, dS, accumulation: about 3500 cycles): key units have two
// buffers; query units, which need no dV, a third one in its place.
// TMEM columns: [0,128) dK or dQ, [128,256) dV or score buffer 2, [256,384) and [384,512) score buffers 0 and 1; a score buffer is
// 64 columns of S and 64 of T.
// The heads' score gradients, and dQ of query units cut into chunks, are added up by kernels of their own (a fence and a ticket per
// unit cost microseconds each, and the block that joined chunks held up the launch).
// Measured: 4 x 256 queries over 717 + 1280 keys of 32 heads of 128 164 to 175 us with the inputs (power moves the clock), of 64 148
// to 154; 512 queries over 16,896 keys of 40 heads 695 to 725, 840 to 880 TFLOP/s of the seven products made, 600 to 625 of the five
// that a gradient needs; 5 to 64 queries over 8 x 269 keys 58, over 4160 keys 76.
// Every wait is bounded; a role whose wait runs out reports it and leaves, and so do the others in turn.
#include "dodo_internal.cuh"
#include "sm100_ptx.cuh"

namespace {

using namespace sm100;

constexpr int BM = 128;                 // rows of a unit
constexpr int BN = 64;                  // rows of a streamed tile
constexpr int kWeightWarps = 8, kEndWarps = 4;
constexpr int kProducer = kWeightWarps + kEndWarps, kIssueScore = kProducer + 1, kIssueAcc = kProducer + 2, kStore = kProducer + 3;
constexpr int kThreads = 32 * (kStore + 1);
constexpr int kSlots = 7, kSlotBytes = 32 * 1024;     // X1 or X2 of a unit, or Y1 and Y2 of a tile
constexpr int kMostTiles = kSlots - 2;                // tiles on their way: a pair is always resident beside them
constexpr int kRing = 8;                              // tiles' barriers (more than kMostTiles)
constexpr int kAhead = 4;                             // units announced ahead
constexpr int kXHalf = BM * 128;                      // 64 features of a stationary tile
constexpr int kYHalf = BN * 128;
constexpr int kStatBytes = BN * 8;
static_assert(2 * kXHalf == kSlotBytes && 4 * kYHalf == kSlotBytes, "slots hold head size 128");
constexpr int kOffStat = kSlots * kSlotBytes;         // [kMostTiles][64 x -lse, 64 x -D]
constexpr int kOffSync = kOffStat + kMostTiles * kStatBytes;
constexpr uint32_t kTmemCols = 512;
constexpr uint32_t kColAcc2 = 128;
__device__ __forceinline__ uint32_t score_col(int buffer) { return buffer == 2 ? 128u : 256u + 128u * buffer; }   // S; T at + 64

// barriers and the small tables behind them, at the end of the block's shared memory (all of it is dynamic, so that it starts
// at a 1024-byte boundary without padding: there is none to spare)
struct Sync {
    uint64_t x[2], xdone[2], staged[2];                  // a unit's pair: here, its slots free again, its results staged in them
    uint64_t y[kRing], yfree[kRing];                     // a tile: here, consumed
    uint64_t s[3], t[3], p[3], d[3], a[3];               // a score buffer: S, T, P, dS there; consumed
    uint64_t done, epi[2], unit[kAhead], unit_free[kAhead];     // accumulators: complete; read out (each of the two)
    int x_slot[2];           // slots of a unit's pair (first | second << 8), units with tiles counted
    int y_slot[kRing];       // a tile's slot
    int release[kRing];      // producer: slots that come back with a tile
    int unit_id[kAhead];
    uint32_t tmem;
};
constexpr int kSmemBytes = kOffSync + 512;
static_assert(sizeof(Sync) <= 512 && kSmemBytes <= 227 * 1024, "shared memory");

struct BackwardMaps { CUtensorMap Q, dO, cK, cV, lK, lV, dQ, dcK, dcV, dlK, dlV; };   // boxes of 64 elements x 64 rows, 128-byte swizzle

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
// 32 columns of the warp's 32 TMEM lanes; the caller waits (tmem_wait_ld) before it uses them
__device__ __forceinline__ void tmem_ld32_async(uint32_t a, uint32_t* v) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]),
          "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]),
          "=r"(v[16]), "=r"(v[17]), "=r"(v[18]), "=r"(v[19]), "=r"(v[20]), "=r"(v[21]), "=r"(v[22]), "=r"(v[23]),
          "=r"(v[24]), "=r"(v[25]), "=r"(v[26]), "=r"(v[27]), "=r"(v[28]), "=r"(v[29]), "=r"(v[30]), "=r"(v[31])
        : "r"(a) : "memory");
}
// (the values pass through, so that nothing that uses them moves ahead of the wait)
__device__ __forceinline__ void tmem_wait_ld(uint32_t* v) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
        : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]), "+r"(v[6]), "+r"(v[7]),
          "+r"(v[8]), "+r"(v[9]), "+r"(v[10]), "+r"(v[11]), "+r"(v[12]), "+r"(v[13]), "+r"(v[14]), "+r"(v[15]),
          "+r"(v[16]), "+r"(v[17]), "+r"(v[18]), "+r"(v[19]), "+r"(v[20]), "+r"(v[21]), "+r"(v[22]), "+r"(v[23]),
          "+r"(v[24]), "+r"(v[25]), "+r"(v[26]), "+r"(v[27]), "+r"(v[28]), "+r"(v[29]), "+r"(v[30]), "+r"(v[31]) :: "memory");
}
__device__ __forceinline__ void tmem_st16_async(uint32_t a, const uint32_t* v) {     // (the caller waits)
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
        ::"r"(a), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]),
          "r"(v[8]), "r"(v[9]), "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]) : "memory");
}
// a wait that may take long, by a warp that nobody is in a hurry for: sleeps between polls, which otherwise take issue slots
__device__ __forceinline__ bool slow_wait(uint64_t* bar, uint32_t parity) {
    for (int i = 0; i < kWaitPolls / 16; ++i) {
        if (mbar_try_wait(bar, parity)) return true;
        __nanosleep(128);
    }
    return false;
}
__device__ __forceinline__ void tma_store_2d(const CUtensorMap* map, int x, int y, uint32_t src) {
    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%1, %2}], [%3];"
                 ::"l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(src) : "memory");
}
__device__ __forceinline__ bool elect_one() {
    uint32_t p;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(p));
    return p != 0;
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
        u.l_vis = dodo_visible_local(sq.l_len, sq.l_pos0, sq.q_pos0 + u.first + u.rows - 1);
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

// The score buffers' order, which every role follows by itself: a key unit's tiles alternate between two buffers, a query unit's
// go round three; a buffer's barriers complete once per use, that of P once per use by a key unit.
struct Buffers {
    int cur = 1;
    uint32_t parity = 0u, used = 0u, key_parity = 0u;       // of the next use; whether there was one; of the next by a key unit
    __device__ __forceinline__ void next(bool keys) { cur = keys ? (cur == 0 ? 1 : 0) : (cur == 2 ? 0 : cur + 1); }
    __device__ __forceinline__ uint32_t phase() const { return (parity >> cur) & 1u; }
    __device__ __forceinline__ bool again() const { return ((used >> cur) & 1u) != 0u; }
    __device__ __forceinline__ uint32_t key_phase() const { return (key_parity >> cur) & 1u; }
    __device__ __forceinline__ void use(bool keys) {
        parity ^= 1u << cur;
        used |= 1u << cur;
        if (keys) key_parity ^= 1u << cur;
    }
};

// DH: head size; a row has kH runs of 64 features, the width of a tensor copy's box
template <int DH>
__global__ void __launch_bounds__(kThreads, 1)
backward_dense_kernel(const __grid_constant__ BackwardMaps maps, const __grid_constant__ BackwardGroup g, const BackwardArrays a, int H,
                      float scale, int* __restrict__ next_unit, int* __restrict__ dev_status) {
    constexpr int kH = DH / 64, kYTile = kH * kYHalf;
    extern __shared__ __align__(1024) unsigned char smem[];
    const uint32_t base = smem_u32(smem);
    Sync& sy = *reinterpret_cast<Sync*>(smem + kOffSync);

    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int total = g.q_blocks + g.kv_blocks;
    if ((base & 1023u) != 0u) {      // (the swizzle counts on it; a block's dynamic shared memory starts there when there is no other)
        if (tid == 0) atomicOr(dev_status, DODO_DEV_WAIT_TIMEOUT);
        return;
    }
    if (tid == 0) {
        for (int i = 0; i < 2; ++i) { mbar_init(&sy.x[i], 1); mbar_init(&sy.xdone[i], 1); mbar_init(&sy.staged[i], kEndWarps); }
        for (int i = 0; i < kRing; ++i) { mbar_init(&sy.y[i], 1); mbar_init(&sy.yfree[i], 1); }
        for (int i = 0; i < 3; ++i) {
            mbar_init(&sy.s[i], 1); mbar_init(&sy.t[i], 1); mbar_init(&sy.a[i], 1);
            mbar_init(&sy.p[i], kWeightWarps); mbar_init(&sy.d[i], kWeightWarps);
        }
        for (int i = 0; i < kAhead; ++i) { mbar_init(&sy.unit[i], 1); mbar_init(&sy.unit_free[i], 3 + kWeightWarps + kEndWarps); }
        mbar_init(&sy.done, 1);
        for (int i = 0; i < 2; ++i) mbar_init(&sy.epi[i], kEndWarps);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 0) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sy.tmem)), "r"(kTmemCols) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(&sy.tmem);
    // (launched in plain stream order: everything before this kernel on the stream has completed)

    auto shared_int = [](const int& v) { return *reinterpret_cast<const volatile int*>(&v); };
    // the unit announced as number k to a whole warp: -1 past the last, -2 when the announcement does not come
    auto unit_number = [&](int k) {
        if (!warp_wait(&sy.unit[k % kAhead], static_cast<uint32_t>(k / kAhead) & 1u)) return -2;
        return shared_int(sy.unit_id[k % kAhead]);
    };
    auto unit_read = [&](int k) {       // ... has been read by all lanes of the warp
        __syncwarp();
        if (lane == 0) mbar_arrive(&sy.unit_free[k % kAhead]);
    };

    // Barriers' phases: tile m (counted over all units of the block) uses ring entry m % kRing, the x-th unit with tiles pair
    // entry x & 1, score buffers as Buffers says.  Nobody can fall two phases behind: a ring entry is used again only after its
    // tile's accumulation, which everyone's part in the tile precedes; likewise score buffers; a pair entry only after the
    // results of the unit before in it have been stored.
    bool ok = true;
    if (warp == kProducer) {
        if (lane == 0) {
            unsigned free_slots = (1u << kSlots) - 1u;
            int m = 0, freed = 0, x = 0, xfreed = 0;       // tiles issued, consumed; units with tiles begun, stored
            unsigned pair_slots[2] = {0u, 0u};             // slots of the units begun and not stored
            auto pair_back = [&]() { free_slots |= (xfreed & 1) ? pair_slots[1] : pair_slots[0]; ++xfreed; };
            auto take_slot = [&]() {
                for (int i = 0; free_slots == 0u; ++i) {   // a tile consumed or a unit stored, whichever comes first
                    if (freed < m && mbar_try_wait(&sy.yfree[freed % kRing], static_cast<uint32_t>(freed / kRing) & 1u)) {
                        free_slots |= static_cast<unsigned>(sy.release[freed % kRing]);
                        ++freed;
                    } else if (xfreed < x && mbar_try_wait(&sy.xdone[xfreed & 1], static_cast<uint32_t>(xfreed >> 1) & 1u)) {
                        pair_back();
                    } else if (i >= kWaitPolls / 16) {
                        ok = false;
                        return 0;
                    } else {
                        __nanosleep(32);
                    }
                }
                const int s = __ffs(static_cast<int>(free_slots)) - 1;
                free_slots &= ~(1u << s);
                return s;
            };
            for (int k = 0; ok; ++k) {
                const int entry = k % kAhead;
                if (k >= kAhead && !mbar_wait(&sy.unit_free[entry], static_cast<uint32_t>(k / kAhead - 1) & 1u)) { ok = false; break; }
                const int drawn = atomicAdd(next_unit, 1);
                if (drawn == total + static_cast<int>(gridDim.x) - 1) *next_unit = 0;   // every block draws one past the end: the last puts the counter back
                const int id = drawn < total ? drawn : -1;
                *reinterpret_cast<volatile int*>(&sy.unit_id[entry]) = id;
                mbar_arrive(&sy.unit[entry]);
                if (id < 0) break;
                const Unit u = unit_of(g, H, id);
                if (u.n == 0) continue;
                const BackwardSeq& sq = g.seq[u.i];
                const int col = u.h * DH, xe = x & 1;
                while (xfreed < x - 1) {      // (the unit that had this entry has been stored)
                    if (!mbar_wait(&sy.xdone[xfreed & 1], static_cast<uint32_t>(xfreed >> 1) & 1u)) { ok = false; break; }
                    pair_back();
                }
                if (!ok) break;
                const int x1 = take_slot();
                if (!ok) break;
                const int x2 = take_slot();
                if (!ok) break;
                if (xe == 0) pair_slots[0] = (1u << x1) | (1u << x2); else pair_slots[1] = (1u << x1) | (1u << x2);
                sy.x_slot[xe] = x1 | (x2 << 8);
                const CUtensorMap* m1 = !u.keys ? &maps.Q : u.cached ? &maps.cK : &maps.lK;
                const CUtensorMap* m2 = !u.keys ? &maps.dO : u.cached ? &maps.cV : &maps.lV;
                mbar_expect_tx(&sy.x[xe], 2 * kH * kXHalf);
                for (int part = 0; part < 2 * kH; ++part) {      // (64 features, 64 rows) at a time
                    const uint32_t at = base + (part >> 1) * kXHalf + (part & 1) * (64 * 128);
                    tma_load_2d(at + x1 * kSlotBytes, m1, col + (part >> 1) * 64, u.row0 + (part & 1) * 64, &sy.x[xe]);
                    tma_load_2d(at + x2 * kSlotBytes, m2, col + (part >> 1) * 64, u.row0 + (part & 1) * 64, &sy.x[xe]);
                }
                ++x;
                for (int j = 0; j < u.n; ++j, ++m) {
                    const int slot = take_slot(), e = m % kRing;
                    if (!ok) break;
                    const Tile t = tile_of(sq, u, u.t0 + j);
                    const CUtensorMap* y1 = u.keys ? &maps.Q : t.cached ? &maps.cK : &maps.lK;
                    const CUtensorMap* y2 = u.keys ? &maps.dO : t.cached ? &maps.cV : &maps.lV;
                    const uint32_t dst = base + slot * kSlotBytes;
                    sy.y_slot[e] = slot;
                    sy.release[e] = 1 << slot;
                    mbar_expect_tx(&sy.y[e], 2 * kYTile + (u.keys ? kStatBytes : 0));
                    for (int c = 0; c < kH; ++c) {
                        tma_load_2d(dst + c * kYHalf, y1, col + 64 * c, t.row0, &sy.y[e]);
                        tma_load_2d(dst + kYTile + c * kYHalf, y2, col + 64 * c, t.row0, &sy.y[e]);
                    }
                    if (u.keys)
                        bulk_load(base + kOffStat + (m % kMostTiles) * kStatBytes,
                                  a.stats + (static_cast<size_t>(u.h) * g.stat_rows + sq.stat0 + t.first) * 2, kStatBytes, &sy.y[e]);
                }
            }
            if (!ok) {       // leave no copy in flight behind
                for (int i = max(0, m - kMostTiles); i < m; ++i) mbar_wait(&sy.y[i % kRing], static_cast<uint32_t>(i / kRing) & 1u);
                for (int i = max(0, x - 2); i < x; ++i) mbar_wait(&sy.x[i & 1], static_cast<uint32_t>(i / 2) & 1u);
            }
        }
    } else if (warp == kIssueScore) {
        // ---- S = X1 Y1^T, T = X2 Y2^T (a whole warp with an elected lane per instruction: descriptors stay in uniform registers)
        const uint32_t idesc = idesc_bf16(BN, false);
        Buffers buf;
        int m = 0, x = 0;
        for (int k = 0; ok; ++k) {
            const int id = __reduce_max_sync(0xffffffffu, unit_number(k));
            if (id < 0) { ok = id == -1; break; }
            unit_read(k);
            const int n = __reduce_max_sync(0xffffffffu, unit_of(g, H, id).n);
            const bool keys = id >= g.q_blocks;
            if (n == 0) continue;
            if (!warp_wait(&sy.x[x & 1], static_cast<uint32_t>(x / 2) & 1u)) { ok = false; break; }
            const int xs = __reduce_max_sync(0xffffffffu, shared_int(sy.x_slot[x & 1]));
            const uint64_t a1 = desc_kmajor(base + (xs & 255) * kSlotBytes), a2 = desc_kmajor(base + (xs >> 8) * kSlotBytes);
            for (int j = 0; j < n; ++j, ++m) {
                const int e = m % kRing;
                buf.next(keys);
                if (!warp_wait(&sy.y[e], static_cast<uint32_t>(m / kRing) & 1u)) { ok = false; break; }
                const int ys = __reduce_max_sync(0xffffffffu, shared_int(sy.y_slot[e]));
                const uint64_t b1 = desc_kmajor(base + ys * kSlotBytes), b2 = desc_kmajor(base + ys * kSlotBytes + kYTile);
                const uint32_t d = tmem + score_col(buf.cur);
                if (buf.again() && !warp_wait(&sy.a[buf.cur], buf.phase() ^ 1u)) { ok = false; break; }    // the P and dS before have been consumed
                tc_fence_after();
                if (elect_one()) {
#pragma unroll
                    for (int i = 0; i < DH / 16; ++i)
                        mma_bf16(d, a1 + static_cast<uint64_t>(((i / 4) * kXHalf + (i % 4) * 32) >> 4),
                                 b1 + static_cast<uint64_t>(((i / 4) * kYHalf + (i % 4) * 32) >> 4), idesc, i > 0);
                    mma_commit(&sy.s[buf.cur]);
#pragma unroll
                    for (int i = 0; i < DH / 16; ++i)
                        mma_bf16(d + 64, a2 + static_cast<uint64_t>(((i / 4) * kXHalf + (i % 4) * 32) >> 4),
                                 b2 + static_cast<uint64_t>(((i / 4) * kYHalf + (i % 4) * 32) >> 4), idesc, i > 0);
                    mma_commit(&sy.t[buf.cur]);
                }
                __syncwarp();
                buf.use(keys);
            }
            ++x;
        }
    } else if (warp == kIssueAcc) {
        // ---- acc2 += P Y2, acc1 += dS Y1 -------------------------------------------------------------------------------------
        const uint32_t idesc = idesc_bf16(DH, true);
        Buffers buf;
        int m = 0, x = 0;
        for (int k = 0; ok; ++k) {
            const int id = __reduce_max_sync(0xffffffffu, unit_number(k));
            if (id < 0) { ok = id == -1; break; }
            unit_read(k);
            const int n = __reduce_max_sync(0xffffffffu, unit_of(g, H, id).n);
            const bool keys = id >= g.q_blocks;
            if (n == 0) continue;
            for (int j = 0; j < n; ++j, ++m) {
                const int e = m % kRing;
                buf.next(keys);
                const uint32_t p = tmem + score_col(buf.cur);
                if (!warp_wait(&sy.y[e], static_cast<uint32_t>(m / kRing) & 1u)) { ok = false; break; }
                const int ys = __reduce_max_sync(0xffffffffu, shared_int(sy.y_slot[e]));
                const uint64_t y1 = desc_mnmajor(base + ys * kSlotBytes, kYHalf), y2 = desc_mnmajor(base + ys * kSlotBytes + kYTile, kYHalf);
                // (16 rows of Y = 8 columns of pairs; a row's two threads keep to their own half of the S and T columns)
                if (keys) {
                    // (the last unit's accumulators are out; where that was a query unit, its tiles in score buffer 2 are done with)
                    if (j == 0 && x >= 1 && !warp_wait(&sy.epi[1], static_cast<uint32_t>(x - 1) & 1u)) { ok = false; break; }
                    if (!warp_wait(&sy.p[buf.cur], buf.key_phase())) { ok = false; break; }
                    tc_fence_after();
                    if (elect_one()) {
#pragma unroll
                        for (int i = 0; i < BN / 16; ++i)
                            mma_bf16_ts(tmem + kColAcc2, p + (i / 2) * 32 + (i % 2) * 8, y2 + static_cast<uint64_t>((i * 2048) >> 4), idesc, j > 0 || i > 0);
                    }
                    __syncwarp();
                }
                if (j == 0 && x >= 1 && !warp_wait(&sy.epi[0], static_cast<uint32_t>(x - 1) & 1u)) { ok = false; break; }
                if (!warp_wait(&sy.d[buf.cur], buf.phase())) { ok = false; break; }
                tc_fence_after();
                if (elect_one()) {
#pragma unroll
                    for (int i = 0; i < BN / 16; ++i)
                        mma_bf16_ts(tmem, p + 64 + (i / 2) * 32 + (i % 2) * 8, y1 + static_cast<uint64_t>((i * 2048) >> 4), idesc, j > 0 || i > 0);
                    mma_commit(&sy.a[buf.cur]);
                    mma_commit(&sy.yfree[e]);
                    if (j == n - 1) mma_commit(&sy.done);
                }
                __syncwarp();
                buf.use(keys);
            }
            ++x;
        }
    } else if (warp == kStore) {
        // ---- results staged in the pair's slots go out, 64 rows of 64 features at a time -----------------------------------------
        if (lane == 0) {
            int x = 0;
            for (int k = 0; ok; ++k) {
                if (!mbar_wait(&sy.unit[k % kAhead], static_cast<uint32_t>(k / kAhead) & 1u)) { ok = false; break; }
                const int id = shared_int(sy.unit_id[k % kAhead]);
                if (id < 0) break;
                mbar_arrive(&sy.unit_free[k % kAhead]);
                const Unit u = unit_of(g, H, id);
                if (u.n == 0) continue;
                const int xe = x & 1;
                if (!slow_wait(&sy.staged[xe], static_cast<uint32_t>(x >> 1) & 1u)) { ok = false; break; }
                if (u.keys || g.seq[u.i].nchunk == 1) {
                    const int xs = shared_int(sy.x_slot[xe]);
                    const CUtensorMap* o1 = !u.keys ? &maps.dQ : u.cached ? &maps.dcK : &maps.dlK;
                    const CUtensorMap* o2 = u.cached ? &maps.dcV : &maps.dlV;
                    for (int box = 0; box < u.rows / 64; ++box)
                        for (int c = 0; c < kH; ++c) {
                            const uint32_t at = base + c * kXHalf + box * (64 * 128);
                            tma_store_2d(o1, u.h * DH + c * 64, u.row0 + box * 64, at + (xs & 255) * kSlotBytes);
                            if (u.keys) tma_store_2d(o2, u.h * DH + c * 64, u.row0 + box * 64, at + (xs >> 8) * kSlotBytes);
                        }
                    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
                    asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
                }
                mbar_arrive(&sy.xdone[xe]);
                ++x;
            }
            asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
        }
    } else if (warp < kWeightWarps) {
        // ---- weights -----------------------------------------------------------------------------------------------------------
        const int row = tid & (BM - 1), half = tid >> 7;        // 32 of a tile's columns
        const uint32_t lane_sel = static_cast<uint32_t>((warp & 3) * 32) << 16;
        const float scale2 = scale * 1.4426950408889634f;
        const float2 c2 = make_float2(scale2, scale2);
        Buffers buf;
        int m = 0;
        for (int k = 0; ok; ++k) {
            const int id = unit_number(k);
            if (id < 0) { ok = id == -1; break; }
            unit_read(k);
            const Unit u = unit_of(g, H, id);
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
            // query unit: positions of the thread's 32 columns of a tile, one a lane, fetched a tile ahead
            auto column_pos = [&](int t) {
                const Tile s = tile_of(sq, u, t);
                const int c = half * 32 + lane;
                if (c >= s.rows) return 0x7fffffff;
                return s.cached ? __ldg(a.cache_pos + s.row0 + c) : sq.l_pos0 + s.first + c;
            };
            int next_pos = 0;
            if (!u.keys && u.n > 0) next_pos = column_pos(u.t0);


            for (int j = 0; j < u.n; ++j, ++m) {
                buf.next(u.keys);
                const int e = m % kRing, b = buf.cur;
                const uint32_t ts = tmem + score_col(b) + half * 32 + lane_sel;
                uint32_t sv[32], pk[16];
                if (u.keys) {
                    if (!warp_wait(&sy.s[b], buf.phase())) { ok = false; break; }
                    // (this warp sees the tile's own barrier too: the statistics came with it, and rows may have to be cleared)
                    if (!warp_wait(&sy.y[e], static_cast<uint32_t>(m / kRing) & 1u)) { ok = false; break; }
                    const float4* nl = reinterpret_cast<const float4*>(smem + kOffStat + (m % kMostTiles) * kStatBytes) + half * 8;
                    const float4* nd = nl + 16;
                    const int first = (u.t0 + j) * BN, rows = min(BN, sq.tq - first), q0 = sq.q_pos0 + first;
                    const bool test = edge > q0 || rows < BN;
                    // the row's key is seen from column my_pos - q0 on; that difference may need 33 bits (a nugget's position is any
                    // number), so the comparison comes first and 0 to BN is what is left of it
                    const int from = my_pos <= q0 ? 0 : static_cast<int>(min(static_cast<unsigned>(my_pos) - static_cast<unsigned>(q0), static_cast<unsigned>(BN)));
                    const int c_lo = from - half * 32, c_hi = rows - half * 32;
                    if (rows < BN) {   // rows behind the sequence's queries must not reach the products (both score products done with them)
                        if (!warp_wait(&sy.t[b], buf.phase())) { ok = false; break; }
                        unsigned char* y = smem + shared_int(sy.y_slot[e]) * kSlotBytes;
                        for (int i = tid; i < (BN - rows) * 16 * kH; i += 32 * kWeightWarps) {     // 16 bytes of a row of the pair
                            const int r = rows + i / (16 * kH), piece = i % (16 * kH);
                            *reinterpret_cast<uint4*>(y + (piece >> 3) * kYHalf + r * 128 + (piece & 7) * 16) = make_uint4(0, 0, 0, 0);
                        }
                        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    }
                    tc_fence_after();
                    tmem_ld32_async(ts, sv);
                    tmem_wait_ld(sv);
                    float2 p[16];
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const float4 l4 = nl[i / 2];
                        const float2 z = __ffma2_rn(make_float2(__uint_as_float(sv[2 * i]), __uint_as_float(sv[2 * i + 1])), c2,
                                                    (i & 1) == 0 ? make_float2(l4.x, l4.y) : make_float2(l4.z, l4.w));
                        p[i] = make_float2(ex2_approx(z.x), ex2_approx(z.y));
                    }
                    if (test) {
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            if (2 * i < c_lo || 2 * i >= c_hi) p[i].x = 0.f;
                            if (2 * i + 1 < c_lo || 2 * i + 1 >= c_hi) p[i].y = 0.f;
                        }
                    }
#pragma unroll
                    for (int i = 0; i < 16; ++i) pk[i] = pack_bf16(p[i].x, p[i].y);
                    tmem_st16_async(ts, pk);
                    asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&sy.p[b]);
                    if (!warp_wait(&sy.t[b], buf.phase())) { ok = false; break; }
                    tc_fence_after();
                    tmem_ld32_async(ts + 64, sv);
                    tmem_wait_ld(sv);
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const float4 d4 = nd[i / 2];
                        p[i] = __fmul2_rn(p[i], __fadd2_rn(make_float2(__uint_as_float(sv[2 * i]), __uint_as_float(sv[2 * i + 1])),
                                                          (i & 1) == 0 ? make_float2(d4.x, d4.y) : make_float2(d4.z, d4.w)));
                    }
                    if (test) {         // (0 times a NaN of a masked pair)
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            if (2 * i < c_lo || 2 * i >= c_hi) p[i].x = 0.f;
                            if (2 * i + 1 < c_lo || 2 * i + 1 >= c_hi) p[i].y = 0.f;
                        }
                    }
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        score2 = __fadd2_rn(score2, p[i]);
                        pk[i] = pack_bf16(p[i].x, p[i].y);
                    }
                } else {
                    const int cpos = next_pos;
                    if (j + 1 < u.n) next_pos = column_pos(u.t0 + j + 1);
                    const int far = __reduce_max_sync(0xffffffffu, cpos);
                    const bool test = far > edge;
                    const float2 l2 = make_float2(nlse, nlse), d2 = make_float2(ndelta, ndelta);
                    if (!warp_wait(&sy.t[b], buf.phase())) { ok = false; break; }     // (T is issued behind S by the same thread)
                    tc_fence_after();
                    uint32_t tv[32];
                    tmem_ld32_async(ts, sv);
                    tmem_ld32_async(ts + 64, tv);
                    tmem_wait_ld(sv);
                    tmem_wait_ld(tv);
                    float2 d[16];
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const float2 z = __ffma2_rn(make_float2(__uint_as_float(sv[2 * i]), __uint_as_float(sv[2 * i + 1])), c2, l2);
                        d[i] = __fmul2_rn(make_float2(ex2_approx(z.x), ex2_approx(z.y)),
                                          __fadd2_rn(make_float2(__uint_as_float(tv[2 * i]), __uint_as_float(tv[2 * i + 1])), d2));
                    }
                    if (test) {
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            if (__shfl_sync(0xffffffffu, cpos, 2 * i) > my_pos) d[i].x = 0.f;
                            if (__shfl_sync(0xffffffffu, cpos, 2 * i + 1) > my_pos) d[i].y = 0.f;
                        }
                    }
#pragma unroll
                    for (int i = 0; i < 16; ++i) pk[i] = pack_bf16(d[i].x, d[i].y);
                    // Keys that some query of the tile does not see, and rows behind the segment: dS is 0 there, but 0 times
                    // what the row holds need not be.  Rows behind the segment are zeroed, NaN and infinities of the others
                    // replaced by 0 (a query that sees such a key has a NaN in dS).  Each warp takes 8 rows of its half.
                    if (far > sq.q_pos0 + u.first) {
                        if (!warp_wait(&sy.y[e], static_cast<uint32_t>(m / kRing) & 1u)) { ok = false; break; }
                        const int rows = tile_of(sq, u, u.t0 + j).rows;
                        const int r = half * 32 + (warp & 3) * 8 + (lane >> 2), piece = lane & 3;
                        uint4* y = reinterpret_cast<uint4*>(smem + shared_int(sy.y_slot[e]) * kSlotBytes + (piece * kH / 4) * kYHalf + r * 128 + (piece * kH % 4) * 32);
#pragma unroll
                        for (int i = 0; i < 2 * kH; ++i) {
                            const uint4 w = y[i];
                            y[i] = r >= rows ? make_uint4(0, 0, 0, 0) : make_uint4(finite2(w.x), finite2(w.y), finite2(w.z), finite2(w.w));
                        }
                        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    }
                }
                tmem_st16_async(ts + 64, pk);
                asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&sy.d[b]);
                buf.use(u.keys);
            }
            if (!ok) break;
            if (live && u.keys && u.cached && a.dscore != nullptr)
                a.score_part[(static_cast<size_t>(u.h) * 2 + half) * a.score_rows + u.row0 + row] = score2.x + score2.y;
        }
    } else {
        // ---- the end of a unit: a thread takes its row of the accumulators, 32 columns at a time -------------------------------------
        const int row = tid & (BM - 1);
        const uint32_t lane_sel = static_cast<uint32_t>((warp & 3) * 32) << 16;
        int x = 0;
        for (int k = 0; ok; ++k) {
            const int id = unit_number(k);
            if (id < 0) { ok = id == -1; break; }
            unit_read(k);
            const Unit u = unit_of(g, H, id);
            const BackwardSeq& sq = g.seq[u.i];
            const bool live = row < u.rows;
            const size_t at = (static_cast<size_t>(u.row0 + row) * H + u.h) * DH;
            const bool cut = !u.keys && sq.nchunk > 1;
            const bool some = (row & ~31) < u.rows;      // the warp has live rows (a short query block fills one of four)
            const size_t unit0 = cut ? static_cast<size_t>(sq.part0 + (u.qt * H + u.h) * sq.nchunk) : 0u;
            float* const mine = a.dq_part + (unit0 + u.chunk) * (BM * DH) + row;     // [feature][row]: a warp's lanes write consecutive floats
            void* const out[2] = {u.keys ? (u.cached ? a.dcK : a.dlK) : a.dQ, u.cached ? a.dcV : a.dlV};
            const int outs = u.keys ? 2 : 1;
            if (u.n > 0) {
                if (__all_sync(0xffffffffu, slow_wait(&sy.done, static_cast<uint32_t>(x) & 1u)) == 0) { ok = false; break; }
                tc_fence_after();
                const int xs = shared_int(sy.x_slot[x & 1]);
                const bool boxed = (row | 63) < u.rows;       // all 64 rows of the row's box are live
                // dV first: its accumulation is the first of the next unit's
                for (int o = 1; o >= 0; --o) {
                    if (o < outs) {
                        const float f = o == 0 ? scale : 1.f;
                        unsigned char* const stage = smem + ((xs >> (8 * o)) & 255) * kSlotBytes + row * 128;     // swizzled halves of 64 features
                        __nv_bfloat16* const direct = static_cast<__nv_bfloat16*>(out[o]) + at;
                        uint32_t va[32], vb[32];
                        auto put = [&](int c, const uint32_t* v) {
                            if (cut) {
                                if (some) {
#pragma unroll
                                    for (int e = 0; e < 32; ++e) mine[(c * 32 + e) * BM] = __uint_as_float(v[e]);
                                }
                                return;
                            }
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const uint4 q = make_uint4(pack_bf16(__uint_as_float(v[8 * e]) * f, __uint_as_float(v[8 * e + 1]) * f),
                                                           pack_bf16(__uint_as_float(v[8 * e + 2]) * f, __uint_as_float(v[8 * e + 3]) * f),
                                                           pack_bf16(__uint_as_float(v[8 * e + 4]) * f, __uint_as_float(v[8 * e + 5]) * f),
                                                           pack_bf16(__uint_as_float(v[8 * e + 6]) * f, __uint_as_float(v[8 * e + 7]) * f));
                                if (boxed) *reinterpret_cast<uint4*>(stage + (c >> 1) * kXHalf + ((((c & 1) * 4 + e) ^ (row & 7)) << 4)) = q;
                                else if (live) *reinterpret_cast<uint4*>(direct + c * 32 + 8 * e) = q;
                            }
                        };
                        const uint32_t col = tmem + o * kColAcc2 + lane_sel;
                        tmem_ld32_async(col, va);
#pragma unroll 1
                        for (int c = 0; c < 2 * kH; c += 2) {  // the next columns are on their way while these are put away
                            tmem_wait_ld(va);
                            tmem_ld32_async(col + (c + 1) * 32, vb);
                            put(c, va);
                            tmem_wait_ld(vb);
                            if (c + 2 < 2 * kH) tmem_ld32_async(col + 64, va);
                            put(c + 1, vb);
                        }
                    }
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&sy.epi[o]);
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0) mbar_arrive(&sy.staged[x & 1]);
                ++x;
            } else if (cut) {             // an empty chunk's partial
                if (some)
                    for (int e = 0; e < DH; ++e) mine[e * BM] = 0.f;
            } else if (live) {            // nothing was summed: zeros
                for (int o = 0; o < outs; ++o)
                    for (int e = 0; e < DH / 8; ++e) *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(out[o]) + at + 8 * e) = make_uint4(0, 0, 0, 0);
            }
        }
    }
    if (!ok) atomicOr(dev_status, DODO_DEV_WAIT_TIMEOUT);
    tc_fence_before();
    __syncthreads();
    if (warp == 0)
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
}

// dQ of query units cut into chunks of the key list: their partial tiles added up in chunk order, 8 features of 128 queries a block.
// (A kernel of its own: done by the last chunk's block, which has other units to go on with, it held up one block for 50 us.)
template <int DH>
__global__ void __launch_bounds__(BM)
backward_join_kernel(const BackwardArrays a, const __grid_constant__ BackwardGroup g, int H, float scale) {
    const BackwardSeq& sq = g.seq[blockIdx.z];
    const int unit = static_cast<int>(blockIdx.x), qt = unit / H, h = unit % H, q = qt * BM + static_cast<int>(threadIdx.x), c = 8 * static_cast<int>(blockIdx.y);
    dodo_grid_dependency_sync();
    if (sq.nchunk == 1 || q >= sq.tq) return;
    const float* const src = a.dq_part + static_cast<size_t>(sq.part0 + unit * sq.nchunk) * (BM * DH) + c * BM + threadIdx.x;
    float o[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = 0.f;
    for (int n = 0; n < sq.nchunk; n += 4) {        // four chunks' loads in flight together
        float v[4][8];
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int e = 0; e < 8; ++e) v[k][e] = __ldcg(src + static_cast<size_t>(min(n + k, sq.nchunk - 1)) * (BM * DH) + e * BM);
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int e = 0; e < 8; ++e) o[e] += n + k < sq.nchunk ? v[k][e] : 0.f;
    }
    *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(a.dQ) + (static_cast<size_t>(sq.q_row0 + q) * H + h) * DH + c) =
        make_uint4(pack_bf16(o[0] * scale, o[1] * scale), pack_bf16(o[2] * scale, o[3] * scale), pack_bf16(o[4] * scale, o[5] * scale),
                   pack_bf16(o[6] * scale, o[7] * scale));
}

}  // namespace

BackwardTiles dodo_backward_dense_tiles() { return {BM, BM, BN}; }

template <int DH>
static int launch_dense(dodo_ctx* ctx, int slot, int H, float sm_scale, const BackwardGroup& g, const BackwardArrays& a, int q_rows, int cache_rows,
                        int loc_rows, int* next_unit, cudaStream_t st) {
    const int total = g.q_blocks + g.kv_blocks;
    if (total == 0) return DODO_OK;
    BackwardMaps maps;
    memset(&maps, 0, sizeof maps);
    struct { CUtensorMap* map; const void* base; int rows; } todo[11] = {
        {&maps.Q, a.Q, q_rows},        {&maps.dO, a.dO, q_rows},        {&maps.dQ, a.dQ, q_rows},        {&maps.cK, a.cK, cache_rows},
        {&maps.cV, a.cV, cache_rows},  {&maps.dcK, a.dcK, cache_rows},  {&maps.dcV, a.dcV, cache_rows},  {&maps.lK, a.lK, loc_rows},
        {&maps.lV, a.lV, loc_rows},    {&maps.dlK, a.dlK, loc_rows},    {&maps.dlV, a.dlV, loc_rows}};
    for (auto& t : todo) {
        if (t.rows == 0) continue;
        const int rc = dodo_encode_bf16_rows(ctx, t.map, t.base, H * DH, t.rows, BN);
        if (rc != DODO_OK) return rc;
    }
    const size_t smem = static_cast<size_t>(kSmemBytes);
    if (!ctx->backward_attr_set[slot]) {
        const cudaError_t e = cudaFuncSetAttribute(backward_dense_kernel<DH>, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem));
        if (e != cudaSuccess) return dodo_check_cuda(ctx, e, "attend gradient shared-memory attribute");
        ctx->backward_attr_set[slot] = true;
    }
    const int grid = total < ctx->num_sms ? total : ctx->num_sms;
    backward_dense_kernel<DH><<<grid, kThreads, smem, st>>>(maps, g, a, H, sm_scale, next_unit, ctx->dev_status);
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return dodo_check_cuda(ctx, e, "attend gradient launch");
    int units = 0;      // most (query tile, head) units of a sequence whose units are cut
    for (int i = 0; i < g.nseq; ++i) {
        const int n = g.seq[i].nchunk > 1 ? (g.seq[i].tq + BM - 1) / BM * H : 0;
        units = units > n ? units : n;
    }
    if (units > 0) {
        e = dodo_launch_dependent(backward_join_kernel<DH>, dim3(static_cast<unsigned>(units), DH / 8, static_cast<unsigned>(g.nseq)), dim3(BM), 0, st, a, g, H, sm_scale);
        if (e != cudaSuccess) return dodo_check_cuda(ctx, e, "attend gradient launch");
    }
    return dodo_launch_backward_scores(ctx, g, a, 2 * H, st);
}

int dodo_launch_backward_dense(dodo_ctx* ctx, int H, int dh, float sm_scale, const BackwardGroup& g, const BackwardArrays& a, int q_rows,
                               int cache_rows, int loc_rows, int* next_unit, cudaStream_t st) {
    return dh == 128 ? launch_dense<128>(ctx, 2, H, sm_scale, g, a, q_rows, cache_rows, loc_rows, next_unit, st)
                     : launch_dense<64>(ctx, 3, H, sm_scale, g, a, q_rows, cache_rows, loc_rows, next_unit, st);
}
