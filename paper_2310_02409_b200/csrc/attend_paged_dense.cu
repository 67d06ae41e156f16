// Attention of many rows over a paged cache on the 5th-generation tensor cores (bf16; rows = query tokens x query heads of a KV head).
// 4 x 256 queries of 32 heads on 8 KV heads over 717 + 1280 keys: 43.7 us, 718 TFLOP/s; 512 queries of 40 heads over 16,896 keys: 164 to
// 179 us by the clock, 0.98 to 1.06 PFLOP/s (call after call, at the power limit, 214: 0.81); with heads of 64 the two take 36 us (435 TFLOP/s)
// and 132 (661): the same rounds for half the products.  Bound by a tile's round, scores -> softmax -> weights -> values: about 3000 cycles for 128
// keys of 256 rows, of which the matrix products are 2048; short lists by a unit's begin and end, about three rounds.
//
// Work is counted in slots, one per tile of 128 keys of a unit (sequence, KV head, tile of rows) and, where units differ, a few ahead of
// them for the unit's begin and end; the units are laid end to end and
// thread block c of G, one per SM, takes the slots [c T / G, (c+1) T / G) whatever units they fall in.  A unit that a block boundary
// cuts is finished through partial results in the workspace; the last of its blocks to arrive joins them.  Nobody waits for anybody.
//
// A block holds two score streams: S = Q K^T [128 rows x 128 keys] of stream s in tensor-memory columns [128 s, 128 s + 128), its
// P (bf16 pairs) over the first 64 of them, O at [256 + DH s, ...).  With more than 128 rows the streams are the two halves of a tile
// of 256 rows, which share every K and V tile (half the operand traffic from L2); with fewer they take the key tiles in turn and are
// added at the end.  While one stream's softmax runs, the tensor core works for the other.  Roles, each a warp or more:
//   scout (warp 8)  walks the key list: 32 lanes look four keys each up (page, position), skip tiles that no query sees, and leave a
//       tile's rows and positions in shared memory.
//   producer (warp 10)  brings K and V by tensor copies with the 128-byte swizzle, a box as many rows high as the power of two that
//       divides the page's (a page's rows lie side by side), up to the tile's 128; where that is less than eight, four rows at a time by
//       gather copies (tile::gather4), about 10,000 cycles a tile: the 512 queries in pages of one row 367 us, the four
//       chunks in pages of five 59.  Local tokens are boxes of 128.
//   cleaner (warp 11)  writes zeros over V rows of keys that are not there or that no query of the tile sees.
//   matrix issuer (warp 9)  the whole warp walks the same list, one elected lane issues: every operand of an instruction then lies in
//       uniform registers.  Per tile and stream O += P V, in halves of 64 keys, then S = Q K^T of the stream's next tile.
//   softmax (warps 0-3 and 4-7)  a thread is a row: its 128 scores in registers, a reference maximum and the sum in 32 bits.  A tile's
//       weights are made with the reference of the tiles before while its own maximum is found beside them; only where a score passes the
//       reference by 2^24 (the first tile among these) is the tile begun again and O rescaled in tensor memory.  The first 64 keys' weights
//       go to the matrix unit ahead of the others'.  Weights are rounded to bf16 for P V (the sum is not): at most 2^-8 of each, the rounding
//       of the result itself.  When a unit ends, the next one's Q is brought before its results go out.
// Masked scores are -infinity; in the product their weight 0 times a NaN or an infinity of V is a NaN all the same (keys that some
// rows of a tile see and others do not), so results that are not finite are summed again on the FMA units over what their row sees.
// Every wait is bounded: on time-out a role leaves its loop, the status word is set, tensor memory is freed.
#include "paged.cuh"
#include "sm100_ptx.cuh"

namespace {

using namespace sm100;
using namespace dodo_paged;

constexpr int BM = 128, BN = 128;
constexpr int kSoftmaxWarps = 8, kThreads = 32 * (kSoftmaxWarps + 4);
constexpr int kPosReaders = kSoftmaxWarps + 3;      // softmax, issuer, producer, cleaner
// Registers of a thread: the launch's 168 a thread (384 threads), shared out anew between two warpgroups of softmax threads (a row's 128
// scores) and the one of the others: 216 + 216 + 72 = 3 x 168
constexpr int kSoftmaxRegs = 216, kOtherRegs = 72;
constexpr int kPosSlots = 4;
// A row's reference maximum moves only when a score passes it by this many octaves: weights of up to 2^24 cost no digit in bf16 or fp32
constexpr float kRescaleStep = 24.f;
enum { kMasked = 1, kEnd = 2, kLocal = 4, kHoles = 8 };     // of a tile; kHoles: some of its keys are not there or seen by nobody

template <int DH, int TILES>
struct Layout {
    static constexpr int kHalves = DH / 64;
    static constexpr int kTile = BN * DH * 2;                 // bytes of 128 rows
    static constexpr int kHalf = BN * 128;                    // 64 columns of them
    static constexpr int kKStages = TILES == 1 || DH == 64 ? 3 : 2, kVStages = TILES == 1 && DH == 128 ? 2 : kKStages;
    static constexpr int kOffK = TILES * kTile, kOffV = kOffK + kKStages * kTile, kOffPos = kOffV + kVStages * kTile;
    static constexpr int kOffXch = kOffPos + 2 * kPosSlots * BN * 4;      // maxima and sums that the streams of one tile of rows exchange
    static constexpr int kOffOut = kOffXch + (TILES == 1 ? 2 * 2 * BM * 4 : 0);      // results on their way out: 32 rows x 32 features a warp
    static constexpr int kBytes = kOffOut + kSoftmaxWarps * 2048;
    static constexpr int kRows = TILES * BM;
    static constexpr size_t kPartFloats = static_cast<size_t>(kRows) * (DH + 2);
};

struct DenseShare {
    int total;                      // slots
    int ahead;                      // slots of a unit ahead of its tiles', for what its begin and end cost
    int whole;                      // slots that a block takes or leaves together: 1, or a unit's where blocks take whole units
    int slot0[DODO_GROUP + 1];      // first slot of each sequence
    int nt[DODO_GROUP];             // tiles of a unit of the sequence
    int tiles[DODO_GROUP];          // tiles of rows
};

__device__ __forceinline__ bool elect_one() {
    uint32_t p;
    asm volatile("{\n\t.reg .pred P;\n\telect.sync _|P, 0xffffffff;\n\tselp.u32 %0, 1, 0, P;\n\t}" : "=r"(p));
    return p != 0;
}
__device__ __forceinline__ void gather4(uint32_t dst, const CUtensorMap* map, int x, int4 r, uint64_t* bar) {
    asm volatile(
        "cp.async.bulk.tensor.2d.shared::cluster.global.tile::gather4.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5, %6}], [%7];"
        ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(r.x), "r"(r.y), "r"(r.z), "r"(r.w), "r"(smem_u32(bar))
        : "memory");
}
#define DODO_REGS64(v) \
    "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]), "+r"(v[6]), "+r"(v[7]), "+r"(v[8]), "+r"(v[9]), "+r"(v[10]), "+r"(v[11]), \
    "+r"(v[12]), "+r"(v[13]), "+r"(v[14]), "+r"(v[15]), "+r"(v[16]), "+r"(v[17]), "+r"(v[18]), "+r"(v[19]), "+r"(v[20]), "+r"(v[21]), "+r"(v[22]), \
    "+r"(v[23]), "+r"(v[24]), "+r"(v[25]), "+r"(v[26]), "+r"(v[27]), "+r"(v[28]), "+r"(v[29]), "+r"(v[30]), "+r"(v[31]), "+r"(v[32]), "+r"(v[33]), \
    "+r"(v[34]), "+r"(v[35]), "+r"(v[36]), "+r"(v[37]), "+r"(v[38]), "+r"(v[39]), "+r"(v[40]), "+r"(v[41]), "+r"(v[42]), "+r"(v[43]), "+r"(v[44]), \
    "+r"(v[45]), "+r"(v[46]), "+r"(v[47]), "+r"(v[48]), "+r"(v[49]), "+r"(v[50]), "+r"(v[51]), "+r"(v[52]), "+r"(v[53]), "+r"(v[54]), "+r"(v[55]), \
    "+r"(v[56]), "+r"(v[57]), "+r"(v[58]), "+r"(v[59]), "+r"(v[60]), "+r"(v[61]), "+r"(v[62]), "+r"(v[63])
// the wait for a tmem_ld64: it names the registers, so that nothing reads them ahead of it
__device__ __forceinline__ void tmem_wait64(uint32_t* v) { asm volatile("tcgen05.wait::ld.sync.aligned;" : DODO_REGS64(v)::"memory"); }
// 64 columns of this warp's 32 lanes
__device__ __forceinline__ void tmem_ld64(uint32_t taddr, uint32_t* v) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x64.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, "
        "%32, %33, %34, %35, %36, %37, %38, %39, %40, %41, %42, %43, %44, %45, %46, %47, "
        "%48, %49, %50, %51, %52, %53, %54, %55, %56, %57, %58, %59, %60, %61, %62, %63}, [%64];"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]), "=r"(v[10]),
          "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]), "=r"(v[16]), "=r"(v[17]), "=r"(v[18]), "=r"(v[19]), "=r"(v[20]),
          "=r"(v[21]), "=r"(v[22]), "=r"(v[23]), "=r"(v[24]), "=r"(v[25]), "=r"(v[26]), "=r"(v[27]), "=r"(v[28]), "=r"(v[29]), "=r"(v[30]),
          "=r"(v[31]), "=r"(v[32]), "=r"(v[33]), "=r"(v[34]), "=r"(v[35]), "=r"(v[36]), "=r"(v[37]), "=r"(v[38]), "=r"(v[39]), "=r"(v[40]),
          "=r"(v[41]), "=r"(v[42]), "=r"(v[43]), "=r"(v[44]), "=r"(v[45]), "=r"(v[46]), "=r"(v[47]), "=r"(v[48]), "=r"(v[49]), "=r"(v[50]),
          "=r"(v[51]), "=r"(v[52]), "=r"(v[53]), "=r"(v[54]), "=r"(v[55]), "=r"(v[56]), "=r"(v[57]), "=r"(v[58]), "=r"(v[59]), "=r"(v[60]),
          "=r"(v[61]), "=r"(v[62]), "=r"(v[63])
        : "r"(taddr)
        : "memory");
}
__device__ __forceinline__ float max3(float a, float b, float c) {
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}

// a wait of the whole warp: the same answer in every lane
__device__ __forceinline__ bool warp_wait(uint64_t* bar, uint32_t parity) { return __all_sync(0xffffffffu, mbar_wait(bar, parity)); }
// barrier of the softmax threads that tells each whether any of them said so
__device__ __forceinline__ bool any_softmax(bool mine) {
    uint32_t r;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\tbar.red.or.pred q, 1, 256, p;\n\tselp.u32 %0, 1, 0, q;\n\t}" : "=r"(r) : "r"(mine ? 1u : 0u) : "memory");
    return r != 0u;
}

// the first slot of block c of G, and, where shares are single slots, the block whose range holds slot x
__device__ __forceinline__ int block_start(const DenseShare& w, int G, int c) { return static_cast<int>(static_cast<long long>(c) * (w.total / w.whole) / G) * w.whole; }
__device__ __forceinline__ int block_of(int T, int G, int x) { return static_cast<int>(((static_cast<long long>(x) + 1) * G - 1) / T); }

// A unit's share of a block: its rows, its key list, the tiles [t0, t1) of it
struct Segment {
    int b, head, tile;
    int first_slot, nt, t0, t1;     // slot of the unit's first tile; tiles of the unit
    int rows, r0;                   // rows of this tile of rows and the first
    int min_pos, last_pos;          // positions of its first and last row
    int l_vis, c_tiles;             // local tokens that its last row sees; tiles of the cache's rows, which the local ones follow
};
// walks the segments of slots [x, end)
__device__ __forceinline__ bool next_segment(const PagedGroup& g, const PagedArrays& a, const DenseShare& w, int tile_rows, int& x, int end, Segment& q) {
    if (x >= end) return false;
    int lo = 0, hi = g.nseq;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (w.slot0[mid] <= x) lo = mid; else hi = mid;
    }
    const PagedSeq& s = g.seq[lo];
    const int off = x - w.slot0[lo], unit = off / (w.nt[lo] + w.ahead), begin = x - (off - unit * (w.nt[lo] + w.ahead));
    if (end - begin <= w.ahead) return false;       // the next block has its first tile
    q.b = lo;
    q.tile = unit % w.tiles[lo];
    q.head = unit / w.tiles[lo];
    q.nt = w.nt[lo];
    q.first_slot = begin + w.ahead;
    q.t0 = max(0, x - q.first_slot);
    q.t1 = min(q.nt, end - q.first_slot);
    q.r0 = q.tile * tile_rows;
    q.rows = min(tile_rows, s.tq * a.group - q.r0);
    q.min_pos = s.q_pos0 + token_of(a, q.r0);
    q.last_pos = s.q_pos0 + token_of(a, q.r0 + q.rows - 1);
    q.c_tiles = (s.c_len + BN - 1) / BN;
    q.l_vis = dodo_visible_local(s.l_len, s.l_pos0, q.last_pos);
    x = q.first_slot + q.t1;
    return true;
}

// a hint to L2 for row r of the segment's Q
template <int DH>
__device__ __forceinline__ void hint_row(const PagedArrays& a, const PagedSeq& s, const Segment& q, int r) {
    if (r >= q.rows) return;
    const __nv_bfloat16* const p = static_cast<const __nv_bfloat16*>(a.Q) + out_row(a, s, q.head, q.r0 + r) * DH;
#pragma unroll
    for (int c = 0; c < DH; c += 64) asm volatile("prefetch.global.L2 [%0];" ::"l"(p + c));
}

// hints for the positions, K and V rows of the segment's first tile: a warp, four keys a lane
template <int DH>
__device__ __forceinline__ void hint_keys(const PagedArrays& a, const PagedSeq& s, const Segment& q, int lane) {
    const size_t pitch = static_cast<size_t>(a.Hkv) * DH;
    const int v = q.t0 * BN + 4 * lane;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int entry = page_entry(a, s, v + e, s.c_len);
        if (q.t0 >= q.c_tiles || v + e >= s.c_len || static_cast<unsigned>(entry) >= static_cast<unsigned>(a.pages)) continue;
        const int row = entry * a.page + (v + e - page_of(a, v + e) * a.page);
        const size_t at = static_cast<size_t>(row) * pitch + static_cast<size_t>(q.head) * DH;
        if (e == 0) asm volatile("prefetch.global.L2 [%0];" ::"l"(a.pos + row));
#pragma unroll
        for (int c = 0; c < DH; c += 64) {
            asm volatile("prefetch.global.L2 [%0];" ::"l"(static_cast<const __nv_bfloat16*>(a.cK) + at + c));
            asm volatile("prefetch.global.L2 [%0];" ::"l"(static_cast<const __nv_bfloat16*>(a.cV) + at + c));
        }
    }
}

template <int DH, int TILES>
__global__ void __launch_bounds__(kThreads, 1)
attend_paged_dense_kernel(const __grid_constant__ PagedBoxes maps, const __grid_constant__ PagedGroup g, const __grid_constant__ PagedArrays a,
                          const __grid_constant__ DenseShare work) {
    using L = Layout<DH, TILES>;
    extern __shared__ unsigned char smem_raw[];
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    unsigned char* const base_ptr = smem_raw + (base - smem_u32(smem_raw));
    __shared__ __align__(8) uint64_t bar_q, bar_o, bar_drain, bar_s[2], bar_p[2][2], bar_kfull[L::kKStages], bar_kfree[L::kKStages], bar_vfull[L::kVStages],
        bar_vfree[L::kVStages], bar_vclean[L::kVStages], bar_posfull[kPosSlots], bar_posfree[kPosSlots];
    __shared__ uint32_t s_tmem;
    __shared__ int s_kind[kPosSlots], s_last;
    int* const s_pos = reinterpret_cast<int*>(base_ptr + L::kOffPos);
    int* const s_row = s_pos + kPosSlots * BN;

    const int tid = static_cast<int>(threadIdx.x), lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
    const int T = work.total, G = static_cast<int>(gridDim.x), bid = static_cast<int>(blockIdx.x);
    const int slot_end = block_start(work, G, bid + 1);
    int x = block_start(work, G, bid);
    Segment q;

    // Hints to L2 while the block sets itself up: the rows of Q that it begins with (behind the first keys of all blocks they would come
    // late), and, as their look-up is a chain of reads from memory, positions and rows of the first keys.
    if (warp <= kSoftmaxWarps) {
        int ahead = x;
        if (next_segment(g, a, work, L::kRows, ahead, slot_end, q)) {
            const PagedSeq& s = g.seq[q.b];
            if (warp < kSoftmaxWarps) {
                hint_row<DH>(a, s, q, tid);
            } else {
                dodo_grid_dependency_sync();
                hint_keys<DH>(a, s, q, lane);
            }
        }
    }
    if (tid == 0) {
        mbar_init(&bar_q, kSoftmaxWarps);
        mbar_init(&bar_o, 1);
        mbar_init(&bar_drain, 1);
        for (int i = 0; i < 2; ++i) { mbar_init(&bar_s[i], 1); mbar_init(&bar_p[i][0], 4); mbar_init(&bar_p[i][1], 4); }
        for (int i = 0; i < L::kKStages; ++i) { mbar_init(&bar_kfull[i], 1); mbar_init(&bar_kfree[i], 1); }
        for (int i = 0; i < L::kVStages; ++i) { mbar_init(&bar_vfull[i], 1); mbar_init(&bar_vfree[i], 1); mbar_init(&bar_vclean[i], 1); }
        for (int i = 0; i < kPosSlots; ++i) { mbar_init(&bar_posfull[i], 1); mbar_init(&bar_posfree[i], kPosReaders); }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 0) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&s_tmem)), "r"(512u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    if (warp != kSoftmaxWarps || x >= slot_end) dodo_grid_dependency_sync();
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = s_tmem;
    bool stuck = false;

    if (warp == kSoftmaxWarps) {
        // ================================================ scout ===================================================
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs));
        int c = 0;                     // tiles and ends of segments so far
        while (!stuck && next_segment(g, a, work, L::kRows, x, slot_end, q)) {
            const PagedSeq& s = g.seq[q.b];
            // a lane's four keys of tile t: page entries first, rows and positions a tile later
            int entry[4], row[4], pos[4];
            auto entries = [&](int t) {
                const int v = t * BN + 4 * lane;
#pragma unroll
                for (int e = 0; e < 4; ++e) entry[e] = t < q.t1 && t < q.c_tiles ? page_entry(a, s, v + e, s.c_len) : 0;
            };
            auto keys = [&](int t) {
                const int v = t * BN + 4 * lane, j = v - q.c_tiles * BN;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    row[e] = -1; pos[e] = kNoPos;
                    if (t >= q.t1) continue;
                    if (t >= q.c_tiles) {
                        if (j + e < q.l_vis) { row[e] = s.l_row0 + j + e; pos[e] = s.l_pos0 + j + e; }
                    } else {
                        const Key k = key_at(a, s, v + e, s.c_len, entry[e]);
                        row[e] = k.row; pos[e] = k.pos;
                    }
                }
            };
            for (int r = lane; r < q.rows; r += 32) hint_row<DH>(a, s, q, r);     // the segment's Q, while others are at the one before
            entries(q.t0);
            keys(q.t0);
            entries(q.t0 + 1);
            for (int t = q.t0; t <= q.t1; ++t) {           // q.t1: the segment's end
                int r[4], p[4], hi = static_cast<int>(0x80000000);
                bool any = false;      // rows where there are keys, positions only where somebody sees them
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const bool there = row[e] >= 0 && pos[e] <= q.last_pos;
                    r[e] = row[e];
                    p[e] = there ? pos[e] : kNoPos;
                    hi = max(hi, p[e]);
                    any = any || there;
                }
                if (t < q.t1) {
                    keys(t + 1);
                    entries(t + 2);
                    if (!__any_sync(0xffffffffu, any)) continue;                // nobody sees a key of this tile
                }
                const bool masked = __any_sync(0xffffffffu, hi > q.min_pos);
                const int ps = c % kPosSlots;
                if (!warp_wait(&bar_posfree[ps], static_cast<uint32_t>(c / kPosSlots + 1) & 1u)) { stuck = true; break; }
                *reinterpret_cast<int4*>(s_pos + ps * BN + 4 * lane) = make_int4(p[0], p[1], p[2], p[3]);
                *reinterpret_cast<int4*>(s_row + ps * BN + 4 * lane) = make_int4(r[0], r[1], r[2], r[3]);
                const bool holes = __any_sync(0xffffffffu, hi == kNoPos);
                if (lane == 0) s_kind[ps] = t == q.t1 ? kEnd : (masked ? kMasked : 0) | (t >= q.c_tiles ? kLocal : 0) | (holes ? kHoles : 0);
                __syncwarp();
                if (lane == 0) mbar_arrive(&bar_posfull[ps]);
                ++c;
            }
        }
    } else if (warp == kSoftmaxWarps + 2) {
        // ================================================ producer ================================================
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs));
        int c = 0, n = 0;              // tiles and ends so far; tiles
        // the rows of a tile to stage n of a ring: boxes whose first key is there
        auto bring = [&](uint32_t ring, uint64_t* full, uint64_t* free, int stages, const CUtensorMap* cache, const CUtensorMap* loc, bool local, int col, const int* rows) {
            const int stage = n % stages;
            if (!warp_wait(&free[stage], static_cast<uint32_t>(n / stages + 1) & 1u)) return false;
            uint64_t* const bar = &full[stage];
            const uint32_t dst = ring + stage * L::kTile;
            if (local) {
                const int r = rows[0];
                if (elect_one()) {
                    mbar_expect_tx(bar, L::kTile);
#pragma unroll
                    for (int h = 0; h < L::kHalves; ++h) tma_load_2d(dst + h * L::kHalf, loc, col + 64 * h, r, bar);
                }
            } else if (const int box = maps.rows; box >= 8) {
                int count = 0;
                for (int k = lane * box; k < BN; k += 32 * box) count += rows[k] >= 0 ? 1 : 0;
                count = __reduce_add_sync(0xffffffffu, count);
                if (elect_one()) mbar_expect_tx(bar, static_cast<uint32_t>(count * box * DH * 2));
                for (int k = 0; k < BN; k += box) {
                    const int r = rows[k];
                    if (r >= 0 && elect_one()) {
#pragma unroll
                        for (int h = 0; h < L::kHalves; ++h) tma_load_2d(dst + h * L::kHalf + k * 128, cache, col + 64 * h, r, bar);
                    }
                }
            } else {
                int4 r = *reinterpret_cast<const int4*>(rows + 4 * lane);
                const int some = max(max(r.x, r.y), max(r.z, r.w));       // in the place of rows that are not there
                const uint32_t has = __ballot_sync(0xffffffffu, some >= 0);
                if (lane == 0) mbar_expect_tx(bar, static_cast<uint32_t>(__popc(has) * 4 * DH * 2));
                __syncwarp();
                if (some >= 0) {
                    r.x = r.x < 0 ? some : r.x; r.y = r.y < 0 ? some : r.y; r.z = r.z < 0 ? some : r.z; r.w = r.w < 0 ? some : r.w;
#pragma unroll
                    for (int h = 0; h < L::kHalves; ++h) gather4(dst + h * L::kHalf + lane * 512, cache, col + 64 * h, r, bar);
                }
            }
            __syncwarp();
            return true;
        };
        while (!stuck && next_segment(g, a, work, L::kRows, x, slot_end, q)) {
            const int col = q.head * DH;
            while (true) {
                const int ps = c % kPosSlots;
                if (!warp_wait(&bar_posfull[ps], static_cast<uint32_t>(c / kPosSlots) & 1u)) { stuck = true; break; }
                const int kind = s_kind[ps];
                ++c;
                if (kind != kEnd) {
                    const bool local = (kind & kLocal) != 0;
                    const int* const rows = s_row + ps * BN;
                    if (!bring(base + L::kOffK, bar_kfull, bar_kfree, L::kKStages, &maps.cK, &maps.lK, local, col, rows) ||
                        !bring(base + L::kOffV, bar_vfull, bar_vfree, L::kVStages, &maps.cV, &maps.lV, local, col, rows)) { stuck = true; break; }
                    ++n;
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(&bar_posfree[ps]);
                if (kind == kEnd) break;
            }
        }
        if (stuck) {         // copies in flight land before the block's shared memory goes
            for (int i = max(0, n - L::kKStages + 1); i <= n; ++i) mbar_wait(&bar_kfull[i % L::kKStages], static_cast<uint32_t>(i / L::kKStages) & 1u);
            for (int i = max(0, n - L::kVStages + 1); i <= n; ++i) mbar_wait(&bar_vfull[i % L::kVStages], static_cast<uint32_t>(i / L::kVStages) & 1u);
        }
    } else if (warp == kSoftmaxWarps + 3) {
        // ================================================ cleaner =================================================
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs));
        constexpr int kPieces = DH / 8;                    // 16-byte pieces of a row
        int c = 0, n = 0;
        while (!stuck && next_segment(g, a, work, L::kRows, x, slot_end, q)) {
            while (true) {
                const int ps = c % kPosSlots, stage = n % L::kVStages;
                if (!warp_wait(&bar_posfull[ps], static_cast<uint32_t>(c / kPosSlots) & 1u)) { stuck = true; break; }
                const int kind = s_kind[ps];
                ++c;
                if (kind != kEnd) {
                    if (!warp_wait(&bar_vfull[stage], static_cast<uint32_t>(n / L::kVStages) & 1u)) { stuck = true; break; }
                    if ((kind & kHoles) != 0) {
                        unsigned char* const v = base_ptr + L::kOffV + stage * L::kTile + (lane % kPieces / 8) * L::kHalf + lane % 8 * 16;
#pragma unroll
                        for (int r0 = 0; r0 < BN; r0 += 32) {
                            // bit r: row r0 + r; as many rows at a time as lanes hold pieces for
                            uint32_t holes = __ballot_sync(0xffffffffu, s_pos[ps * BN + r0 + lane] == kNoPos);
                            holes >>= lane / kPieces;
#pragma unroll
                            for (int r = 0; r < 32; r += 32 / kPieces)
                                if ((holes >> r & 1u) != 0u) *reinterpret_cast<uint4*>(v + (r0 + r + lane / kPieces) * 128) = make_uint4(0u, 0u, 0u, 0u);
                        }
                        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    }
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&bar_vclean[stage]);
                    ++n;
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(&bar_posfree[ps]);
                if (kind == kEnd) break;
            }
        }
    } else if (warp == kSoftmaxWarps + 1) {
        // ================================================ matrix issuer ===========================================
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs));
        int c_pos = 0, ck = 0, cv = 0, np[2] = {0, 0}, segs = 0;     // tiles and ends; K tiles; V tiles; P of the streams
        const uint32_t idesc_s = idesc_bf16(BN, false), idesc_o = idesc_bf16(DH, true);
        auto next_tile = [&]() {        // whether the segment has another tile (or a wait ran out)
            const int ps = c_pos % kPosSlots;
            if (!warp_wait(&bar_posfull[ps], static_cast<uint32_t>(c_pos / kPosSlots) & 1u)) { stuck = true; return false; }
            const int kind = s_kind[ps];
            __syncwarp();
            if (lane == 0) mbar_arrive(&bar_posfree[ps]);
            ++c_pos;
            return kind != kEnd;
        };
        auto wait_k = [&](int c) { if (!warp_wait(&bar_kfull[c % L::kKStages], static_cast<uint32_t>(c / L::kKStages) & 1u)) stuck = true; };
        auto scores = [&](int st, int qtile, int c, bool last_user) {
            tc_fence_after();
            const uint64_t da = desc_kmajor(base + qtile * L::kTile), db = desc_kmajor(base + L::kOffK + (c % L::kKStages) * L::kTile);
            if (elect_one()) {
#pragma unroll
                for (int i = 0; i < DH / 16; ++i) {
                    const uint64_t step = static_cast<uint64_t>(((i / 4) * L::kHalf + (i % 4) * 32) >> 4);
                    mma_bf16(tmem + st * BN, da + step, db + step, idesc_s, i > 0);
                }
                mma_commit(&bar_s[st]);
                if (last_user) mma_commit(&bar_kfree[c % L::kKStages]);
            }
            __syncwarp();
        };
        // the product of a tile's weights and values, in halves of 64 keys as the softmax publishes them; `between` runs while the first is
        // being worked on
        auto values = [&](int st, int c, bool add, bool last_user, auto between) {
            const uint64_t db = desc_mnmajor(base + L::kOffV + (c % L::kVStages) * L::kTile, L::kHalf);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                if (!warp_wait(&bar_p[st][h], static_cast<uint32_t>(np[st]) & 1u)) stuck = true;
                tc_fence_after();
                if (elect_one()) {
#pragma unroll
                    for (int i = h * BN / 32; i < (h + 1) * BN / 32; ++i)       // 16 keys of P = 8 columns of bf16 pairs
                        mma_bf16_ts(tmem + 2 * BN + st * DH, tmem + st * BN + i * 8, db + static_cast<uint64_t>((i * 2048) >> 4), idesc_o, add || i > 0);
                    if (h == 1 && last_user) mma_commit(&bar_vfree[c % L::kVStages]);
                }
                __syncwarp();
                if (h == 0) between();
            }
            ++np[st];
        };
        auto wait_v = [&](int c) { if (!warp_wait(&bar_vclean[c % L::kVStages], static_cast<uint32_t>(c / L::kVStages) & 1u)) stuck = true; };
        // nobody sees a key of the segment: the softmax warps, which bring the next Q behind this, come no further ahead than that
        auto empty = [&]() {
            if (lane == 0) mbar_arrive(&bar_o);
            __syncwarp();
        };
        while (!stuck && next_segment(g, a, work, L::kRows, x, slot_end, q)) {
            if (!warp_wait(&bar_q, static_cast<uint32_t>(segs) & 1u)) { stuck = true; break; }
            ++segs;
            if constexpr (TILES == 2) {
                const int streams = q.rows > BM ? 2 : 1;
                bool more = next_tile();
                if (!more) { empty(); continue; }
                wait_k(ck);
                for (int st = 0; st < streams; ++st) scores(st, st, ck, st == streams - 1);
                ++ck;
                more = next_tile();
                bool add = false, ended = false, v_there = false;
                while (!ended && !stuck) {
                    const bool now = more;             // a tile follows this one
                    if (!v_there) wait_v(cv);
                    for (int st = 0; st < streams; ++st) {
                        values(st, cv, add, st == streams - 1, [&] {
                            if (now && st == 0) wait_k(ck);
                            if (now && st == streams - 1) {
                                more = next_tile();
                                v_there = __all_sync(0xffffffffu, mbar_try_wait(&bar_vclean[(cv + 1) % L::kVStages], static_cast<uint32_t>((cv + 1) / L::kVStages) & 1u));
                            }
                        });
                        if (now) scores(st, st, ck, st == streams - 1);
                    }
                    ++cv;
                    ck += now ? 1 : 0;
                    add = true;
                    ended = !now;
                }
            } else {
                // tile i of the segment belongs to stream i & 1; scores run two tiles ahead of the values
                int i = 0, ahead = 0;
                bool ended = false;
                auto next_scores = [&]() {
                    if (ended) return;
                    if (!next_tile()) { ended = true; return; }
                    wait_k(ck);
                    scores(ahead & 1, 0, ck, true);
                    ++ahead;
                    ++ck;
                };
                next_scores();
                next_scores();
                if (ahead == 0) { empty(); continue; }
                while (!stuck && i < ahead) {
                    wait_v(cv);
                    values(i & 1, cv, i >= 2, true, [] {});
                    ++cv;
                    ++i;
                    next_scores();
                }
            }
            if (elect_one()) mma_commit(&bar_o);
            __syncwarp();
        }
        if (stuck) {         // products in flight end before the block's tensor and shared memory go
            if (elect_one()) mma_commit(&bar_drain);
            __syncwarp();
            mbar_wait(&bar_drain, 0u);
        }
    } else {
        // ================================================ softmax =================================================
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftmaxRegs));
        const int st = warp >> 2, row = tid & (BM - 1);
        const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16, t_s = tmem + st * BN + lanes, t_o = tmem + 2 * BN + lanes;
        float* const xch = reinterpret_cast<float*>(base_ptr + L::kOffXch);
        const float2 c2 = make_float2(a.scale_log2, a.scale_log2);
        // Q in the layout of the matrix unit's operands (128-byte rows of 64 features, 16-byte pieces swizzled): a warp brings its 32 rows
        // (with one tile of rows, its stream's half of their features), neighbouring lanes neighbouring pieces
        constexpr int kPieces = (TILES == 2 ? DH : DH / 2) / 8, kAtOnce = 32 / kPieces;
        const int warp_row = (TILES == 2 ? st * BM : 0) + (row & ~31), piece = (TILES == 2 ? 0 : st * kPieces) + lane % kPieces;
        unsigned char* const q_tile = base_ptr + (TILES == 2 ? st * L::kTile : 0) + (piece / 8) * L::kHalf + (row & ~31) * 128;
        auto bring_q = [&](const Segment& u) {
            uint4 v[32 / kAtOnce];
#pragma unroll
            for (int i = 0; i < 32 / kAtOnce; ++i) {        // (rows behind the last are the last one again)
                const int r = min(warp_row + i * kAtOnce + lane / kPieces, u.rows - 1);
                v[i] = __ldg(reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(a.Q) + out_row(a, g.seq[u.b], u.head, u.r0 + r) * DH) + piece);
            }
#pragma unroll
            for (int i = 0; i < 32 / kAtOnce; ++i) {
                const int r = i * kAtOnce + lane / kPieces;
                *reinterpret_cast<uint4*>(q_tile + r * 128 + (((piece % 8) ^ (r & 7)) << 4)) = v[i];
            }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) mbar_arrive(&bar_q);
        };
        unsigned char* const out_tile = base_ptr + L::kOffOut + warp * 2048;
        int ck = 0, ns = 0, os = 0;
        bool first_seg = true;
        // (a wait that has run out ends the waiting, not the walk: the barriers of these warps count all of them)
        bool more = next_segment(g, a, work, L::kRows, x, slot_end, q);
        if (more) bring_q(q);
        while (more) {
            const PagedSeq& s = g.seq[q.b];
            const int my = (TILES == 2 ? st * BM : 0) + row;               // this thread's row of the tile of rows
            const bool live = my < q.rows, stream_live = TILES == 1 || st * BM < q.rows, warp_live = (TILES == 2 ? st * BM : 0) + (row & ~31) < q.rows;
            const int qpos = s.q_pos0 + token_of(a, q.r0 + min(my, q.rows - 1));
            float m = -INFINITY, l = 0.f;
            int mine = 0, tiles = 0;         // tiles of this stream; of the segment
            while (!stuck) {
                const int ps = ck % kPosSlots;
                if (!warp_wait(&bar_posfull[ps], static_cast<uint32_t>(ck / kPosSlots) & 1u)) { stuck = true; break; }
                const int kind = s_kind[ps];
                ++ck;
                if (kind == kEnd || !stream_live || (TILES == 1 && (tiles & 1) != st)) {
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&bar_posfree[ps]);
                    if (kind == kEnd) break;
                    ++tiles;
                    continue;
                }
                ++tiles;
                if (!warp_wait(&bar_s[st], static_cast<uint32_t>(ns) & 1u)) { stuck = true; break; }
                ++ns;
                tc_fence_after();
                if (warp_live) {
                    uint32_t sv[BN];
                    auto load_half = [&](int h) {
                        if (h == 0) tmem_ld64(t_s, sv);
                        else tmem_ld64(t_s + 64, sv + 64);
                    };
                    auto mask_half = [&](int h) {
#pragma unroll
                        for (int c = h * 64; c < h * 64 + 64; c += 4) {
                            const int4 kp = *reinterpret_cast<const int4*>(s_pos + ps * BN + c);
                            if (kp.x > qpos) sv[c] = 0xff800000u;
                            if (kp.y > qpos) sv[c + 1] = 0xff800000u;
                            if (kp.z > qpos) sv[c + 2] = 0xff800000u;
                            if (kp.w > qpos) sv[c + 3] = 0xff800000u;
                        }
                    };
                    load_half(0);
                    tmem_wait64(sv);
                    load_half(1);
                    if ((kind & kMasked) != 0) mask_half(0);
                    tmem_wait64(sv + 64);
                    if ((kind & kMasked) != 0) mask_half(1);
                    float2 sum0 = make_float2(0.f, 0.f), sum1 = make_float2(0.f, 0.f);
                    float2 nm2 = make_float2(m == -INFINITY ? 0.f : -m, m == -INFINITY ? 0.f : -m);
                    // weights of scores c to c + 3, packed where scores have been read
                    auto weights = [&](int c) {
                        const float2 x0 = __ffma2_rn(make_float2(__uint_as_float(sv[c]), __uint_as_float(sv[c + 1])), c2, nm2);
                        const float2 x1 = __ffma2_rn(make_float2(__uint_as_float(sv[c + 2]), __uint_as_float(sv[c + 3])), c2, nm2);
                        const float2 p0 = make_float2(exp2_fast(x0.x), exp2_fast(x0.y));
                        const float2 p1 = make_float2(exp2_fast(x1.x), exp2_fast(x1.y));
                        sv[c / 2] = pack_bf16(p0.x, p0.y);
                        sv[c / 2 + 1] = pack_bf16(p1.x, p1.y);
                        sum0 = __fadd2_rn(sum0, p0);
                        sum1 = __fadd2_rn(sum1, p1);
                    };
                    auto publish = [&](int h) {
                        tmem_st32(t_s + h * 32, sv + h * 32);
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(&bar_p[st][h]);
                    };
                    // The first half's weights by the reference maximum that there is; the tile's own is found beside them, and only where
                    // it has grown too far (the first tile among these) is the tile begun again.
                    float t4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                    for (int c = 0; c < BN / 2; c += 4) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) t4[e] = max3(t4[e], __uint_as_float(sv[c + e]), __uint_as_float(sv[BN / 2 + c + e]));
                        weights(c);
                    }
                    float top = fmaxf(max3(t4[0], t4[1], t4[2]), t4[3]) * a.scale_log2;      // -infinity stays what it is: the scale is positive
                    const bool grow = top > m + kRescaleStep;
                    if (__any_sync(0xffffffffu, grow)) {
                        const float m_new = grow ? top : m;
                        if (mine > 0) {
                            // P V of this stream's tile before is complete: its scores of this tile were issued behind it
                            const float corr = grow ? part_weight(m, m_new) : 1.f;
                            l *= corr;
#pragma unroll 1
                            for (int c = 0; c < DH; c += 32) {
                                uint32_t ov[32];
                                tmem_ld32(t_o + st * DH + c, ov);
#pragma unroll
                                for (int e = 0; e < 32; ++e) ov[e] = __float_as_uint(__uint_as_float(ov[e]) * corr);
                                tmem_st32(t_o + st * DH + c, ov);
                            }
                        }
                        m = m_new;
                        nm2.x = nm2.y = m == -INFINITY ? 0.f : -m;
                        sum0 = sum1 = make_float2(0.f, 0.f);
                        load_half(0);
                        tmem_wait64(sv);
                        if ((kind & kMasked) != 0) mask_half(0);
#pragma unroll
                        for (int c = 0; c < BN / 2; c += 4) weights(c);
                    }
                    publish(0);
#pragma unroll
                    for (int c = BN / 2; c < BN; c += 4) weights(c);
                    publish(1);
                    l += (sum0.x + sum0.y) + (sum1.x + sum1.y);
                } else if (lane == 0) {
                    mbar_arrive(&bar_p[st][0]);
                    mbar_arrive(&bar_p[st][1]);
                }
                ++mine;
                __syncwarp();
                if (lane == 0) mbar_arrive(&bar_posfree[ps]);
            }
            if (!stuck && !warp_wait(&bar_o, static_cast<uint32_t>(os) & 1u)) stuck = true;
            ++os;
            tc_fence_after();
            if (l != l) m = INFINITY;        // a NaN among the logits that the row sees: the whole row's, wherever its maximum stands
            // The matrix unit is through with Q: it gets the next segment's now, and has work while this one's results go out.
            Segment next;
            more = next_segment(g, a, work, L::kRows, x, slot_end, next);
            if (more) bring_q(next);
            // ---- a row's result: of its stream, or of both, each thread then half of the features
            constexpr int kFeat = TILES == 2 ? DH : DH / 2;
            const int f0 = TILES == 2 ? 0 : st * kFeat;
            float w0 = 1.f, w1 = 0.f, M = m, S = l;        // weights of stream 0 (or the own one) and 1
            if constexpr (TILES == 1) {
                xch[st * 2 * BM + row] = m;
                xch[st * 2 * BM + BM + row] = l;
                asm volatile("bar.sync 1, 256;" ::: "memory");
                const float om = xch[(st ^ 1) * 2 * BM + row], ol = xch[(st ^ 1) * 2 * BM + BM + row];
                M = fmaxf(m, om);
                const float a0 = part_weight(m, M), a1 = part_weight(om, M);
                S = __fadd_rn(a0 != 0.f ? __fmul_rn(a0, l) : 0.f, a1 != 0.f ? __fmul_rn(a1, ol) : 0.f);      // the same number in both
                w0 = st == 0 ? a0 : a1;
                w1 = st == 0 ? a1 : a0;
            }
            auto own = [&](int c, float* o) {              // 32 features of this block's piece, not divided by the sum
                if (TILES == 2 ? mine == 0 : tiles == 0) {
#pragma unroll
                    for (int e = 0; e < 32; ++e) o[e] = 0.f;
                    return;
                }
                uint32_t ov[32];
                tmem_ld32(t_o + (TILES == 2 ? st * DH : 0) + c, ov);
#pragma unroll
                for (int e = 0; e < 32; ++e) o[e] = TILES == 2 ? __uint_as_float(ov[e]) : w0 != 0.f ? w0 * __uint_as_float(ov[e]) : 0.f;
                if (TILES == 1 && tiles > 1) {
                    tmem_ld32(t_o + DH + c, ov);
#pragma unroll
                    for (int e = 0; e < 32; ++e) o[e] = w1 != 0.f ? fmaf(w1, __uint_as_float(ov[e]), o[e]) : o[e];
                }
            };
            // A unit that is cut: whoever finds all other pieces there joins them with its own, which stays in tensor memory; the
            // others write theirs.  Pieces: four features of a row side by side, then maxima and sums.
            int c_first = bid, c_last = bid;
            bool done = true;
            if (q.t0 != 0 || q.t1 != q.nt) {
                c_first = block_of(T, G, q.first_slot);
                c_last = block_of(T, G, q.first_slot + q.nt - 1);
                // a block's last unit is the only one that begins in it and goes on: the block's number names it
                int* const ticket = a.tickets + c_first;
                if (tid == 0) s_last = ld_acquire_gpu(ticket) == c_last - c_first;
                asm volatile("bar.sync 1, 256;" ::: "memory");
                done = s_last != 0;
                if (!done) {
                    float* const part = a.part + static_cast<size_t>(2 * bid + (first_seg ? 0 : 1)) * L::kPartFloats;
#pragma unroll 1
                    for (int c = f0; c < f0 + kFeat && warp_live; c += 32) {
                        float o[32];
                        own(c, o);
#pragma unroll
                        for (int e = 0; e < 32; e += 4)
                            reinterpret_cast<float4*>(part)[static_cast<size_t>((c + e) / 4) * L::kRows + my] = make_float4(o[e], o[e + 1], o[e + 2], o[e + 3]);
                    }
                    if (TILES == 2 || st == 0) reinterpret_cast<float2*>(part + static_cast<size_t>(DH) * L::kRows)[my] = make_float2(M, S);
                    __threadfence();
                    asm volatile("bar.sync 1, 256;" ::: "memory");
                    if (tid == 0) s_last = atomicAdd(ticket, 1) == c_last - c_first;
                    asm volatile("bar.sync 1, 256;" ::: "memory");
                    done = s_last != 0;
                }
                if (done) {
                    if (tid == 0) *ticket = 0;             // clean for the next launch
                    __threadfence();
                }
            }
            bool odd = false;                              // a result that is not finite
            if (done && warp_live) {
                // out through shared memory, 32 features at a time: four lanes a row, eight rows an instruction
                uint4* at[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int r = min(warp_row + i * 8 + lane / 4, q.rows - 1);
                    at[i] = reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(a.O) + out_row(a, s, q.head, q.r0 + r) * DH + f0) + lane % 4;
                }
                float2 zero = make_float2(0.f, 0.f);
                auto emit = [&](int f, const float2* o) {
                    uint32_t w[16];
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        zero = __ffma2_rn(o[e], make_float2(0.f, 0.f), zero);
                        w[e] = pack_bf16(o[e].x, o[e].y);
                    }
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        *reinterpret_cast<uint4*>(out_tile + lane * 64 + ((e ^ (lane >> 1 & 3)) << 4)) = make_uint4(w[4 * e], w[4 * e + 1], w[4 * e + 2], w[4 * e + 3]);
                    __syncwarp();
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int r = i * 8 + lane / 4;
                        if (warp_row + r < q.rows) at[i][f / 8] = *reinterpret_cast<const uint4*>(out_tile + r * 64 + ((lane % 4 ^ (r >> 1 & 3)) << 4));
                    }
                    __syncwarp();
                };
                float MM = M, SS = S;
                if (c_first == c_last) {
                    const float inv = S != 0.f ? 1.f / S : 0.f;
                    const float2 k0 = make_float2(w0 * inv, w0 * inv), k1 = make_float2(w1 * inv, w1 * inv);
                    const bool some = TILES == 2 ? mine > 0 : tiles > 0;
#pragma unroll
                    for (int f = 0; f < kFeat; f += 32) {
                        uint32_t ov[32];
                        float2 o[16];
#pragma unroll
                        for (int e = 0; e < 16; ++e) o[e] = make_float2(0.f, 0.f);
                        if (some) {
                            tmem_ld32(t_o + (TILES == 2 ? st * DH : 0) + f0 + f, ov);
#pragma unroll
                            for (int e = 0; e < 16; ++e) o[e] = __fmul2_rn(k0, make_float2(__uint_as_float(ov[2 * e]), __uint_as_float(ov[2 * e + 1])));
                        }
                        if (TILES == 1 && tiles > 1) {
                            tmem_ld32(t_o + DH + f0 + f, ov);
#pragma unroll
                            for (int e = 0; e < 16; ++e) o[e] = __ffma2_rn(k1, make_float2(__uint_as_float(ov[2 * e]), __uint_as_float(ov[2 * e + 1])), o[e]);
                        }
                        emit(f, o);
                    }
                } else {
                    // the unit is the first of every block but the one that it begins in
                    const int begun = block_start(work, G, c_first) < q.first_slot - work.ahead ? 1 : 0;
                    auto part_of = [&](int c) { return a.part + static_cast<size_t>(2 * c + (c == c_first ? begun : 0)) * L::kPartFloats; };
                    auto max_sum = [&](int c) { return c == bid ? make_float2(M, S) : __ldcg(reinterpret_cast<const float2*>(part_of(c) + static_cast<size_t>(DH) * L::kRows) + my); };
                    MM = -INFINITY, SS = 0.f;
                    for (int c = c_first; c <= c_last; ++c) {
                        const float2 ms = max_sum(c);
                        const float top = fmaxf(MM, ms.x), a0 = part_weight(MM, top), a1 = part_weight(ms.x, top);
                        SS = (a0 != 0.f ? a0 * SS : 0.f) + (a1 != 0.f ? a1 * ms.y : 0.f);
                        MM = top;
                    }
                    const float inv = SS != 0.f ? 1.f / SS : 0.f;
                    float2 o[kFeat / 2];
#pragma unroll
                    for (int e = 0; e < kFeat / 2; ++e) o[e] = make_float2(0.f, 0.f);
#pragma unroll 1
                    for (int c = c_first; c <= c_last; ++c) {
                        const float w = part_weight(max_sum(c).x, MM);
                        const float2 k = make_float2(w * inv, w * inv);
#pragma unroll
                        for (int f = 0; f < kFeat; f += 32) {
                            float v[32];
                            if (c == bid) {
                                own(f0 + f, v);
                            } else {
                                const float4* const src = reinterpret_cast<const float4*>(part_of(c)) + static_cast<size_t>((f0 + f) / 4) * L::kRows + my;
#pragma unroll
                                for (int e = 0; e < 32; e += 4) {
                                    const float4 x4 = __ldcg(src + static_cast<size_t>(e / 4) * L::kRows);
                                    v[e] = x4.x; v[e + 1] = x4.y; v[e + 2] = x4.z; v[e + 3] = x4.w;
                                }
                            }
#pragma unroll
                            for (int e = 0; e < 16; ++e) o[f / 2 + e] = __ffma2_rn(k, make_float2(v[2 * e], v[2 * e + 1]), o[f / 2 + e]);
                        }
                    }
#pragma unroll
                    for (int f = 0; f < kFeat; f += 32) emit(f, o + f / 2);
                }
                odd = !(zero.x + zero.y == 0.f);
                if (live && a.lse != nullptr && (TILES == 2 || st == 0)) a.lse[out_row(a, s, q.head, q.r0 + my)] = SS != 0.f ? (MM + log2f(SS)) * 0.6931471805599453f : -INFINITY;
            }
            // ---- results that are not finite, once more over what their rows see
            if (any_softmax(odd && live && done)) {            // (behind it, both streams' O are read too)
                for (int r = warp; r < q.rows; r += kSoftmaxWarps) {
                    __nv_bfloat16* const out = static_cast<__nv_bfloat16*>(a.O) + out_row(a, s, q.head, q.r0 + r) * DH;
                    bool bad = false;
                    for (int f = lane; f < DH; f += 32) bad = bad || !isfinite(__bfloat162float(out[f]));
                    if (__any_sync(0xffffffffu, bad)) sum_again<__nv_bfloat16, DH>(a, s, q.head, q.r0 + r, out);
                }
            }
            first_seg = false;
            q = next;
        }
    }
    if (stuck && lane == 0) atomicOr(a.status, DODO_DEV_WAIT_TIMEOUT);
    tc_fence_before();
    __syncthreads();
    if (warp == 0) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
}

template <int DH, int TILES>
int launch(dodo_ctx* ctx, const PagedBoxes& maps, const PagedGroup& g, const PagedArrays& a, const DenseShare& w, int grid, cudaStream_t st) {
    auto kern = attend_paged_dense_kernel<DH, TILES>;
    const int smem = Layout<DH, TILES>::kBytes + 1024;
    bool& set = ctx->paged_attr_set[(DH == 128 ? 2 : 0) + TILES - 1];
    if (!set) {
        const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
        if (e != cudaSuccess) return dodo_check_cuda(ctx, e, "paged dense attend shared-memory attribute");
        set = true;
    }
    return dodo_check_cuda(ctx, dodo_launch_dependent(kern, dim3(static_cast<unsigned>(grid)), dim3(kThreads), static_cast<size_t>(smem), st, maps, g, a, w),
                           "paged dense attend launch");
}

}  // namespace

size_t dodo_paged_dense_workspace_bytes(int num_sms, int dh) { return static_cast<size_t>(2) * num_sms * 2 * BM * (dh + 2) * sizeof(float); }

int dodo_launch_paged_dense(dodo_ctx* ctx, int dh, int max_rows, int loc_rows, const PagedGroup& g, const PagedArrays& a, cudaStream_t st) {
    const int tiles = max_rows > BM ? 2 : 1, tile_rows = tiles * BM;
    DenseShare w;
    int64_t total = 0, units = 0;
    bool alike = true;
    int nt = 0;
    for (int i = 0; i < g.nseq; ++i) {
        const PagedSeq& s = g.seq[i];
        const int64_t rows = static_cast<int64_t>(s.tq) * a.group, rt = (rows + tile_rows - 1) / tile_rows;
        const int l_vis = s.tq > 0 ? dodo_visible_local(s.l_len, s.l_pos0, s.q_pos0 + s.tq - 1) : 0, n = (s.c_len + BN - 1) / BN + (l_vis + BN - 1) / BN;
        w.nt[i] = n > 0 ? n : 1;
        w.tiles[i] = static_cast<int>(rt > 0 ? rt : 1);
        total += rt * a.Hkv * w.nt[i];
        units += rt * a.Hkv;
        if (s.tq > 0) { alike = alike && (nt == 0 || nt == w.nt[i]); nt = w.nt[i]; }
    }
    if (total == 0) return DODO_OK;
    // A unit begun and ended costs about three tiles' times (Q, a pipeline filled and emptied, results), pieces joined another three.  Where
    // units differ in length they count so much longer, or blocks with many short ones would work longest (8 x 18 to 26 queries of two heads a
    // KV head over lists of 30 to 3178 keys, 27 KV heads: 58 us, 38 so).  Not with four-row gather copies, whose tiles take as long as that.
    // One block per SM, but none for less than four tiles (with one tile of rows two: the streams take them side by side; 7 x 12 to 16
    // queries of eight heads a KV head over up to 2296 keys took 29 us with four, 25 with two) or a unit.  Where all units are alike there
    // is also the share of a k-th of a unit each (no block then works for two units) and that of whole units (none is joined: 256 units of
    // 64 rows over 264 keys took 36 us with equal shares, 26 so), by the slowest block's count of tiles' times.
    constexpr int kUnit = 3;
    const int64_t shares = tiles == 1 ? (total + 1) / 2 : (total + 3) / 4, most = shares > units ? shares : units;
    int64_t grid = most < ctx->num_sms ? most : ctx->num_sms;
    w.whole = 1;
    const int box = dodo_paged_box(a.page, BN);
    w.ahead = alike || box == 0 ? 0 : kUnit;
    if (alike) {
        const int64_t each = (total + grid - 1) / grid, most_units = (units + ctx->num_sms - 1) / ctx->num_sms;
        int64_t cost = each + kUnit * ((each + nt - 1) / nt + 1) + kUnit;
        if (units > ctx->num_sms && most_units * (nt + kUnit) < cost) { grid = ctx->num_sms; w.whole = nt; }
        for (int64_t k = 1; k <= ctx->num_sms / units && k <= (nt + 3) / 4; ++k) {
            const int64_t c = (nt + k - 1) / k + kUnit + (k > 1 ? kUnit : 0);
            if (c < cost) { cost = c; grid = units * k; }
        }
    }
    int64_t slots = 0;
    for (int i = 0; i < g.nseq; ++i) {
        const int64_t rows = static_cast<int64_t>(g.seq[i].tq) * a.group;
        w.slot0[i] = static_cast<int>(slots);
        slots += (rows + tile_rows - 1) / tile_rows * a.Hkv * (w.nt[i] + w.ahead);
        if (slots > 0x7fffffff) return dodo_fail(ctx, DODO_ERR_UNSUPPORTED, "more than 2^31 tiles of keys in 64 sequences");
    }
    w.slot0[g.nseq] = static_cast<int>(slots);
    w.total = static_cast<int>(slots);
    PagedBoxes maps;
    const int rc = dodo_paged_boxes(ctx, a, dh, loc_rows, box > 0 ? box : 1, BN, maps);
    if (rc != DODO_OK) return rc;
    if (dh == 128) return tiles == 2 ? launch<128, 2>(ctx, maps, g, a, w, static_cast<int>(grid), st) : launch<128, 1>(ctx, maps, g, a, w, static_cast<int>(grid), st);
    return tiles == 2 ? launch<64, 2>(ctx, maps, g, a, w, static_cast<int>(grid), st) : launch<64, 1>(ctx, maps, g, a, w, static_cast<int>(grid), st);
}
