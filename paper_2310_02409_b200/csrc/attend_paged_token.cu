// Attention of few rows (query tokens x query heads of a KV head) over a paged cache, bf16: what a decode step asks for.  Bound by HBM:
// every K and V row is read once, and the arithmetic has to stay out of its way.  16 tokens of 32 heads on 8 KV heads over 122,000 keys: 84 us,
// 6.0 TB/s; one token over 16,448 keys of 40 heads: 57 us, 5.9 TB/s; 8 tokens over 269 keys of 32 heads: 10.3 us, 3.4 TB/s, of which half is
// a chain of latencies (page, rows, scores, values, results).
//
// A block works through a chunk of the key list in stages of 64 keys.  A producer warp looks keys up (page, position), skips stages that
// no query sees, and brings K and V by tensor copies, a box as many rows high as the power of two that divides the page's, into a ring
// with the 128-byte swizzle; the first stages' copies go out ahead of their positions (11.1 -> 10.1 us at 8 tokens).  Four consumer warps take 16 keys of a stage each, by warp-level matrix products in which keys are the rows
// and queries the eight columns, so that few queries waste little:
//   S^T [16 keys x 8 queries] = K Q^T      K's fragments by ldmatrix as they lie, Q's in registers from the start
//   O^T [16 features x 8 queries] += V^T P^T      V's by ldmatrix.trans, P^T by transposing S^T's packed fragments (movmatrix)
// Softmax: a row's reference maximum is its first stage's, and moves only when a score passes it by 2^24 (weights of up to that cost no
// digit); sums in 32 bits.  A weight meets V as the sum of two bf16 numbers, its rounding and the rounding of what that left: 16 bits of it
// (at most 2^-16 of it is lost) for a second product with fragments that are there already: 0.1 to 0.5 us of the 10 to 84 us of the cases above, 1.7 %
// at most (8 queries of 2 heads a KV head over 8 x 2064 keys, 23.2 -> 23.6 us).  V rows of keys that are not there, or seen by no query, are set
// to zero in shared memory; what some queries of a tile see and others do not is left to the check of the results at the end (finish).
#include "paged.cuh"
#include "sm100_ptx.cuh"

namespace {

using namespace sm100;
using namespace dodo_paged;

constexpr int BN = 64;                        // keys of a stage
constexpr int kConsumers = 4, kThreads = 32 * (kConsumers + 1);
constexpr float kRescaleStep = 24.f;
constexpr int kAhead = 4;                     // stages whose keys are looked up at once
// (Tiles of 32 rows, Q's fragments from shared memory, read a cache of 17 to 32 rows once instead of twice and were slower all the same: 20 of
// 8 x 1000 keys 22.3 us against 21.4, 32 rows of them 26.9 against 21.7.)
enum { kMasked = 1, kEnd = 2, kLocal = 4, kHoles = 8 };      // of a stage; kHoles: some of its keys are not there or seen by nobody

template <int DH>
struct Ring {
    static constexpr int kHalves = DH / 64, kHalf = BN * 128, kTile = kHalves * kHalf, kStage = 2 * kTile;
    static constexpr int kStages = DH == 128 ? 3 : 6;        // 96 KB: two blocks an SM, 100 KB and more on their way at any time
    static constexpr int kBytes = kStages * kStage;
};

__device__ __forceinline__ void ldmatrix4(uint32_t addr, uint32_t* r) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldmatrix4_trans(uint32_t addr, uint32_t* r) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ uint32_t transpose8(uint32_t v) {
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}
__device__ __forceinline__ void mma16816(float* c, const uint32_t* a, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}
// two floats as bf16, and what the rounding left of them as bf16 again
__device__ __forceinline__ void split_bf16(float a, float b, uint32_t& whole, uint32_t& rest) {
    whole = pack_bf16(a, b);
    rest = pack_bf16(a - __uint_as_float(whole << 16), b - __uint_as_float(whole & 0xffff0000u));
}

// NQ: tiles of eight rows
template <int DH, int NQ>
__global__ void __launch_bounds__(kThreads, 2)
attend_paged_token_kernel(const __grid_constant__ PagedBoxes boxes, const __grid_constant__ PagedGroup g, const __grid_constant__ PagedArrays a) {
    using L = Ring<DH>;
    constexpr int kRows = 8 * NQ, KK = DH / 16;
    extern __shared__ unsigned char smem_raw[];
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    unsigned char* const base_ptr = smem_raw + (base - smem_u32(smem_raw));
    __shared__ __align__(8) uint64_t full[L::kStages], empty[L::kStages];
    __shared__ __align__(16) int s_pos[L::kStages][BN];
    __shared__ int s_kind[L::kStages];
    __shared__ float s_max[kConsumers * kRows], s_sum[kConsumers * kRows];
    const int tid = static_cast<int>(threadIdx.x), lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0);
    if (tid == 0) {
        for (int i = 0; i < L::kStages; ++i) { mbar_init(&full[i], 1); mbar_init(&empty[i], kConsumers); }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    const Place p = place_of(g, a.Hkv, static_cast<int>(blockIdx.x));
    const PagedSeq& s = g.seq[p.b];
    const int R = s.tq * a.group, r0 = p.tile * kRows, rows = min(kRows, R - r0);
    const int first_pos = s.q_pos0 + token_of(a, r0), last_pos = s.q_pos0 + token_of(a, r0 + rows - 1);
    const int l_vis = dodo_visible_local(s.l_len, s.l_pos0, last_pos);
    // the chunk: stages of cached rows, then stages of local tokens
    const int c_stages = (s.c_len + BN - 1) / BN, t_end = min((p.chunk + 1) * (s.chunk_keys / BN), c_stages + (l_vis + BN - 1) / BN);
    const int t_begin = p.chunk * (s.chunk_keys / BN);
    bool stuck = false;
    // ahead of the dependency wait, hints to L2 only: the first page entries, the rows of Q
    if (warp == kConsumers) {
        const int first = t_begin * BN + 16 * lane;
        if (first < s.c_len) asm volatile("prefetch.global.L2 [%0];" ::"l"(a.table + s.page0 + page_of(a, first)));
    } else if (tid < rows) {
        const __nv_bfloat16* const q = static_cast<const __nv_bfloat16*>(a.Q) + out_row(a, s, p.head, r0 + tid) * DH;
#pragma unroll
        for (int c = 0; c < DH; c += 64) asm volatile("prefetch.global.L2 [%0];" ::"l"(q + c));
    }
    __syncthreads();
    dodo_grid_dependency_sync();

    if (warp == kConsumers) {
        // ================================================ producer ================================================
        const int col = p.head * DH;
        // Look-ups go ahead by fours: the page entries of four stages at once, then their positions, while the four before are brought.
        // (One stage at a time, a short list would take a round trip to memory for each.)
        int entry[kAhead][2], row[kAhead][2], pos[kAhead][2];
        auto entries = [&](int t) {
#pragma unroll
            for (int u = 0; u < kAhead; ++u)
#pragma unroll
                for (int e = 0; e < 2; ++e) entry[u][e] = t + u < t_end && t + u < c_stages ? page_entry(a, s, (t + u) * BN + 2 * lane + e, s.c_len) : 0;
        };
        auto keys = [&](int t) {
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const int v = (t + u) * BN + 2 * lane, j = v - c_stages * BN;
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    row[u][e] = -1; pos[u][e] = kNoPos;
                    if (t + u >= t_end) continue;
                    if (t + u >= c_stages) {
                        if (j + e < l_vis) { row[u][e] = s.l_row0 + j + e; pos[u][e] = s.l_pos0 + j + e; }
                    } else {
                        const Key k = key_at(a, s, v + e, s.c_len, entry[u][e]);
                        row[u][e] = k.row; pos[u][e] = k.pos;
                    }
                }
            }
        };
        entries(t_begin);
        keys(t_begin);
        entries(t_begin + kAhead);
        int n = 0;                     // stages filled so far
        // A stage's copies need its rows alone; what the consumers wait for beside them are its positions, and the word that they are there.
        auto copy = [&](int st, int t, int r0) {
            // a box starts with an even key: the lane that holds it copies it, if its first row is there
            const bool local = t >= c_stages;
            const int box = local ? BN : boxes.rows;
            const bool mine = 2 * lane % box == 0 && r0 >= 0;
            const uint32_t have = __popc(__ballot_sync(0xffffffffu, mine));
            if (lane == 0)
                asm volatile("mbarrier.expect_tx.relaxed.cta.shared::cta.b64 [%0], %1;" ::"r"(smem_u32(&full[st])), "r"(have * box * DH * 4) : "memory");
            __syncwarp();
            if (mine) {
                const CUtensorMap* const mk = local ? &boxes.lK : &boxes.cK;
                const CUtensorMap* const mv = local ? &boxes.lV : &boxes.cV;
                const uint32_t dst = base + st * L::kStage + 2 * lane * 128;
#pragma unroll
                for (int h = 0; h < L::kHalves; ++h) tma_load_2d(dst + h * L::kHalf, mk, col + 64 * h, r0, &full[st]);
#pragma unroll
                for (int h = 0; h < L::kHalves; ++h) tma_load_2d(dst + L::kTile + h * L::kHalf, mv, col + 64 * h, r0, &full[st]);
            }
        };
        auto publish = [&](int st, int p0, int p1, bool end) {
            const int hi = max(p0, p1);
            const bool masked = __any_sync(0xffffffffu, hi > first_pos), holes = __any_sync(0xffffffffu, hi == kNoPos);
            *reinterpret_cast<int2*>(&s_pos[st][2 * lane]) = make_int2(p0, p1);
            if (lane == 0) s_kind[st] = end ? kEnd : (masked ? kMasked : 0) | (holes ? kHoles : 0);
            __syncwarp();
            if (lane == 0) mbar_arrive(&full[st]);
            ++n;
        };
        auto wait_empty = [&]() { return __all_sync(0xffffffffu, mbar_wait(&empty[n % L::kStages], static_cast<uint32_t>(n / L::kStages + 1) & 1u)); };
        // the first stages go out ahead of their positions
        constexpr int kFirst = L::kStages < kAhead ? L::kStages : kAhead;
#pragma unroll
        for (int u = 0; u < kFirst; ++u)
            if (t_begin + u < t_end) copy(u, t_begin + u, row[u][0]);
        for (int t = t_begin; t < t_end && !stuck; t += kAhead) {
            int r0[kAhead], q[kAhead][2];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                r0[u] = row[u][0];
#pragma unroll
                for (int e = 0; e < 2; ++e) q[u][e] = row[u][e] >= 0 && pos[u][e] <= last_pos ? pos[u][e] : kNoPos;
            }
            keys(t + kAhead);
            entries(t + 2 * kAhead);
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                if (stuck || t + u >= t_end) continue;
                if (u < kFirst && t == t_begin) {
                    publish(u, q[u][0], q[u][1], false);
                } else if (__any_sync(0xffffffffu, min(q[u][0], q[u][1]) != kNoPos)) {      // (else nobody sees a key of this stage)
                    if (!wait_empty()) { stuck = true; continue; }
                    const int st = n % L::kStages;
                    copy(st, t + u, r0[u]);
                    publish(st, q[u][0], q[u][1], false);
                }
            }
        }
        if (!stuck && !wait_empty()) stuck = true;
        if (!stuck) publish(n % L::kStages, kNoPos, kNoPos, true);
        if (stuck)          // copies in flight land before the block's shared memory goes
            for (int i = max(0, n - L::kStages); i < n; ++i) mbar_wait(&full[i % L::kStages], static_cast<uint32_t>(i / L::kStages) & 1u);
    } else {
        // ================================================ consumers ===============================================
        // fragments: lane = 4 i + j holds, of S^T and O^T, rows i and i + 8 of columns (queries) 2 j and 2 j + 1
        const int i = lane / 4, j = lane % 4;
        uint32_t qf[NQ][KK][2];
        int qpos[NQ][2];
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
            // Q^T's columns: column i of this lane, features 2 j, 2 j + 1 (+ 8) of each sixteen
            const __nv_bfloat16* const q = static_cast<const __nv_bfloat16*>(a.Q) + out_row(a, s, p.head, r0 + min(8 * n + i, rows - 1)) * DH + 2 * j;
#pragma unroll
            for (int k = 0; k < KK; ++k) {
                qf[n][k][0] = __ldg(reinterpret_cast<const unsigned int*>(q + 16 * k));
                qf[n][k][1] = __ldg(reinterpret_cast<const unsigned int*>(q + 16 * k + 8));
            }
#pragma unroll
            for (int e = 0; e < 2; ++e) qpos[n][e] = s.q_pos0 + token_of(a, r0 + min(8 * n + 2 * j + e, rows - 1));
        }
        float o[NQ][KK][4], m[NQ][2], l[NQ][2];
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
#pragma unroll
            for (int k = 0; k < KK; ++k)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[n][k][e] = 0.f;
            m[n][0] = m[n][1] = -INFINITY;
            l[n][0] = l[n][1] = 0.f;
        }
        // ldmatrix: lane's row of the warp's 16 keys and the piece within a pair of 16-byte pieces.  K's fragment wants keys 0-7, 8-15 of the
        // lower piece, then of the upper; V^T's wants the lower piece's keys 0-7 and the upper's, then keys 8-15 of both
        const int key0 = warp * 16, kr = key0 + (lane & 15), kp = lane >> 4, vr = key0 + (lane & 7) + ((lane >> 4) << 3), vp = lane >> 3 & 1;
        for (int c = 0;; ++c) {
            const int st = c % L::kStages;
            if (!__all_sync(0xffffffffu, mbar_wait(&full[st], static_cast<uint32_t>(c / L::kStages) & 1u))) { stuck = true; break; }
            const int kind = s_kind[st];
            if (kind == kEnd) break;
            const uint32_t sk = base + st * L::kStage, sv = sk + L::kTile;
            float x[NQ][2][4];         // two chains of sums
#pragma unroll
            for (int n = 0; n < NQ; ++n)
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[n][h][e] = 0.f;
#pragma unroll
            for (int k = 0; k < KK; ++k) {
                uint32_t f[4];
                ldmatrix4(sk + (k / 4) * L::kHalf + kr * 128 + (((2 * (k % 4) + kp) ^ (kr & 7)) << 4), f);
#pragma unroll
                for (int n = 0; n < NQ; ++n) mma16816(x[n][k & 1], f, qf[n][k][0], qf[n][k][1]);
            }
            bool grow = false;
#pragma unroll
            for (int n = 0; n < NQ; ++n) {
#pragma unroll
                for (int e = 0; e < 4; ++e) x[n][0][e] = (x[n][0][e] + x[n][1][e]) * a.scale_log2;
                if ((kind & kMasked) != 0) {
                    const int p0 = s_pos[st][key0 + i], p1 = s_pos[st][key0 + i + 8];
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        if (p0 > qpos[n][e]) x[n][0][e] = -INFINITY;
                        if (p1 > qpos[n][e]) x[n][0][2 + e] = -INFINITY;
                    }
                }
#pragma unroll
                for (int e = 0; e < 2; ++e) grow = grow || fmaxf(x[n][0][e], x[n][0][2 + e]) > m[n][e] + kRescaleStep;
            }
            if (__any_sync(0xffffffffu, grow)) {
#pragma unroll
                for (int n = 0; n < NQ; ++n)
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        float top = fmaxf(x[n][0][e], x[n][0][2 + e]);
#pragma unroll
                        for (int d = 4; d < 32; d <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
                        const float to = fmaxf(top, m[n][e]), corr = part_weight(m[n][e], to);
                        m[n][e] = to;
                        l[n][e] *= corr;
#pragma unroll
                        for (int k = 0; k < KK; ++k) { o[n][k][e] *= corr; o[n][k][2 + e] *= corr; }
                    }
            }
            uint32_t pf[NQ][2][2];     // keys 0-7 and 8-15; a weight's two pieces
#pragma unroll
            for (int n = 0; n < NQ; ++n) {
                float w[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) w[e] = exp2_fast(x[n][0][e] - (m[n][e & 1] == -INFINITY ? 0.f : m[n][e & 1]));
                l[n][0] += w[0] + w[2];
                l[n][1] += w[1] + w[3];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    split_bf16(w[2 * h], w[2 * h + 1], pf[n][h][0], pf[n][h][1]);
                    pf[n][h][0] = transpose8(pf[n][h][0]);
                    pf[n][h][1] = transpose8(pf[n][h][1]);
                }
            }
            if ((kind & kHoles) != 0) {
                unsigned char* const v = base_ptr + st * L::kStage + L::kTile;
                for (int r = key0; r < key0 + 16; ++r)
                    if (s_pos[st][r] == kNoPos && lane < DH / 8) *reinterpret_cast<uint4*>(v + (lane / 8) * L::kHalf + r * 128 + (lane & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");      // ahead of the next copy to this place
                __syncwarp();
            }
#pragma unroll
            for (int k = 0; k < KK; ++k) {
                uint32_t f[4];
                ldmatrix4_trans(sv + (k / 4) * L::kHalf + vr * 128 + (((2 * (k % 4) + vp) ^ (vr & 7)) << 4), f);
#pragma unroll
                for (int n = 0; n < NQ; ++n)
#pragma unroll
                    for (int e = 0; e < 2; ++e) mma16816(o[n][k], f, pf[n][0][e], pf[n][1][e]);
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(&empty[st]);
        }
        asm volatile("bar.sync 1, 128;" ::: "memory");       // nobody reads the ring any more
        float* const acc = reinterpret_cast<float*>(base_ptr);
#pragma unroll
        for (int n = 0; n < NQ; ++n)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                float sum = l[n][e];
#pragma unroll
                for (int d = 4; d < 32; d <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
                const int at = warp * kRows + 8 * n + 2 * j + e;
                if (i == 0) {
                    s_sum[at] = sum;
                    s_max[at] = sum != sum ? INFINITY : m[n][e];       // a NaN among the logits that the row sees: the whole row's
                }
#pragma unroll
                for (int k = 0; k < KK; ++k) {
                    acc[at * (DH + 4) + 16 * k + i] = o[n][k][e];
                    acc[at * (DH + 4) + 16 * k + i + 8] = o[n][k][2 + e];
                }
            }
    }
    if (stuck && lane == 0) atomicOr(a.status, DODO_DEV_WAIT_TIMEOUT);
    __syncthreads();
    finish<__nv_bfloat16, DH, kThreads, true>(a, s, p, kRows, rows, kConsumers, reinterpret_cast<float*>(base_ptr), DH + 4, s_max, s_sum);
}

template <int DH, int NQ>
int launch(dodo_ctx* ctx, const PagedBoxes& m, const PagedGroup& g, const PagedArrays& a, cudaStream_t st) {
    auto kern = attend_paged_token_kernel<DH, NQ>;
    const int smem = Ring<DH>::kBytes + 1024;
    bool& set = ctx->paged_token_attr_set[(DH == 128 ? 2 : 0) + NQ - 1];
    if (!set) {
        const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
        if (e != cudaSuccess) return dodo_check_cuda(ctx, e, "paged token attend shared-memory attribute");
        set = true;
    }
    return dodo_check_cuda(ctx, dodo_launch_dependent(kern, dim3(static_cast<unsigned>(g.cta0[g.nseq])), dim3(kThreads), static_cast<size_t>(smem), st, m, g, a),
                           "paged token attend launch");
}

}  // namespace

int dodo_paged_box(int page, int most) {
    int box = 1;
    while (box < most && page % (2 * box) == 0) box *= 2;
    return box < 8 ? 0 : box;
}

int dodo_paged_boxes(dodo_ctx* ctx, const PagedArrays& a, int dh, int loc_rows, int box, int local_box, PagedBoxes& m) {
    memset(&m, 0, sizeof m);
    m.rows = box;
    const int width = a.Hkv * dh, rows = a.pages * a.page;
    int rc = DODO_OK;
    if (a.cK != nullptr) {
        rc = dodo_encode_bf16_rows(ctx, &m.cK, a.cK, width, rows, box);
        if (rc == DODO_OK) rc = dodo_encode_bf16_rows(ctx, &m.cV, a.cV, width, rows, box);
    }
    if (rc == DODO_OK && a.lK != nullptr) {
        rc = dodo_encode_bf16_rows(ctx, &m.lK, a.lK, width, loc_rows, local_box);
        if (rc == DODO_OK) rc = dodo_encode_bf16_rows(ctx, &m.lV, a.lV, width, loc_rows, local_box);
    }
    return rc;
}

PagedCut dodo_paged_token_cut(const dodo_ctx* ctx, int max_rows) { return {max_rows <= 8 ? 8 : 16, BN, 2 * ctx->num_sms, 4 * BN, 0}; }

int dodo_launch_paged_token(dodo_ctx* ctx, int dh, int max_rows, int loc_rows, const PagedGroup& g, const PagedArrays& a, cudaStream_t st) {
    PagedBoxes m;
    const int rc = dodo_paged_boxes(ctx, a, dh, loc_rows, dodo_paged_box(a.page, BN), BN, m);
    if (rc != DODO_OK) return rc;
    if (dh == 128) return max_rows <= 8 ? launch<128, 1>(ctx, m, g, a, st) : launch<128, 2>(ctx, m, g, a, st);
    return max_rows <= 8 ? launch<64, 1>(ctx, m, g, a, st) : launch<64, 2>(ctx, m, g, a, st);
}
