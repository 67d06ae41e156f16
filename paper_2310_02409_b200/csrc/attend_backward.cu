// Gradient of attention over [nugget cache ; local tokens].  With x = scale q.k (the softmax's argument) on visible
// (query, key) pairs, and the forward's output O and log-sum-exp at hand,
//   P = exp(x - lse),  D = sum(dO * O) per query,  dP = dO . V,  dS = P (dP - D)
//   dQ = scale dS K,   dK = scale dS^T Q,   dV = P^T dO,   dscore_j = sum over queries and heads of dS_j
// The probabilities are recomputed, nothing of size queries x keys is stored.  dscore is the straight-through gradient
// (Eq. 16-18): the paper adds s_j - StopGrad(s_j) to every logit of nugget j, so what reaches its score is the sum of
// the gradients at its logits.  Every output row is summed by one owner in a fixed order (no atomics): results repeat
// bit for bit.
//
// Two kernels here, a third (blocks of bf16 queries) on the tensor cores in attend_backward_dense.cu:
//   backward_stream_kernel  up to four queries per sequence (single-token steps), eight for fp32 rows of 128.  All traffic, no reuse: one pass reads
//       K and V once, writes dK and dV once and sums dQ, the queries and their dQ in registers.
//   backward_tile_kernel    fp32 blocks: key blocks and query blocks side by side in one launch,
//       64 keys x 32 queries at a time in shared memory, fp32 FMAs on register tiles.
#include "dodo_internal.cuh"

namespace {

constexpr int kThreads = 256;
constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ float ex2_approx(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t two_bf16(float lo, float hi) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}
template <typename T> __device__ __forceinline__ uint4 pack16(const float* f);
template <> __device__ __forceinline__ uint4 pack16<float>(const float* f) {
    return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
}
template <> __device__ __forceinline__ uint4 pack16<__nv_bfloat16>(const float* f) {
    return make_uint4(two_bf16(f[0], f[1]), two_bf16(f[2], f[3]), two_bf16(f[4], f[5]), two_bf16(f[6], f[7]));
}
__device__ __forceinline__ float4 load4(const float* p) { return __ldg(reinterpret_cast<const float4*>(p)); }
__device__ __forceinline__ void store4(float* p, float4 v) { *reinterpret_cast<float4*>(p) = v; }
// a query's statistic: minus the log-sum-exp in base 2, -inf (every weight comes out 0) where the query sees nothing
__device__ __forceinline__ float minus_lse2(float lse) { return lse == -INFINITY ? -INFINITY : -lse * kLog2e; }

// One more of `n` arrivals on a counter that is zero between launches; true for the last, which finds the others' writes
// visible.  All threads of the block call it.
__device__ __forceinline__ bool last_arrival(int* counter, int n, int* flag) {
    __threadfence();
    __syncthreads();
    if (threadIdx.x == 0) {
        const int t = atomicAdd(counter, 1);
        *flag = t == n - 1;
        if (t == n - 1) *counter = 0;
    }
    __syncthreads();
    const bool last = *flag != 0;
    if (last) __threadfence();
    __syncthreads();
    return last;
}

// Gradient of the scores of cache rows [row, row + n): the heads' sums added up in head order by the last head to arrive.
__device__ __forceinline__ void finish_scores(const BackwardArrays& a, int H, int row, int n, int* counter, int* flag) {
    if (!last_arrival(counter, H, flag)) return;
    for (int i = threadIdx.x; i < n; i += kThreads) {
        float s = 0.f;
        for (int h = 0; h < H; ++h) s += __ldcg(a.score_part + static_cast<size_t>(h) * a.score_rows + row + i);
        a.dscore[row + i] = s;
    }
}

// =============================================== few queries ============================================================
template <typename T, int DH, int QT, int U>
__global__ void __launch_bounds__(kThreads)
backward_stream_kernel(const BackwardArrays a, const __grid_constant__ BackwardGroup g, int H, float scale) {
    constexpr int E = Vec16<T>::kElems, LPR = DH / E, NB = kThreads / LPR;
    __shared__ float red[NB][DH + 4];
    __shared__ int s_flag;
    const int tid = threadIdx.x, bundle = tid / LPR, lig = tid % LPR;
    int b = 0;
    for (int i = 1; i < g.nseq; ++i) b += g.seq[i].kv0 <= static_cast<int>(blockIdx.x) ? 1 : 0;
    const BackwardSeq sq = g.seq[b];
    const int r = static_cast<int>(blockIdx.x) - sq.kv0;
    const int chunk = r % sq.nchunk, h = r / sq.nchunk;
    const int n_keys = sq.c_len + sq.l_len;
    const int k0 = min(n_keys, chunk * sq.ctiles * NB), k1 = min(n_keys, k0 + sq.ctiles * NB);
    const size_t row_elems = static_cast<size_t>(H) * DH;
    const size_t col = static_cast<size_t>(h) * DH + lig * E;
    // ahead of the dependency wait, hints to L2 for the rows of the first batches (a hint brings nothing into the SM, and L2 is
    // where writes of the kernel before would land too)
    if (lig % 8 == 0) {
#pragma unroll
        for (int u = 0; u < 2 * U; ++u) {
            const int j = k0 + u * NB + bundle;
            if (j < k1) {
                const bool cached = j < sq.c_len;
                const size_t at = static_cast<size_t>(cached ? sq.c_row0 + j : sq.l_row0 + (j - sq.c_len)) * row_elems + col;
                asm volatile("prefetch.global.L2 [%0];" :: "l"(static_cast<const T*>(cached ? a.cK : a.lK) + at));
                asm volatile("prefetch.global.L2 [%0];" :: "l"(static_cast<const T*>(cached ? a.cV : a.lV) + at));
            }
        }
    }
    dodo_grid_dependency_sync();

    float q[QT][E], go[QT][E], dq[QT][E], nlse[QT], delta[QT];
    int qpos[QT];
#pragma unroll
    for (int i = 0; i < QT; ++i) {
        float o[E];
#pragma unroll
        for (int e = 0; e < E; ++e) q[i][e] = go[i][e] = o[e] = dq[i][e] = 0.f;
        nlse[i] = -INFINITY;
        qpos[i] = static_cast<int>(0x80000000);
        if (i < sq.tq) {
            const size_t at = static_cast<size_t>(sq.q_row0 + i) * row_elems + col;
            Vec16<T>::unpack(*reinterpret_cast<const uint4*>(static_cast<const T*>(a.Q) + at), q[i]);
            Vec16<T>::unpack(*reinterpret_cast<const uint4*>(static_cast<const T*>(a.dO) + at), go[i]);
            Vec16<T>::unpack(*reinterpret_cast<const uint4*>(static_cast<const T*>(a.O) + at), o);
            nlse[i] = minus_lse2(a.lse[static_cast<size_t>(sq.q_row0 + i) * H + h]);
            qpos[i] = sq.q_pos0 + i;
        }
        float d = 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) d = fmaf(go[i][e], o[e], d);
#pragma unroll
        for (int s = LPR / 2; s > 0; s >>= 1) d += __shfl_xor_sync(0xffffffffu, d, s);
        delta[i] = d;
    }
    const float scale2 = scale * kLog2e;

    uint4 kv[U], vv[U];
    int kpos[U];
    auto load = [&](int base) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int j = base + u * NB + bundle;
            kv[u] = vv[u] = make_uint4(0, 0, 0, 0);
            kpos[u] = 0x7fffffff;
            if (j < k1) {
                const bool cached = j < sq.c_len;
                const int row = cached ? sq.c_row0 + j : sq.l_row0 + (j - sq.c_len);
                const size_t at = static_cast<size_t>(row) * row_elems + col;
                kv[u] = ld_stream16(static_cast<const T*>(cached ? a.cK : a.lK) + at);
                vv[u] = ld_stream16(static_cast<const T*>(cached ? a.cV : a.lV) + at);
                kpos[u] = cached ? __ldg(a.cache_pos + row) : sq.l_pos0 + (j - sq.c_len);
            }
        }
    };
    load(k0);
    for (int base = k0; base < k1; base += NB * U) {
        uint4 kc[U], vc[U];
        int pc[U];
#pragma unroll
        for (int u = 0; u < U; ++u) { kc[u] = kv[u]; vc[u] = vv[u]; pc[u] = kpos[u]; }
        load(base + NB * U);
        // logits and dP of the batch; the sums over a row's lanes for all keys and queries together
        float s[QT][U], t[QT][U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float k[E], v[E];
            Vec16<T>::unpack(kc[u], k);
            Vec16<T>::unpack(vc[u], v);
#pragma unroll
            for (int i = 0; i < QT; ++i) {
                float2 x = make_float2(0.f, 0.f), y = make_float2(0.f, 0.f);
#pragma unroll
                for (int e = 0; e < E; e += 2) {
                    x = __ffma2_rn(make_float2(q[i][e], q[i][e + 1]), make_float2(k[e], k[e + 1]), x);
                    y = __ffma2_rn(make_float2(go[i][e], go[i][e + 1]), make_float2(v[e], v[e + 1]), y);
                }
                s[i][u] = x.x + x.y;
                t[i][u] = y.x + y.y;
            }
        }
#pragma unroll
        for (int o = LPR / 2; o > 0; o >>= 1)
#pragma unroll
            for (int i = 0; i < QT; ++i)
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    s[i][u] += __shfl_xor_sync(0xffffffffu, s[i][u], o);
                    t[i][u] += __shfl_xor_sync(0xffffffffu, t[i][u], o);
                }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int j = base + u * NB + bundle;
            float k[E], dk[E], dv[E], ds_sum = 0.f;
            Vec16<T>::unpack(kc[u], k);
#pragma unroll
            for (int e = 0; e < E; ++e) dk[e] = dv[e] = 0.f;
#pragma unroll
            for (int i = 0; i < QT; ++i) {
                const bool see = pc[u] <= qpos[i];       // a masked key takes no part, whatever its row holds
                const float p = see ? ex2_approx(fmaf(s[i][u], scale2, nlse[i])) : 0.f;
                const float ds = see ? p * (t[i][u] - delta[i]) : 0.f;
                ds_sum += ds;
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    dk[e] = fmaf(ds, q[i][e], dk[e]);
                    dv[e] = fmaf(p, go[i][e], dv[e]);
                    dq[i][e] = see ? fmaf(ds, k[e], dq[i][e]) : dq[i][e];
                }
            }
            if (j < k1) {
#pragma unroll
                for (int e = 0; e < E; ++e) dk[e] *= scale;
                const bool cached = j < sq.c_len;
                const int row = cached ? sq.c_row0 + j : sq.l_row0 + (j - sq.c_len);
                const size_t at = static_cast<size_t>(row) * row_elems + col;
                *reinterpret_cast<uint4*>(static_cast<T*>(cached ? a.dcK : a.dlK) + at) = pack16<T>(dk);
                *reinterpret_cast<uint4*>(static_cast<T*>(cached ? a.dcV : a.dlV) + at) = pack16<T>(dv);
                if (cached && a.dscore != nullptr && lig == 0) a.score_part[static_cast<size_t>(h) * a.score_rows + row] = ds_sum;
            }
        }
    }

    // ---- dQ: the bundles' sums, then the chunks' --------------------------------------------------------------
#pragma unroll 1
    for (int i = 0; i < QT; ++i) {
        if (i >= sq.tq) break;
        float mine[E];
#pragma unroll
        for (int e = 0; e < E; ++e) {
            mine[e] = 0.f;
#pragma unroll
            for (int k = 0; k < QT; ++k) mine[e] = k == i ? dq[k][e] : mine[e];
            red[bundle][lig * E + e] = mine[e];
        }
        __syncthreads();
        if (tid < DH) {
            float sum = 0.f;
#pragma unroll
            for (int n = 0; n < NB; ++n) sum += red[n][tid];
            if (sq.nchunk == 1) {
                const float v = sum * scale;
                T* out = static_cast<T*>(a.dQ) + static_cast<size_t>(sq.q_row0 + i) * row_elems + static_cast<size_t>(h) * DH + tid;
                if constexpr (sizeof(T) == 4) *out = v; else *out = __float2bfloat16_rn(v);
            } else {
                a.dq_part[(static_cast<size_t>(sq.part0 + h * sq.nchunk + chunk) * QT + i) * DH + tid] = sum;
            }
        }
        __syncthreads();
    }
    // cache rows of this chunk: their score gradients, once every head has been here
    const int c1 = min(sq.c_len, k1);
    if (a.dscore != nullptr && k0 < c1) finish_scores(a, H, sq.c_row0 + k0, c1 - k0, a.tickets + sq.stick0 + chunk, &s_flag);
    if (sq.nchunk > 1 && sq.tq > 0 && last_arrival(a.tickets + sq.qtick0 + h, sq.nchunk, &s_flag)) {
        for (int i = tid; i < sq.tq * DH; i += kThreads) {
            float sum = 0.f;
            for (int c = 0; c < sq.nchunk; ++c)
                sum += __ldcg(a.dq_part + (static_cast<size_t>(sq.part0 + h * sq.nchunk + c) * QT + i / DH) * DH + i % DH);
            const float v = sum * scale;
            T* out = static_cast<T*>(a.dQ) + static_cast<size_t>(sq.q_row0 + i / DH) * row_elems + static_cast<size_t>(h) * DH + i % DH;
            if constexpr (sizeof(T) == 4) *out = v; else *out = __float2bfloat16_rn(v);
        }
    }
}

// =============================================== statistics =============================================================
// (for the tensor-core kernel, whose statistics travel with its tiles; the others make their own)
// -(log-sum-exp in base 2) and -(sum of dO * O) of every query, one row per head so that a tile's entries are contiguous;
// entries behind a sequence's last query, up to a multiple of 64, are -inf and 0: such a column's weights come out 0.
__global__ void __launch_bounds__(kThreads)
backward_stats_kernel(const BackwardArrays a, const __grid_constant__ BackwardGroup g, int H, int DH) {
    constexpr int E = Vec16<__nv_bfloat16>::kElems;
    const int lpr = DH / E;                             // lanes per row: 8 or 16
    const int per_block = kThreads / lpr;
    const long long unit = static_cast<long long>(blockIdx.x) * per_block + threadIdx.x / lpr;   // (entry, head), heads fastest
    const int entry = static_cast<int>(unit / H), h = static_cast<int>(unit % H), lig = threadIdx.x % lpr;
    int b = 0;
    for (int i = 1; i < g.nseq; ++i) b += g.seq[i].stat0 <= entry ? 1 : 0;
    const int q = entry - g.seq[b].stat0;
    dodo_grid_dependency_sync();
    const bool live = entry < g.stat_rows && q < g.seq[b].tq;
    float d = 0.f;
    const size_t row = static_cast<size_t>(g.seq[b].q_row0 + q) * H + h;
    if (live) {
        float x[E], y[E];
        Vec16<__nv_bfloat16>::unpack(ld_stream16(static_cast<const __nv_bfloat16*>(a.dO) + row * DH + lig * E), x);
        Vec16<__nv_bfloat16>::unpack(ld_stream16(static_cast<const __nv_bfloat16*>(a.O) + row * DH + lig * E), y);
#pragma unroll
        for (int e = 0; e < E; ++e) d = fmaf(x[e], y[e], d);
    }
    for (int s = lpr / 2; s > 0; s >>= 1) d += __shfl_xor_sync(0xffffffffu, d, s);
    if (entry < g.stat_rows && lig == 0) {
        float* s = a.stats + (static_cast<size_t>(h) * g.stat_rows + (entry & ~63)) * 2 + (entry & 63);
        s[0] = live ? minus_lse2(a.lse[row]) : -INFINITY;
        s[64] = live ? -d : 0.f;
    }
}

// =============================================== score gradients =========================================================
// dscore of 32 cache rows per block: a warp adds up every eighth of the parts, then the warps' sums are added in warp order.
__global__ void __launch_bounds__(kThreads)
backward_scores_kernel(const BackwardArrays a, const __grid_constant__ BackwardGroup g, int parts) {
    __shared__ float sums[kThreads / 32][32];
    const int b = blockIdx.y, row = static_cast<int>(blockIdx.x) * 32 + (threadIdx.x & 31), warp = threadIdx.x >> 5;
    dodo_grid_dependency_sync();
    if (static_cast<int>(blockIdx.x) * 32 >= g.seq[b].c_len) return;
    float s = 0.f;
    if (row < g.seq[b].c_len) {
        const float* p = a.score_part + g.seq[b].c_row0 + row;
#pragma unroll 8
        for (int i = warp; i < parts; i += kThreads / 32) s += __ldcg(p + static_cast<size_t>(i) * a.score_rows);
    }
    sums[warp][threadIdx.x & 31] = s;
    __syncthreads();
    if (warp == 0 && row < g.seq[b].c_len) {
#pragma unroll
        for (int w = 1; w < kThreads / 32; ++w) s += sums[w][threadIdx.x];
        a.dscore[g.seq[b].c_row0 + row] = s;
    }
}

// =============================================== fp32 tiles ==============================================================
constexpr int TK = 64, TQ = 32;     // keys and queries of a tile
constexpr int LDP = TK + 4;         // row of the weight tiles

template <int DH> struct TileSmem {
    static constexpr int LD = DH + 4;   // rows 4 banks apart: eight rows' 16-byte pieces cover all banks
    float K[TK][LD], V[TK][LD], Q[TQ][LD], G[TQ][LD];
    float P[TQ][LDP], S[TQ][LDP];       // weights and dS, [query][key]
    float2 stat[TQ];
    int kpos[TK];
    int flag;
};

// statistics of queries [q0, q0 + nq) of a sequence and head: eight threads a query
template <int DH>
__device__ __forceinline__ void tile_stats(float2* dst, const BackwardArrays& a, int H, int h, int row0, int nq) {
    const int q = threadIdx.x / 8, part = threadIdx.x % 8;
    float d = 0.f;
    const size_t row = static_cast<size_t>(row0 + q) * H + h;
    if (q < nq) {
#pragma unroll
        for (int i = 0; i < DH / 32; ++i) {
            const float4 x = load4(static_cast<const float*>(a.dO) + row * DH + 4 * (part + 8 * i));
            const float4 y = load4(static_cast<const float*>(a.O) + row * DH + 4 * (part + 8 * i));
            d = fmaf(x.x, y.x, fmaf(x.y, y.y, fmaf(x.z, y.z, fmaf(x.w, y.w, d))));
        }
    }
#pragma unroll
    for (int s = 4; s > 0; s >>= 1) d += __shfl_xor_sync(0xffffffffu, d, s);
    if (part == 0) dst[q] = q < nq ? make_float2(minus_lse2(__ldg(a.lse + row)), -d) : make_float2(-INFINITY, 0.f);
}

// N rows of a head's matrix on their way to shared memory, those from `rows` on as zeros
template <int N, int DH> struct RowPieces {
    static constexpr int V4 = DH / 4, kIter = N * V4 / kThreads;
    static_assert(N * V4 % kThreads == 0, "whole passes");
    float4 v[kIter];
    __device__ __forceinline__ void fetch(const float* src, size_t row_elems, int row0, int rows) {
#pragma unroll
        for (int i = 0; i < kIter; ++i) {
            const int at = threadIdx.x + i * kThreads, r = at / V4, c = at % V4;
            v[i] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (r < rows) v[i] = load4(src + static_cast<size_t>(row0 + r) * row_elems + 4 * c);
        }
    }
    __device__ __forceinline__ void put(float (*dst)[DH + 4]) const {
#pragma unroll
        for (int i = 0; i < kIter; ++i) {
            const int at = threadIdx.x + i * kThreads;
            *reinterpret_cast<float4*>(&dst[at / V4][4 * (at % V4)]) = v[i];
        }
    }
};
// Dot products of a tile, 32 keys x 8 queries per warp (warp w: keys from 32 (w & 1), queries from 8 (w / 2)).  A thread sums a quarter
// of the features for 8 keys x 4 queries, so that a load of 16 bytes feeds 21 products (with all the features of 4 x 2 pairs a thread
// it was 5, and shared memory the bound); the four quarters are added up by exchanges that leave a lane 4 keys x 2 queries:
// keys lane_key + 4 i, queries lane_query + 2 j.  The quarters start two pieces apart, which spreads a load over all banks.
template <int DH>
__device__ __forceinline__ void tile_dots(const float (*A)[DH + 4], const float (*B)[DH + 4], float (&out)[4][2]) {
    constexpr int kPieces = DH / 16;                // 16-byte pieces of a quarter
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, quarter = lane >> 3;
    const float* const a = A[32 * (warp & 1) + (lane >> 1 & 3)] + quarter * (DH / 4);
    const float* const b = B[8 * (warp >> 1) + (lane & 1)] + quarter * (DH / 4);
    // head size 128: pairs of features in packed sums; 64, where registers decide whether two blocks fit an SM: single ones
    constexpr bool kPacked = DH == 128;
    float2 s[8][4];
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) s[i][j] = make_float2(0.f, 0.f);
#pragma unroll kPacked ? 2 : 1
    for (int c = 0; c < kPieces; ++c) {
        const int at = 4 * ((c + 2 * quarter) & (kPieces - 1));
        float4 x[8], y[4];
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = *reinterpret_cast<const float4*>(a + 4 * i * (DH + 4) + at);
#pragma unroll
        for (int j = 0; j < 4; ++j) y[j] = *reinterpret_cast<const float4*>(b + 2 * j * (DH + 4) + at);
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if constexpr (kPacked) {
                    s[i][j] = __ffma2_rn(make_float2(x[i].x, x[i].y), make_float2(y[j].x, y[j].y), s[i][j]);
                    s[i][j] = __ffma2_rn(make_float2(x[i].z, x[i].w), make_float2(y[j].z, y[j].w), s[i][j]);
                } else {
                    s[i][j].x = fmaf(x[i].x, y[j].x, fmaf(x[i].y, y[j].y, fmaf(x[i].z, y[j].z, fmaf(x[i].w, y[j].w, s[i][j].x))));
                }
            }
    }
    const bool up16 = (lane & 16) != 0, up8 = (lane & 8) != 0;
    float h[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float low = s[i][j].x + s[i][j].y, high = s[i + 4][j].x + s[i + 4][j].y;
            h[i][j] = (up16 ? high : low) + __shfl_xor_sync(0xffffffffu, up16 ? low : high, 16);
        }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j)
            out[i][j] = (up8 ? h[i][j + 2] : h[i][j]) + __shfl_xor_sync(0xffffffffu, up8 ? h[i][j] : h[i][j + 2], 8);
}
// weights and dS of a tile (a warp whose queries are all behind the last has nothing to do)
template <int DH>
__device__ __forceinline__ void tile_weights(TileSmem<DH>& sm, int nq, int qpos0, float scale2) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (8 * (warp >> 1) >= nq) return;
    float s[4][2], t[4][2];
    tile_dots<DH>(sm.K, sm.Q, s);
    tile_dots<DH>(sm.V, sm.G, t);
    const int key0 = 32 * (warp & 1) + (lane >> 1 & 3) + (lane >> 4) * 16, q0 = 8 * (warp >> 1) + (lane & 1) + (lane >> 3 & 1) * 4;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int key = key0 + 4 * i, q = q0 + 2 * j;
            const bool see = q < nq && sm.kpos[key] <= qpos0 + q;
            const float2 st = sm.stat[q];
            const float p = see ? ex2_approx(fmaf(s[i][j], scale2, st.x)) : 0.f;
            sm.P[q][key] = p;
            sm.S[q][key] = see ? p * (t[i][j] + st.y) : 0.f;
        }
}

template <int DH>
__global__ void __launch_bounds__(kThreads, DH == 64 ? 2 : 1)
backward_tile_kernel(const BackwardArrays a, const __grid_constant__ BackwardGroup g, int H, float scale) {
    extern __shared__ __align__(16) unsigned char raw[];
    TileSmem<DH>& sm = *reinterpret_cast<TileSmem<DH>*>(raw);
    const int tid = threadIdx.x;
    const size_t row_elems = static_cast<size_t>(H) * DH;
    const float scale2 = scale * kLog2e;
    // query blocks first: they are the longer ones
    const bool own_queries = static_cast<int>(blockIdx.x) < g.q_blocks;
    const int bid = static_cast<int>(blockIdx.x) - (own_queries ? 0 : g.q_blocks);
    int b = 0;
    for (int i = 1; i < g.nseq; ++i) b += (own_queries ? g.seq[i].q0 : g.seq[i].kv0) <= bid ? 1 : 0;
    const BackwardSeq sq = g.seq[b];
    const int tx = tid % 16, ty = tid / 16;
    constexpr int ND = DH / 64;       // a thread owns 4 consecutive features in each run of 64
    dodo_grid_dependency_sync();

    if (!own_queries) {
        const int r = bid - sq.kv0;
        const int h = r % H, tile = r / H;
        const int nt_c = (sq.c_len + TK - 1) / TK;
        const bool cached = tile < nt_c;
        const int first = (cached ? tile : tile - nt_c) * TK;
        const int rows = min(TK, (cached ? sq.c_len : sq.l_len) - first);
        const int row0 = (cached ? sq.c_row0 : sq.l_row0) + first;
        const float* gk = static_cast<const float*>(cached ? a.cK : a.lK) + static_cast<size_t>(h) * DH;
        const float* gv = static_cast<const float*>(cached ? a.cV : a.lV) + static_cast<size_t>(h) * DH;
        {
            RowPieces<TK, DH> k, v;
            k.fetch(gk, row_elems, row0, rows);
            v.fetch(gv, row_elems, row0, rows);
            k.put(sm.K);
            v.put(sm.V);
        }
        if (tid < TK) sm.kpos[tid] = tid >= rows ? 0x7fffffff : cached ? __ldg(a.cache_pos + row0 + tid) : sq.l_pos0 + first + tid;
        float2 dk[4][2 * ND], dv[4][2 * ND];
        float score[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            score[i] = 0.f;
#pragma unroll
            for (int e = 0; e < 2 * ND; ++e) dk[i][e] = dv[i][e] = make_float2(0.f, 0.f);
        }
        RowPieces<TQ, DH> next_q, next_g;
        auto fetch_queries = [&](int q0) {
            const int n = min(TQ, sq.tq - q0);
            next_q.fetch(static_cast<const float*>(a.Q) + static_cast<size_t>(h) * DH, row_elems, sq.q_row0 + q0, n);
            next_g.fetch(static_cast<const float*>(a.dO) + static_cast<size_t>(h) * DH, row_elems, sq.q_row0 + q0, n);
        };
        // queries from the first one that can see a key of a local tile
        const int q_start = cached ? 0 : max(0, sq.l_pos0 + first - sq.q_pos0) / TQ * TQ;
        if (q_start < sq.tq) fetch_queries(q_start);
        for (int q0 = q_start; q0 < sq.tq; q0 += TQ) {
            const int nq = min(TQ, sq.tq - q0);
            if (q0 > q_start) __syncthreads();      // (the first queries come with the keys)
            next_q.put(sm.Q);
            next_g.put(sm.G);
            tile_stats<DH>(sm.stat, a, H, h, sq.q_row0 + q0, nq);
            __syncthreads();
            if (q0 + TQ < sq.tq) fetch_queries(q0 + TQ);
            tile_weights<DH>(sm, nq, sq.q_pos0 + q0, scale2);
            __syncthreads();
#pragma unroll 2
            for (int q = 0; q < nq; ++q) {
                const float4 p = *reinterpret_cast<const float4*>(&sm.P[q][4 * ty]), s = *reinterpret_cast<const float4*>(&sm.S[q][4 * ty]);
                const float pa[4] = {p.x, p.y, p.z, p.w}, sa[4] = {s.x, s.y, s.z, s.w};
#pragma unroll
                for (int i = 0; i < 4; ++i) score[i] += sa[i];
#pragma unroll
                for (int d = 0; d < ND; ++d) {
                    const float4 o = *reinterpret_cast<const float4*>(&sm.G[q][64 * d + 4 * tx]);
                    const float4 x = *reinterpret_cast<const float4*>(&sm.Q[q][64 * d + 4 * tx]);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float2 p2 = make_float2(pa[i], pa[i]), s2 = make_float2(sa[i], sa[i]);
                        dv[i][2 * d] = __ffma2_rn(p2, make_float2(o.x, o.y), dv[i][2 * d]);
                        dv[i][2 * d + 1] = __ffma2_rn(p2, make_float2(o.z, o.w), dv[i][2 * d + 1]);
                        dk[i][2 * d] = __ffma2_rn(s2, make_float2(x.x, x.y), dk[i][2 * d]);
                        dk[i][2 * d + 1] = __ffma2_rn(s2, make_float2(x.z, x.w), dk[i][2 * d + 1]);
                    }
                }
            }
        }
        float* ok = static_cast<float*>(cached ? a.dcK : a.dlK) + static_cast<size_t>(h) * DH;
        float* ov = static_cast<float*>(cached ? a.dcV : a.dlV) + static_cast<size_t>(h) * DH;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int key = 4 * ty + i;
            if (key >= rows) continue;
            const size_t at = static_cast<size_t>(row0 + key) * row_elems;
#pragma unroll
            for (int d = 0; d < ND; ++d) {
                store4(ok + at + 64 * d + 4 * tx, make_float4(dk[i][2 * d].x * scale, dk[i][2 * d].y * scale, dk[i][2 * d + 1].x * scale, dk[i][2 * d + 1].y * scale));
                store4(ov + at + 64 * d + 4 * tx, make_float4(dv[i][2 * d].x, dv[i][2 * d].y, dv[i][2 * d + 1].x, dv[i][2 * d + 1].y));
            }
            if (cached && a.dscore != nullptr && tx == 0) a.score_part[static_cast<size_t>(h) * a.score_rows + row0 + key] = score[i];
        }
        if (cached && a.dscore != nullptr) finish_scores(a, H, row0, rows, a.tickets + sq.stick0 + tile, &sm.flag);
        return;
    }

    // ---- a query tile (or a chunk of its key list) -------------------------------------------------------------------
    int r = bid - sq.q0;
    const int chunk = r % sq.nchunk; r /= sq.nchunk;
    const int h = r % H, qt = r / H;
    const int q0 = qt * TQ, nq = min(TQ, sq.tq - q0);
    const int l_vis = dodo_visible_local(sq.l_len, sq.l_pos0, sq.q_pos0 + q0 + nq - 1);
    const int nt_c = (sq.c_len + TK - 1) / TK, nt = nt_c + (l_vis + TK - 1) / TK;
    const int t0 = min(nt, chunk * sq.ctiles), t1 = min(nt, t0 + sq.ctiles);
    {
        RowPieces<TQ, DH> q, g2;
        q.fetch(static_cast<const float*>(a.Q) + static_cast<size_t>(h) * DH, row_elems, sq.q_row0 + q0, nq);
        g2.fetch(static_cast<const float*>(a.dO) + static_cast<size_t>(h) * DH, row_elems, sq.q_row0 + q0, nq);
        q.put(sm.Q);
        g2.put(sm.G);
    }
    tile_stats<DH>(sm.stat, a, H, h, sq.q_row0 + q0, nq);
    // a warp owns four queries, a lane DH / 32 consecutive features of theirs
    const int lane = tid & 31, qw = 4 * (tid >> 5);
    float2 dq[4][ND];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int e = 0; e < ND; ++e) dq[i][e] = make_float2(0.f, 0.f);
    // the next keys are on their way while these are worked on
    RowPieces<TK, DH> next_k, next_v;
    int next_pos = 0;
    auto fetch_keys = [&](int t) {
        const bool cached = t < nt_c;
        const int first = (cached ? t : t - nt_c) * TK;
        const int rows = min(TK, (cached ? sq.c_len : l_vis) - first);
        const int row0 = (cached ? sq.c_row0 : sq.l_row0) + first;
        next_k.fetch(static_cast<const float*>(cached ? a.cK : a.lK) + static_cast<size_t>(h) * DH, row_elems, row0, rows);
        next_v.fetch(static_cast<const float*>(cached ? a.cV : a.lV) + static_cast<size_t>(h) * DH, row_elems, row0, rows);
        if (tid < TK) next_pos = tid >= rows ? 0x7fffffff : cached ? __ldg(a.cache_pos + row0 + tid) : sq.l_pos0 + first + tid;
    };
    if (t0 < t1) fetch_keys(t0);
    for (int t = t0; t < t1; ++t) {
        if (t > t0) __syncthreads();
        next_k.put(sm.K);
        next_v.put(sm.V);
        if (tid < TK) sm.kpos[tid] = next_pos;
        __syncthreads();
        if (t + 1 < t1) fetch_keys(t + 1);
        tile_weights<DH>(sm, nq, sq.q_pos0 + q0, scale2);
        __syncthreads();
        if (qw < nq) {
#pragma unroll 2
            for (int k = 0; k < TK; k += 4) {
                float w[4][4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float4 u = *reinterpret_cast<const float4*>(&sm.S[qw + i][k]);
                    w[i][0] = u.x; w[i][1] = u.y; w[i][2] = u.z; w[i][3] = u.w;
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    float2 x[ND];
                    const float2* const row = reinterpret_cast<const float2*>(&sm.K[k + e][2 * ND * lane]);
                    if constexpr (ND == 2) {
                        const float4 v = *reinterpret_cast<const float4*>(row);
                        x[0] = make_float2(v.x, v.y);
                        x[1] = make_float2(v.z, v.w);
                    } else {
                        x[0] = *row;
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (w[i][e] != 0.f) {   // a key that some queries of the tile do not see may hold anything: its dS is exactly 0 there
#pragma unroll
                            for (int d = 0; d < ND; ++d) dq[i][d] = __ffma2_rn(make_float2(w[i][e], w[i][e]), x[d], dq[i][d]);
                        }
                }
            }
        }
    }
    float* out = static_cast<float*>(a.dQ) + static_cast<size_t>(sq.q_row0 + q0) * row_elems + static_cast<size_t>(h) * DH;
    const size_t part = static_cast<size_t>(sq.part0 + (qt * H + h) * sq.nchunk);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int q = qw + i;
        if (q >= nq) continue;
        float* const row = (sq.nchunk == 1 ? out + q * row_elems : a.dq_part + ((part + chunk) * TQ + q) * DH) + 2 * ND * lane;
        const float f = sq.nchunk == 1 ? scale : 1.f;
#pragma unroll
        for (int d = 0; d < ND; ++d) *reinterpret_cast<float2*>(row + 2 * d) = make_float2(dq[i][d].x * f, dq[i][d].y * f);
    }
    if (sq.nchunk == 1 || !last_arrival(a.tickets + sq.qtick0 + qt * H + h, sq.nchunk, &sm.flag)) return;
    for (int i = tid; i < nq * (DH / 4); i += kThreads) {
        const int q = i / (DH / 4), c = 4 * (i % (DH / 4));
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int n = 0; n < sq.nchunk; ++n) {
            const float4 x = __ldcg(reinterpret_cast<const float4*>(a.dq_part + ((part + n) * TQ + q) * DH + c));
            v.x += x.x; v.y += x.y; v.z += x.z; v.w += x.w;
        }
        store4(out + q * row_elems + c, make_float4(v.x * scale, v.y * scale, v.z * scale, v.w * scale));
    }
}

template <typename T, int DH>
int launch_stream(dodo_ctx* ctx, int H, float scale, int max_tq, const BackwardGroup& g, const BackwardArrays& a, cudaStream_t st) {
    const dim3 grid(static_cast<unsigned>(g.kv_blocks)), block(kThreads);
    cudaError_t e;
    if constexpr (sizeof(T) == 4 && DH == 128)
        if (max_tq > 4)
            return dodo_check_cuda(ctx, dodo_launch_dependent(backward_stream_kernel<T, DH, 8, 2>, grid, block, 0, st, a, g, H, scale), "attend gradient launch");
    e = max_tq <= 1 ? dodo_launch_dependent(backward_stream_kernel<T, DH, 1, 4>, grid, block, 0, st, a, g, H, scale)
                        : max_tq <= 2 ? dodo_launch_dependent(backward_stream_kernel<T, DH, 2, 2>, grid, block, 0, st, a, g, H, scale)
                                      : dodo_launch_dependent(backward_stream_kernel<T, DH, 4, 2>, grid, block, 0, st, a, g, H, scale);
    return dodo_check_cuda(ctx, e, "attend gradient launch");
}

template <int DH>
int launch_tile(dodo_ctx* ctx, int slot, int H, float scale, const BackwardGroup& g, const BackwardArrays& a, cudaStream_t st) {
    auto kern = backward_tile_kernel<DH>;
    const size_t smem = sizeof(TileSmem<DH>);
    if (!ctx->backward_attr_set[slot]) {
        const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem));
        if (e != cudaSuccess) return dodo_check_cuda(ctx, e, "attend gradient shared-memory attribute");
        ctx->backward_attr_set[slot] = true;
    }
    return dodo_check_cuda(ctx, dodo_launch_dependent(kern, dim3(static_cast<unsigned>(g.q_blocks + g.kv_blocks)), dim3(kThreads), smem, st, a, g, H, scale),
                           "attend gradient launch");
}

}  // namespace

// The streaming kernel beats the others up to four queries everywhere (4 queries over 8 x 269 keys of 32 heads of 128: bf16 33.5
// against 58 us on the tensor cores, fp32 36 against 124; 4160 keys: 53 / 76, 62 / 197; head size 64: bf16 22 / 51, fp32 with 8
// heads 12 / 18).  With eight it still does for fp32 rows of 128 (66 to 72 against 124 us; 106 to 112 against 197); at 64
// the tiles are as fast (20 to 23 against 18 to 20), and bf16 has twice the features a lane, whose sums eight queries do not fit.
int dodo_backward_stream_queries(int dtype, int dh) { return dtype == DODO_F32 && dh == 128 ? 8 : 4; }

BackwardTiles dodo_backward_tiles(int variant, int dtype, int dh) {
    const int bundles = kThreads / (dh * static_cast<int>(dodo_elem_bytes(dtype)) / 16);
    if (variant == DODO_BWD_STREAM) return {bundles, dodo_backward_stream_queries(dtype, dh), bundles};
    if (variant == DODO_BWD_DENSE) return dodo_backward_dense_tiles();
    return {TK, TQ, TK};
}

int dodo_launch_backward_stream(dodo_ctx* ctx, int dtype, int H, int dh, float sm_scale, int max_tq, const BackwardGroup& g,
                                const BackwardArrays& a, cudaStream_t st) {
    if (g.kv_blocks == 0) return DODO_OK;
    if (dtype == DODO_BF16 && dh == 128) return launch_stream<__nv_bfloat16, 128>(ctx, H, sm_scale, max_tq, g, a, st);
    if (dtype == DODO_BF16) return launch_stream<__nv_bfloat16, 64>(ctx, H, sm_scale, max_tq, g, a, st);
    if (dh == 128) return launch_stream<float, 128>(ctx, H, sm_scale, max_tq, g, a, st);
    return launch_stream<float, 64>(ctx, H, sm_scale, max_tq, g, a, st);
}

int dodo_launch_backward_stats(dodo_ctx* ctx, int H, int dh, const BackwardGroup& g, const BackwardArrays& a, cudaStream_t st) {
    if (g.stat_rows == 0) return DODO_OK;
    const int per_block = kThreads / (dh / 8);
    const long long units = static_cast<long long>(g.stat_rows) * H;
    const cudaError_t e = dodo_launch_dependent(backward_stats_kernel, dim3(static_cast<unsigned>((units + per_block - 1) / per_block)), dim3(kThreads), 0,
                                                st, a, g, H, dh);
    return dodo_check_cuda(ctx, e, "attend gradient statistics launch");
}

int dodo_launch_backward_scores(dodo_ctx* ctx, const BackwardGroup& g, const BackwardArrays& a, int parts, cudaStream_t st) {
    int most = 0;
    for (int i = 0; i < g.nseq; ++i) most = most > g.seq[i].c_len ? most : g.seq[i].c_len;
    if (a.dscore == nullptr || most == 0) return DODO_OK;
    return dodo_check_cuda(ctx, dodo_launch_dependent(backward_scores_kernel, dim3(static_cast<unsigned>((most + 31) / 32), static_cast<unsigned>(g.nseq)),
                                                      dim3(kThreads), 0, st, a, g, parts),
                           "attend gradient score launch");
}

int dodo_launch_backward_tile(dodo_ctx* ctx, int H, int dh, float sm_scale, const BackwardGroup& g, const BackwardArrays& a,
                              cudaStream_t st) {
    if (g.q_blocks + g.kv_blocks == 0) return DODO_OK;
    if (dh == 128) return launch_tile<128>(ctx, 0, H, sm_scale, g, a, st);
    return launch_tile<64>(ctx, 1, H, sm_scale, g, a, st);
}
