// Attention of many fp32 rows (query tokens x query heads of a KV head) over a paged cache, on the FMA units.  Four sequences
// of 128 queries over 1128 keys, 8 heads of 128: 98 us, 24 TFLOP/s, a third of the units' rate (a row or a few rows a warp, as for few rows: 204
// us).  What stands between: two blocks an SM are two warps a scheduler, which meet at four barriers of the block a step, and the softmax between
// the two products has nothing beside it.  By their counts neither the FMA units nor shared memory's reads are full.
//
// A block takes a tile of 64 (or 32) rows through a chunk of the key list, 48 (64) keys a step: as many as let an SM hold two blocks (four
// sequences of 64 rows over 1064 keys: 70 us, with 64 keys and one block 81).  Scores and results are made by 8 x 16 threads
// of eight (four) rows and three (four) keys, or DH / 16 features, each: operands from shared memory are then used several times from
// registers, and the multiplications outweigh the loads.  Rows of keys lie DH + 4 floats apart, so that the sixteen threads that read
// sixteen keys' features at once meet no bank twice.  The next tile's K is on its way while weights meet V, its V during the next scores,
// its keys' pages and positions are looked up a tile ahead.  Softmax: a row's maximum over its sixteen threads, sums kept by each of them
// to the end.  What some rows of a tile see and others do not has weight 0 in the product; results that are not finite are summed again
// over what their row sees (finish).
#include "paged.cuh"
#include "sm100_ptx.cuh"

namespace {

using namespace dodo_paged;

constexpr int kThreads = 128;

template <int DH, int TM>
struct Tile {
    static constexpr int BN = TM == 8 ? 48 : 64;               // keys of a step: as many as let an SM hold two blocks
    static constexpr int kRows = 8 * TM, kPitch = DH + 4, kWeights = BN + 4;
    static constexpr int kFloats = (kRows + 2 * BN) * kPitch + kRows * kWeights;
};

__device__ __forceinline__ void copy16(float* dst, const float* src, bool there) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(sm100::smem_u32(dst)), "l"(src), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ void commit_copies() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void wait_copies() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

template <int DH, int TM>
__global__ void __launch_bounds__(kThreads, 2)
attend_paged_tile_kernel(const __grid_constant__ PagedGroup g, const __grid_constant__ PagedArrays a) {
    using L = Tile<DH, TM>;
    constexpr int BN = L::BN, KJ = BN / 16;                    // keys of a step, of a thread
    constexpr int FV = DH / 64;                                // quadruples of features of a thread
    extern __shared__ float4 smem4[];
    float* const sQ = reinterpret_cast<float*>(smem4);
    float* const sK = sQ + L::kRows * L::kPitch;
    float* const sV = sK + BN * L::kPitch;
    float* const sP = sV + BN * L::kPitch;
    __shared__ int s_row[2][BN], s_pos[2][BN];                 // a key's row: of the cache, -2 - row of the local tokens, -1 where there is none
    const int tid = static_cast<int>(threadIdx.x), tx = tid % 16, ty = tid / 16;
    dodo_grid_dependency_sync();
    const Place p = place_of(g, a.Hkv, static_cast<int>(blockIdx.x));
    const PagedSeq& s = g.seq[p.b];
    const int r0 = p.tile * L::kRows, rows = min(L::kRows, s.tq * a.group - r0);
    const int last_pos = s.q_pos0 + token_of(a, r0 + rows - 1);
    const int end_all = s.c_len + dodo_visible_local(s.l_len, s.l_pos0, last_pos);
    const int begin = p.chunk * s.chunk_keys, end = min(begin + s.chunk_keys, end_all);
    const size_t pitch = static_cast<size_t>(a.Hkv) * DH, at = static_cast<size_t>(p.head) * DH;
    const int steps = end > begin ? (end - begin + BN - 1) / BN : 0;

    int row = -1, pos = kNoPos;
    auto look_up = [&](int t) {
        if (tid >= BN) return;
        const int j = begin + t * BN + tid;
        const Key k = key_at(a, s, j, end, page_entry(a, s, j, end));
        const bool there = k.row >= 0 && k.pos <= last_pos;
        row = there ? (k.local ? -2 - k.row : k.row) : -1;
        pos = there ? k.pos : kNoPos;
    };
    auto publish = [&](int t) {
        if (tid < BN) { s_row[t & 1][tid] = row; s_pos[t & 1][tid] = pos; }
    };
    constexpr int kLanes = DH / 4;                             // threads of a row's copy
    auto bring = [&](float* dst, const void* cache, const void* local, int t) {
        for (int r = tid / kLanes; r < BN; r += kThreads / kLanes) {
            const int from = s_row[t & 1][r];
            const float* const base = static_cast<const float*>(from >= 0 ? cache : local) + static_cast<size_t>(from >= 0 ? from : -2 - from) * pitch + at;
            copy16(dst + r * L::kPitch + tid % kLanes * 4, from != -1 ? base + tid % kLanes * 4 : static_cast<const float*>(a.Q), from != -1);
        }
        commit_copies();
    };

    if (steps > 0) {
        look_up(0);
        publish(0);
    }
    for (int r = tid / kLanes; r < L::kRows && steps > 0; r += kThreads / kLanes)
        copy16(sQ + r * L::kPitch + tid % kLanes * 4, static_cast<const float*>(a.Q) + out_row(a, s, p.head, r0 + min(r, rows - 1)) * DH + tid % kLanes * 4, true);
    __syncthreads();
    if (steps > 0) {
        bring(sK, a.cK, a.lK, 0);                              // (Q's copies belong to the same group)
        bring(sV, a.cV, a.lV, 0);
    }
    // this thread's rows are ty + 8 i, its keys tx + 16 j, its features 4 tx + 64 v
    int qpos[TM];
    float m[TM], l[TM];
    float2 o[TM][2 * FV];
#pragma unroll
    for (int i = 0; i < TM; ++i) {
        qpos[i] = s.q_pos0 + token_of(a, r0 + min(ty + 8 * i, rows - 1));
        m[i] = -INFINITY;
        l[i] = 0.f;
#pragma unroll
        for (int v = 0; v < 2 * FV; ++v) o[i][v] = make_float2(0.f, 0.f);
    }
    for (int t = 0; t < steps; ++t) {
        if (t + 1 < steps) look_up(t + 1);
        wait_copies<1>();
        __syncthreads();                                       // K is there for all
        float2 x[TM][KJ];
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < KJ; ++j) x[i][j] = make_float2(0.f, 0.f);
#pragma unroll 4
        for (int f = 0; f < DH; f += 4) {
            float4 k[KJ];
#pragma unroll
            for (int j = 0; j < KJ; ++j) k[j] = *reinterpret_cast<const float4*>(sK + (tx + 16 * j) * L::kPitch + f);
#pragma unroll
            for (int i = 0; i < TM; ++i) {
                const float4 q = *reinterpret_cast<const float4*>(sQ + (ty + 8 * i) * L::kPitch + f);
#pragma unroll
                for (int j = 0; j < KJ; ++j) {
                    x[i][j] = __ffma2_rn(make_float2(q.x, q.y), make_float2(k[j].x, k[j].y), x[i][j]);
                    x[i][j] = __ffma2_rn(make_float2(q.z, q.w), make_float2(k[j].z, k[j].w), x[i][j]);
                }
            }
        }
        int kpos[KJ];
#pragma unroll
        for (int j = 0; j < KJ; ++j) kpos[j] = s_pos[t & 1][tx + 16 * j];
        if (t + 1 < steps) publish(t + 1);
        __syncthreads();                                       // nobody reads this K any more
        if (t + 1 < steps) bring(sK, a.cK, a.lK, t + 1); else commit_copies();
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            float w[KJ], top = m[i];
#pragma unroll
            for (int j = 0; j < KJ; ++j) {
                w[j] = kpos[j] <= qpos[i] ? (x[i][j].x + x[i][j].y) * a.scale_log2 : -INFINITY;
                top = fmaxf(top, w[j]);
            }
#pragma unroll
            for (int d = 1; d < 16; d <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
            const float ref = top == -INFINITY ? 0.f : top, corr = part_weight(m[i], ref);
            m[i] = top;
            l[i] *= corr;
#pragma unroll
            for (int v = 0; v < 2 * FV; ++v) o[i][v] = __fmul2_rn(o[i][v], make_float2(corr, corr));
#pragma unroll
            for (int j = 0; j < KJ; ++j) {
                w[j] = exp2_fast(w[j] - ref);
                l[i] += w[j];
                sP[(ty + 8 * i) * L::kWeights + tx + 16 * j] = w[j];
            }
        }
        wait_copies<1>();
        __syncthreads();                                       // V and the weights are there for all
#pragma unroll 2
        for (int k = 0; k < BN; k += 4) {
            float4 v[4][FV];
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int h = 0; h < FV; ++h) v[e][h] = *reinterpret_cast<const float4*>(sV + (k + e) * L::kPitch + 4 * tx + 64 * h);
#pragma unroll
            for (int i = 0; i < TM; ++i) {
                const float4 w4 = *reinterpret_cast<const float4*>(sP + (ty + 8 * i) * L::kWeights + k);
                const float w[4] = {w4.x, w4.y, w4.z, w4.w};
#pragma unroll
                for (int e = 0; e < 4; ++e)
#pragma unroll
                    for (int h = 0; h < FV; ++h) {
                        o[i][2 * h] = __ffma2_rn(make_float2(w[e], w[e]), make_float2(v[e][h].x, v[e][h].y), o[i][2 * h]);
                        o[i][2 * h + 1] = __ffma2_rn(make_float2(w[e], w[e]), make_float2(v[e][h].z, v[e][h].w), o[i][2 * h + 1]);
                    }
            }
        }
        __syncthreads();                                       // nobody reads this V any more
        if (t + 1 < steps) bring(sV, a.cV, a.lV, t + 1); else commit_copies();
    }
    wait_copies<0>();
    __syncthreads();                                           // Q's place takes the results, the weights' their maxima and sums
    float* const mx = sP;
    float* const sum = sP + L::kRows;
#pragma unroll
    for (int i = 0; i < TM; ++i) {
        const int r = ty + 8 * i;
#pragma unroll
        for (int d = 1; d < 16; d <<= 1) l[i] += __shfl_xor_sync(0xffffffffu, l[i], d);
        if (tx == 0) {
            mx[r] = l[i] != l[i] ? INFINITY : m[i];            // a NaN among the logits that the row sees: the whole row's
            sum[r] = l[i];
        }
#pragma unroll
        for (int h = 0; h < FV; ++h)
            *reinterpret_cast<float4*>(sQ + r * L::kPitch + 4 * tx + 64 * h) = make_float4(o[i][2 * h].x, o[i][2 * h].y, o[i][2 * h + 1].x, o[i][2 * h + 1].y);
    }
    __syncthreads();
    finish<float, DH, kThreads, true>(a, s, p, L::kRows, rows, 1, sQ, L::kPitch, mx, sum);
}

template <int DH, int TM>
int launch(dodo_ctx* ctx, const PagedGroup& g, const PagedArrays& a, cudaStream_t st) {
    auto kern = attend_paged_tile_kernel<DH, TM>;
    const int smem = Tile<DH, TM>::kFloats * static_cast<int>(sizeof(float));
    bool& set = ctx->paged_tile_attr_set[(DH == 128 ? 2 : 0) + TM / 8];
    if (!set) {
        const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
        if (e != cudaSuccess) return dodo_check_cuda(ctx, e, "paged tile attend shared-memory attribute");
        set = true;
    }
    return dodo_check_cuda(ctx, dodo_launch_dependent(kern, dim3(static_cast<unsigned>(g.cta0[g.nseq])), dim3(kThreads), static_cast<size_t>(smem), st, g, a),
                           "paged tile attend launch");
}

}  // namespace

// 64 rows a tile where every block has eight steps of 48 keys or more to take with them, else 32: twice the units, so that lists are cut less and
// the last block of one joins fewer and shorter pieces (40 rows of 8 heads over 11,454 keys: 140 us with 64, 94 with 32; 167 rows of 25
// heads over three lists of 545 to 1728 keys: 145, 191).
PagedCut dodo_paged_tile_cut(const dodo_ctx* ctx, const PagedGroup& g, int group, int Hkv, int max_rows) {
    constexpr int keys64 = Tile<128, 8>::BN, keys32 = Tile<128, 4>::BN;
    int64_t steps = 0;
    for (int i = 0; i < g.nseq; ++i) {
        const PagedSeq& s = g.seq[i];
        steps += (static_cast<int64_t>(s.tq) * group + 63) / 64 * Hkv * ((static_cast<int64_t>(s.c_len) + s.l_len + keys64 - 1) / keys64);
    }
    const bool wide = max_rows > 32 && steps >= 8 * 2 * static_cast<int64_t>(ctx->num_sms);
    return {wide ? 64 : 32, wide ? keys64 : keys32, 2 * ctx->num_sms, 2 * (wide ? keys64 : keys32), 0};
}

int dodo_launch_paged_tile(dodo_ctx* ctx, int dh, const PagedCut& cut, const PagedGroup& g, const PagedArrays& a, cudaStream_t st) {
    if (dh == 128) return cut.rows == 32 ? launch<128, 4>(ctx, g, a, st) : launch<128, 8>(ctx, g, a, st);
    return cut.rows == 32 ? launch<64, 4>(ctx, g, a, st) : launch<64, 8>(ctx, g, a, st);
}
