// Attention over a paged cache: tables of a launch, the walk through a sequence's key list, and how a block's results are joined.
//
// A unit of work is (sequence, tile of rows, KV head).  Its rows are the (query token, query head of the KV head's group) pairs of
// the sequence, tokens first: row r is token r / group, head r % group, so that query heads which share a KV head share what is
// read of it.  Its keys are one list: the rows in use of the cache, then the local tokens that its last query sees.  A long list is
// cut into chunks, one block each; the blocks of a unit leave partial results in the workspace and the last to arrive joins them,
// in the chunks' order.
#pragma once

#include "dodo_internal.cuh"

struct PagedSeq {
    int q_row0, tq, q_pos0;
    int c_len, page0;           // rows in use; first entry in the page table
    int l_row0, l_len, l_pos0;
    int nchunk, chunk_keys;     // chunks of the key list and the keys of each
    int part0, tick0;           // first partial row in the workspace, first arrival counter
};
struct PagedGroup {
    int nseq;
    int cta0[DODO_GROUP + 1];
    PagedSeq seq[DODO_GROUP];
};
struct PagedArrays {
    const void *Q, *cK, *cV, *lK, *lV;
    const int32_t *pos, *table;
    int pages, page;
    uint32_t page_mul;          // n / page = n * page_mul >> page_shift for n < 2^31
    int page_shift;
    int H, Hkv, group;          // query heads, KV heads, H / Hkv
    uint32_t group_mul;         // n / group = n * group_mul >> group_shift for n < 2^31
    int group_shift;
    float scale_log2;
    void* O;
    float* lse;
    float* part;                // partial rows: [rows][dh], then (maximum, sum) of each
    int* tickets;
    int* status;
};
// How a launch cuts its work: rows of a tile, keys a chunk is a multiple of, blocks to aim at, keys a chunk has at least, rows of a warp
struct PagedCut { int rows, keys, target, least, warp_rows; };
void dodo_paged_plan(const PagedCut& cut, PagedGroup& g, int group, int Hkv, bool may_cut);
static inline size_t dodo_paged_part_rows(const PagedCut& cut) { return static_cast<size_t>(2) * cut.target * cut.rows; }
// floats of a partial row: dh sums, a maximum and a sum, and two more so that every row of every tile starts on 16 bytes
static constexpr int dodo_paged_part_floats(int dh) { return dh + 4; }

constexpr int kPagedRowsMost = 32;          // rows of a tile of the kernel on the FMA units, at most
static inline int dodo_paged_rows_blocks(const dodo_ctx* ctx) { return 4 * ctx->num_sms; }      // blocks that it aims at
PagedCut dodo_paged_rows_cut(const dodo_ctx* ctx, const PagedGroup& g, int group, int Hkv, int max_rows);
// many bf16 rows, on the tensor cores; scale of DODO_DENSE_LEAST_SCALE or more
size_t dodo_paged_dense_workspace_bytes(int num_sms, int dh);
int dodo_launch_paged_dense(dodo_ctx* ctx, int dh, int max_rows, int loc_rows, const PagedGroup& g, const PagedArrays& a, cudaStream_t st);
// few bf16 rows, on the warp-level matrix units; pages that are multiples of eight rows
struct PagedBoxes { int rows; CUtensorMap cK, cV, lK, lV; };     // tensor maps of 64 features x `rows` rows, of local tokens as many as a tile has
int dodo_paged_box(int page, int most);       // rows that a tensor copy may take at once: the power of two that divides the page's, 0 below 8
int dodo_paged_boxes(dodo_ctx* ctx, const PagedArrays& a, int dh, int loc_rows, int box, int local_box, PagedBoxes& m);
PagedCut dodo_paged_token_cut(const dodo_ctx* ctx, int max_rows);
int dodo_launch_paged_token(dodo_ctx* ctx, int dh, int max_rows, int loc_rows, const PagedGroup& g, const PagedArrays& a, cudaStream_t st);
// many fp32 rows, on the FMA units
PagedCut dodo_paged_tile_cut(const dodo_ctx* ctx, const PagedGroup& g, int group, int Hkv, int max_rows);
int dodo_launch_paged_tile(dodo_ctx* ctx, int dh, const PagedCut& cut, const PagedGroup& g, const PagedArrays& a, cudaStream_t st);
int dodo_launch_paged_rows(dodo_ctx* ctx, int dtype, int dh, const PagedCut& cut, const PagedGroup& g, const PagedArrays& a, cudaStream_t st);

#ifdef __CUDACC__
namespace dodo_paged {

// where this block works: sequence, tile of rows, KV head, chunk
struct Place { int b, tile, head, chunk; };
__device__ __forceinline__ Place place_of(const PagedGroup& g, int Hkv, int bid) {
    int lo = 0, hi = g.nseq;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (g.cta0[mid] <= bid) lo = mid; else hi = mid;
    }
    Place p;
    p.b = lo;
    const int r = bid - g.cta0[lo], n = g.seq[lo].nchunk;
    p.chunk = r % n;
    p.head = r / n % Hkv;
    p.tile = r / n / Hkv;
    return p;
}

// A key of the list: `row` of the cache's or the local tokens' arrays, its position; none: row < 0
struct Key { int row, pos; bool local; };
constexpr int kNoPos = 0x7fffffff;

// entry of the page table that key j needs, 0 for local tokens
__device__ __forceinline__ int page_of(const PagedArrays& a, int j) { return static_cast<int>(static_cast<uint64_t>(j) * a.page_mul >> a.page_shift); }
__device__ __forceinline__ int page_entry(const PagedArrays& a, const PagedSeq& s, int j, int end) {
    return j < min(end, s.c_len) ? __ldg(a.table + s.page0 + page_of(a, j)) : 0;
}
// the key itself, with its page's number at hand
__device__ __forceinline__ Key key_at(const PagedArrays& a, const PagedSeq& s, int j, int end, int entry) {
    Key k;
    k.row = -1; k.pos = kNoPos; k.local = j >= s.c_len;
    if (j >= end) return k;
    if (k.local) {
        k.row = s.l_row0 + (j - s.c_len);
        k.pos = s.l_pos0 + (j - s.c_len);
    } else if (static_cast<unsigned>(entry) < static_cast<unsigned>(a.pages)) {
        k.row = entry * a.page + (j - page_of(a, j) * a.page);
        k.pos = __ldg(a.pos + k.row);
    } else {
        atomicOr(a.status, DODO_DEV_BAD_INDEX);
    }
    return k;
}

__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// weight of a part whose maximum is m in a whole whose maximum is M
__device__ __forceinline__ float part_weight(float m, float M) { return m == -INFINITY ? 0.f : exp2_fast(m - M); }

template <typename T> __device__ __forceinline__ void store4(T* p, const float* f);
template <> __device__ __forceinline__ void store4<float>(float* p, const float* f) { *reinterpret_cast<float4*>(p) = make_float4(f[0], f[1], f[2], f[3]); }
template <> __device__ __forceinline__ void store4<__nv_bfloat16>(__nv_bfloat16* p, const float* f) {
    const __nv_bfloat162 a = __floats2bfloat162_rn(f[0], f[1]), b = __floats2bfloat162_rn(f[2], f[3]);
    *reinterpret_cast<uint2*>(p) = make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
}

// token of row r, and the row of Q and O that it is
__device__ __forceinline__ int token_of(const PagedArrays& a, int r) { return static_cast<int>(static_cast<uint64_t>(r) * a.group_mul >> a.group_shift); }
__device__ __forceinline__ size_t out_row(const PagedArrays& a, const PagedSeq& s, int head, int r) {
    const int t = token_of(a, r);
    return static_cast<size_t>(s.q_row0 + t) * a.H + head * a.group + (r - t * a.group);
}

// One row's result again over all of the unit's keys that it sees, whatever the others hold: a warp, a key a lane for the scores, four (two)
// features a lane for the sums.  For results of products of tiles that are not finite, where a weight of 0 may have met a NaN.
template <typename T, int DH>
__device__ __noinline__ void sum_again(const PagedArrays& a, const PagedSeq& s, int head, int r, T* out) {
    constexpr int F = DH / 32, E = 16 / static_cast<int>(sizeof(T));
    const int lane = static_cast<int>(threadIdx.x) & 31;
    const size_t pitch = static_cast<size_t>(a.Hkv) * DH, at = static_cast<size_t>(head) * DH;
    const T* const q = static_cast<const T*>(a.Q) + out_row(a, s, head, r) * DH;
    const int qpos = s.q_pos0 + token_of(a, r), end = s.c_len + dodo_visible_local(s.l_len, s.l_pos0, qpos);
    float m = -INFINITY, l = 0.f, acc[F];
#pragma unroll
    for (int f = 0; f < F; ++f) acc[f] = 0.f;
#pragma unroll 1
    for (int j0 = 0; j0 < end; j0 += 32) {
        const Key k = key_at(a, s, j0 + lane, end, page_entry(a, s, j0 + lane, end));
        float x = -INFINITY;
        if (k.row >= 0 && k.pos <= qpos) {
            const T* const kr = static_cast<const T*>(k.local ? a.lK : a.cK) + static_cast<size_t>(k.row) * pitch + at;
            x = 0.f;
#pragma unroll 4
            for (int c = 0; c < DH; c += E) {
                float kf[E], qf[E];
                Vec16<T>::unpack(__ldg(reinterpret_cast<const uint4*>(kr + c)), kf);
                Vec16<T>::unpack(__ldg(reinterpret_cast<const uint4*>(q + c)), qf);
#pragma unroll
                for (int e = 0; e < E; ++e) x = fmaf(kf[e], qf[e], x);
            }
            x *= a.scale_log2;
        }
        const bool sees = x != -INFINITY;         // a logit of -infinity is as good as none
        float top = fmaxf(m, x);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        const float ref = top == -INFINITY ? 0.f : top, corr = part_weight(m, ref), w = exp2_fast(x - ref);
        m = top;
        l = fmaf(l, corr, w);
#pragma unroll
        for (int f = 0; f < F; ++f) acc[f] *= corr;
        uint32_t seen = __ballot_sync(0xffffffffu, sees);
        while (seen != 0u) {
            const int e = __ffs(seen) - 1;
            seen &= seen - 1u;
            const int row = __shfl_sync(0xffffffffu, k.row, e);
            const bool local = __shfl_sync(0xffffffffu, k.local ? 1 : 0, e) != 0;
            const float c = __shfl_sync(0xffffffffu, w, e);
            const T* const vr = static_cast<const T*>(local ? a.lV : a.cV) + static_cast<size_t>(row) * pitch + at + lane * F;
#pragma unroll
            for (int f = 0; f < F; ++f) acc[f] = fmaf(c, static_cast<float>(vr[f]), acc[f]);
        }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
    const float inv = l != 0.f ? 1.f / l : 0.f;
#pragma unroll
    for (int f = 0; f < F; ++f) out[lane * F + f] = static_cast<T>(acc[f] * inv);
}

// The end of a block of kThreads threads: `parts` partial results of `rows` rows in shared memory (sums of weighted V [part][row][DH]
// with pitch floats a row, maxima and sums of weights [part][row]) joined into results, or, where the unit is cut, into a partial
// result of the workspace; the last block of the unit joins those.  Called by all threads, behind a barrier.  kMixed: the sums may hold
// what some rows do not see; results that are not finite are then summed again.
template <typename T, int DH, int kThreads, bool kMixed = false>
__device__ __forceinline__ void finish(const PagedArrays& a, const PagedSeq& s, const Place& p, int tile_rows, int rows, int parts, float* acc,
                                       int pitch, float* mx, float* sum) {
    constexpr int kPieces = DH / 4;
    __shared__ int s_last;
    const int tid = static_cast<int>(threadIdx.x), r0 = p.tile * tile_rows;
    const size_t unit = static_cast<size_t>(p.tile) * a.Hkv + p.head;
    // partial rows of a chunk: tile_rows rows of DH floats, then a pair of floats each
    const size_t chunk_floats = static_cast<size_t>(tile_rows) * dodo_paged_part_floats(DH);
    float* const base = a.part + static_cast<size_t>(s.part0) * dodo_paged_part_floats(DH) + unit * s.nchunk * chunk_floats;
    float* const mine = base + p.chunk * chunk_floats;
    bool whole = s.nchunk == 1, odd = false;
    for (;;) {
        for (int i = tid; i < rows * kPieces; i += kThreads) {
            const int r = i / kPieces, c = i % kPieces * 4;
            float M = -INFINITY, L = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
            for (int w = 0; w < parts; ++w) M = fmaxf(M, mx[w * tile_rows + r]);
            for (int w = 0; w < parts; ++w) {
                const float k = part_weight(mx[w * tile_rows + r], M);
                if (k == 0.f) continue;
                L = fmaf(k, sum[w * tile_rows + r], L);
                const float4 v = *reinterpret_cast<const float4*>(acc + (static_cast<size_t>(w) * tile_rows + r) * pitch + c);
                o[0] = fmaf(k, v.x, o[0]); o[1] = fmaf(k, v.y, o[1]); o[2] = fmaf(k, v.z, o[2]); o[3] = fmaf(k, v.w, o[3]);
            }
            if (whole) {
                const size_t at = out_row(a, s, p.head, r0 + r);
                const float inv = L != 0.f ? 1.f / L : 0.f;
#pragma unroll
                for (int e = 0; e < 4; ++e) { o[e] *= inv; odd = odd || !(o[e] * 0.f == 0.f); }
                store4(static_cast<T*>(a.O) + at * DH + c, o);
                if (c == 0 && a.lse != nullptr) a.lse[at] = L != 0.f ? (M + log2f(L)) * 0.6931471805599453f : -INFINITY;
            } else {
                *reinterpret_cast<float4*>(mine + static_cast<size_t>(r) * DH + c) = make_float4(o[0], o[1], o[2], o[3]);
                if (c == 0) *reinterpret_cast<float2*>(mine + static_cast<size_t>(tile_rows) * DH + 2 * r) = make_float2(M, L);
            }
        }
        if (whole) break;
        __threadfence();
        __syncthreads();
        if (tid == 0) {
            int* const t = a.tickets + s.tick0 + unit;
            const int arrived = atomicAdd(t, 1);
            s_last = arrived == s.nchunk - 1;
            if (s_last) *t = 0;        // clean for the next launch
        }
        __syncthreads();
        if (!s_last) return;
        __threadfence();
        // The chunks' partial rows, back to where the parts were: of as many parts as leave each about eight chunks, part w takes every
        // parts-th, in order.  Warps share parts and rows out (kLanes lanes a row, four features each); two rows of four chunks each are
        // on their way at a time.
        constexpr int kLanes = kPieces, kRowsAtOnce = 32 / kLanes, kWarps = kThreads / 32;
        parts = min(parts, (s.nchunk + 7) / 8);
        const int warp = tid >> 5, lane = tid & 31, teams = kWarps / parts;       // warps of a part
        if (warp < teams * parts) {
            const int w = warp % parts, c = lane % kLanes * 4, step = teams * kRowsAtOnce;
            for (int first = warp / parts * kRowsAtOnce + lane / kLanes; first < rows; first += 2 * step) {
                float M[2] = {-INFINITY, -INFINITY}, L[2] = {0.f, 0.f}, o[2][4] = {};
                for (int k = w; k < s.nchunk; k += 4 * parts) {
                    float2 q[2][4];
                    float4 v[2][4];
#pragma unroll
                    for (int h = 0; h < 2; ++h)
#pragma unroll
                        for (int u = 0; u < 4; ++u) {
                            const int r = min(first + h * step, rows - 1);
                            const float* const from = base + static_cast<size_t>(min(k + u * parts, s.nchunk - 1)) * chunk_floats;
                            q[h][u] = __ldcg(reinterpret_cast<const float2*>(from + static_cast<size_t>(tile_rows) * DH + 2 * r));
                            v[h][u] = __ldcg(reinterpret_cast<const float4*>(from + static_cast<size_t>(r) * DH + c));
                        }
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        float top = M[h];
#pragma unroll
                        for (int u = 0; u < 4; ++u) top = k + u * parts < s.nchunk ? fmaxf(top, q[h][u].x) : top;
                        const float old = part_weight(M[h], top);
                        M[h] = top;
                        L[h] = old != 0.f ? L[h] * old : 0.f;
#pragma unroll
                        for (int e = 0; e < 4; ++e) o[h][e] = old != 0.f ? o[h][e] * old : 0.f;
#pragma unroll
                        for (int u = 0; u < 4; ++u) {
                            const float x = k + u * parts < s.nchunk ? part_weight(q[h][u].x, top) : 0.f;
                            if (x == 0.f) continue;
                            L[h] = fmaf(x, q[h][u].y, L[h]);
                            o[h][0] = fmaf(x, v[h][u].x, o[h][0]); o[h][1] = fmaf(x, v[h][u].y, o[h][1]);
                            o[h][2] = fmaf(x, v[h][u].z, o[h][2]); o[h][3] = fmaf(x, v[h][u].w, o[h][3]);
                        }
                    }
                }
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    if (first + h * step >= rows) continue;
                    const int at = w * tile_rows + first + h * step;
                    *reinterpret_cast<float4*>(acc + static_cast<size_t>(at) * pitch + c) = make_float4(o[h][0], o[h][1], o[h][2], o[h][3]);
                    if (c == 0) { mx[at] = M[h]; sum[at] = L[h]; }
                }
            }
        }
        __syncthreads();
        whole = true;
    }
    if constexpr (kMixed) {
        if (__syncthreads_or(odd ? 1 : 0) == 0) return;
        for (int r = tid / 32; r < rows; r += kThreads / 32) {
            T* const out = static_cast<T*>(a.O) + out_row(a, s, p.head, r0 + r) * DH;
            bool bad = false;
            for (int f = tid % 32; f < DH; f += 32) bad = bad || !isfinite(static_cast<float>(out[f]));
            if (__any_sync(0xffffffffu, bad)) sum_again<T, DH>(a, s, p.head, r0 + r, out);
        }
    }
}

}  // namespace dodo_paged
#endif
