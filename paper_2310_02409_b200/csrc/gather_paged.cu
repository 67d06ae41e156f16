// Append to a paged nugget cache: the selected tokens' K and V rows (or all tokens') copied to the rows that the page table names, K
// rotated at its position on the way.  Bound by HBM: a thread block of 128 threads per appended row, whose first two pieces of K and four of V a
// thread are requested before the block makes the sines and cosines of its one position: the whole row up to 8 KB of K and 8 KB of V (32 heads of
// 128 in bf16).  What a longer row has beyond comes piece by piece behind that.  205 of 2048 tokens of each of 8 sequences, 32 heads of 128: 11.2 us,
// 4.8 TB/s, bound by the chain index -> row -> loads -> stores in the 1.4 waves that the blocks make (V by bulk copies: 10.95); 40 heads 14.9 us,
// 4.5 TB/s; 32 fp32 heads 20.1 us, 5.3 TB/s; a token of each: 2.5 us, the launch.  K of rotations whose halves are no multiple of 16 bytes goes element
// by element: 32 bf16 heads of 96 with 24 features turned 34 us, where their bytes take 6.
#include "rope.cuh"

namespace {

using namespace dodo_rotary;

struct PagedAppend {
    int nseq;
    int idx0[DODO_GROUP + 1];   // prefix of appended rows (slots in idx, absolute)
    int src_row0[DODO_GROUP];   // first row of the sequence in K and V
    int n[DODO_GROUP];          // tokens: an index outside [0, n) is reported, not followed
    int len[DODO_GROUP];        // rows in use before the append
    int page0[DODO_GROUP];      // first entry of the sequence in the page table
    int pos_base[DODO_GROUP];
};

// row r of a sequence whose entries in the table start at page0: a row of the pool, or -1 where the table's entry is no page
__device__ __forceinline__ int pool_row(const int32_t* table, int page0, int pages, int page, int r) {
    const int p = __ldg(table + page0 + r / page);
    return static_cast<unsigned>(p) < static_cast<unsigned>(pages) ? p * page + r % page : -1;
}

constexpr int kThreads = 128;
constexpr int kAhead = 2;       // slots of K (a piece or two each) and twice as many pieces of V that a thread requests before anything else

template <typename T, int VEC, bool INTER>
__global__ void __launch_bounds__(512)
gather_paged_kernel(const T* __restrict__ K, const T* __restrict__ V, long long kv_row, const int32_t* __restrict__ idx,
                    const __grid_constant__ PagedAppend g, const __grid_constant__ Rotation p, int H, int dh, int slots, int lanes,
                    T* __restrict__ cacheK, T* __restrict__ cacheV, int32_t* __restrict__ cache_pos, const int32_t* __restrict__ table, int pages,
                    int page, int* __restrict__ dev_status) {
    __shared__ float2 cs[DODO_ROPE_MAX / 2];
    const int tid = static_cast<int>(threadIdx.x), threads = static_cast<int>(blockDim.x);
    const int j = g.idx0[0] + static_cast<int>(blockIdx.x);
    int b = 0, hi = g.nseq;
    while (hi - b > 1) {
        const int mid = (b + hi) >> 1;
        if (g.idx0[mid] <= j) b = mid; else hi = mid;
    }
    const int slot = tid % slots, lane = tid / slots, vecs = H * dh * static_cast<int>(sizeof(T)) / 16;
    dodo_grid_dependency_sync();   // the indices come from the kernel before
    const int token = idx != nullptr ? __ldg(idx + j) : j - g.idx0[b];
    const int row = pool_row(table, g.page0[b], pages, page, g.len[b] + j - g.idx0[b]);
    if (static_cast<unsigned>(token) >= static_cast<unsigned>(g.n[b]) || row < 0) {
        if (tid == 0) atomicOr(dev_status, DODO_DEV_BAD_INDEX);
        return;
    }
    const T* const sk = K + (g.src_row0[b] + static_cast<long long>(token)) * kv_row;
    const uint4* const sv = reinterpret_cast<const uint4*>(V + (g.src_row0[b] + static_cast<long long>(token)) * kv_row);
    T* const dk = cacheK + static_cast<long long>(row) * H * dh;
    uint4* const dv = reinterpret_cast<uint4*>(cacheV + static_cast<long long>(row) * H * dh);
    const int pos = g.pos_base[b] + token;

    Slot<T, VEC, INTER> k[kAhead];
    uint4 v[2 * kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
        const int h = lane + u * lanes;
        if (lane < lanes && h < H) k[u].load(sk + h * dh, slot, p.half);
    }
#pragma unroll
    for (int u = 0; u < 2 * kAhead; ++u) {
        const int c = tid + u * threads;
        if (c < vecs) v[u] = ld_stream16(sv + c);
    }
    for (int i = tid; i < p.half; i += threads) cs[i] = cos_sin(p, i, pos);
    if (tid == 0) cache_pos[row] = pos;
#pragma unroll
    for (int u = 0; u < 2 * kAhead; ++u) {
        const int c = tid + u * threads;
        if (c < vecs) dv[c] = v[u];
    }
    for (int c = tid + 2 * kAhead * threads; c < vecs; c += threads) dv[c] = ld_stream16(sv + c);
    __syncthreads();
    if (lane >= lanes) return;
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
        const int h = lane + u * lanes;
        if (h < H) k[u].store(dk + h * dh, slot, p.half, cs);
    }
    for (int h = lane + kAhead * lanes; h < H; h += lanes) {
        Slot<T, VEC, INTER> s;
        s.load(sk + h * dh, slot, p.half);
        s.store(dk + h * dh, slot, p.half, cs);
    }
}

struct Append {
    const void *K, *V;
    long long kv_row;
    const int32_t* idx;
    const dodo_paged_cache* cache;
};

template <typename T, int VEC, bool INTER>
cudaError_t launch(const dodo_ctx* ctx, const Append& a, const PagedAppend& g, const Rotation& p, cudaStream_t st) {
    const dodo_paged_cache& c = *a.cache;
    const int slots = slots_of<VEC, INTER>(c.dh, p.half), most = slots >= kThreads ? 1 : kThreads / slots;
    const int lanes = most < c.H ? most : c.H;
    const int threads = (slots * lanes + 31) / 32 * 32;
    return dodo_launch_dependent(gather_paged_kernel<T, VEC, INTER>, dim3(static_cast<unsigned>(g.idx0[g.nseq] - g.idx0[0])),
                                 dim3(static_cast<unsigned>(threads)), 0, st, static_cast<const T*>(a.K), static_cast<const T*>(a.V), a.kv_row, a.idx, g, p,
                                 c.H, c.dh, slots, lanes, static_cast<T*>(c.K), static_cast<T*>(c.V), c.pos, c.table, c.pages, c.page, ctx->dev_status);
}

}  // namespace

// What every call that takes a paged cache asks of it and of its tables; `rows`: whether any row of it will be touched
int dodo_check_paged(dodo_ctx* ctx, const dodo_paged_cache* c, const int32_t* page_off, const int32_t* cache_len, int B, bool rows) {
    if (c == nullptr) return dodo_fail(ctx, DODO_ERR_INVALID_ARG, "cache must not be NULL");
    if (c->dtype != DODO_F32 && c->dtype != DODO_BF16) return dodo_fail(ctx, DODO_ERR_UNSUPPORTED, "dtype %d", c->dtype);
    if (c->H <= 0 || c->dh <= 0 || c->page <= 0 || c->pages < 0 || static_cast<int64_t>(c->pages) * c->page > 0x7fffffff)
        return dodo_fail(ctx, DODO_ERR_INVALID_ARG, "cache of %d pages of %d rows, %d heads of %d", c->pages, c->page, c->H, c->dh);
    if (!dodo_valid_offsets(page_off, B)) return dodo_fail(ctx, DODO_ERR_INVALID_ARG, "page_off must start at 0 and be non-decreasing");
    if (B > 0 && cache_len == nullptr) return dodo_fail(ctx, DODO_ERR_INVALID_ARG, "cache_len must not be NULL");
    for (int b = 0; b < B; ++b)
        if (cache_len[b] < 0 || cache_len[b] > static_cast<int64_t>(page_off[b + 1] - page_off[b]) * c->page)
            return dodo_fail(ctx, DODO_ERR_INVALID_ARG, "sequence %d: cache_len %d outside its pages", b, cache_len[b]);
    if (!rows) return DODO_OK;
    if (c->K == nullptr || c->V == nullptr || c->pos == nullptr || c->table == nullptr || !dodo_aligned16(c->K) || !dodo_aligned16(c->V))
        return dodo_fail(ctx, DODO_ERR_INVALID_ARG, "the cache's K, V, pos and table must be non-NULL, K and V 16-byte aligned");
    return DODO_OK;
}

extern "C" int dodo_gather_kv_paged(dodo_ctx* ctx, const void* K, const void* V, int64_t kv_row, const int32_t* seq_off, const int32_t* idx,
                                    const int32_t* nug_off, const int32_t* pos_base, int B, const dodo_rope_spec* rope,
                                    const dodo_paged_cache* cache, const int32_t* page_off, int32_t* cache_len, void* stream) {
    if (ctx == nullptr) return DODO_ERR_INVALID_ARG;
    if (B < 0) return dodo_fail(ctx, DODO_ERR_INVALID_ARG, "B = %d is negative", B);
    if (idx == nullptr) nug_off = seq_off;
    if (!dodo_valid_offsets(seq_off, B) || !dodo_valid_offsets(nug_off, B))
        return dodo_fail(ctx, DODO_ERR_INVALID_ARG, "seq_off and nug_off must start at 0 and be non-decreasing");
    int rc = dodo_check_paged(ctx, cache, page_off, cache_len, B, nug_off[B] > 0);
    if (rc != DODO_OK) return rc;
    dodo_rope_spec none;
    if (rope == nullptr) {      // no pair is turned: every piece of K is copied
        memset(&none, 0, sizeof none);
        none.layout = DODO_ROPE_INTERLEAVED;
        none.scale = 1.f;
        none.ready = 1u;
    }
    const dodo_rope_spec* const turn = rope != nullptr ? rope : &none;
    if ((rc = dodo_check_rope(ctx, turn, cache->dh)) != DODO_OK) return rc;
    const int64_t e = static_cast<int64_t>(dodo_elem_bytes(cache->dtype)), row = static_cast<int64_t>(cache->H) * cache->dh;
    if (row * e % 16 != 0 || kv_row * e % 16 != 0)
        return dodo_fail(ctx, DODO_ERR_INVALID_ARG, "a K/V row (%lld bytes) and kv_row must be multiples of 16 bytes", static_cast<long long>(row * e));
    if (row > 0x7fffffff / 4) return dodo_fail(ctx, DODO_ERR_UNSUPPORTED, "%d heads of %d", cache->H, cache->dh);
    if (B > 0 && pos_base == nullptr) return dodo_fail(ctx, DODO_ERR_INVALID_ARG, "pos_base must not be NULL");
    for (int b = 0; b < B; ++b) {
        const int n = seq_off[b + 1] - seq_off[b], k = nug_off[b + 1] - nug_off[b];
        if (k > n) return dodo_fail(ctx, DODO_ERR_INVALID_ARG, "sequence %d: k = %d exceeds its tokens", b, k);
        if (k > 0 && static_cast<int64_t>(pos_base[b]) + n > (int64_t{1} << 31))
            return dodo_fail(ctx, DODO_ERR_INVALID_ARG, "sequence %d: positions from %d pass 2^31", b, pos_base[b]);
        if (cache_len[b] + static_cast<int64_t>(k) > static_cast<int64_t>(page_off[b + 1] - page_off[b]) * cache->page)
            return dodo_fail(ctx, DODO_ERR_CAPACITY, "sequence %d: %d cached + %d new nuggets exceed its %d pages of %d rows", b, cache_len[b], k,
                             page_off[b + 1] - page_off[b], cache->page);
    }
    if (nug_off[B] == 0) return DODO_OK;
    if (K == nullptr || V == nullptr || !dodo_aligned16(K) || !dodo_aligned16(V))
        return dodo_fail(ctx, DODO_ERR_INVALID_ARG, "K and V must be non-NULL and 16-byte aligned");
    if ((rc = dodo_check_device(ctx)) != DODO_OK) return rc;
    const Append a = {K, V, kv_row, idx, cache};
    const Rotation p = dodo_rotation(turn, false);
    const bool wide = wide_fits(cache->dtype, turn->layout, cache->dh, turn->rot), inter = turn->layout == DODO_ROPE_INTERLEAVED;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    for (int b0 = 0; b0 < B; b0 += DODO_GROUP) {
        PagedAppend g;
        g.nseq = B - b0 < DODO_GROUP ? B - b0 : DODO_GROUP;
        for (int i = 0; i < g.nseq; ++i) {
            const int b = b0 + i;
            g.idx0[i] = nug_off[b];
            g.src_row0[i] = seq_off[b];
            g.n[i] = seq_off[b + 1] - seq_off[b];
            g.len[i] = cache_len[b];
            g.page0[i] = page_off[b];
            g.pos_base[i] = pos_base[b];
        }
        g.idx0[g.nseq] = nug_off[b0 + g.nseq];
        if (g.idx0[g.nseq] == g.idx0[0]) continue;
        ctx->cache_clean = false;   // the next attend must not read cache rows ahead of its dependency wait
        cudaError_t err;
        if (cache->dtype == DODO_F32)
            err = wide ? (inter ? launch<float, 4, true>(ctx, a, g, p, st) : launch<float, 4, false>(ctx, a, g, p, st))
                       : (inter ? launch<float, 2, true>(ctx, a, g, p, st) : launch<float, 1, false>(ctx, a, g, p, st));
        else
            err = wide ? (inter ? launch<__nv_bfloat16, 8, true>(ctx, a, g, p, st) : launch<__nv_bfloat16, 8, false>(ctx, a, g, p, st))
                       : (inter ? launch<__nv_bfloat16, 2, true>(ctx, a, g, p, st) : launch<__nv_bfloat16, 1, false>(ctx, a, g, p, st));
        if (err != cudaSuccess) return dodo_check_cuda(ctx, err, "paged append launch");
    }
    for (int b = 0; b < B; ++b) cache_len[b] += nug_off[b + 1] - nug_off[b];
    return DODO_OK;
}
