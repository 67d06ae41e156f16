// Attention of few rows over a paged cache on the FMA units (fp32, and bf16 in pages that tensor copies cannot take): a warp holds a few rows (their queries and running results in registers, spread over
// the lanes by features) and streams the keys from memory straight into registers, a key's K and V row as one coalesced access.
// Per step it takes U keys a group of lanes: partial products of all (row, key) pairs, summed over the lanes by halving exchanges so
// that each lane ends up with one pair's logit, one exponential a lane, and the weights handed back by shuffles.  Table entries,
// positions and rows of the following steps are on their way meanwhile (three steps deep, as each needs the one before).  A block's
// four warps share the keys where there are rows for all of them (the rows they read then come from L1) and split them where not.
// Bound by memory's latency for a row or two (16 fp32 queries over 68 keys of 4 heads: 5.4 us), by HBM for long lists, by the FMA units and
// the exchanges between lanes from four rows a KV head on (four over 8 x 4001 keys of 8 heads: 64 us, 4.1 TB/s of K and V).
#include "paged.cuh"

namespace {

using namespace dodo_paged;

constexpr int kWarps = 4, kThreads = 32 * kWarps;

// A logit of -infinity or no key: weight 0.  QR: rows of a warp; row_warps of the block's warps have rows of their own
template <typename T, int DH, int QR>
__global__ void __launch_bounds__(kThreads)
attend_paged_rows_kernel(const __grid_constant__ PagedGroup g, const __grid_constant__ PagedArrays a, int row_warps) {
    constexpr int E = 16 / static_cast<int>(sizeof(T));     // features of a lane
    constexpr int LK = DH / E, KP = 32 / LK;                // lanes of a key, keys side by side
    constexpr int U = LK / QR < 4 ? LK / QR : 4;            // keys a group of lanes takes per step
    constexpr int N = QR * U, COPY = LK / N, KS = U * KP;   // pairs of a group, lanes that share a pair, keys of a step
    static_assert(U >= 1 && N <= LK, "a lane owns at most one pair");
    extern __shared__ float4 smem4[];
    float* const smem = reinterpret_cast<float*>(smem4);
    const int lane = static_cast<int>(threadIdx.x) & 31, warp = static_cast<int>(threadIdx.x) >> 5;
    const int grp = lane / LK, feat = lane % LK * E;
    const int key_warps = kWarps / row_warps, tile_rows = row_warps * QR;
    dodo_grid_dependency_sync();
    const Place p = place_of(g, a.Hkv, static_cast<int>(blockIdx.x));
    const PagedSeq& s = g.seq[p.b];
    const int R = s.tq * a.group, r0 = p.tile * tile_rows, rows = min(tile_rows, R - r0);
    const int wr = warp % row_warps, wk = warp / row_warps, w0 = r0 + wr * QR;          // this warp's first row
    const int live = min(QR, R - w0);                                                   // its rows, none where <= 0
    const int last_pos = s.q_pos0 + token_of(a, min(r0 + rows, R) - 1);
    const int end_all = s.c_len + dodo_visible_local(s.l_len, s.l_pos0, last_pos);
    const int begin = p.chunk * s.chunk_keys, end = min(begin + s.chunk_keys, end_all);
    const size_t pitch = static_cast<size_t>(a.Hkv) * DH;

    float q[QR][E], acc[QR][E];
#pragma unroll
    for (int r = 0; r < QR; ++r) {
        const int row = min(w0 + r, R - 1);
        const uint4 v = __ldg(reinterpret_cast<const uint4*>(static_cast<const T*>(a.Q) + out_row(a, s, p.head, row) * DH + feat));
        Vec16<T>::unpack(v, q[r]);
#pragma unroll
        for (int e = 0; e < E; ++e) { q[r][e] *= a.scale_log2; acc[r][e] = 0.f; }
    }
    const int my_pair = lane % LK / COPY, my_row = my_pair / U, my_u = my_pair % U;
    const int my_qpos = s.q_pos0 + token_of(a, w0 + my_row);
    const bool my_live = my_row < live;
    const int most_pos = live > 0 ? s.q_pos0 + token_of(a, w0 + live - 1) : static_cast<int>(0x80000000);
    float m = -INFINITY, l = 0.f;

    // step t of this warp: keys first(t) .. first(t) + KS - 1, key first(t) + i with lane i
    auto first = [&](int t) { return begin + (wk + t * key_warps) * KS; };
    const int steps = live > 0 && end > begin ? ((end - begin + KS - 1) / KS - wk + key_warps - 1) / key_warps : 0;
    auto entry_for = [&](int t) { return lane < KS ? page_entry(a, s, first(t) + lane, end) : 0; };
    auto key_for = [&](int t, int entry) {
        Key k;
        k.row = -1; k.pos = kNoPos; k.local = false;
        if (lane < KS) k = key_at(a, s, first(t) + lane, end, entry);
        if (k.pos > most_pos) k.row = -1;          // nobody here sees it
        return k;
    };
    uint4 kreg[U], vreg[U];
    auto fetch = [&](const Key& k) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int row = __shfl_sync(0xffffffffu, k.row, u * KP + grp);
            const bool local = __shfl_sync(0xffffffffu, k.local ? 1 : 0, u * KP + grp) != 0;
            kreg[u] = vreg[u] = make_uint4(0u, 0u, 0u, 0u);
            if (row >= 0) {
                const size_t at = static_cast<size_t>(row) * pitch + static_cast<size_t>(p.head) * DH + feat;
                kreg[u] = __ldg(reinterpret_cast<const uint4*>(static_cast<const T*>(local ? a.lK : a.cK) + at));
                vreg[u] = __ldg(reinterpret_cast<const uint4*>(static_cast<const T*>(local ? a.lV : a.cV) + at));
            }
        }
    };
    Key k0, k1;                    // of this step and the next
    int entry = 0;
    if (steps > 0) {
        k0 = key_for(0, entry_for(0));
        k1 = key_for(1, entry_for(1));
        entry = entry_for(2);
        fetch(k0);
    }
    for (int t = 0; t < steps; ++t) {
        uint4 kw[U], vw[U];
#pragma unroll
        for (int u = 0; u < U; ++u) { kw[u] = kreg[u]; vw[u] = vreg[u]; }
        const int key_row = __shfl_sync(0xffffffffu, k0.row, my_u * KP + grp), key_pos = __shfl_sync(0xffffffffu, k0.pos, my_u * KP + grp);
        if (t + 1 < steps) fetch(k1);
        k0 = k1;
        k1 = key_for(t + 2, entry);
        entry = entry_for(t + 3);

        float part[N];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float f[E];
            Vec16<T>::unpack(kw[u], f);
#pragma unroll
            for (int r = 0; r < QR; ++r) {
                float d = q[r][0] * f[0];
#pragma unroll
                for (int e = 1; e < E; ++e) d = fmaf(q[r][e], f[e], d);
                part[r * U + u] = d;
            }
        }
#pragma unroll
        for (int o = LK / 2, n = N / 2; o > 0; o >>= 1, n >>= 1) {
            if (n == 0) {
                part[0] += __shfl_xor_sync(0xffffffffu, part[0], o);
            } else {
                const bool upper = (lane & o) != 0;
#pragma unroll
                for (int j = 0; j < n; ++j) {
                    const float give = upper ? part[j] : part[j + n], keep = upper ? part[j + n] : part[j];
                    part[j] = keep + __shfl_xor_sync(0xffffffffu, give, o);
                }
            }
        }
        const bool there = key_row >= 0 && my_live;
        const float x = there && key_pos <= my_qpos ? part[0] : -INFINITY;
        const bool sees = x != -INFINITY;              // (a logit of -infinity is as good as none: its V may hold anything too)
        float top = fmaxf(m, x);
#pragma unroll
        for (int o = COPY; o < COPY * U; o <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
#pragma unroll
        for (int o = LK; o < 32; o <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        const float ref = top == -INFINITY ? 0.f : top;
        const float corr = part_weight(m, ref), w = exp2_fast(x - ref);
        if (__any_sync(0xffffffffu, top > m)) {
            l *= corr;
#pragma unroll
            for (int r = 0; r < QR; ++r) {
                const float c = __shfl_sync(0xffffffffu, corr, r * U * COPY, LK);
#pragma unroll
                for (int e = 0; e < E; ++e) acc[r][e] *= c;
            }
        }
        m = top;
        l += w;
        // keys that some rows see and others do not: a row adds up what it sees, whatever lies in the others
        const bool mixed = __any_sync(0xffffffffu, there && !sees);
        const uint32_t seen = __ballot_sync(0xffffffffu, sees);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float f[E];
            Vec16<T>::unpack(vw[u], f);
#pragma unroll
            for (int r = 0; r < QR; ++r) {
                const int from = (r * U + u) * COPY;
                const float c = __shfl_sync(0xffffffffu, w, from, LK);
                if (!mixed || (seen >> (grp * LK + from) & 1u) != 0u) {
#pragma unroll
                    for (int e = 0; e < E; ++e) acc[r][e] = fmaf(c, f[e], acc[r][e]);
                }
            }
        }
    }
    // groups of lanes and lanes of a row add up; the block's warps meet in shared memory, [key warp][row]
#pragma unroll
    for (int o = LK; o < 32; o <<= 1) {
        l += __shfl_xor_sync(0xffffffffu, l, o);
#pragma unroll
        for (int r = 0; r < QR; ++r)
#pragma unroll
            for (int e = 0; e < E; ++e) acc[r][e] += __shfl_xor_sync(0xffffffffu, acc[r][e], o);
    }
#pragma unroll
    for (int o = COPY; o < COPY * U; o <<= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
    if (l != l) m = INFINITY;        // a NaN among the logits that the row sees: the whole row's, wherever its maximum stands
    constexpr int kPitch = DH + 4;
    float* const mx = smem + static_cast<size_t>(key_warps) * tile_rows * kPitch;
    float* const sum = mx + key_warps * tile_rows;
    if (grp == 0) {
#pragma unroll
        for (int r = 0; r < QR; ++r) {
            const int at = wk * tile_rows + wr * QR + r;
#pragma unroll
            for (int e = 0; e < E; e += 4) *reinterpret_cast<float4*>(smem + static_cast<size_t>(at) * kPitch + feat + e) = make_float4(acc[r][e], acc[r][e + 1], acc[r][e + 2], acc[r][e + 3]);
        }
        if (lane % COPY == 0 && my_u == 0) {
            mx[wk * tile_rows + wr * QR + my_row] = m;
            sum[wk * tile_rows + wr * QR + my_row] = l;
        }
    }
    __syncthreads();
    finish<T, DH, kThreads>(a, s, p, tile_rows, rows, key_warps, smem, kPitch, mx, sum);
}


template <typename T, int DH>
cudaError_t launch(const PagedCut& cut, const PagedGroup& g, const PagedArrays& a, cudaStream_t st) {
    const size_t smem = sizeof(float) * static_cast<size_t>(kWarps) * cut.warp_rows * (DH + 4 + 2);
    const dim3 grid(static_cast<unsigned>(g.cta0[g.nseq])), block(kThreads);
    const int row_warps = cut.rows / cut.warp_rows;
    if (cut.warp_rows == 1) return dodo_launch_dependent(attend_paged_rows_kernel<T, DH, 1>, grid, block, smem, st, g, a, row_warps);
    if (cut.warp_rows == 4) return dodo_launch_dependent(attend_paged_rows_kernel<T, DH, 4>, grid, block, smem, st, g, a, row_warps);
    return dodo_launch_dependent(attend_paged_rows_kernel<T, DH, 8>, grid, block, smem, st, g, a, row_warps);
}

}  // namespace

// As many rows a warp and a block as there are (their keys are then read once), up to eight and 32, while that leaves blocks enough for the
// device; a small batch takes fewer, down to a row a warp, and its keys are split over more warps and blocks instead (16 queries over 52 + 16
// keys of 4 heads: 11.2 us with 16 rows a block, 5.4 with one).
PagedCut dodo_paged_rows_cut(const dodo_ctx* ctx, const PagedGroup& g, int group, int Hkv, int max_rows) {
    static const int shapes[][2] = {{8, 32}, {8, 16}, {8, 8}, {4, 4}, {1, 1}};
    PagedCut cut = {1, 32, dodo_paged_rows_blocks(ctx), 128, 1};
    for (const auto& s : shapes) {
        if (s[1] > 1 && 2 * max_rows <= s[1]) continue;
        cut.warp_rows = s[0];
        cut.rows = s[1];
        // blocks: as many as registers let an SM hold, but with eight rows a warp, bound by arithmetic, twice as many (256 fp32 queries over
        // 2256 keys, in tiles of 64 rows by now: 265 us, with half as many blocks 327; four rows over 8 x 4001 keys 64 us, with a third more blocks 85)
        cut.target = s[0] == 4 ? 3 * ctx->num_sms : dodo_paged_rows_blocks(ctx);
        int64_t blocks = 0;
        for (int i = 0; i < g.nseq; ++i) {
            const PagedSeq& q = g.seq[i];
            const int64_t units = (static_cast<int64_t>(q.tq) * group + cut.rows - 1) / cut.rows * Hkv, chunks = (static_cast<int64_t>(q.c_len) + q.l_len) / cut.least;
            blocks += units * (chunks > 1 ? chunks : 1);
        }
        if (blocks >= ctx->num_sms) break;
    }
    return cut;
}

int dodo_launch_paged_rows(dodo_ctx* ctx, int dtype, int dh, const PagedCut& cut, const PagedGroup& g, const PagedArrays& a, cudaStream_t st) {
    cudaError_t e;
    if (dtype == DODO_F32) e = dh == 64 ? launch<float, 64>(cut, g, a, st) : launch<float, 128>(cut, g, a, st);
    else e = dh == 64 ? launch<__nv_bfloat16, 64>(cut, g, a, st) : launch<__nv_bfloat16, 128>(cut, g, a, st);
    return dodo_check_cuda(ctx, e, "paged attend launch");
}
