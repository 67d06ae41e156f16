// C ABI entry point of attend's gradient: checks, which kernel, key and query blocks, launches.
#include <stdlib.h>

#include "dodo_internal.cuh"

namespace {

constexpr int kStatAlign = 64;         // a sequence's statistics start at a multiple of this
constexpr int kPartFloats = 128 * 128; // largest partial tile of dQ

size_t round256(size_t n) { return (n + 255) & ~static_cast<size_t>(255); }
int ceil_div(int a, int b) { return (a + b - 1) / b; }

// workspace: statistics of one launch group, the heads' score gradients, partial tiles of dQ
struct Layout { size_t stats, scores, parts, total; };
Layout layout(const dodo_ctx* ctx, int q_rows, int H, int cache_rows) {
    Layout l;
    l.stats = 0;
    l.scores = round256(static_cast<size_t>(H) * (static_cast<size_t>(q_rows) + DODO_GROUP * kStatAlign) * 2 * sizeof(float));
    l.parts = l.scores + round256(static_cast<size_t>(H) * 2 * cache_rows * sizeof(float));
    l.total = l.parts + static_cast<size_t>(2) * ctx->num_sms * kPartFloats * sizeof(float);
    return l;
}

struct Interval { int lo, hi; };
int by_lo(const void* a, const void* b) {
    const int x = static_cast<const Interval*>(a)->lo, y = static_cast<const Interval*>(b)->lo;
    return x < y ? -1 : x > y ? 1 : 0;
}
// Every local row's gradient belongs to one sequence: windows that share rows cannot be served.
int check_windows(dodo_ctx* ctx, const int32_t* loc_off, const int32_t* loc_len, int B) {
    Interval* v = static_cast<Interval*>(malloc(sizeof(Interval) * static_cast<size_t>(B)));
    if (v == nullptr) return dodo_fail(ctx, DODO_ERR_CUDA, "out of host memory");
    int n = 0;
    for (int b = 0; b < B; ++b)
        if (loc_len[b] > 0) { v[n].lo = loc_off[b]; v[n].hi = loc_off[b] + loc_len[b]; ++n; }
    qsort(v, static_cast<size_t>(n), sizeof *v, by_lo);
    int bad = -1;
    for (int i = 1; i < n && bad < 0; ++i)
        if (v[i].lo < v[i - 1].hi) bad = v[i].lo;
    free(v);
    if (bad >= 0) return dodo_fail(ctx, DODO_ERR_INVALID_ARG, "local row %d belongs to two sequences' windows", bad);
    return DODO_OK;
}

// Tables of one launch group.  Query tiles are cut into chunks of their key list only while there are too few of them
// for the device; a sequence's share of the target goes by its part of the work, rounded down, so that the partial tiles
// stay below the target.  The streaming kernel has no query blocks: its key chunks sum dQ too.
int plan_group(dodo_ctx* ctx, const AttendShape& s, int variant, int b0, int nb, BackwardGroup& g) {
    const BackwardTiles t = dodo_backward_tiles(variant, s.dtype, s.dh);
    memset(&g, 0, sizeof g);
    g.nseq = nb;
    int64_t work = 0;
    for (int i = 0; i < nb; ++i) {
        const int b = b0 + i;
        BackwardSeq& q = g.seq[i];
        q.q_row0 = s.q_off[b];
        q.tq = s.q_off[b + 1] - s.q_off[b];
        q.q_pos0 = s.q_pos0[b];
        q.c_len = s.cache_len ? s.cache_len[b] : 0;
        q.c_row0 = q.c_len > 0 ? s.cache_off[b] : 0;
        q.l_len = s.loc_len ? s.loc_len[b] : 0;
        q.l_row0 = q.l_len > 0 ? s.loc_off[b] : 0;
        q.l_pos0 = q.l_len > 0 ? s.loc_pos0[b] : 0;
        const int64_t steps = ceil_div(q.c_len, t.step) + ceil_div(q.l_len, t.step);
        work += steps * s.H * (variant == DODO_BWD_STREAM ? 1 : ceil_div(q.tq, t.queries));
    }
    const int64_t target = 2 * static_cast<int64_t>(ctx->num_sms);
    int64_t kv = 0, qb = 0, parts = 0, qticks = 0, sticks = 0, stat = 0;
    for (int i = 0; i < nb; ++i) {
        BackwardSeq& q = g.seq[i];
        const int steps = ceil_div(q.c_len, t.step) + ceil_div(q.l_len, t.step);
        const int qtiles = variant == DODO_BWD_STREAM ? 1 : ceil_div(q.tq, t.queries);
        int64_t n = work > 0 ? target * steps / work : 1;
        const int most = ceil_div(steps, variant == DODO_BWD_TILE ? 2 : 4);    // chunks of two (fp32 tiles) or four steps at least
        if (n > most) n = most;
        if (n < 1) n = 1;
        q.ctiles = steps > 0 ? ceil_div(steps, static_cast<int>(n)) : 1;
        q.nchunk = steps > 0 ? ceil_div(steps, q.ctiles) : 1;
        q.stat0 = static_cast<int>(stat);
        q.kv0 = static_cast<int>(kv);
        q.q0 = static_cast<int>(qb);
        q.part0 = static_cast<int>(parts);
        q.qtick0 = static_cast<int>(qticks);
        stat += ceil_div(q.tq, kStatAlign) * static_cast<int64_t>(kStatAlign);
        const int64_t units = static_cast<int64_t>(qtiles) * s.H;
        if (variant == DODO_BWD_STREAM) {
            if (steps > 0 || q.tq > 0) kv += units * q.nchunk;
        } else {
            kv += static_cast<int64_t>(ceil_div(q.c_len, t.keys) + ceil_div(q.l_len, t.keys)) * s.H;
            qb += units * q.nchunk;
        }
        if (q.nchunk > 1) {
            parts += units * q.nchunk;
            if (variant != DODO_BWD_DENSE) qticks += units;       // (the tensor-core kernel leaves joins and scores to kernels of their own)
        }
    }
    for (int i = 0; i < nb; ++i) {
        g.seq[i].stick0 = static_cast<int>(qticks + sticks);
        sticks += variant == DODO_BWD_STREAM ? g.seq[i].nchunk : variant == DODO_BWD_TILE ? ceil_div(g.seq[i].c_len, t.keys) : 0;
    }
    if (qticks + sticks > DODO_NUM_TICKETS - 1)      // (the last counter hands out the tensor-core kernel's units)
        return dodo_fail(ctx, DODO_ERR_CAPACITY, "too many key tiles and split query tiles (%lld) in one group of sequences", static_cast<long long>(qticks + sticks));
    if (kv + qb > 0x7fffffff || stat > 0x7fffffff)
        return dodo_fail(ctx, DODO_ERR_CAPACITY, "too many thread blocks (%lld)", static_cast<long long>(kv + qb));
    g.kv_blocks = static_cast<int>(kv);
    g.q_blocks = static_cast<int>(qb);
    g.stat_rows = static_cast<int>(stat);
    return DODO_OK;
}

bool usable(const void* p) { return p != nullptr && dodo_aligned16(p); }

}  // namespace

extern "C" {

size_t dodo_attend_backward_workspace_bytes(const dodo_ctx* ctx, int q_rows, int H, int dh, int cache_rows) {
    if (ctx == nullptr || q_rows < 0 || H <= 0 || dh <= 0 || cache_rows < 0) return 0;
    return layout(ctx, q_rows, H, cache_rows).total;
}

int dodo_attend_backward(dodo_ctx* ctx, const void* Q, const int32_t* q_off, const int32_t* q_pos0, int dtype, int H, int dh,
                         float sm_scale, const void* cacheK, const void* cacheV, const int32_t* cache_pos,
                         const int32_t* cache_off, const int32_t* cache_len, const void* locK, const void* locV,
                         const int32_t* loc_off, const int32_t* loc_len, const int32_t* loc_pos0, int loc_rows, int B,
                         const void* O, const float* lse, const void* dO, void* dQ, void* dcacheK, void* dcacheV, void* dlocK,
                         void* dlocV, float* dscore, void* workspace, size_t workspace_bytes, void* stream) {
    if (ctx == nullptr) return DODO_ERR_INVALID_ARG;
    int rc = dodo_check_attend_queries(ctx, q_off, q_pos0, dtype, H, dh, B);
    if (rc != DODO_OK) return rc;
    bool any_cache = false, any_local = false;
    rc = dodo_check_attend_keys(ctx, cache_off, cache_len, loc_off, loc_len, loc_pos0, loc_rows, B, &any_cache, &any_local);
    if (rc != DODO_OK) return rc;
    if ((rc = dodo_check_positions(ctx, q_off, q_pos0, loc_len, loc_pos0, B)) != DODO_OK) return rc;
    if (B == 0 || (q_off[B] == 0 && !any_cache && !any_local)) return DODO_OK;
    if (q_off[B] > 0 && (!usable(Q) || !usable(O) || !usable(dO) || !usable(dQ) || lse == nullptr))
        return dodo_fail(ctx, DODO_ERR_INVALID_ARG, "Q, O, dO, dQ and lse must be non-NULL, all but lse 16-byte aligned");
    if (any_cache && (!usable(cacheK) || !usable(cacheV) || cache_pos == nullptr || !usable(dcacheK) || !usable(dcacheV)))
        return dodo_fail(ctx, DODO_ERR_INVALID_ARG, "cacheK, cacheV, cache_pos, dcacheK and dcacheV must be non-NULL, all but cache_pos 16-byte aligned");
    if (any_local && (!usable(locK) || !usable(locV) || !usable(dlocK) || !usable(dlocV)))
        return dodo_fail(ctx, DODO_ERR_INVALID_ARG, "locK, locV, dlocK and dlocV must be non-NULL and 16-byte aligned");
    if (any_local && (rc = check_windows(ctx, loc_off, loc_len, B)) != DODO_OK) return rc;
    const Layout lay = layout(ctx, q_off[B], H, any_cache ? cache_off[B] : 0);
    if (!usable(workspace) || workspace_bytes < lay.total)
        return dodo_fail(ctx, DODO_ERR_CAPACITY, "workspace of %zu bytes is too small or misaligned (need %zu)", workspace_bytes, lay.total);
    if ((rc = dodo_check_device(ctx)) != DODO_OK) return rc;

    int max_tq = 0;
    for (int b = 0; b < B; ++b) max_tq = max_tq > q_off[b + 1] - q_off[b] ? max_tq : q_off[b + 1] - q_off[b];
    const int variant = max_tq <= dodo_backward_stream_queries(dtype, dh) ? DODO_BWD_STREAM : dtype == DODO_BF16 ? DODO_BWD_DENSE : DODO_BWD_TILE;
    unsigned char* ws = static_cast<unsigned char*>(workspace);
    BackwardArrays a;
    a.Q = Q; a.O = O; a.dO = dO; a.cK = cacheK; a.cV = cacheV; a.lK = locK; a.lV = locV;
    a.cache_pos = cache_pos; a.lse = lse;
    a.dQ = dQ; a.dcK = dcacheK; a.dcV = dcacheV; a.dlK = dlocK; a.dlV = dlocV;
    a.dscore = any_cache ? dscore : nullptr;
    a.stats = reinterpret_cast<float*>(ws + lay.stats);
    a.score_part = reinterpret_cast<float*>(ws + lay.scores);
    a.dq_part = reinterpret_cast<float*>(ws + lay.parts);
    a.score_rows = any_cache ? cache_off[B] : 0;
    a.tickets = ctx->tickets;
    const AttendShape shp = {q_off, q_pos0, cache_off, cache_len, loc_off, loc_len, loc_pos0, B, H, dh, dtype};
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    // two passes over the launch groups, so that a capacity error comes before any launch
    for (int pass = 0; pass < 2; ++pass) {
        for (int b0 = 0; b0 < B; b0 += DODO_GROUP) {
            BackwardGroup g;
            rc = plan_group(ctx, shp, variant, b0, B - b0 < DODO_GROUP ? B - b0 : DODO_GROUP, g);
            if (rc != DODO_OK) return rc;
            if (pass == 0) continue;
            if (variant == DODO_BWD_STREAM) {
                rc = dodo_launch_backward_stream(ctx, dtype, H, dh, sm_scale, max_tq, g, a, st);
            } else if (variant == DODO_BWD_TILE) {
                rc = dodo_launch_backward_tile(ctx, H, dh, sm_scale, g, a, st);
            } else {
                rc = dodo_launch_backward_stats(ctx, H, dh, g, a, st);
                if (rc == DODO_OK)
                    rc = dodo_launch_backward_dense(ctx, H, dh, sm_scale, g, a, q_off[B], a.score_rows, any_local ? loc_rows : 0,
                                                    ctx->tickets + DODO_NUM_TICKETS - 1, st);
            }
            if (rc != DODO_OK) return rc;
        }
    }
    return DODO_OK;
}

}  // extern "C"
