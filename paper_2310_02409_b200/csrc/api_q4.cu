// C ABI entry points of the 4-bit nugget cache: append, expansion, attention.
#include <stdlib.h>

#include "dodo_internal.cuh"

namespace {

bool q4_head(int dh) { return dh == 64 || dh == 128; }
size_t round16(size_t n) { return (n + 15) & ~static_cast<size_t>(15); }

int check_cache_arrays(dodo_ctx* ctx, const void* cache_q4, const uint32_t* cache_scale) {
    if (cache_q4 == nullptr || cache_scale == nullptr || !dodo_aligned16(cache_q4) || !dodo_aligned16(cache_scale))
        return dodo_fail(ctx, DODO_ERR_INVALID_ARG, "cache_q4 and cache_scale must be non-NULL and 16-byte aligned");
    return DODO_OK;
}

// expansion of the rows in use, sequence by sequence, into arrays laid out like the cache
int expand_rows(dodo_ctx* ctx, const void* cache_q4, const uint32_t* cache_scale, int H, int dh, int dtype,
                const int32_t* cache_off, const int32_t* cache_len, int B, void* K, void* V, cudaStream_t st) {
    for (int b0 = 0; b0 < B; b0 += DODO_GROUP) {
        ExpandGroup g;
        memset(&g, 0, sizeof g);
        g.nseq = B - b0 < DODO_GROUP ? B - b0 : DODO_GROUP;
        for (int i = 0; i < g.nseq; ++i) {
            g.row0[i] = cache_off[b0 + i];
            g.out0[i + 1] = g.out0[i] + cache_len[b0 + i];
        }
        const int rc = dodo_launch_expand_q4(ctx, cache_q4, cache_scale, H, dh, dtype, g, K, V, st);
        if (rc != DODO_OK) return rc;
    }
    return DODO_OK;
}

}  // namespace

extern "C" {

int dodo_gather_kv_q4(dodo_ctx* ctx, const void* K, const void* V, int dtype, int H, int dh, const int32_t* seq_off,
                      const int32_t* idx, const int32_t* nug_off, const int32_t* pos_base, int B, void* cache_q4,
                      uint32_t* cache_scale, int32_t* cache_pos, const int32_t* cache_off, int32_t* cache_len, void* stream) {
    if (ctx == nullptr) return DODO_ERR_INVALID_ARG;
    size_t row_bytes = 0;
    int rc = dodo_check_gather(ctx, dtype, H, dh, seq_off, nug_off, pos_base, B, cache_off, cache_len, &row_bytes);
    if (rc != DODO_OK) return rc;
    if (!q4_head(dh)) return dodo_fail(ctx, DODO_ERR_UNSUPPORTED, "head size %d (supported: 64, 128)", dh);
    if (nug_off[B] > 0) {
        if (K == nullptr || V == nullptr || idx == nullptr || cache_pos == nullptr || !dodo_aligned16(K) || !dodo_aligned16(V))
            return dodo_fail(ctx, DODO_ERR_INVALID_ARG, "K, V, idx and cache_pos must be non-NULL, K and V 16-byte aligned");
        if ((rc = check_cache_arrays(ctx, cache_q4, cache_scale)) != DODO_OK) return rc;
    }
    if ((rc = dodo_check_device(ctx)) != DODO_OK) return rc;
    for (int b0 = 0; b0 < B; b0 += DODO_GROUP) {
        GatherGroup g;
        dodo_fill_gather_group(g, b0, B, seq_off, nug_off, pos_base, cache_off, cache_len);
        ctx->cache_clean = false;   // the next attend must not read cache rows ahead of its dependency wait
        rc = dodo_launch_gather_q4(ctx, K, V, dtype, H, dh, idx, g, cache_q4, cache_scale, cache_pos, ctx->dev_status,
                                   static_cast<cudaStream_t>(stream));
        if (rc != DODO_OK) return rc;
    }
    for (int b = 0; b < B; ++b) cache_len[b] += nug_off[b + 1] - nug_off[b];
    return DODO_OK;
}

int dodo_expand_kv_q4(dodo_ctx* ctx, const void* cache_q4, const uint32_t* cache_scale, int H, int dh, const int32_t* cache_off,
                      const int32_t* cache_len, int B, int dtype, void* K, void* V, void* stream) {
    if (ctx == nullptr) return DODO_ERR_INVALID_ARG;
    if (B < 0) return dodo_fail(ctx, DODO_ERR_INVALID_ARG, "B = %d is negative", B);
    if (dtype != DODO_F32 && dtype != DODO_BF16) return dodo_fail(ctx, DODO_ERR_UNSUPPORTED, "dtype %d", dtype);
    if (!q4_head(dh)) return dodo_fail(ctx, DODO_ERR_UNSUPPORTED, "head size %d (supported: 64, 128)", dh);
    if (H <= 0) return dodo_fail(ctx, DODO_ERR_INVALID_ARG, "H = %d", H);
    if (cache_off == nullptr || cache_len == nullptr) return dodo_fail(ctx, DODO_ERR_INVALID_ARG, "cache_off and cache_len must not be NULL");
    bool any_cache = false, any_local = false;
    int rc = dodo_check_attend_keys(ctx, cache_off, cache_len, nullptr, nullptr, nullptr, 0, B, &any_cache, &any_local);
    if (rc != DODO_OK || !any_cache) return rc;
    if ((rc = check_cache_arrays(ctx, cache_q4, cache_scale)) != DODO_OK) return rc;
    if (K == nullptr || V == nullptr || !dodo_aligned16(K) || !dodo_aligned16(V))
        return dodo_fail(ctx, DODO_ERR_INVALID_ARG, "K and V must be non-NULL and 16-byte aligned");
    if ((rc = dodo_check_device(ctx)) != DODO_OK) return rc;
    ctx->cache_clean = false;       // K and V may be a nugget cache that the next attend reads
    return expand_rows(ctx, cache_q4, cache_scale, H, dh, dtype, cache_off, cache_len, B, K, V, static_cast<cudaStream_t>(stream));
}

size_t dodo_attend_q4_workspace_bytes(const dodo_ctx* ctx, int H, int dh, int cache_rows) {
    if (ctx == nullptr || H <= 0 || dh <= 0 || cache_rows < 0) return 0;
    return round16(dodo_attend_workspace_bytes(ctx, dh)) + 2 * static_cast<size_t>(cache_rows) * H * dh * dodo_elem_bytes(DODO_BF16);
}

int dodo_attend_q4(dodo_ctx* ctx, const void* Q, const int32_t* q_off, const int32_t* q_pos0, int dtype, int H, int dh,
                   float sm_scale, const void* cache_q4, const uint32_t* cache_scale, const int32_t* cache_pos,
                   const int32_t* cache_off, const int32_t* cache_len, const void* locK, const void* locV,
                   const int32_t* loc_off, const int32_t* loc_len, const int32_t* loc_pos0, int loc_rows, int B, void* O,
                   float* lse, void* workspace, size_t workspace_bytes, void* stream) {
    if (ctx == nullptr) return DODO_ERR_INVALID_ARG;
    int rc = dodo_check_attend_queries(ctx, q_off, q_pos0, dtype, H, dh, B);
    if (rc != DODO_OK || q_off[B] == 0) return rc;
    if (Q == nullptr || O == nullptr || !dodo_aligned16(Q) || !dodo_aligned16(O))
        return dodo_fail(ctx, DODO_ERR_INVALID_ARG, "Q and O must be non-NULL and 16-byte aligned");
    bool any_cache = false, any_local = false;
    rc = dodo_check_attend_keys(ctx, cache_off, cache_len, loc_off, loc_len, loc_pos0, loc_rows, B, &any_cache, &any_local);
    if (rc != DODO_OK) return rc;
    if ((rc = dodo_check_positions(ctx, q_off, q_pos0, loc_len, loc_pos0, B)) != DODO_OK) return rc;
    if (any_cache) {
        if ((rc = check_cache_arrays(ctx, cache_q4, cache_scale)) != DODO_OK) return rc;
        if (cache_pos == nullptr) return dodo_fail(ctx, DODO_ERR_INVALID_ARG, "cache_pos must not be NULL");
    }
    if (any_local && (locK == nullptr || locV == nullptr || !dodo_aligned16(locK) || !dodo_aligned16(locV)))
        return dodo_fail(ctx, DODO_ERR_INVALID_ARG, "locK and locV must be non-NULL and 16-byte aligned");
    if ((rc = dodo_check_device(ctx)) != DODO_OK) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(stream);

    // A block of many bf16 queries is a contraction: expand the rows in use once and attend them on the tensor cores,
    // if the caller's workspace has room for them.
    int max_tq = 0;
    for (int b = 0; b < B; ++b) max_tq = max_tq > q_off[b + 1] - q_off[b] ? max_tq : q_off[b + 1] - q_off[b];
    const int cache_rows = any_cache ? cache_off[B] : 0;
    if (dtype == DODO_BF16 && dh == 128 && sm_scale >= DODO_DENSE_LEAST_SCALE && max_tq >= ctx->dense_min_tq && workspace != nullptr &&
        dodo_aligned16(workspace) && workspace_bytes >= dodo_attend_q4_workspace_bytes(ctx, H, dh, cache_rows)) {
        const size_t head = round16(dodo_attend_workspace_bytes(ctx, dh));
        unsigned char* K = static_cast<unsigned char*>(workspace) + head;
        unsigned char* V = K + static_cast<size_t>(cache_rows) * H * dh * dodo_elem_bytes(dtype);
        if (any_cache) {
            rc = expand_rows(ctx, cache_q4, cache_scale, H, dh, dtype, cache_off, cache_len, B, K, V, st);
            if (rc != DODO_OK) return rc;
            ctx->cache_clean = false;
        }
        return dodo_attend(ctx, Q, q_off, q_pos0, dtype, H, dh, sm_scale, K, V, cache_pos, cache_off, cache_len, locK, locV, loc_off,
                           loc_len, loc_pos0, loc_rows, B, O, lse, workspace, head, stream);
    }

    AttendShape shp = {q_off, q_pos0, cache_off, cache_len, loc_off, loc_len, loc_pos0, B, H, dh, dtype};
    AttendPlan plan;
    AttendTotals tot;
    dodo_attend_plan_begin(shp, ctx->attend_target_ctas, plan, tot, dodo_attend_q4_tile_queries(dtype, max_tq));
    // A sequence whose key list is longer than a block's share of the work is cut even when there are units enough for the
    // device (one long sequence of a ragged batch would outlast all others), but never into chunks of less than four tiles,
    // whose merge costs more than it saves (8 x 269 keys of 32 heads in two chunks each: 11.8 against 6.6 us).
    tot.split = tot.work > tot.units;
    tot.min_chunk = 4;
    tot.target = dodo_attend_q4_target(ctx->attend_target_ctas);
    const int ngroups = (B + DODO_GROUP - 1) / DODO_GROUP;
    AttendGroup one;
    AttendGroup* groups = &one;
    if (ngroups > 1) {
        groups = static_cast<AttendGroup*>(malloc(sizeof(AttendGroup) * static_cast<size_t>(ngroups)));
        if (groups == nullptr) return dodo_fail(ctx, DODO_ERR_CUDA, "out of host memory");
    }
    for (int gi = 0; gi < ngroups; ++gi) {
        const int b0 = gi * DODO_GROUP;
        dodo_attend_plan_group(shp, plan, tot, b0, B - b0 < DODO_GROUP ? B - b0 : DODO_GROUP, groups[gi]);
    }
    const size_t need = static_cast<size_t>(tot.part_rows) * (dh + 2) * sizeof(float);
    if (tot.part_rows > 0 && (workspace == nullptr || !dodo_aligned16(workspace) || need > workspace_bytes))
        rc = dodo_fail(ctx, DODO_ERR_CAPACITY, "workspace of %zu bytes is too small or misaligned (need %zu)", workspace_bytes, need);
    else if (tot.tick_rows > DODO_NUM_TICKETS)
        rc = dodo_fail(ctx, DODO_ERR_CAPACITY, "too many split units (%lld)", static_cast<long long>(tot.tick_rows));
    const unsigned long long capture = dodo_capture_id(st);
    for (int gi = 0; gi < ngroups && rc == DODO_OK; ++gi) {
        if (groups[gi].cta0[groups[gi].nseq] == 0) continue;      // no query in it, nothing launched: it settles nothing
        const bool early = dodo_cache_settled(ctx, capture);
        rc = dodo_launch_attend_q4(ctx, dtype, H, dh, sm_scale, plan, groups[gi], Q, cache_q4, cache_scale, cache_rows, cache_pos, locK, locV, O, lse,
                                   static_cast<float*>(workspace), ctx->tickets, early, st);
        if (rc == DODO_OK) dodo_attend_launched(ctx, capture);
    }
    if (groups != &one) free(groups);
    return rc;
}

}  // extern "C"
