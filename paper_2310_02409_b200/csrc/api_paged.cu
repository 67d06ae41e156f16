// C ABI entry point of attention over a paged cache: checks, tables, choice of kernel.
#include <algorithm>

#include "paged.cuh"

int dodo_check_paged(dodo_ctx* ctx, const dodo_paged_cache* c, const int32_t* page_off, const int32_t* cache_len, int B, bool rows);

// Chunks of each sequence's key list, blocks, partial rows and arrival counters.  A list is cut where it is longer than a block's share of
// all the work (units times keys over the blocks to aim at), into chunks of about that share, all alike.  A cut list has more than one share,
// so its chunks are fewer than twice its shares and the chunks of all cut units fewer than twice the target: dodo_paged_part_rows.
// Without room for partial rows no list is cut.
void dodo_paged_plan(const PagedCut& cut, PagedGroup& g, int group, int Hkv, bool may_cut) {
    auto tiles_of = [&](const PagedSeq& s) {
        // (tiles of cached rows, then tiles of local tokens: one more than there are keys for, at most)
        return (static_cast<int64_t>(s.c_len) + cut.keys - 1) / cut.keys + (dodo_visible_local(s.l_len, s.l_pos0, s.q_pos0 + s.tq - 1) + cut.keys - 1) / cut.keys;
    };
    auto units_of = [&](const PagedSeq& s) { return (static_cast<int64_t>(s.tq) * group + cut.rows - 1) / cut.rows * Hkv; };
    int64_t work = 0;
    for (int i = 0; i < g.nseq; ++i) work += units_of(g.seq[i]) * tiles_of(g.seq[i]);
    int64_t share = (work + cut.target - 1) / cut.target;
    if (share < cut.least / cut.keys) share = cut.least / cut.keys;
    // chunks of whole tiles may come to a few blocks more than the device holds at once, whose turn would come behind all others:
    // larger chunks then, unless the whole units alone are that many.  Lists shorter than a share count as the part of one that they are, and
    // come last, where they fill what the others leave (7 x 4 or 5 tokens of 34 heads of 64 over lists of 10 to 3976 keys: 56 us where they
    // counted whole, 36 so).
    int64_t blocks = 0;
    for (int turn = 0; turn < 16; ++turn) {
        int64_t parts = 0, whole = 0;      // sixteenths of a share's block
        blocks = 0;
        for (int i = 0; i < g.nseq; ++i) {
            const int64_t u = units_of(g.seq[i]), n = tiles_of(g.seq[i]), of = n > share ? 16 * ((n + share - 1) / share) : 1 + 15 * n / share;
            parts += u * of;
            whole += u * (of < 16 ? of : 16);
            blocks += u * (n > share ? (n + share - 1) / share : 1);
        }
        if (parts <= 16 * static_cast<int64_t>(cut.target) || whole >= 16 * static_cast<int64_t>(cut.target)) break;
        share += 1 + (parts - 16 * static_cast<int64_t>(cut.target)) * share / (4 * parts);
    }
    if (blocks > cut.target)
        std::stable_sort(g.seq, g.seq + g.nseq, [](const PagedSeq& a, const PagedSeq& b) {
            return static_cast<int64_t>(a.c_len) + a.l_len > static_cast<int64_t>(b.c_len) + b.l_len;
        });
    int64_t part = 0, tick = 0, cta = 0;
    for (int i = 0; i < g.nseq; ++i) {
        PagedSeq& s = g.seq[i];
        const int64_t tiles = tiles_of(s), units = units_of(s);
        const int64_t n = may_cut && tiles > share ? (tiles + share - 1) / share : 1, each = (tiles + n - 1) / n;
        s.nchunk = static_cast<int>(tiles > 0 ? (tiles + each - 1) / each : 1);
        s.chunk_keys = static_cast<int>((tiles > 0 ? each : 1) * cut.keys);
        s.part0 = static_cast<int>(part);
        s.tick0 = static_cast<int>(tick);
        if (s.nchunk > 1) { part += units * s.nchunk * cut.rows; tick += units; }
        g.cta0[i] = static_cast<int>(cta);
        cta += units * s.nchunk;
    }
    g.cta0[g.nseq] = static_cast<int>(cta);
}

namespace {
// Whether a batch is worth the tensor cores' kernel, whose blocks take longer to begin and to end, or the one for few rows takes it in
// tiles of 16.  By what both take for stages of keys per SM: about 6 us and 1.6 us for each 64 keys of 16 rows that two blocks of an SM have,
// against 14 us and 2.4 us for each 128 keys of a tile of rows.  (16 queries of four heads a KV head, 4 x 4000 keys, 8 KV heads: 46 us there,
// 32 here; 6 queries over 2000 keys of one sequence: 19 there, 22 here.)  More tiles of 16 rows than blocks at a time take turns: four
// sequences of 64 rows and 264 keys, 32 KV heads, 25 us there and 15 here.  Up to 16 rows there is nothing to gain here.  Pages that are no
// multiple of eight rows are not weighed: the other kernel does not take them, and the FMA units would have to, so more than 16 rows go here.
bool is_contraction(const PagedGroup& g, int group, int Hkv, int max_rows, int num_sms) {
    const int tile_rows = max_rows > 128 ? 256 : 128;
    int64_t few = 0, many = 0, units = 0;
    for (int i = 0; i < g.nseq; ++i) {
        const PagedSeq& s = g.seq[i];
        if (s.tq == 0) continue;
        const int64_t rows = static_cast<int64_t>(s.tq) * group, local = dodo_visible_local(s.l_len, s.l_pos0, s.q_pos0 + s.tq - 1);
        units += (rows + 15) / 16 * Hkv;
        few += (rows + 15) / 16 * Hkv * ((s.c_len + 63) / 64 + (local + 63) / 64);
        many += (rows + tile_rows - 1) / tile_rows * Hkv * ((s.c_len + 127) / 128 + (local + 127) / 128);
    }
    const double turns = units > 2 * num_sms ? static_cast<double>((units + 2 * num_sms - 1) / (2 * num_sms)) / units : 0.5 / num_sms;
    return 1.6 * few * turns > 8.0 + 2.4 * many / num_sms;
}
// Whether fp32 rows are taken in tiles: where tiles of 128 keys and up to 64 rows are blocks enough for the device.  Fewer are spread over more
// blocks by the kernel for few rows (64 rows over 124 keys of 8 heads: 9 us there, 27 in tiles; four times 64 rows over 1064 keys: 111, 70).
bool is_tiled(const PagedGroup& g, int group, int Hkv, int max_rows, int num_sms) {
    const int tile_rows = max_rows <= 32 ? 32 : 64;
    int64_t blocks = 0;
    for (int i = 0; i < g.nseq; ++i) {
        const PagedSeq& s = g.seq[i];
        const int64_t chunks = (static_cast<int64_t>(s.c_len) + s.l_len) / 128;
        blocks += (static_cast<int64_t>(s.tq) * group + tile_rows - 1) / tile_rows * Hkv * (chunks > 1 ? chunks : 1);
    }
    return blocks >= num_sms;
}
// n / d = n * mul >> shift for 0 <= n < 2^31: mul = ceil(2^shift / d) with 2^(shift - 31) >= d is at most d / 2^shift too large
void divide_by(int d, uint32_t& mul, int& shift) {
    shift = 31;
    while ((int64_t{1} << (shift - 31)) < d) ++shift;
    mul = static_cast<uint32_t>(((uint64_t{1} << shift) + d - 1) / d);
}
}  // namespace

extern "C" {

size_t dodo_attend_paged_workspace_bytes(const dodo_ctx* ctx, int dh) {
    if (ctx == nullptr || dh <= 0) return 0;
    const size_t rows = dodo_paged_part_rows({kPagedRowsMost, 0, dodo_paged_rows_blocks(ctx), 0, 0}) * dodo_paged_part_floats(dh) * sizeof(float);
    const size_t dense = dodo_paged_dense_workspace_bytes(ctx->num_sms, dh);
    return rows > dense ? rows : dense;
}

int dodo_attend_paged(dodo_ctx* ctx, const void* Q, const int32_t* q_off, const int32_t* q_pos0, int H, float sm_scale,
                      const dodo_paged_cache* cache, const int32_t* page_off, const int32_t* cache_len, const void* locK, const void* locV,
                      const int32_t* loc_off, const int32_t* loc_len, const int32_t* loc_pos0, int loc_rows, int B, void* O, float* lse,
                      void* workspace, size_t workspace_bytes, void* stream) {
    if (ctx == nullptr) return DODO_ERR_INVALID_ARG;
    if (cache == nullptr) return dodo_fail(ctx, DODO_ERR_INVALID_ARG, "cache must not be NULL");
    const int dtype = cache->dtype, dh = cache->dh, Hkv = cache->H;
    int rc = dodo_check_attend_queries(ctx, q_off, q_pos0, dtype, H, dh, B);
    if (rc != DODO_OK) return rc;
    if (Hkv <= 0 || H % Hkv != 0) return dodo_fail(ctx, DODO_ERR_INVALID_ARG, "%d query heads over %d heads of the cache", H, Hkv);
    if ((rc = dodo_check_paged(ctx, cache, page_off, cache_len, B, false)) != DODO_OK) return rc;
    bool any_rows = false, any_cache = false, any_local = false;
    for (int b = 0; b < B; ++b) any_rows = any_rows || cache_len[b] > 0;
    if (any_rows && (rc = dodo_check_paged(ctx, cache, page_off, cache_len, B, true)) != DODO_OK) return rc;
    if ((rc = dodo_check_attend_keys(ctx, nullptr, nullptr, loc_off, loc_len, loc_pos0, loc_rows, B, &any_cache, &any_local)) != DODO_OK) return rc;
    if ((rc = dodo_check_positions(ctx, q_off, q_pos0, loc_len, loc_pos0, B)) != DODO_OK) return rc;
    if (q_off[B] == 0) return DODO_OK;
    if (Q == nullptr || O == nullptr || !dodo_aligned16(Q) || !dodo_aligned16(O))
        return dodo_fail(ctx, DODO_ERR_INVALID_ARG, "Q and O must be non-NULL and 16-byte aligned");
    if (any_local && (locK == nullptr || locV == nullptr || !dodo_aligned16(locK) || !dodo_aligned16(locV)))
        return dodo_fail(ctx, DODO_ERR_INVALID_ARG, "locK and locV must be non-NULL and 16-byte aligned");
    for (int b = 0; b < B; ++b)
        if (static_cast<int64_t>(cache_len[b]) + (loc_len != nullptr ? loc_len[b] : 0) > 0x7ff00000)
            return dodo_fail(ctx, DODO_ERR_UNSUPPORTED, "sequence %d: more than 2^31 - 2^20 keys", b);
    if (!dodo_aligned16(workspace)) return dodo_fail(ctx, DODO_ERR_INVALID_ARG, "workspace must be 16-byte aligned");
    if ((rc = dodo_check_device(ctx)) != DODO_OK) return rc;
    cudaStream_t st = static_cast<cudaStream_t>(stream);

    PagedArrays a;
    memset(&a, 0, sizeof a);
    a.Q = Q; a.O = O;
    const bool any_page = any_rows && cache->pages > 0;      // (a pool of no pages: no entry of the table is one)
    a.cK = any_page ? cache->K : nullptr; a.cV = any_page ? cache->V : nullptr;
    a.lK = any_local ? locK : nullptr; a.lV = any_local ? locV : nullptr;
    a.pos = cache->pos; a.table = cache->table;
    a.pages = cache->pages; a.page = cache->page;
    a.H = H; a.Hkv = Hkv; a.group = H / Hkv;
    divide_by(cache->page, a.page_mul, a.page_shift);
    divide_by(a.group, a.group_mul, a.group_shift);
    a.scale_log2 = sm_scale * 1.4426950408889634f;
    a.lse = lse;
    a.part = static_cast<float*>(workspace);
    a.tickets = ctx->tickets;
    a.status = ctx->dev_status;
    for (int b0 = 0; b0 < B; b0 += DODO_GROUP) {
        PagedGroup g;
        g.nseq = B - b0 < DODO_GROUP ? B - b0 : DODO_GROUP;
        int64_t most = 0;
        for (int i = 0; i < g.nseq; ++i) {
            const int b = b0 + i, l = loc_len != nullptr ? loc_len[b] : 0;
            g.seq[i] = {q_off[b], q_off[b + 1] - q_off[b], q_pos0[b], cache_len[b], page_off[b], l > 0 ? loc_off[b] : 0, l, l > 0 ? loc_pos0[b] : 0, 1, 1, 0, 0};
            most = most > static_cast<int64_t>(g.seq[i].tq) * a.group ? most : static_cast<int64_t>(g.seq[i].tq) * a.group;
        }
        if (most == 0) continue;
        const int max_rows = most > 0x7fffffff ? 0x7fffffff : static_cast<int>(most);
        const bool boxes = dodo_paged_box(cache->page, 8) > 0;       // pages that tensor copies can take by boxes
        // Many bf16 rows are a contraction: the tensor cores.  (Row maxima are taken before scaling, so the scale must be positive.)
        if (dtype == DODO_BF16 && sm_scale >= DODO_DENSE_LEAST_SCALE && workspace != nullptr &&
            workspace_bytes >= dodo_paged_dense_workspace_bytes(ctx->num_sms, dh) && ctx->paged_dense != 2 &&
            (ctx->paged_dense == 1 || (max_rows > 16 && (!boxes || is_contraction(g, a.group, Hkv, max_rows, ctx->num_sms))))) {
            if ((rc = dodo_launch_paged_dense(ctx, dh, max_rows, any_local ? loc_rows : 0, g, a, st)) != DODO_OK) return rc;
            continue;
        }
        const bool token = dtype == DODO_BF16 && boxes, tile = dtype == DODO_F32 && max_rows > 16 && is_tiled(g, a.group, Hkv, max_rows, ctx->num_sms);
        const PagedCut cut = token ? dodo_paged_token_cut(ctx, max_rows) : tile ? dodo_paged_tile_cut(ctx, g, a.group, Hkv, max_rows) : dodo_paged_rows_cut(ctx, g, a.group, Hkv, max_rows);
        const size_t need = dodo_paged_part_rows(cut) * dodo_paged_part_floats(dh) * sizeof(float);
        dodo_paged_plan(cut, g, a.group, Hkv, workspace != nullptr && workspace_bytes >= need);
        if (token) rc = dodo_launch_paged_token(ctx, dh, max_rows, any_local ? loc_rows : 0, g, a, st);
        else if (tile) rc = dodo_launch_paged_tile(ctx, dh, cut, g, a, st);
        else rc = dodo_launch_paged_rows(ctx, dtype, dh, cut, g, a, st);
        if (rc != DODO_OK) return rc;
    }
    return DODO_OK;
}

}  // extern "C"
