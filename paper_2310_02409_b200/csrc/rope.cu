// Rotary positions of whole arrays (a layer's queries and keys) and their gradient.  A copy with a few operations an element: bound
// by HBM (16,384 tokens of 40 + 40 heads: 110 us, 6.1 TB/s; gradient of 5120 tokens of 32 + 32 interleaved heads: 34 us, 4.9 TB/s, the
// launch's begin and end inside it; a token: 2.1 us, the launch).  A block takes a few tokens; its threads make the sines and cosines of the tokens' pairs once, in shared memory (made by
// every head they would cost as much as the copy), and then run over the heads of all arrays, 16 bytes of each half of a head at
// a time: two such pieces (eight of the interleaved layout) are requested together, then turned and stored, the first ones while sines and
// cosines are made; what covers the others' way is the SM's other warps.  Rotations whose halves are no multiple of 16 bytes go element by element:
// 16,384 tokens of 40 + 40 bf16 heads of 96 with 24 features turned take 487 us (0.16 of their bytes' time), of 80 with 20 as long, fp32 too.
#include <math.h>

#include "rope.cuh"

namespace {

using namespace dodo_rotary;

struct RopeArrays {
    int n, heads;                                // arrays; heads of all of them
    const void* in[DODO_ROPE_ARRAYS];
    void* out[DODO_ROPE_ARRAYS];
    int first[DODO_ROPE_ARRAYS];                 // first head of the array in the count of all heads
    long long in_row[DODO_ROPE_ARRAYS], in_head[DODO_ROPE_ARRAYS], out_row[DODO_ROPE_ARRAYS], out_head[DODO_ROPE_ARRAYS];
};
struct RopeRows {
    int nseq;
    int row0[DODO_GROUP + 1];
    int pos0[DODO_GROUP];
};

__device__ __forceinline__ int sequence_of(const int* row0, int nseq, int row) {
    int lo = 0, hi = nseq;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (row0[mid] <= row) lo = mid; else hi = mid;
    }
    return lo;
}

// slots: pieces of a head; blockDim.x >= slots * lanes, thread = (lane, slot), lanes run over the heads
template <typename T, int VEC, bool INTER>
__global__ void __launch_bounds__(512)
rope_kernel(const __grid_constant__ RopeArrays a, const __grid_constant__ Rotation p, const __grid_constant__ RopeRows g, int dh, int slots,
            int lanes, int tokens) {
    extern __shared__ float2 cs[];               // [tokens][half]
    const int tid = static_cast<int>(threadIdx.x), slot = tid % slots, lane = tid / slots;
    const int row_first = g.row0[0] + static_cast<int>(blockIdx.x) * tokens, row_end = row_first + min(tokens, g.row0[g.nseq] - row_first);
    const int step = lanes * static_cast<int>(gridDim.y), head0 = lane < lanes ? lane + lanes * static_cast<int>(blockIdx.y) : a.heads;
    const int per_row = head0 < a.heads ? (a.heads - head0 + step - 1) / step : 0;      // this thread's pieces of a row
    const int items = per_row * (row_end - row_first);
    constexpr int kBatch = INTER ? 8 : 2;        // pieces (of one or two loads) on their way at a time

    auto array_of = [&](int head) {
        int k = 0;
#pragma unroll
        for (int i = 1; i < DODO_ROPE_ARRAYS; ++i) k += i < a.n && head >= a.first[i] ? 1 : 0;
        return k;
    };
    int load_row = row_first, load_head = head0, row = row_first, head = head0;
    Slot<T, VEC, INTER> piece[kBatch];
    auto fetch = [&](int first) {
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            if (first + u >= items) return;
            const int k = array_of(load_head);
            piece[u].load(static_cast<const T*>(a.in[k]) + load_row * a.in_row[k] + (load_head - a.first[k]) * a.in_head[k], slot, p.half);
            load_head += step;
            if (load_head >= a.heads) { load_head = head0; ++load_row; }
        }
    };
    dodo_grid_dependency_sync();
    fetch(0);
    for (int i = tid; i < (row_end - row_first) * p.half; i += static_cast<int>(blockDim.x)) {
        const int r = row_first + i / p.half, b = sequence_of(g.row0, g.nseq, r);
        cs[i] = cos_sin(p, i % p.half, g.pos0[b] + (r - g.row0[b]));
    }
    __syncthreads();
    for (int it = 0; it < items; it += kBatch) {
        if (it > 0) fetch(it);
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            if (it + u >= items) return;
            const int k = array_of(head);
            piece[u].store(static_cast<T*>(a.out[k]) + row * a.out_row[k] + (head - a.first[k]) * a.out_head[k], slot, p.half,
                           cs + static_cast<size_t>(row - row_first) * p.half);
            head += step;
            if (head >= a.heads) { head = head0; ++row; }
        }
    }
}

template <typename T, int VEC, bool INTER>
cudaError_t launch(const dodo_ctx* ctx, const RopeArrays& a, const Rotation& p, const RopeRows& g, int dh, cudaStream_t st) {
    const int slots = slots_of<VEC, INTER>(dh, p.half), rows = g.row0[g.nseq] - g.row0[0];
    const int lanes = slots >= 128 ? 1 : min(128 / slots, a.heads);
    // Two tokens a block of 128 threads once there are blocks enough for the device that way, so that sines and cosines are made while the
    // first rows are on their way (16,384 tokens of 40 + 40 heads: 110 us; one token 140, four 113); else one, and where tokens are few
    // their heads are spread over blocks as well
    const int tokens = rows >= 2 * 8 * ctx->num_sms ? 2 : 1;
    const int split = rows >= 4 * ctx->num_sms ? 1 : (a.heads + lanes - 1) / lanes;
    const int threads = (slots * lanes + 31) / 32 * 32;
    return dodo_launch_dependent(rope_kernel<T, VEC, INTER>, dim3(static_cast<unsigned>((rows - 1) / tokens + 1), static_cast<unsigned>(split)),
                                 dim3(static_cast<unsigned>(threads)), sizeof(float2) * tokens * p.half, st, a, p, g, dh, slots, lanes, tokens);
}

// Whether two heads of dh elements each, of `rows` rows and `heads` heads at these distances, share an element
bool lie_over_one_another(int rows, int heads, int64_t row, int64_t head, int dh) {
    const __int128 r = row < 0 ? -static_cast<__int128>(row) : row, h = head < 0 ? -static_cast<__int128>(head) : head;
    if (heads > 0 && ((rows > 1 && r < dh) || (heads > 1 && h < dh))) return true;
    if (rows <= 1 || heads <= 1 || r >= h * (heads - 1) + dh || h >= r * (rows - 1) + dh) return false;
    // neither lies whole within a step of the other: heads k apart against the rows next to them
    for (int k = 1; k < heads; ++k) {
        const __int128 at = h * k, n = at / r;
        if ((n < rows && at - n * r < dh) || (n + 1 < rows && (n + 1) * r - at < dh)) return true;
    }
    return false;
}

int rope_impl(dodo_ctx* ctx, const dodo_rope_spec* rope, const dodo_rope_array* arrays, int n, int dtype, int dh, const int32_t* row_off,
              const int32_t* pos0, int B, bool back, cudaStream_t st) {
    if (ctx == nullptr) return DODO_ERR_INVALID_ARG;
    if (B < 0) return dodo_fail(ctx, DODO_ERR_INVALID_ARG, "B = %d is negative", B);
    if (dtype != DODO_F32 && dtype != DODO_BF16) return dodo_fail(ctx, DODO_ERR_UNSUPPORTED, "dtype %d", dtype);
    int rc = dodo_check_rope(ctx, rope, dh);
    if (rc != DODO_OK) return rc;
    if (n < 0 || n > DODO_ROPE_ARRAYS || (n > 0 && arrays == nullptr)) return dodo_fail(ctx, DODO_ERR_INVALID_ARG, "%d arrays (0 to %d)", n, DODO_ROPE_ARRAYS);
    if (!dodo_valid_offsets(row_off, B)) return dodo_fail(ctx, DODO_ERR_INVALID_ARG, "row_off must start at 0 and be non-decreasing");
    if (B > 0 && pos0 == nullptr) return dodo_fail(ctx, DODO_ERR_INVALID_ARG, "pos0 must not be NULL");
    for (int b = 0; b < B; ++b)
        if (static_cast<int64_t>(pos0[b]) + (row_off[b + 1] - row_off[b]) > (int64_t{1} << 31))
            return dodo_fail(ctx, DODO_ERR_INVALID_ARG, "sequence %d: positions from %d pass 2^31", b, pos0[b]);
    const size_t e = dodo_elem_bytes(dtype);
    RopeArrays a;
    memset(&a, 0, sizeof a);
    bool wide = wide_fits(dtype, rope->layout, dh, rope->rot);
    for (int i = 0; i < n; ++i) {
        const dodo_rope_array& v = arrays[i];
        if (v.heads < 0) return dodo_fail(ctx, DODO_ERR_INVALID_ARG, "array %d: %d heads", i, v.heads);
        if (v.heads == 0 || row_off[B] == 0) continue;
        if (v.in == nullptr || v.out == nullptr) return dodo_fail(ctx, DODO_ERR_INVALID_ARG, "array %d: in and out must not be NULL", i);
        if (reinterpret_cast<uintptr_t>(v.in) % e != 0 || reinterpret_cast<uintptr_t>(v.out) % e != 0)
            return dodo_fail(ctx, DODO_ERR_INVALID_ARG, "array %d is not aligned to its type", i);
        // 16-byte pieces need every row and head to start on 16 bytes
        wide = wide && dodo_aligned16(v.in) && dodo_aligned16(v.out) && v.in_row * static_cast<int64_t>(e) % 16 == 0 && v.in_head * static_cast<int64_t>(e) % 16 == 0 &&
               v.out_row * static_cast<int64_t>(e) % 16 == 0 && v.out_head * static_cast<int64_t>(e) % 16 == 0;
        a.in[a.n] = v.in; a.out[a.n] = v.out;
        a.first[a.n] = a.heads;
        a.in_row[a.n] = v.in_row; a.in_head[a.n] = v.in_head; a.out_row[a.n] = v.out_row; a.out_head[a.n] = v.out_head;
        if (v.heads > 65535 - a.heads) return dodo_fail(ctx, DODO_ERR_UNSUPPORTED, "more than 65,535 heads");
        a.heads += v.heads;
        ++a.n;
    }
    if (a.heads == 0) return DODO_OK;
    for (int i = 0; i < n; ++i)
        if (lie_over_one_another(row_off[B], arrays[i].heads, arrays[i].out_row, arrays[i].out_head, dh))
            return dodo_fail(ctx, DODO_ERR_INVALID_ARG, "array %d: rows and heads of the output lie over one another", i);
    if ((rc = dodo_check_device(ctx)) != DODO_OK) return rc;
    const Rotation p = dodo_rotation(rope, back);
    const bool inter = rope->layout == DODO_ROPE_INTERLEAVED;
    for (int b0 = 0; b0 < B; b0 += DODO_GROUP) {
        RopeRows g;
        g.nseq = B - b0 < DODO_GROUP ? B - b0 : DODO_GROUP;
        for (int i = 0; i < g.nseq; ++i) { g.row0[i] = row_off[b0 + i]; g.pos0[i] = pos0[b0 + i]; }
        g.row0[g.nseq] = row_off[b0 + g.nseq];
        if (g.row0[g.nseq] == g.row0[0]) continue;
        ctx->cache_clean = false;        // an output may be a nugget cache
        cudaError_t err;
        if (dtype == DODO_F32)
            err = wide ? (inter ? launch<float, 4, true>(ctx, a, p, g, dh, st) : launch<float, 4, false>(ctx, a, p, g, dh, st))
                       : (inter ? launch<float, 2, true>(ctx, a, p, g, dh, st) : launch<float, 1, false>(ctx, a, p, g, dh, st));
        else
            err = wide ? (inter ? launch<__nv_bfloat16, 8, true>(ctx, a, p, g, dh, st) : launch<__nv_bfloat16, 8, false>(ctx, a, p, g, dh, st))
                       : (inter ? launch<__nv_bfloat16, 2, true>(ctx, a, p, g, dh, st) : launch<__nv_bfloat16, 1, false>(ctx, a, p, g, dh, st));
        if (err != cudaSuccess) return dodo_check_cuda(ctx, err, "rope launch");
    }
    return DODO_OK;
}

}  // namespace

int dodo_check_rope(dodo_ctx* ctx, const dodo_rope_spec* rope, int dh) {
    if (rope == nullptr || rope->ready != 1u) return dodo_fail(ctx, DODO_ERR_INVALID_ARG, "the rotation has not been made by dodo_rope_init");
    if (dh < 2 || dh > 512 || dh % 2 != 0) return dodo_fail(ctx, DODO_ERR_UNSUPPORTED, "head size %d (supported: even, 2 to 512)", dh);
    if (rope->rot > dh) return dodo_fail(ctx, DODO_ERR_INVALID_ARG, "%d features to rotate, the head has %d", rope->rot, dh);
    return DODO_OK;
}

dodo_rotary::Rotation dodo_rotation(const dodo_rope_spec* rope, bool back) {
    Rotation p;
    p.half = rope->rot / 2;
    p.scale = rope->scale;
    p.sign = back ? -1.f : 1.f;
    memcpy(p.turn, rope->turn, sizeof p.turn);
    return p;
}

extern "C" {

int dodo_rope_frequencies(int rot, double base, int scaling, double factor, int trained, double low, double high, double* freq) {
    if (rot < 2 || rot > DODO_ROPE_MAX || rot % 2 != 0 || freq == nullptr || !(base > 0.0) || !isfinite(base)) return DODO_ERR_INVALID_ARG;
    if (scaling < DODO_ROPE_PLAIN || scaling > DODO_ROPE_PARTS) return DODO_ERR_INVALID_ARG;
    if (scaling != DODO_ROPE_PLAIN && (!(factor > 0.0) || !isfinite(factor))) return DODO_ERR_INVALID_ARG;
    if (scaling == DODO_ROPE_PARTS && (trained <= 0 || !isfinite(low) || !isfinite(high) || !(low < high))) return DODO_ERR_INVALID_ARG;
    if (scaling == DODO_ROPE_BASE && rot > 2) base *= pow(factor, static_cast<double>(rot) / (rot - 2));
    for (int i = 0; i < rot / 2; ++i) {
        double f = pow(base, -2.0 * i / rot);
        if (scaling == DODO_ROPE_LINEAR) f /= factor;
        if (scaling == DODO_ROPE_PARTS) {
            double keep = (trained * f / 6.283185307179586477 - low) / (high - low);
            keep = keep < 0.0 ? 0.0 : keep > 1.0 ? 1.0 : keep;
            f *= keep + (1.0 - keep) / factor;
        }
        freq[i] = f;
    }
    return DODO_OK;
}

int dodo_rope_init(dodo_rope_spec* rope, int rot, int layout, float scale, const double* freq) {
    if (rope == nullptr) return DODO_ERR_INVALID_ARG;
    memset(rope, 0, sizeof *rope);
    if (rot < 2 || rot > DODO_ROPE_MAX || rot % 2 != 0 || freq == nullptr || !isfinite(scale)) return DODO_ERR_INVALID_ARG;
    if (layout != DODO_ROPE_HALF && layout != DODO_ROPE_INTERLEAVED) return DODO_ERR_INVALID_ARG;
    for (int i = 0; i < rot / 2; ++i) {
        if (!isfinite(freq[i])) return DODO_ERR_INVALID_ARG;
        // 64 bits of the fraction of a turn: long double has as many
        long double t = static_cast<long double>(freq[i]) * 0.159154943091895335768883763372514362L;
        t -= floorl(t);
        const long double v = t * 18446744073709551616.0L;
        rope->turn[i] = v >= 18446744073709551615.0L ? 0ull : static_cast<uint64_t>(v + 0.5L);
    }
    rope->rot = rot;
    rope->layout = layout;
    rope->scale = scale;
    rope->ready = 1u;
    return DODO_OK;
}

int dodo_rope(dodo_ctx* ctx, const dodo_rope_spec* rope, const dodo_rope_array* arrays, int n, int dtype, int dh, const int32_t* row_off,
              const int32_t* pos0, int B, void* stream) {
    return rope_impl(ctx, rope, arrays, n, dtype, dh, row_off, pos0, B, false, static_cast<cudaStream_t>(stream));
}

int dodo_rope_backward(dodo_ctx* ctx, const dodo_rope_spec* rope, const dodo_rope_array* arrays, int n, int dtype, int dh,
                       const int32_t* row_off, const int32_t* pos0, int B, void* stream) {
    return rope_impl(ctx, rope, arrays, n, dtype, dh, row_off, pos0, B, true, static_cast<cudaStream_t>(stream));
}

}  // extern "C"
