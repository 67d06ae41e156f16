// Attention of query tokens over [4-bit nugget cache ; local tokens] (Eq. 4, Eq. 9, Eq. 13): the streaming kernel of
// attend.cu for a cache in the format of cache_q4.cu.  Softmax, masking, split over key chunks and log-sum-exp are as
// there; the values are those the codes stand for, m + c s, never materialised:
//   q . k   = sum over groups of  s (sum_i q_i c_i) + m (sum_i q_i)
//   sum_j p_j v_j = sum_j (p_j s_j) c_j + (sum_j p_j m_j)   per feature, the second sum once per group
// so that a group costs one extra multiply-add per key on either side.
//
// A cached key is 160 bytes a head (dh 128) where bf16 has 512, so the bound moves towards instruction issue: what counts
// is instructions per code.  Three kernels:
//   attend_q4_kernel        fp32, and single bf16 queries at head size 64: fp32 FMAs, exact codes as floats.  (For those attend_q4_few_kernel
//                           takes 6.5 against 5.3 us over 8 x 205 cached and 64 local keys of 32 heads, 28.9 against 27.8 over a ragged
//                           batch of 52 to 3277 rows, and 25.4 against 29.4 over 16,384 rows of 40 heads: the kernel for the usual lists.)
//   attend_q4_token_kernel  single bf16 queries at head size 128: the codes go to the matrix units as they are
//   attend_q4_few_kernel    bf16, tiles of eight queries: likewise
//
// attend_q4_kernel: a lane owns a run of 16 features of a head (half a group: 8 bytes of codes, one word each of K and V
// steps); eight lanes share a key of 128.  A code is turned into a float in place, without a shift: masking nibble i of a
// word and or-ing in the exponent of 2^23 gives 2^23 + c 16^i exactly, one packed subtraction per two codes takes the 2^23
// off, and the weight 16^i is folded into the query feature (for K) and divided out of the accumulator at the end (for V),
// both powers of two and exact.  That is 2.1 instructions per code and product, and instruction issue bounds it: one bf16 query
// over 8 x 205 cached and 64 local keys of 32 heads of 64 takes 5.2 us, one of fp32 of 128 8.3 (four queries 19.5).
#include "dodo_internal.cuh"
#include "sm100_ptx.cuh"
#include <type_traits>

namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kHintKeys = 32;         // local rows requested into L2 ahead of the dependency wait
constexpr float kNeg = -1.0e30f;      // finite stand-in for -inf in running maxima

__device__ __forceinline__ float ex2_approx(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ void store_out(float* p, float v) { *p = v; }
__device__ __forceinline__ void store_out(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }

// power of 16 that nibble i of a word carries after extraction (the word is shifted once, by 12, for nibbles 5 to 7)
__device__ __forceinline__ constexpr int nibble_at(int i) { return i < 5 ? i : i - 3; }
__device__ __forceinline__ constexpr float nibble_scale(int i) { return static_cast<float>(1 << (4 * nibble_at(i))); }

// eight codes of a word as c 16^nibble_at(i)
__device__ __forceinline__ void codes_of(uint32_t w, float2* c) {
    const uint32_t hi = w >> 12;
    const float2 base = make_float2(-8388608.f, -8388608.f);
    float f[8];
#pragma unroll
    for (int i = 0; i < 8; ++i)
        f[i] = __uint_as_float(((i < 5 ? w : hi) & (15u << (4 * nibble_at(i)))) | 0x4B000000u);
#pragma unroll
    for (int i = 0; i < 4; ++i) c[i] = __fadd2_rn(make_float2(f[2 * i], f[2 * i + 1]), base);
}

struct Codes { uint32_t w[2]; };
__device__ __forceinline__ Codes load_codes(const uint32_t* p) {
    Codes c;
    asm volatile("ld.global.nc.L1::no_allocate.v2.u32 {%0,%1}, [%2];" : "=r"(c.w[0]), "=r"(c.w[1]) : "l"(p));
    return c;
}

template <typename T, int DH>
__device__ __forceinline__ void write_out(T* O, float* lse, size_t orow, int dim, float M, float L, float o) {
    store_out(O + orow * DH + dim, L != 0.f ? o / L : 0.f);   // (a NaN sum stays one)
    if (lse != nullptr && dim == 0) lse[orow] = L != 0.f ? (M + log2f(L)) * 0.6931471805599453f : -INFINITY;
}

// The last chunk of a (query tile, head) to arrive merges the partials of all of them by log-sum-exp; nobody waits.
template <typename T, int DH>
__device__ __forceinline__ void merge_chunks(const AttendSeq& sq, int H, int qtile, int h, int q_first, int nq,
                                             int nchunk, const float* partials, int* tickets, int* flag, T* O, float* lse) {
    constexpr int RED = DH + 2;
    __threadfence();
    __syncthreads();
    if (threadIdx.x == 0) {
        int* tk = tickets + sq.tick0 + qtile * H + h;
        const int t = atomicAdd(tk, 1);
        *flag = t == nchunk - 1;
        if (t == nchunk - 1) *tk = 0;  // leave the counter clean for the next launch
    }
    __syncthreads();
    if (*flag == 0) return;
    __threadfence();
    for (int i = threadIdx.x; i < nq * DH; i += blockDim.x) {
        const int q2 = i / DH, dim = i % DH;
        const float* pr = partials + (static_cast<size_t>(sq.part0) + (static_cast<size_t>(q_first + q2) * H + h) * nchunk) * RED;
        float M = kNeg, L = 0.f, o = 0.f;
        for (int c0 = 0; c0 < nchunk; c0 += 8) {   // eight chunks' loads in flight together
            float mv[8], lv[8], ov[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const bool live = c0 + u < nchunk;
                const float* pc = pr + static_cast<size_t>(live ? c0 + u : 0) * RED;
                mv[u] = live ? __ldcg(pc + DH) : kNeg;
                lv[u] = live ? __ldcg(pc + DH + 1) : 0.f;
                ov[u] = live ? __ldcg(pc + dim) : 0.f;
            }
            float M_new = M;
#pragma unroll
            for (int u = 0; u < 8; ++u) M_new = fmaxf(M_new, mv[u]);
            const float corr = ex2_approx(M - M_new);
            M = M_new;
            L *= corr;
            o *= corr;
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const float wgt = ex2_approx(mv[u] - M);
                L = fmaf(lv[u], wgt, L);
                o = fmaf(ov[u], wgt, o);
            }
        }
        write_out<T, DH>(O, lse, static_cast<size_t>(sq.q_row0 + q_first + q2) * H + h, dim, M, L, o);
    }
}

struct Q4Source {
    const uint32_t* q4;       // codes, dh / 4 words per (row, head): K's then V's
    const uint32_t* scale;    // 2 dh / 32 words per (row, head): K's then V's
    const void *lK, *lV;
};

// U keys per lane bundle and batch: 4 for one query, 2 for tiles of queries, whose accumulators take the registers
template <typename T, int DH, int QT, int U>
__global__ void __launch_bounds__(kThreads, QT == 1 ? 2 : 1)
attend_q4_kernel(const T* __restrict__ Q, const Q4Source src, const __grid_constant__ AttendGroup g,
                 const int32_t* __restrict__ cache_pos, int H, float scale_log2, int TK, T* __restrict__ O,
                 float* __restrict__ lse, float* __restrict__ partials, int* __restrict__ tickets, int early_cache) {
    constexpr int FPL = 16, LPR = DH / FPL, BPW = 32 / LPR, NB = kWarps * BPW;   // lanes per key, bundles per warp and per block
    constexpr int W = FPL / 8;                                         // words of codes per lane and row
    constexpr int RED = DH + 2;
    constexpr int kLocVec = FPL * static_cast<int>(sizeof(T)) / 16;    // 16-byte loads of a local row per lane
    constexpr int E = Vec16<T>::kElems;

    __shared__ float red[kWarps][QT][RED];
    __shared__ int s_flag;

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int bundle = tid / LPR, lig = tid % LPR;
    const int bid = static_cast<int>(blockIdx.x);
    int b;
    if (g.uniform_ctas > 0) {
        b = bid / g.uniform_ctas;
    } else {
        b = 0;
#pragma unroll 8
        for (int i = 1; i < DODO_GROUP; ++i) b += (i < g.nseq && g.cta0[i] <= bid) ? 1 : 0;
    }
    const AttendSeq sq = g.seq[b];
    int r0 = bid - g.cta0[b];
    const int nchunk = sq.nchunk;
    const int chunk = r0 % nchunk; r0 /= nchunk;
    const int h = r0 % H;
    const int qtile = r0 / H;
    const int q_first = qtile * QT;
    const int nq = min(QT, sq.tq - q_first);
    const int l_vis = dodo_visible_local(sq.l_len, sq.l_pos0, sq.q_pos0 + q_first + nq - 1);
    // this chunk's slice of the key list [nuggets ; local], in granules of TK keys per segment
    const int nt_c = (sq.c_len + TK - 1) / TK;
    const int t_begin = chunk * sq.ctiles, t_end = t_begin + sq.ctiles;
    const int c_begin = min(sq.c_len, t_begin * TK), c_end = min(sq.c_len, t_end * TK);
    const int l_begin = min(l_vis, max(0, t_begin - nt_c) * TK), l_end = min(l_vis, max(0, t_end - nt_c) * TK);
    const int n_c = c_end - c_begin, n_l = l_end - l_begin;
    const int c_row = sq.c_row0 + c_begin, l_row = sq.l_row0 + l_begin, l_pos = sq.l_pos0 + l_begin;

    // ---- cached keys: batches of NB * U, the next one's loads in flight while one is reduced ----------------
    const uint32_t* const q4_0 = src.q4 + (static_cast<size_t>(c_row) * H + h) * (DH / 4) + lig * W;
    const uint32_t* const sc_0 = src.scale + (static_cast<size_t>(c_row) * H + h) * (2 * DH / DODO_Q4_GROUP) + lig * FPL / DODO_Q4_GROUP;
    struct Batch { Codes k[U], v[U]; uint32_t ks[U], vs[U]; int pos[U]; };
    auto load_batch = [&](int base, Batch& t) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int j = base + u * NB + bundle;
            t.pos[u] = 0x7fffffff;
            t.ks[u] = t.vs[u] = 0u;
#pragma unroll
            for (int i = 0; i < W; ++i) t.k[u].w[i] = t.v[u].w[i] = 0u;
            if (j < n_c) {
                const size_t at = static_cast<size_t>(j) * H;
                t.k[u] = load_codes(q4_0 + at * (DH / 4));
                t.v[u] = load_codes(q4_0 + at * (DH / 4) + DH / 8);
                t.ks[u] = __ldg(sc_0 + at * (2 * DH / DODO_Q4_GROUP));
                t.vs[u] = __ldg(sc_0 + at * (2 * DH / DODO_Q4_GROUP) + DH / DODO_Q4_GROUP);
                t.pos[u] = __ldg(cache_pos + c_row + j);
            }
        }
    };
    // Ahead of the dependency wait (see attend.cu): cache rows are loaded when nothing in flight writes a cache; hints to
    // L2 for the query rows and the first local rows always.
    auto hint_rows = [&](const T* base, int row, int rows) {
        constexpr int kLines = DH * static_cast<int>(sizeof(T)) / 128;
        for (int i = tid; i < rows * kLines; i += kThreads) {
            const char* line = reinterpret_cast<const char*>(base + (static_cast<size_t>(row + i / kLines) * H + h) * DH) + (i % kLines) * 128;
            asm volatile("prefetch.global.L2 [%0];" :: "l"(line));
        }
    };
    hint_rows(Q, sq.q_row0 + q_first, nq);
    hint_rows(static_cast<const T*>(src.lK), l_row, min(n_l, kHintKeys));
    hint_rows(static_cast<const T*>(src.lV), l_row, min(n_l, kHintKeys));
    Batch A, B;
    if (early_cache) {
        load_batch(0, A);
        load_batch(NB * U, B);
    }
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (!early_cache) {
        load_batch(0, A);
        load_batch(NB * U, B);
    }

    // ---- the queries, in base 2, each feature divided by the power of 16 its codes carry ------------------------
    float2 qf[QT][FPL / 2], acc[QT][FPL / 2];
    float qsum[QT], accm[QT], m[QT], l[QT];
    int qpos[QT];
#pragma unroll
    for (int qi = 0; qi < QT; ++qi) {
        qpos[qi] = static_cast<int>(0x80000000);   // a dead slot sees nothing
        float f[FPL];
#pragma unroll
        for (int i = 0; i < FPL; ++i) f[i] = 0.f;
        if (qi < nq) {
            const T* row = Q + (static_cast<size_t>(sq.q_row0 + q_first + qi) * H + h) * DH + lig * FPL;
#pragma unroll
            for (int i = 0; i < kLocVec; ++i) Vec16<T>::unpack(*reinterpret_cast<const uint4*>(row + i * E), f + i * E);
            qpos[qi] = sq.q_pos0 + q_first + qi;
        }
        qsum[qi] = 0.f;
#pragma unroll
        for (int i = 0; i < FPL; ++i) {
            f[i] *= scale_log2;
            qsum[qi] += f[i];
            f[i] *= 1.f / nibble_scale(i % 8);
        }
        m[qi] = kNeg; l[qi] = 0.f; accm[qi] = 0.f;
#pragma unroll
        for (int i = 0; i < FPL / 2; ++i) {
            qf[qi][i] = make_float2(f[2 * i], f[2 * i + 1]);
            acc[qi][i] = make_float2(0.f, 0.f);
        }
    }

    // running maximum, sum and weights of N keys whose logits are in s; a masked key's weight is exactly 0
    auto weigh = [&](auto count, int qi, float* s, const int* pos, bool fast) {
        constexpr int N = decltype(count)::value;
        float m_new = m[qi];
#pragma unroll
        for (int u = 0; u < N; ++u) {
            if (!fast) s[u] = pos[u] <= qpos[qi] ? s[u] : kNeg;
            m_new = fmaxf(m_new, s[u]);
        }
        const float corr = ex2_approx(m[qi] - m_new);
        m[qi] = m_new;
        l[qi] *= corr;
        accm[qi] *= corr;
        const float2 c2 = make_float2(corr, corr);
#pragma unroll
        for (int i = 0; i < FPL / 2; ++i) acc[qi][i] = __fmul2_rn(acc[qi][i], c2);
#pragma unroll
        for (int u = 0; u < N; ++u) {
            const float p = ex2_approx(s[u] - m_new);
            s[u] = fast || pos[u] <= qpos[qi] ? p : 0.f;
            l[qi] += s[u];
        }
    };
    auto all_visible = [&](auto count, int qi, const int* pos) {
        bool v = true;
#pragma unroll
        for (int u = 0; u < decltype(count)::value; ++u) v = v && pos[u] <= qpos[qi];
        return __all_sync(0xffffffffu, v) != 0;
    };

    auto reduce = [&](const Batch& t) {
        using N = std::integral_constant<int, U>;
        float s[QT][U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float2 d[QT];
#pragma unroll
            for (int qi = 0; qi < QT; ++qi) d[qi] = make_float2(0.f, 0.f);
#pragma unroll
            for (int w = 0; w < W; ++w) {
                float2 c[4];
                codes_of(t.k[u].w[w], c);
#pragma unroll
                for (int qi = 0; qi < QT; ++qi)
#pragma unroll
                    for (int i = 0; i < 4; ++i) d[qi] = __ffma2_rn(qf[qi][w * 4 + i], c[i], d[qi]);
            }
            const float step = __uint_as_float(t.ks[u] << 16), low = __uint_as_float(t.ks[u] & 0xffff0000u);
#pragma unroll
            for (int qi = 0; qi < QT; ++qi) s[qi][u] = fmaf(step, d[qi].x + d[qi].y, low * qsum[qi]);
        }
#pragma unroll
        for (int o = LPR / 2; o > 0; o >>= 1)
#pragma unroll
            for (int qi = 0; qi < QT; ++qi)
#pragma unroll
                for (int u = 0; u < U; ++u) s[qi][u] += __shfl_xor_sync(0xffffffffu, s[qi][u], o);
        bool fast[QT];
#pragma unroll
        for (int qi = 0; qi < QT; ++qi) {
            fast[qi] = all_visible(N(), qi, t.pos);
            weigh(N(), qi, s[qi], t.pos, fast[qi]);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const float step = __uint_as_float(t.vs[u] << 16), low = __uint_as_float(t.vs[u] & 0xffff0000u);
            float2 ps[QT];
#pragma unroll
            for (int qi = 0; qi < QT; ++qi) {
                // (a masked key's group words may hold anything, NaN included)
                const bool see = fast[qi] || t.pos[u] <= qpos[qi];
                const float p = see ? s[qi][u] * step : 0.f;
                accm[qi] = see ? fmaf(s[qi][u], low, accm[qi]) : accm[qi];
                ps[qi] = make_float2(p, p);
            }
#pragma unroll
            for (int w = 0; w < W; ++w) {
                float2 c[4];
                codes_of(t.v[u].w[w], c);
#pragma unroll
                for (int qi = 0; qi < QT; ++qi)
#pragma unroll
                    for (int i = 0; i < 4; ++i) acc[qi][w * 4 + i] = __ffma2_rn(ps[qi], c[i], acc[qi][w * 4 + i]);
            }
        }
    };
    for (int base = 0; base < n_c; base += 2 * NB * U) {
        reduce(A);
        load_batch(base + 2 * NB * U, A);
        if (base + NB * U < n_c) reduce(B);
        load_batch(base + 3 * NB * U, B);
    }

    // ---- from the codes' scale to that of plain values ------------------------------------------------------------
#pragma unroll
    for (int qi = 0; qi < QT; ++qi) {
#pragma unroll
        for (int i = 0; i < FPL / 2; ++i) {
            const float a = nibble_scale((2 * i) % 8), c = nibble_scale((2 * i + 1) % 8);
            qf[qi][i].x *= a; qf[qi][i].y *= c;
            acc[qi][i].x = fmaf(acc[qi][i].x, 1.f / a, accm[qi]);
            acc[qi][i].y = fmaf(acc[qi][i].y, 1.f / c, accm[qi]);
        }
        accm[qi] = 0.f;
    }

    // ---- local keys, one per bundle and step, uncompressed -----------------------------------------------------------
    for (int base = 0; base < n_l; base += NB) {
        const int j = base + bundle;
        uint4 kv[kLocVec], vv[kLocVec];
        int pos = 0x7fffffff;
#pragma unroll
        for (int i = 0; i < kLocVec; ++i) kv[i] = vv[i] = make_uint4(0, 0, 0, 0);
        if (j < n_l) {
            const size_t at = (static_cast<size_t>(l_row + j) * H + h) * DH + lig * FPL;
#pragma unroll
            for (int i = 0; i < kLocVec; ++i) kv[i] = __ldg(reinterpret_cast<const uint4*>(static_cast<const T*>(src.lK) + at) + i);
#pragma unroll
            for (int i = 0; i < kLocVec; ++i) vv[i] = __ldg(reinterpret_cast<const uint4*>(static_cast<const T*>(src.lV) + at) + i);
            pos = l_pos + j;
        }
        using One = std::integral_constant<int, 1>;
        float s[QT][1];
        float2 d[QT];
#pragma unroll
        for (int qi = 0; qi < QT; ++qi) d[qi] = make_float2(0.f, 0.f);
#pragma unroll
        for (int i = 0; i < kLocVec; ++i) {
            float f[E];
            Vec16<T>::unpack(kv[i], f);
#pragma unroll
            for (int qi = 0; qi < QT; ++qi)
#pragma unroll
                for (int e = 0; e < E; e += 2)
                    d[qi] = __ffma2_rn(qf[qi][(i * E + e) / 2], make_float2(f[e], f[e + 1]), d[qi]);
        }
#pragma unroll
        for (int qi = 0; qi < QT; ++qi) s[qi][0] = d[qi].x + d[qi].y;
#pragma unroll
        for (int o = LPR / 2; o > 0; o >>= 1)
#pragma unroll
            for (int qi = 0; qi < QT; ++qi) s[qi][0] += __shfl_xor_sync(0xffffffffu, s[qi][0], o);
        bool fast[QT];
#pragma unroll
        for (int qi = 0; qi < QT; ++qi) {
            fast[qi] = all_visible(One(), qi, &pos);
            weigh(One(), qi, s[qi], &pos, fast[qi]);
        }
#pragma unroll
        for (int i = 0; i < kLocVec; ++i) {
            float f[E];
            Vec16<T>::unpack(vv[i], f);
#pragma unroll
            for (int qi = 0; qi < QT; ++qi) {
                const float2 p = make_float2(s[qi][0], s[qi][0]);
                if (fast[qi] || pos <= qpos[qi]) {   // (a masked key's row may hold anything)
#pragma unroll
                    for (int e = 0; e < E; e += 2)
                        acc[qi][(i * E + e) / 2] = __ffma2_rn(p, make_float2(f[e], f[e + 1]), acc[qi][(i * E + e) / 2]);
                }
            }
        }
    }

    // ---- merge: the bundles of a warp by halving exchanges, then the warps through shared memory -----------------------
#pragma unroll
    for (int qi = 0; qi < QT; ++qi) {
        float M = m[qi];
#pragma unroll
        for (int o = LPR; o < 32; o <<= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, o));
        const float f = ex2_approx(m[qi] - M);
        float L = l[qi] * f;
#pragma unroll
        for (int o = LPR; o < 32; o <<= 1) L += __shfl_xor_sync(0xffffffffu, L, o);
        float v[FPL];
#pragma unroll
        for (int i = 0; i < FPL / 2; ++i) { v[2 * i] = acc[qi][i].x * f; v[2 * i + 1] = acc[qi][i].y * f; }
        // at each step a lane gives away one half of its features and keeps the sums of the other
        int first = 0;
#pragma unroll
        for (int o = LPR, n = FPL; o < 32; o <<= 1, n >>= 1) {
            const bool upper = (lane & o) != 0;
#pragma unroll
            for (int i = 0; i < n / 2; ++i) {
                const float give = upper ? v[i] : v[n / 2 + i], keep = upper ? v[n / 2 + i] : v[i];
                v[i] = keep + __shfl_xor_sync(0xffffffffu, give, o);
            }
            if (upper) first += n / 2;
        }
        constexpr int kLeft = FPL / BPW;   // features left per lane
#pragma unroll
        for (int i = 0; i < kLeft; ++i) red[warp][qi][lig * FPL + first + i] = v[i];
        if (lane == 0) { red[warp][qi][DH] = M; red[warp][qi][DH + 1] = L; }
    }
    __syncthreads();

    const int qrow0 = sq.q_row0 + q_first;
    for (int i = tid; i < QT * DH; i += kThreads) {
        const int q2 = i / DH, dim = i % DH;
        if (q2 >= nq) continue;
        float M = kNeg;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) M = fmaxf(M, red[w][q2][DH]);
        float L = 0.f, o = 0.f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            const float wgt = ex2_approx(red[w][q2][DH] - M);
            L = fmaf(red[w][q2][DH + 1], wgt, L);
            o = fmaf(red[w][q2][dim], wgt, o);
        }
        if (nchunk == 1) {
            write_out<T, DH>(O, lse, static_cast<size_t>(qrow0 + q2) * H + h, dim, M, L, o);
        } else {
            float* pr = partials + (static_cast<size_t>(sq.part0) + (static_cast<size_t>(q_first + q2) * H + h) * nchunk + chunk) * RED;
            pr[dim] = o;
            if (dim == 0) { pr[DH] = M; pr[DH + 1] = L; }
        }
    }
    if (nchunk == 1) return;

    merge_chunks<T, DH>(sq, H, qtile, h, q_first, nq, nchunk, partials, tickets, &s_flag, O, lse);
}

// ---- one bf16 query per sequence, head size 128 --------------------------------------------------------------------------
// The kernel above spends 40 warp instructions per cached key and head, most of them on turning codes into floats and
// multiplying them one by one.  Here the warp-level matrix instruction takes the codes nearly as they lie in memory: a pair of
// nibbles masked out of a word, read as two bf16 numbers, is c 2^-133 (low nibble of a byte) or 16 c 2^-133 (high nibble) exactly,
// since bf16 bit patterns below 256 are the multiples of 2^-133; so five instructions (four masks, one shift) make eight codes
// into operands.  Scale: the other operand carries a power of two, the products stay in the normal range of fp32.
//   Q.K   A = 16 keys x 16 features of codes, B = the query in up to four columns, column n holding only the features of group n
//         (lane quad t owns group t's features, so a column's lanes are zero elsewhere): one accumulator gathers the four groups'
//         sums of q c apart, exact products summed in fp32; steps and minima enter afterwards.
//   P.V   A = 16 features x 16 keys (words of two keys interleaved by byte permutation), B = p s per key: column n holds group
//         n & 3, its bf16 value for n < 4 and what that rounding left for n >= 4, so that p s keeps 16 bits.  Of the accumulators a
//         row's own group is used, the rest is ignored.
// That is about 14 instructions and one matrix instruction (8.4 cycles of a scheduler's pipe, measured) per key and head.
// Rows come through shared memory: a fifth warp brings 64 keys at a time (their codes and group words of this head, 10 KB) with two
// tensor copies into a ring of four stages, so that 120 KB per SM are on their way whatever the consumers do; loads into
// registers a tile or two ahead left HBM at 2.5 TB/s.  Four consumers and three blocks per SM: with more warps a block two blocks
// fit, registers are rounded down to 96 (five warps on one scheduler) and a ragged batch balances worse (16 sequences, 52 to 3277
// rows: 25.4 against 28.4 us).  What bounds it is instruction issue next to HBM: the same kernel without the arithmetic takes 20 us
// for 16,384 rows of 40 heads (5.4 TB/s) where this takes 25.
constexpr int kQExp = 64;        // the query is shifted to a largest feature near 2^64
constexpr int kMostExp = 57;     // ... where that feature is below 2^58: what undoes the shift, 2^(133 - 64 + 57), is near the largest power there is
constexpr int kPExp = 72;        // power of two on p s, p below 2^8: fits for steps below 2^47, products are normal numbers down to p s of 2^-65

__device__ __forceinline__ void mma16816(float* c, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t two_bf16(float lo, float hi) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
}

// exponent of a number, and a power of two put together bit by bit (both for normal numbers)
__device__ __forceinline__ int exponent_of(float x) { return static_cast<int>((__float_as_uint(x) >> 23) & 255u) - 127; }
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float(static_cast<uint32_t>(e + 127) << 23); }

__device__ __forceinline__ uint32_t lds32(uint32_t a) { uint32_t v; asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(a)); return v; }
__device__ __forceinline__ uint2 lds64(uint32_t a) { uint2 v; asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(a)); return v; }
__device__ __forceinline__ uint4 lds128(uint32_t a) {
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a));
    return v;
}

struct TokenMaps { CUtensorMap q4, scale; };   // boxes of 128 and 32 bytes x kRound rows
constexpr int kTokenWarps = 4;                // consumers; one more warp brings the rows
constexpr int kConsumers = 32 * kTokenWarps, kTokenThreads = kConsumers + 32;
constexpr int kRound = 16 * kTokenWarps;       // keys of a stage: 16 per warp
constexpr int kTokenStages = 4, kTokenBlocks = 3;
// a stage: the codes of its keys' rows (dh bytes each, swizzled), then their group words (dh / 4 bytes)
constexpr int code_bytes(int dh) { return kRound * dh; }
constexpr int stage_bytes(int dh) { return (code_bytes(dh) + kRound * dh / 4 + 1023) / 1024 * 1024; }
constexpr int kCodeBytes = code_bytes(128), kStageBytes = stage_bytes(128);

// The producer's part, one thread: `rounds` stages of rows from c_row on through the ring.  Ahead of the dependency wait (see
// attend.cu) it copies only when nothing in flight writes a cache.  False when a wait ran out.
template <int DH>
__device__ __forceinline__ bool bring_rows(const TokenMaps& maps, uint32_t ring, uint64_t* bar_full, uint64_t* bar_free, int h, int c_row, int rounds,
                                           int early_cache) {
    using namespace sm100;
    bool ok = true;
    auto load_round = [&](int i) {
        const int st = i % kTokenStages;
        const uint32_t dst = ring + st * stage_bytes(DH);
        mbar_expect_tx(&bar_full[st], code_bytes(DH) + kRound * DH / 4);
        tma_load_2d(dst, &maps.q4, h * DH, c_row + i * kRound, &bar_full[st]);
        tma_load_2d(dst + code_bytes(DH), &maps.scale, h * (DH / 4), c_row + i * kRound, &bar_full[st]);
    };
    const int ahead = min(rounds, kTokenStages);
    if (early_cache)
        for (int i = 0; i < ahead; ++i) load_round(i);
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (!early_cache)
        for (int i = 0; i < ahead; ++i) load_round(i);
    int done = ahead;
    for (int i = kTokenStages; i < rounds; ++i) {
        const int st = i % kTokenStages;
        if (!mbar_wait(&bar_free[st], static_cast<uint32_t>(i / kTokenStages - 1) & 1u)) { ok = false; break; }
        load_round(i);
        done = i + 1;
    }
    // leave no copy in flight behind (when consumers have given up)
    for (int i = max(0, done - kTokenStages); i < done; ++i) ok = mbar_wait(&bar_full[i % kTokenStages], static_cast<uint32_t>(i / kTokenStages) & 1u) && ok;
    return ok;
}

__global__ void __launch_bounds__(kTokenThreads, kTokenBlocks)
attend_q4_token_kernel(const __nv_bfloat16* __restrict__ Q, const __grid_constant__ TokenMaps maps, const Q4Source src,
                       const __grid_constant__ AttendGroup g, const int32_t* __restrict__ cache_pos, int H, float scale_log2, int TK,
                       __nv_bfloat16* __restrict__ O, float* __restrict__ lse, float* __restrict__ partials, int* __restrict__ tickets,
                       int early_cache, int* __restrict__ dev_status) {
    using namespace sm100;
    constexpr int DH = 128, RED = DH + 2;
    extern __shared__ unsigned char smem_raw[];
    __shared__ float red[2 * kTokenWarps][RED];                 // a warp's cached keys, its local keys
    __shared__ float up[kTokenWarps];                           // a huge query's power of two
    __shared__ __align__(8) uint64_t bar_full[kTokenStages], bar_free[kTokenStages];
    __shared__ int s_flag;
    const uint32_t ring = (smem_u32(smem_raw) + 1023u) & ~1023u;

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int r = lane >> 2, t = lane & 3;                 // fragment row (key, feature word or column) and quad lane
    const int bid = static_cast<int>(blockIdx.x);
    int b;
    if (g.uniform_ctas > 0) {
        b = bid / g.uniform_ctas;
    } else {
        b = 0;
#pragma unroll 8
        for (int i = 1; i < DODO_GROUP; ++i) b += (i < g.nseq && g.cta0[i] <= bid) ? 1 : 0;
    }
    const AttendSeq sq = g.seq[b];
    const int r0 = bid - g.cta0[b];
    const int nchunk = sq.nchunk, chunk = r0 % nchunk, h = r0 / nchunk;    // one query: H units of nchunk blocks
    const int qpos = sq.q_pos0;
    const int l_vis = dodo_visible_local(sq.l_len, sq.l_pos0, qpos);
    const int nt_c = (sq.c_len + TK - 1) / TK;                             // planning tiles of TK keys
    const int t_begin = chunk * sq.ctiles, t_end = t_begin + sq.ctiles;
    const int c_begin = min(sq.c_len, t_begin * TK), c_end = min(sq.c_len, t_end * TK);
    const int l_begin = min(l_vis, max(0, t_begin - nt_c) * TK), l_end = min(l_vis, max(0, t_end - nt_c) * TK);
    const int n_c = c_end - c_begin, n_l = l_end - l_begin;
    const int c_row = sq.c_row0 + c_begin, l_row = sq.l_row0 + l_begin;
    const int rounds = (n_c + kRound - 1) / kRound;

    if (tid == 0) {
        for (int i = 0; i < kTokenStages; ++i) { mbar_init(&bar_full[i], 1); mbar_init(&bar_free[i], kTokenWarps); }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    __syncthreads();
    bool ok = true;
    if (warp == kTokenWarps) {
        if (lane == 0 && !bring_rows<128>(maps, ring, bar_full, bar_free, h, c_row, rounds, early_cache)) atomicOr(dev_status, DODO_DEV_WAIT_TIMEOUT);
    } else {
    auto hint_rows = [&](const __nv_bfloat16* base, int row, int rows) {
        for (int i = tid; i < rows * 2; i += kConsumers)
            asm volatile("prefetch.global.L2 [%0];" :: "l"(reinterpret_cast<const char*>(base + (static_cast<size_t>(row + i / 2) * H + h) * DH) + (i % 2) * 128));
    };
    hint_rows(Q, sq.q_row0, 1);
    hint_rows(static_cast<const __nv_bfloat16*>(src.lK), l_row, min(n_l, kHintKeys));
    hint_rows(static_cast<const __nv_bfloat16*>(src.lV), l_row, min(n_l, kHintKeys));
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

    // a warp's tile of a stage: keys 16 warp + ..., in the swizzled rows of 128 bytes (16-byte piece p of row j lies at p ^ (j & 7))
    const int key0 = 16 * warp;
    const uint32_t k_at = static_cast<uint32_t>((key0 + r) * 128 + ((t ^ r) << 4));             // row r; row r + 8 is 1024 bytes on
    const uint32_t s_at = static_cast<uint32_t>(kCodeBytes + (key0 + r) * 32 + (t & 1) * 8);    // row r + 8: 256 bytes on
    uint32_t v_at[2][2];                                                                        // rows 2 t, 2 t + 1; words r, r + 8
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            const int row = 2 * t + i, piece = 4 + 2 * w + (r >> 2);
            v_at[i][w] = static_cast<uint32_t>((key0 + row) * 128 + ((piece ^ row) << 4) + (r & 3) * 4);
        }
    auto positions = [&](int i, int* pos) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int j = i * kRound + key0 + r + 8 * e;
            pos[e] = j < n_c ? __ldg(cache_pos + c_row + j) : 0x7fffffff;
        }
    };
    // ---- the query as B fragments: lane (n = r, t) holds column n, nonzero where n = t: group t's features -------------------
    const __nv_bfloat16* const qrow = Q + (static_cast<size_t>(sq.q_row0) * H + h) * DH;
    uint32_t qb[4][2][2];
    float qsum[2], q_back;      // sums of q over groups 2 (t & 1) + {0, 1}, lanes t < 2; what undoes the shifts, with the softmax scale
    bool huge;                  // ... but for a query beyond 2^58, which leaves a power of two to its logits
    {
        float f[32], top = 0.f, mine = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) Vec16<__nv_bfloat16>::unpack(*reinterpret_cast<const uint4*>(qrow + 32 * t + 8 * i), f + 8 * i);
#pragma unroll
        for (int i = 0; i < 32; ++i) top = fmaxf(top, fabsf(f[i]));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
        // exponent of the largest feature, as powers of two put together bit by bit; a query below 2^-62 is shifted less, so that both
        // powers stay normal numbers
        int e = max(exponent_of(top), -62);
        huge = e > kMostExp;
        if (huge) {
            const float down = power_of_two(kMostExp - e);
#pragma unroll
            for (int i = 0; i < 32; ++i) f[i] *= down;
            up[warp] = power_of_two(e - kMostExp);     // (all lanes the same)
            e = kMostExp;
        }
#pragma unroll
        for (int i = 0; i < 32; ++i) mine += f[i];
        const float shift = power_of_two(kQExp - e);
        q_back = power_of_two(133 - kQExp + e) * scale_log2;
        const float at0 = __shfl_sync(0xffffffffu, mine, (t & 1) * 2), at1 = __shfl_sync(0xffffffffu, mine, (t & 1) * 2 + 1);
        qsum[0] = t < 2 ? at0 * scale_log2 : 0.f;
        qsum[1] = t < 2 ? at1 * scale_log2 : 0.f;
        const float s1 = r == t ? shift : 0.f, s16 = s1 * 0.0625f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float* w = f + 8 * i;
            qb[i][0][0] = two_bf16(w[0] * s1, w[4] * s1);
            qb[i][0][1] = two_bf16(w[1] * s16, w[5] * s16);
            qb[i][1][0] = two_bf16(w[2] * s1, w[6] * s1);
            qb[i][1][1] = two_bf16(w[3] * s16, w[7] * s16);
        }
    }

    const float kPScale = __uint_as_float(static_cast<uint32_t>(kPExp + 127) << 23);
    const int from = 8 * t + (r < 4 ? 2 : 0) + ((r & 3) >> 1);     // lane that holds the p s of key 2 t for column r
    const uint32_t pick = (r & 1) != 0 ? 0x7632u : 0x5410u;
    float m = kNeg, l = 0.f, accm[2] = {0.f, 0.f};             // the maximum is the warp's; l and accm are a lane's own rows'
    float acc[8][4];
#pragma unroll
    for (int j = 0; j < 8; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[j][e] = 0.f;

    // N stages at once (one tile of 16 keys of each): their chains of shuffles and matrix instructions overlap
    auto reduce = [&](auto count, auto all_seen, const int* stage, const int (*pos)[2]) {
        constexpr int N = decltype(count)::value;
        constexpr bool kAll = decltype(all_seen)::value;           // every key of the tiles is visible: no selects
        uint32_t base[N];
        float s[N][2];
        // ---- logits of keys r and r + 8 ----------------------------------------------------------------------------
#pragma unroll
        for (int n = 0; n < N; ++n) {
            base[n] = ring + stage[n] * kStageBytes;
            const uint4 k0 = lds128(base[n] + k_at), k1 = lds128(base[n] + k_at + 1024u);        // group t's codes
            const uint2 w0 = lds64(base[n] + s_at), w1 = lds64(base[n] + s_at + 256u);           // words of groups 2 (t & 1) + {0, 1}
            const uint32_t ka[4] = {k0.x, k0.y, k0.z, k0.w}, kb[4] = {k1.x, k1.y, k1.z, k1.w};
            float d[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t ha = ka[i] >> 8, hb = kb[i] >> 8;
                mma16816(d, ka[i] & 0x000f000fu, kb[i] & 0x000f000fu, ka[i] & 0x00f000f0u, kb[i] & 0x00f000f0u, qb[i][0][0], qb[i][0][1]);
                mma16816(d, ha & 0x000f000fu, hb & 0x000f000fu, ha & 0x00f000f0u, hb & 0x00f000f0u, qb[i][1][0], qb[i][1][1]);
            }
            const uint2 w[2] = {w0, w1};
#pragma unroll
            for (int i = 0; i < 2; ++i) {      // (lanes t >= 2: columns 4 to 7, all zero)
                const float a0 = fmaf(d[2 * i] * q_back, __uint_as_float(w[i].x << 16), __uint_as_float(w[i].x & 0xffff0000u) * qsum[0]);
                const float a1 = fmaf(d[2 * i + 1] * q_back, __uint_as_float(w[i].y << 16), __uint_as_float(w[i].y & 0xffff0000u) * qsum[1]);
                s[n][i] = a0 + a1;
            }
        }
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int i = 0; i < 2; ++i) s[n][i] += __shfl_xor_sync(0xffffffffu, s[n][i], 1);
        float top = kNeg;
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                s[n][i] = __shfl_sync(0xffffffffu, s[n][i], lane & ~3);
                if (huge) s[n][i] *= up[warp];
                if (!kAll) s[n][i] = pos[n][i] <= qpos ? s[n][i] : kNeg;
                top = fmaxf(top, s[n][i]);
            }
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        if (top > m + 8.f) {     // the reference moves only when it pays: weights stay below 2^8
            const float corr = ex2_approx(m - top);
            m = top;
            l *= corr;
            accm[0] *= corr; accm[1] *= corr;
#pragma unroll
            for (int j = 0; j < 8; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[j][e] *= corr;
        }
        // ---- weights; p s of this lane's keys and V groups, rounded to bf16 (lanes t >= 2) or what rounding left (t < 2) ---------
        uint32_t pw[N][2];
#pragma unroll
        for (int n = 0; n < N; ++n)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const uint2 w = lds64(base[n] + s_at + 16u + 256u * i);
                const bool see = kAll || pos[n][i] <= qpos;         // a masked key takes no part, whatever its words hold
                const float p = see ? ex2_approx(s[n][i] - m) : 0.f;
                l += p;
                const float pp = p * kPScale, lo0 = __uint_as_float(w.x & 0xffff0000u), lo1 = __uint_as_float(w.y & 0xffff0000u);
                float a0 = pp * __uint_as_float(w.x << 16), a1 = pp * __uint_as_float(w.y << 16);
                if (!kAll) { a0 = see ? a0 : 0.f; a1 = see ? a1 : 0.f; }
                accm[0] = see ? fmaf(p, lo0, accm[0]) : accm[0];
                accm[1] = see ? fmaf(p, lo1, accm[1]) : accm[1];
                const uint32_t u = two_bf16(a0, a1);
                a0 -= __uint_as_float(u << 16);
                a1 -= __uint_as_float(u & 0xffff0000u);
                pw[n][i] = t < 2 ? two_bf16(a0, a1) : u;
            }
#pragma unroll
        for (int n = 0; n < N; ++n) {
            // B fragments: column r is group r & 3, rounded part for r < 4; keys 2 t, 2 t + 1 and 2 t + 8, 2 t + 9
            const uint32_t b0 = __byte_perm(__shfl_sync(0xffffffffu, pw[n][0], from), __shfl_sync(0xffffffffu, pw[n][0], from + 4), pick);
            const uint32_t b1 = __byte_perm(__shfl_sync(0xffffffffu, pw[n][1], from), __shfl_sync(0xffffffffu, pw[n][1], from + 4), pick);
            uint32_t v[8];
#pragma unroll
            for (int i = 0; i < 4; ++i) {       // keys 2 t, 2 t + 1, 2 t + 8, 2 t + 9: words r and r + 8 of V's codes
                v[2 * i] = lds32(base[n] + v_at[i & 1][0] + 1024u * (i >> 1));
                v[2 * i + 1] = lds32(base[n] + v_at[i & 1][1] + 1024u * (i >> 1));
            }
            // ---- P V: nibble j of words r (rows r) and r + 8 (rows r + 8), keys interleaved -----------------------------------------
#pragma unroll
            for (int hf = 0; hf < 2; ++hf) {
                const uint32_t sel = hf == 0 ? 0x5410u : 0x7632u;
                const uint32_t wa = __byte_perm(v[0], v[2], sel), wb = __byte_perm(v[1], v[3], sel);
                const uint32_t wc = __byte_perm(v[4], v[6], sel), wd = __byte_perm(v[5], v[7], sel);
                mma16816(acc[4 * hf], wa & 0x000f000fu, wb & 0x000f000fu, wc & 0x000f000fu, wd & 0x000f000fu, b0, b1);
                mma16816(acc[4 * hf + 1], wa & 0x00f000f0u, wb & 0x00f000f0u, wc & 0x00f000f0u, wd & 0x00f000f0u, b0, b1);
                const uint32_t ha = wa >> 8, hb = wb >> 8, hc = wc >> 8, hd = wd >> 8;
                mma16816(acc[4 * hf + 2], ha & 0x000f000fu, hb & 0x000f000fu, hc & 0x000f000fu, hd & 0x000f000fu, b0, b1);
                mma16816(acc[4 * hf + 3], ha & 0x00f000f0u, hb & 0x00f000f0u, hc & 0x00f000f0u, hd & 0x00f000f0u, b0, b1);
            }
        }
    };
    const int mine = n_c > key0 ? (n_c - key0 + kRound - 1) / kRound : 0;      // stages that hold keys of this warp's
    int pos[2][2], next_pos[2][2];
    positions(0, next_pos[0]);
    positions(1, next_pos[1]);
    for (int i = 0; i < rounds; i += 2) {
        const int st[2] = {i % kTokenStages, (i + 1) % kTokenStages};
#pragma unroll
        for (int n = 0; n < 2; ++n) { pos[n][0] = next_pos[n][0]; pos[n][1] = next_pos[n][1]; }
        if (i + 2 < rounds) { positions(i + 2, next_pos[0]); positions(i + 3, next_pos[1]); }
        const bool two = i + 1 < rounds;
        bool came = mbar_wait(&bar_full[st[0]], static_cast<uint32_t>(i / kTokenStages) & 1u);
        if (two) came = mbar_wait(&bar_full[st[1]], static_cast<uint32_t>((i + 1) / kTokenStages) & 1u) && came;
        if (__all_sync(0xffffffffu, came) == 0) { ok = false; break; }
        using One = std::integral_constant<int, 1>;
        using Two = std::integral_constant<int, 2>;
        if (i + 1 < mine) {
            const bool all = max(max(pos[0][0], pos[0][1]), max(pos[1][0], pos[1][1])) <= qpos;
            if (__all_sync(0xffffffffu, all)) reduce(Two(), std::true_type(), st, pos);
            else reduce(Two(), std::false_type(), st, pos);
        } else if (i < mine) {
            reduce(One(), std::false_type(), st, pos);
        }
        __syncwarp();
        if (lane == 0) {
            mbar_arrive(&bar_free[st[0]]);
            if (two) mbar_arrive(&bar_free[st[1]]);
        }
    }
    if (!ok && lane == 0) atomicOr(dev_status, DODO_DEV_WAIT_TIMEOUT);

    // ---- the warp's record of its cached keys ----------------------------------------------------------------------------------
    {
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) {
            l += __shfl_xor_sync(0xffffffffu, l, o);
            accm[0] += __shfl_xor_sync(0xffffffffu, accm[0], o);
            accm[1] += __shfl_xor_sync(0xffffffffu, accm[1], o);
        }
        constexpr int kExp = 133 - kPExp;                          // codes come out as c 2^-133 p s 2^kPExp
        const float back = __uint_as_float(static_cast<uint32_t>(kExp + 127) << 23);
        const bool second = r >= 4;                                // of the two groups in this lane's accumulator columns
        const float bias = second ? accm[1] : accm[0];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            // lanes t even hold rows r (groups 0, 1), odd ones rows r + 8 (groups 2, 3); t and t + 2 the two parts of p s
            float v = (t & 1) == 0 ? (second ? acc[j][1] : acc[j][0]) : (second ? acc[j][3] : acc[j][2]);
            v += __shfl_xor_sync(0xffffffffu, v, 2);
            v = fmaf(v * ((j & 1) != 0 ? 0.0625f : 1.f), back, bias);
            if (t < 2) red[warp][8 * (r + 8 * t) + j] = v;
        }
        if (lane == 0) { red[warp][DH] = m; red[warp][DH + 1] = l; }
    }

    // ---- local keys: eight lanes a key, 16 features a lane, two keys a bundle and round ---------------------------------------------
    {
        constexpr int UL = 2, NB = kConsumers / 8;
        const int bundle = tid >> 3, lig = tid & 7;
        float2 q2[8], a2[8];
        {
            float f[16];
            Vec16<__nv_bfloat16>::unpack(*reinterpret_cast<const uint4*>(qrow + 16 * lig), f);
            Vec16<__nv_bfloat16>::unpack(*reinterpret_cast<const uint4*>(qrow + 16 * lig + 8), f + 8);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                q2[i] = make_float2(f[2 * i] * scale_log2, f[2 * i + 1] * scale_log2);
                a2[i] = make_float2(0.f, 0.f);
            }
        }
        float ml = kNeg, ll = 0.f;
        for (int base = 0; base < n_l; base += NB * UL) {
            uint4 kv[UL][2], vv[UL][2];
            float s[UL];
            bool see[UL];
#pragma unroll
            for (int u = 0; u < UL; ++u) {
                const int j = base + u * NB + bundle;
                see[u] = j < n_l;                               // (rows past the query's own position are not in the window)
                kv[u][0] = kv[u][1] = vv[u][0] = vv[u][1] = make_uint4(0, 0, 0, 0);
                if (see[u]) {
                    const size_t at = (static_cast<size_t>(l_row + j) * H + h) * DH + 16 * lig;
                    const uint4* pk = reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(src.lK) + at);
                    const uint4* pv = reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(src.lV) + at);
                    kv[u][0] = __ldg(pk); kv[u][1] = __ldg(pk + 1);
                    vv[u][0] = __ldg(pv); vv[u][1] = __ldg(pv + 1);
                }
            }
#pragma unroll
            for (int u = 0; u < UL; ++u) {
                float f[16];
                Vec16<__nv_bfloat16>::unpack(kv[u][0], f);
                Vec16<__nv_bfloat16>::unpack(kv[u][1], f + 8);
                float2 d = make_float2(0.f, 0.f);
#pragma unroll
                for (int i = 0; i < 8; ++i) d = __ffma2_rn(q2[i], make_float2(f[2 * i], f[2 * i + 1]), d);
                s[u] = d.x + d.y;
            }
#pragma unroll
            for (int o = 4; o > 0; o >>= 1)
#pragma unroll
                for (int u = 0; u < UL; ++u) s[u] += __shfl_xor_sync(0xffffffffu, s[u], o);
            float m_new = ml;
#pragma unroll
            for (int u = 0; u < UL; ++u) {
                if (!see[u]) s[u] = kNeg;
                m_new = fmaxf(m_new, s[u]);
            }
            const float corr = ex2_approx(ml - m_new);
            ml = m_new;
            ll *= corr;
#pragma unroll
            for (int i = 0; i < 8; ++i) a2[i] = __fmul2_rn(a2[i], make_float2(corr, corr));
#pragma unroll
            for (int u = 0; u < UL; ++u) {
                const float p = see[u] ? ex2_approx(s[u] - m_new) : 0.f;
                ll += p;
                float f[16];
                Vec16<__nv_bfloat16>::unpack(vv[u][0], f);
                Vec16<__nv_bfloat16>::unpack(vv[u][1], f + 8);
#pragma unroll
                for (int i = 0; i < 8; ++i) a2[i] = __ffma2_rn(make_float2(p, p), make_float2(f[2 * i], f[2 * i + 1]), a2[i]);
            }
        }
        // the warp's four bundles: halving exchanges over lane bits 3 and 4
        float M = fmaxf(ml, __shfl_xor_sync(0xffffffffu, ml, 8));
        M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, 16));
        const float f = ex2_approx(ml - M);
        ll *= f;
        ll += __shfl_xor_sync(0xffffffffu, ll, 8);
        ll += __shfl_xor_sync(0xffffffffu, ll, 16);
        float v[16];
#pragma unroll
        for (int i = 0; i < 8; ++i) { v[2 * i] = a2[i].x * f; v[2 * i + 1] = a2[i].y * f; }
        const bool up8 = (lane & 8) != 0, up16 = (lane & 16) != 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float give = up8 ? v[i] : v[8 + i], keep = up8 ? v[8 + i] : v[i];
            v[i] = keep + __shfl_xor_sync(0xffffffffu, give, 8);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float give = up16 ? v[i] : v[4 + i], keep = up16 ? v[4 + i] : v[i];
            red[kTokenWarps + warp][16 * lig + (up8 ? 8 : 0) + (up16 ? 4 : 0) + i] = keep + __shfl_xor_sync(0xffffffffu, give, 16);
        }
        if (lane == 0) { red[kTokenWarps + warp][DH] = M; red[kTokenWarps + warp][DH + 1] = ll; }
    }
    }       // (consumers)
    __syncthreads();
    if (tid < DH) {
        float M = kNeg;
#pragma unroll
        for (int w = 0; w < 2 * kTokenWarps; ++w) M = fmaxf(M, red[w][DH]);
        float L = 0.f, o = 0.f;
#pragma unroll
        for (int w = 0; w < 2 * kTokenWarps; ++w) {
            const float wgt = ex2_approx(red[w][DH] - M);
            L = fmaf(red[w][DH + 1], wgt, L);
            o = fmaf(red[w][tid], wgt, o);
        }
        if (nchunk == 1) {
            write_out<__nv_bfloat16, DH>(O, lse, static_cast<size_t>(sq.q_row0) * H + h, tid, M, L, o);
        } else {
            float* pr = partials + (static_cast<size_t>(sq.part0) + static_cast<size_t>(h) * nchunk + chunk) * RED;
            pr[tid] = o;
            if (tid == 0) { pr[DH] = M; pr[DH + 1] = L; }
        }
    }
    if (nchunk == 1) return;
    merge_chunks<__nv_bfloat16, DH>(sq, H, 0, h, 0, 1, nchunk, partials, tickets, &s_flag, O, lse);
}

// ---- blocks of bf16 queries ------------------------------------------------------------------------------------------------
// The same reading of codes as bf16 numbers with up to eight queries at once: the matrix instruction's eight columns are the queries.
// What differs from the kernel above is which codes share an instruction: one group's only, since steps and minima are a group's.
//   Q.K   lane t of a quad takes word 4 g + t of a key's codes for group g: two instructions per group, their sums over the lanes
//         scaled by the key's step and added to the logit with m (sum of q over the group): queries are not rounded, codes are exact.
//   P.V   rows of A = 16 of a group's 32 features, lane r taking half of word 4 g + (r & 3); columns of B = p s of the group, rounded to
//         bf16 plus what that left (two instructions), so that p s keeps 16 bits.  The weights come out of Q.K with keys as rows and
//         have to be columns: a transposition of two 8 x 8 matrices of bf16 halves (weights split into two halves, 16 bits).
// Local keys take the same steps uncompressed, straight from global memory into the operands, into the same accumulators.
// 24 matrix instructions per 16 keys whatever the number of queries, where the kernel above takes 16 for one.  1, 8, 16 queries over
// 16,384 cached and 512 local keys of 40 heads: 34.5 (the kernel above), 52, 100 us; over 8 x 205 cached and 64 local keys of 32
// heads 7.1, 10.9, 18.3; over 4 x 717 and 1280: 29, 37, 61.  (With fp32 FMAs eight queries took 226, 35 and 118.)  Expanding the rows
// first and attending them on the tensor cores takes 188, 21 and 49 whatever the number, which is the better from about 32 on.
// Head size 64, the same three batches: eight queries 32, 6.9, 25 us (FMAs: four queries 58, 12.0), sixteen 64, 12, 37.
constexpr int kFewQueries = DODO_Q4_TILE_QUERIES;

__device__ __forceinline__ uint32_t transpose8(uint32_t v) {       // an 8 x 8 matrix of 16-bit elements, two of row r in lane (r, t)
    uint32_t d;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(v));
    return d;
}
__device__ __forceinline__ bool infinite2(uint32_t w) { return (w & 0x7f80u) == 0x7f80u || (w & 0x7f800000u) == 0x7f800000u; }
__device__ __forceinline__ float low_half(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float high_half(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
// two floats as bf16 and what the rounding left of them
__device__ __forceinline__ void split2(float a, float b, uint32_t& hi, uint32_t& lo) {
    hi = two_bf16(a, b);
    lo = two_bf16(a - low_half(hi), b - high_half(hi));
}

template <int DH>
__global__ void __launch_bounds__(kTokenThreads, kTokenBlocks)
attend_q4_few_kernel(const __nv_bfloat16* __restrict__ Q, const __grid_constant__ TokenMaps maps, const Q4Source src,
                     const __grid_constant__ AttendGroup g, const int32_t* __restrict__ cache_pos, int H, float scale_log2, int TK,
                     __nv_bfloat16* __restrict__ O, float* __restrict__ lse, float* __restrict__ partials, int* __restrict__ tickets,
                     int early_cache, int* __restrict__ dev_status) {
    using namespace sm100;
    constexpr int RED = DH + 2, G = DH / DODO_Q4_GROUP;
    constexpr uint32_t kWordRow = DH / 4, kCodes = code_bytes(DH), kStage = stage_bytes(DH);
    extern __shared__ unsigned char smem_raw[];
    __shared__ float red[kTokenWarps][kFewQueries][RED];
    __shared__ float2 up[kTokenWarps][kFewQueries / 2];         // huge queries' powers of two
    __shared__ __align__(8) uint64_t bar_full[kTokenStages], bar_free[kTokenStages];
    __shared__ int s_flag;
    const uint32_t ring = (smem_u32(smem_raw) + 1023u) & ~1023u;

    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int r = lane >> 2, t = lane & 3;                 // fragment row (key, feature or query) and quad lane
    const int bid = static_cast<int>(blockIdx.x);
    int b;
    if (g.uniform_ctas > 0) {
        b = bid / g.uniform_ctas;
    } else {
        b = 0;
#pragma unroll 8
        for (int i = 1; i < DODO_GROUP; ++i) b += (i < g.nseq && g.cta0[i] <= bid) ? 1 : 0;
    }
    const AttendSeq sq = g.seq[b];
    int r0 = bid - g.cta0[b];
    const int nchunk = sq.nchunk, chunk = r0 % nchunk;
    r0 /= nchunk;
    const int h = r0 % H, qtile = r0 / H;
    const int q_first = qtile * kFewQueries, nq = min(kFewQueries, sq.tq - q_first);
    const int qpos0 = sq.q_pos0 + q_first;
    const int l_vis = dodo_visible_local(sq.l_len, sq.l_pos0, qpos0 + nq - 1);
    const int nt_c = (sq.c_len + TK - 1) / TK;                             // planning tiles of TK keys
    const int t_begin = chunk * sq.ctiles, t_end = t_begin + sq.ctiles;
    const int c_begin = min(sq.c_len, t_begin * TK), c_end = min(sq.c_len, t_end * TK);
    const int l_begin = min(l_vis, max(0, t_begin - nt_c) * TK), l_end = min(l_vis, max(0, t_end - nt_c) * TK);
    const int n_c = c_end - c_begin, n_l = l_end - l_begin;
    const int c_row = sq.c_row0 + c_begin, l_row = sq.l_row0 + l_begin, l_pos = sq.l_pos0 + l_begin;
    const int rounds = (n_c + kRound - 1) / kRound;

    if (tid == 0) {
        for (int i = 0; i < kTokenStages; ++i) { mbar_init(&bar_full[i], 1); mbar_init(&bar_free[i], kTokenWarps); }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    __syncthreads();
    if (warp == kTokenWarps) {
        if (lane == 0 && !bring_rows<DH>(maps, ring, bar_full, bar_free, h, c_row, rounds, early_cache)) atomicOr(dev_status, DODO_DEV_WAIT_TIMEOUT);
    } else {
        auto hint_rows = [&](const __nv_bfloat16* base, int row, int rows) {
            constexpr int kLines = DH / 64;
            for (int i = tid; i < rows * kLines; i += kConsumers)
                asm volatile("prefetch.global.L2 [%0];" :: "l"(reinterpret_cast<const char*>(base + (static_cast<size_t>(row + i / kLines) * H + h) * DH) + (i % kLines) * 128));
        };
        hint_rows(Q, sq.q_row0 + q_first, nq);
        hint_rows(static_cast<const __nv_bfloat16*>(src.lK), l_row, min(n_l, kHintKeys));
        hint_rows(static_cast<const __nv_bfloat16*>(src.lV), l_row, min(n_l, kHintKeys));
        asm volatile("griddepcontrol.wait;" ::: "memory");
        asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

        // a warp's tile of a stage: keys 16 warp + ..., in swizzled rows of DH bytes.  A stage begins at a multiple of 1024, so that
        // piece p of a row is reached by flipping bits 4 to 6 (rows of 128 bytes) or 4 and 5 (of 64) of the address of the piece whose
        // number is the row's swizzle: row & 7, or (row / 2) & 3.
        const int key0 = 16 * warp;
        const uint32_t swz_r = DH == 128 ? r : r >> 1, swz_t = DH == 128 ? 2 * t : t;
        const uint32_t k_at = static_cast<uint32_t>((key0 + r) * DH + t * 4) + (swz_r << 4);             // row r; row r + 8 is 8 DH bytes on
        const uint32_t ks_at = kCodes + (key0 + r) * kWordRow;
        const uint32_t v_at = static_cast<uint32_t>((key0 + 2 * t) * DH + (r & 3) * 4) + (swz_t << 4);   // row 2 t; the next one's swizzle is
        constexpr uint32_t kNextRow = DH == 128 ? 128 + 16 : 64;                                         // one more, or the same
        const uint32_t vs_at = kCodes + (key0 + 2 * t) * kWordRow + 4 * G;
        auto words = [](uint32_t at, uint32_t* w) {       // a key's G group words
            if constexpr (G == 4) {
                const uint4 v = lds128(at);
                w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
            } else {
                const uint2 v = lds64(at);
                w[0] = v.x; w[1] = v.y;
            }
        };
        const uint32_t sel = r < 4 ? 0x5410u : 0x7632u;            // half of the word whose nibbles are this lane's features

        // ---- the queries as B fragments: lane (r, t) holds query r's features 8 t .. 8 t + 7 of each group
        const __nv_bfloat16* const qrow = Q + (static_cast<size_t>(sq.q_row0 + q_first + min(r, nq - 1)) * H + h) * DH + 8 * t;
        uint32_t qb[G][2][2];
        float2 qsum[G], q_back;                 // of queries 2 t, 2 t + 1
        bool huge;                              // one of the tile's queries leaves a power of two to its logits
        {
            float f[G][8], top = 0.f, sum[G];
#pragma unroll
            for (int i = 0; i < G; ++i) {
                Vec16<__nv_bfloat16>::unpack(*reinterpret_cast<const uint4*>(qrow + 32 * i), f[i]);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    if (r >= nq) f[i][e] = 0.f;
                    top = fmaxf(top, fabsf(f[i][e]));
                }
            }
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
            top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
            // (shifts as in the kernel above, a query's own)
            int e = max(exponent_of(top), -62);
            huge = __any_sync(0xffffffffu, e > kMostExp) != 0;
            if (huge) {
                const int over = max(e - kMostExp, 0);
                const float down = power_of_two(-over);
#pragma unroll
                for (int i = 0; i < G; ++i)
#pragma unroll
                    for (int n = 0; n < 8; ++n) f[i][n] *= down;
                reinterpret_cast<float*>(up[warp])[r] = power_of_two(over);      // (a quad's lanes the same)
                e -= over;
                __syncwarp();
            }
#pragma unroll
            for (int i = 0; i < G; ++i) {
                sum[i] = 0.f;
#pragma unroll
                for (int n = 0; n < 8; ++n) sum[i] += f[i][n];
                sum[i] += __shfl_xor_sync(0xffffffffu, sum[i], 1);
                sum[i] += __shfl_xor_sync(0xffffffffu, sum[i], 2);
                sum[i] *= scale_log2;
                qsum[i].x = __shfl_sync(0xffffffffu, sum[i], 8 * t);
                qsum[i].y = __shfl_sync(0xffffffffu, sum[i], 8 * t + 4);
            }
            const float shift = power_of_two(kQExp - e), s16 = shift * 0.0625f;
            const float back = power_of_two(133 - kQExp + e) * scale_log2;
            q_back.x = __shfl_sync(0xffffffffu, back, 8 * t);
            q_back.y = __shfl_sync(0xffffffffu, back, 8 * t + 4);
#pragma unroll
            for (int i = 0; i < G; ++i) {
                qb[i][0][0] = two_bf16(f[i][0] * shift, f[i][4] * shift);
                qb[i][0][1] = two_bf16(f[i][1] * s16, f[i][5] * s16);
                qb[i][1][0] = two_bf16(f[i][2] * shift, f[i][6] * shift);
                qb[i][1][1] = two_bf16(f[i][3] * s16, f[i][7] * s16);
            }
        }
        const float kPScale = __uint_as_float(static_cast<uint32_t>(kPExp + 127) << 23);
        // positions of queries 2 t, 2 t + 1; one that is not there sees nothing
        const int qpos[2] = {2 * t < nq ? qpos0 + 2 * t : static_cast<int>(0x80000000), 2 * t + 1 < nq ? qpos0 + 2 * t + 1 : static_cast<int>(0x80000000)};

        float m[2] = {kNeg, kNeg};               // of queries 2 t, 2 t + 1: the warp's
        float2 l = make_float2(0.f, 0.f), accm[G];   // sums over a lane's own keys
        float acc[G][2][4];                      // [group][features 0, 1 | 2, 3 of the lane's four]: even feature x queries 2 t, 2 t + 1, then the odd one
#pragma unroll
        for (int i = 0; i < G; ++i) {
            accm[i] = make_float2(0.f, 0.f);
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[i][u][e] = 0.f;
        }
        // logits of a tile (keys r, r + 8 x queries 2 t, 2 t + 1) to weights; moves the maxima and what has been summed so far
        auto weigh = [&](auto all_seen, float2* s, const bool (*see)[2]) {
            constexpr bool kAll = decltype(all_seen)::value;
            if (!kAll) {
#pragma unroll
                for (int i = 0; i < 2; ++i) { s[i].x = see[i][0] ? s[i].x : kNeg; s[i].y = see[i][1] ? s[i].y : kNeg; }
            }
            float top[2] = {fmaxf(s[0].x, s[1].x), fmaxf(s[0].y, s[1].y)};
#pragma unroll
            for (int o = 4; o < 32; o <<= 1) {
                top[0] = fmaxf(top[0], __shfl_xor_sync(0xffffffffu, top[0], o));
                top[1] = fmaxf(top[1], __shfl_xor_sync(0xffffffffu, top[1], o));
            }
            if (top[0] > m[0] + 8.f || top[1] > m[1] + 8.f) {     // the reference moves only when it pays: weights stay below 2^8
                float2 corr;
                float to = top[0] > m[0] + 8.f ? top[0] : m[0];
                corr.x = ex2_approx(m[0] - to);
                m[0] = to;
                to = top[1] > m[1] + 8.f ? top[1] : m[1];
                corr.y = ex2_approx(m[1] - to);
                m[1] = to;
                l = __fmul2_rn(l, corr);
#pragma unroll
                for (int i = 0; i < G; ++i) {
                    accm[i] = __fmul2_rn(accm[i], corr);
#pragma unroll
                    for (int u = 0; u < 2; ++u)
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[i][u][e] *= (e & 1) == 0 ? corr.x : corr.y;
                }
            }
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                s[i] = make_float2(ex2_approx(s[i].x - m[0]), ex2_approx(s[i].y - m[1]));
                if (!kAll) { s[i].x = see[i][0] ? s[i].x : 0.f; s[i].y = see[i][1] ? s[i].y : 0.f; }
                l = __fadd2_rn(l, s[i]);
            }
        };

        // ---- cached keys: one tile of 16 per warp and stage -------------------------------------------------------------------
        auto reduce = [&](auto all_seen, uint32_t base, const int* pos) {
            constexpr bool kAll = decltype(all_seen)::value;
            bool see[2][2];
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int c = 0; c < 2; ++c) see[i][c] = kAll || pos[i] <= qpos[c];
            float2 s[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
            {
                uint32_t wa[G], wb[G];
                words(base + ks_at, wa);
                words(base + ks_at + 8 * kWordRow, wb);
#pragma unroll
                for (int i = 0; i < G; ++i) {
                    const uint32_t at = (base + k_at) ^ (16u * i);
                    const uint32_t ka = lds32(at), kb = lds32(at + 8u * DH), ha = ka >> 8, hb = kb >> 8;
                    float d[4] = {0.f, 0.f, 0.f, 0.f};
                    mma16816(d, ka & 0x000f000fu, kb & 0x000f000fu, ka & 0x00f000f0u, kb & 0x00f000f0u, qb[i][0][0], qb[i][0][1]);
                    mma16816(d, ha & 0x000f000fu, hb & 0x000f000fu, ha & 0x00f000f0u, hb & 0x00f000f0u, qb[i][1][0], qb[i][1][1]);
                    s[0] = __ffma2_rn(__fmul2_rn(make_float2(d[0], d[1]), q_back), make_float2(low_half(wa[i]), low_half(wa[i])), s[0]);
                    s[1] = __ffma2_rn(__fmul2_rn(make_float2(d[2], d[3]), q_back), make_float2(low_half(wb[i]), low_half(wb[i])), s[1]);
                    s[0] = __ffma2_rn(qsum[i], make_float2(high_half(wa[i]), high_half(wa[i])), s[0]);
                    s[1] = __ffma2_rn(qsum[i], make_float2(high_half(wb[i]), high_half(wb[i])), s[1]);
                }
            }
            if (huge) {
                const float2 f = up[warp][t];
                s[0] = __fmul2_rn(s[0], f);
                s[1] = __fmul2_rn(s[1], f);
            }
            weigh(all_seen, s, see);
            // minima of the values; a masked key takes no part, whatever its words hold
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                uint32_t wv[G];
                words(base + ks_at + 4 * G + 8 * kWordRow * i, wv);
#pragma unroll
                for (int n = 0; n < G; ++n) {
                    const float2 v = __ffma2_rn(s[i], make_float2(high_half(wv[n]), high_half(wv[n])), accm[n]);
                    accm[n].x = see[i][0] ? v.x : accm[n].x;
                    accm[n].y = see[i][1] ? v.y : accm[n].y;
                }
                if (!kAll) { s[i].x = see[i][0] ? s[i].x : -1.f; s[i].y = see[i][1] ? s[i].y : -1.f; }    // (a mark for the other side)
            }
            // keys as columns: query r's weights of keys 2 t, 2 t + 1, 2 t + 8, 2 t + 9
            float p[4];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                uint32_t hi, lo;
                split2(s[i].x, s[i].y, hi, lo);
                hi = transpose8(hi);
                lo = transpose8(lo);
                p[2 * i] = low_half(hi) + low_half(lo);
                p[2 * i + 1] = high_half(hi) + high_half(lo);
            }
            uint32_t wv[4][G];
            bool hid[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                hid[i] = !kAll && p[i] < 0.f;
                p[i] *= kPScale;
                words(base + vs_at + kWordRow * (i & 1) + 8 * kWordRow * (i >> 1), wv[i]);
            }
#pragma unroll
            for (int n = 0; n < G; ++n) {
                float x[4];
                uint32_t c[4], hi[2], lo[2];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    x[i] = p[i] * low_half(wv[i][n]);
                    if (!kAll) x[i] = hid[i] ? 0.f : x[i];
                    c[i] = lds32(((base + v_at + (i & 1) * kNextRow) ^ (16u * (G + n))) + 8u * DH * (i >> 1));
                }
                split2(x[0], x[1], hi[0], lo[0]);
                split2(x[2], x[3], hi[1], lo[1]);
                uint32_t wa = __byte_perm(c[0], c[1], sel), wc = __byte_perm(c[2], c[3], sel);
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    mma16816(acc[n][u], wa & 0x000f000fu, wa & 0x00f000f0u, wc & 0x000f000fu, wc & 0x00f000f0u, hi[0], hi[1]);
                    mma16816(acc[n][u], wa & 0x000f000fu, wa & 0x00f000f0u, wc & 0x000f000fu, wc & 0x00f000f0u, lo[0], lo[1]);
                    wa >>= 8;
                    wc >>= 8;
                }
            }
        };
        auto positions = [&](int i, int* pos) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int j = i * kRound + key0 + r + 8 * e;
                pos[e] = j < n_c ? __ldg(cache_pos + c_row + j) : 0x7fffffff;
            }
        };
        bool ok = true;
        const int mine = n_c > key0 ? (n_c - key0 + kRound - 1) / kRound : 0;      // stages that hold keys of this warp's
        int next_pos[2];
        positions(0, next_pos);
        for (int i = 0; i < rounds; ++i) {
            const int st = i % kTokenStages;
            const int pos[2] = {next_pos[0], next_pos[1]};
            if (i + 1 < rounds) positions(i + 1, next_pos);
            if (__all_sync(0xffffffffu, mbar_wait(&bar_full[st], static_cast<uint32_t>(i / kTokenStages) & 1u)) == 0) { ok = false; break; }
            if (i < mine) {
                if (__all_sync(0xffffffffu, max(pos[0], pos[1]) <= qpos0)) reduce(std::true_type(), ring + st * kStage, pos);
                else reduce(std::false_type(), ring + st * kStage, pos);
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(&bar_free[st]);
        }
        if (!ok && lane == 0) atomicOr(dev_status, DODO_DEV_WAIT_TIMEOUT);

        // ---- from the codes' scale to that of plain values ------------------------------------------------------------------------
        {
            const float back = __uint_as_float(static_cast<uint32_t>(133 - kPExp + 127) << 23), back16 = back * 0.0625f;
#pragma unroll
            for (int n = 0; n < G; ++n) {
#pragma unroll
                for (int o = 4; o < 32; o <<= 1) {
                    accm[n].x += __shfl_xor_sync(0xffffffffu, accm[n].x, o);
                    accm[n].y += __shfl_xor_sync(0xffffffffu, accm[n].y, o);
                }
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[n][u][e] = fmaf(acc[n][u][e], e < 2 ? back : back16, (e & 1) == 0 ? accm[n].x : accm[n].y);
                accm[n] = make_float2(0.f, 0.f);
            }
        }

        // ---- local keys, 16 a warp: K and V rows as operands, pieces of them straight from global memory -----------------------------
        if (16 * warp < n_l) {
            uint4 qf[G];                        // query r's features 32 g + 8 t + ...
#pragma unroll
            for (int i = 0; i < G; ++i) {
                qf[i] = *reinterpret_cast<const uint4*>(qrow + 32 * i);
                if (r >= nq) qf[i] = make_uint4(0, 0, 0, 0);
            }
            const size_t pitch = static_cast<size_t>(H) * DH;
            const __nv_bfloat16* const lk = static_cast<const __nv_bfloat16*>(src.lK) + static_cast<size_t>(l_row) * pitch + static_cast<size_t>(h) * DH + 8 * t;
            const __nv_bfloat16* const lv = static_cast<const __nv_bfloat16*>(src.lV) + static_cast<size_t>(l_row) * pitch + static_cast<size_t>(h) * DH + 8 * (r & 3) + 4 * (r >> 2);
            for (int first = 16 * warp; first < n_l; first += kRound) {
                bool see[2][2];
                uint4 k[2][G];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const int j = first + r + 8 * i;
#pragma unroll
                    for (int c = 0; c < 2; ++c) see[i][c] = j < n_l && l_pos + j <= qpos[c];
#pragma unroll
                    for (int n = 0; n < G; ++n) {
                        k[i][n] = make_uint4(0, 0, 0, 0);
                        if (j < n_l) k[i][n] = __ldg(reinterpret_cast<const uint4*>(lk + static_cast<size_t>(j) * pitch + 32 * n));
                    }
                }
                uint2 v[4][G];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int j = first + 2 * t + (i & 1) + 8 * (i >> 1);
#pragma unroll
                    for (int n = 0; n < G; ++n) {
                        v[i][n] = make_uint2(0, 0);
                        if (j < n_l) v[i][n] = __ldg(reinterpret_cast<const uint2*>(lv + static_cast<size_t>(j) * pitch + 32 * n));
                    }
                }
                float2 s[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
                for (int n = 0; n < G; n += 2) {
                    float d[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int e = n; e < n + 2; ++e) {
                        mma16816(d, k[0][e].x, k[1][e].x, k[0][e].y, k[1][e].y, qf[e].x, qf[e].y);
                        mma16816(d, k[0][e].z, k[1][e].z, k[0][e].w, k[1][e].w, qf[e].z, qf[e].w);
                    }
                    s[0] = __fadd2_rn(s[0], make_float2(d[0], d[1]));
                    s[1] = __fadd2_rn(s[1], make_float2(d[2], d[3]));
                }
                const float2 scale2 = make_float2(scale_log2, scale_log2);
                s[0] = __fmul2_rn(s[0], scale2);
                s[1] = __fmul2_rn(s[1], scale2);
                weigh(std::false_type(), s, see);
                uint32_t hi[2], lo[2];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    split2(s[i].x, s[i].y, hi[i], lo[i]);
                    hi[i] = transpose8(hi[i]);
                    lo[i] = transpose8(lo[i]);
                }
                // A key behind some of the tile's queries may hold anything, and 0 times that need not be 0: if a value is not finite there,
                // one query at a time, with the rows it does not see as zeros.
                bool apart = false;
                if (l_pos + min(first + 15, n_l - 1) > qpos0) {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
#pragma unroll
                        for (int n = 0; n < G; ++n) apart = apart || infinite2(v[i][n].x) || infinite2(v[i][n].y);
                    apart = __any_sync(0xffffffffu, apart);
                }
                if (!apart) {
#pragma unroll
                    for (int n = 0; n < G; ++n)
#pragma unroll
                        for (int u = 0; u < 2; ++u) {
                            const uint32_t w0 = u == 0 ? v[0][n].x : v[0][n].y, w1 = u == 0 ? v[1][n].x : v[1][n].y;
                            const uint32_t w2 = u == 0 ? v[2][n].x : v[2][n].y, w3 = u == 0 ? v[3][n].x : v[3][n].y;
                            const uint32_t a0 = __byte_perm(w0, w1, 0x5410), a1 = __byte_perm(w0, w1, 0x7632);
                            const uint32_t a2 = __byte_perm(w2, w3, 0x5410), a3 = __byte_perm(w2, w3, 0x7632);
                            mma16816(acc[n][u], a0, a1, a2, a3, hi[0], hi[1]);
                            mma16816(acc[n][u], a0, a1, a2, a3, lo[0], lo[1]);
                        }
                } else {
#pragma unroll 1
                    for (int q = 0; q < nq; ++q) {
                        const uint32_t bh[2] = {r == q ? hi[0] : 0u, r == q ? hi[1] : 0u}, bl[2] = {r == q ? lo[0] : 0u, r == q ? lo[1] : 0u};
                        bool sees[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) sees[i] = l_pos + first + 2 * t + (i & 1) + 8 * (i >> 1) <= qpos0 + q;
#pragma unroll
                        for (int n = 0; n < G; ++n)
#pragma unroll
                            for (int u = 0; u < 2; ++u) {
                                uint32_t w[4];
#pragma unroll
                                for (int i = 0; i < 4; ++i) w[i] = !sees[i] ? 0u : u == 0 ? v[i][n].x : v[i][n].y;
                                const uint32_t a0 = __byte_perm(w[0], w[1], 0x5410), a1 = __byte_perm(w[0], w[1], 0x7632);
                                const uint32_t a2 = __byte_perm(w[2], w[3], 0x5410), a3 = __byte_perm(w[2], w[3], 0x7632);
                                float d[4] = {0.f, 0.f, 0.f, 0.f};
                                mma16816(d, a0, a1, a2, a3, bh[0], bh[1]);
                                mma16816(d, a0, a1, a2, a3, bl[0], bl[1]);
                                if (2 * t == q) { acc[n][u][0] += d[0]; acc[n][u][2] += d[2]; }
                                if (2 * t + 1 == q) { acc[n][u][1] += d[1]; acc[n][u][3] += d[3]; }
                            }
                    }
                }
            }
        }

        // ---- the warp's record ----------------------------------------------------------------------------------------------------
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) {
            l.x += __shfl_xor_sync(0xffffffffu, l.x, o);
            l.y += __shfl_xor_sync(0xffffffffu, l.y, o);
        }
#pragma unroll
        for (int n = 0; n < G; ++n)
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    red[warp][2 * t + (e & 1)][32 * n + 8 * (r & 3) + 4 * (r >> 2) + 2 * u + (e >> 1)] = acc[n][u][e];
        if (r == 0) {
            red[warp][2 * t][DH] = m[0];
            red[warp][2 * t + 1][DH] = m[1];
            red[warp][2 * t][DH + 1] = l.x;
            red[warp][2 * t + 1][DH + 1] = l.y;
        }
    }       // (consumers)
    __syncthreads();
    for (int i = tid; i < nq * DH; i += kTokenThreads) {
        const int q2 = i / DH, dim = i % DH;
        float M = kNeg;
#pragma unroll
        for (int w = 0; w < kTokenWarps; ++w) M = fmaxf(M, red[w][q2][DH]);
        float L = 0.f, o = 0.f;
#pragma unroll
        for (int w = 0; w < kTokenWarps; ++w) {
            const float wgt = ex2_approx(red[w][q2][DH] - M);
            L = fmaf(red[w][q2][DH + 1], wgt, L);
            o = fmaf(red[w][q2][dim], wgt, o);
        }
        if (nchunk == 1) {
            write_out<__nv_bfloat16, DH>(O, lse, static_cast<size_t>(sq.q_row0 + q_first + q2) * H + h, dim, M, L, o);
        } else {
            float* pr = partials + (static_cast<size_t>(sq.part0) + (static_cast<size_t>(q_first + q2) * H + h) * nchunk + chunk) * RED;
            pr[dim] = o;
            if (dim == 0) { pr[DH] = M; pr[DH + 1] = L; }
        }
    }
    if (nchunk == 1) return;
    merge_chunks<__nv_bfloat16, DH>(sq, H, qtile, h, q_first, nq, nchunk, partials, tickets, &s_flag, O, lse);
}

template <typename T, int DH, int QT, int U>
int launch_t(dodo_ctx* ctx, int H, float sm_scale, const AttendGroup& g, const void* Q, const Q4Source& src,
             const int32_t* cache_pos, void* O, float* lse, float* partials, int* tickets, bool early, cudaStream_t st) {
    const int dtype = sizeof(T) == 4 ? DODO_F32 : DODO_BF16;
    const cudaError_t e = dodo_launch_dependent(attend_q4_kernel<T, DH, QT, U>, dim3(static_cast<unsigned>(g.cta0[g.nseq])), dim3(kThreads), 0,
                                                st, static_cast<const T*>(Q), src, g, cache_pos, H, sm_scale * 1.4426950408889634f,
                                                dodo_attend_tile_keys(dtype, DH), static_cast<T*>(O), lse, partials, tickets, early ? 1 : 0);
    return dodo_check_cuda(ctx, e, "4-bit attend launch");
}

template <typename T, int DH>
int launch_qt(dodo_ctx* ctx, int H, float sm_scale, int qt, const AttendGroup& g, const void* Q, const Q4Source& src,
              const int32_t* cache_pos, void* O, float* lse, float* partials, int* tickets, bool early, cudaStream_t st) {
    if (qt == 1) return launch_t<T, DH, 1, 4>(ctx, H, sm_scale, g, Q, src, cache_pos, O, lse, partials, tickets, early, st);
    if (qt == 2) return launch_t<T, DH, 2, 2>(ctx, H, sm_scale, g, Q, src, cache_pos, O, lse, partials, tickets, early, st);
    if (qt == 4) return launch_t<T, DH, 4, 2>(ctx, H, sm_scale, g, Q, src, cache_pos, O, lse, partials, tickets, early, st);
    return dodo_fail(ctx, DODO_ERR_UNSUPPORTED, "4-bit attend: query tile %d is not built", qt);
}

// the kernels on the warp-level matrix units
int launch_mma(dodo_ctx* ctx, int H, int dh, float sm_scale, int qt, const AttendGroup& g, const void* Q, const Q4Source& src, int cache_rows,
               const int32_t* cache_pos, void* O, float* lse, float* partials, int* tickets, bool early, cudaStream_t st) {
    TokenMaps maps;
    memset(&maps, 0, sizeof maps);
    if (cache_rows > 0) {
        int rc = dodo_encode_byte_rows(ctx, &maps.q4, src.q4, H * dh, cache_rows, dh, kRound);
        if (rc == DODO_OK) rc = dodo_encode_byte_rows(ctx, &maps.scale, src.scale, H * dh / 4, cache_rows, dh / 4, kRound);
        if (rc != DODO_OK) return rc;
    }
    const size_t smem = static_cast<size_t>(kTokenStages) * stage_bytes(dh) + 1024;
    auto kern = dh == 64 ? attend_q4_few_kernel<64> : qt == 1 ? attend_q4_token_kernel : attend_q4_few_kernel<128>;
    bool& set = ctx->q4_attr_set[dh == 64 ? 2 : qt == 1 ? 0 : 1];
    if (!set) {
        const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(smem));
        if (e != cudaSuccess) return dodo_check_cuda(ctx, e, "4-bit attend shared-memory attribute");
        set = true;
    }
    return dodo_check_cuda(ctx, dodo_launch_dependent(kern, dim3(static_cast<unsigned>(g.cta0[g.nseq])), dim3(kTokenThreads), smem, st,
                                                      static_cast<const __nv_bfloat16*>(Q), maps, src, g, cache_pos, H, sm_scale * 1.4426950408889634f,
                                                      dodo_attend_tile_keys(DODO_BF16, dh), static_cast<__nv_bfloat16*>(O), lse, partials, tickets, early ? 1 : 0, ctx->dev_status),
                           "4-bit attend launch");
}

}  // namespace

int dodo_launch_attend_q4(dodo_ctx* ctx, int dtype, int H, int dh, float sm_scale, const AttendPlan& plan,
                          const AttendGroup& g, const void* Q, const void* cache_q4, const uint32_t* cache_scale, int cache_rows,
                          const int32_t* cache_pos, const void* locK, const void* locV, void* O, float* lse,
                          float* partials, int* tickets, bool early_cache, cudaStream_t st) {
    if (g.cta0[g.nseq] == 0) return DODO_OK;
    const Q4Source src = {static_cast<const uint32_t*>(cache_q4), cache_scale, locK, locV};
    if (dtype == DODO_BF16 && (dh == 128 || plan.qt > 1))
        return launch_mma(ctx, H, dh, sm_scale, plan.qt, g, Q, src, cache_rows, cache_pos, O, lse, partials, tickets, early_cache, st);
    if (dtype == DODO_BF16 && dh == 64)
        return launch_t<__nv_bfloat16, 64, 1, 4>(ctx, H, sm_scale, g, Q, src, cache_pos, O, lse, partials, tickets, early_cache, st);
    if (dtype == DODO_F32 && dh == 128)
        return launch_qt<float, 128>(ctx, H, sm_scale, plan.qt, g, Q, src, cache_pos, O, lse, partials, tickets, early_cache, st);
    if (dtype == DODO_F32 && dh == 64)
        return launch_qt<float, 64>(ctx, H, sm_scale, plan.qt, g, Q, src, cache_pos, O, lse, partials, tickets, early_cache, st);
    return dodo_fail(ctx, DODO_ERR_UNSUPPORTED, "4-bit attend: dtype %d with head size %d", dtype, dh);
}

int dodo_attend_q4_tile_queries(int dtype, int max_tq) { return dtype == DODO_BF16 && max_tq > 1 ? kFewQueries : 0; }
