// Attention of query tokens over [4-bit nugget cache ; local tokens] (Eq. 4, Eq. 9, Eq. 13): the streaming kernel of
// attend.cu for a cache in the format of cache_q4.cu.  Softmax, masking, split over key chunks and log-sum-exp are as
// there; the values are those the codes stand for, m + c s, never materialised:
//   q . k   = sum over groups of  s (sum_i q_i c_i) + m (sum_i q_i)
//   sum_j p_j v_j = sum_j (p_j s_j) c_j + (sum_j p_j m_j)   per feature, the second sum once per group
// so that a group costs one extra multiply-add per key on either side.
//
// A cached key is 160 bytes a head (dh 128) where bf16 has 512, so the bound moves towards instruction issue: what counts
// is instructions per code.  A lane owns a run of 32 features of a head (one group: 16 bytes of codes, one word each of K
// and V steps), 16 where several queries share the key.  A code is turned into a float in place, without a shift: masking
// nibble i of a word and or-ing in the exponent of 2^23 gives 2^23 + c 16^i exactly, one packed subtraction per two codes
// takes the 2^23 off, and the weight 16^i is folded into the query feature (for K) and divided out of the accumulator at
// the end (for V), both powers of two and exact.  That is 2.1 instructions per code and product.
#include "dodo_internal.cuh"
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

template <int W> struct Codes { uint32_t w[W]; };
template <int W> __device__ __forceinline__ Codes<W> load_codes(const uint32_t* p);
template <> __device__ __forceinline__ Codes<4> load_codes<4>(const uint32_t* p) {
    const uint4 v = ld_stream16(p);
    return {{v.x, v.y, v.z, v.w}};
}
template <> __device__ __forceinline__ Codes<2> load_codes<2>(const uint32_t* p) {
    Codes<2> c;
    asm volatile("ld.global.nc.L1::no_allocate.v2.u32 {%0,%1}, [%2];" : "=r"(c.w[0]), "=r"(c.w[1]) : "l"(p));
    return c;
}

struct Q4Source {
    const uint32_t* q4;       // codes, dh / 4 words per (row, head): K's then V's
    const uint32_t* scale;    // 2 dh / 32 words per (row, head): K's then V's
    const void *lK, *lV;
};

// FPL: features per lane (32 or 16); LPR = DH / FPL lanes share a key.
template <typename T, int DH, int QT, int FPL, int U>
__global__ void __launch_bounds__(kThreads, QT == 1 ? 2 : 1)
attend_q4_kernel(const T* __restrict__ Q, const Q4Source src, const __grid_constant__ AttendGroup g,
                 const int32_t* __restrict__ cache_pos, int H, float scale_log2, int TK, T* __restrict__ O,
                 float* __restrict__ lse, float* __restrict__ partials, int* __restrict__ tickets, int early_cache) {
    constexpr int LPR = DH / FPL, BPW = 32 / LPR, NB = kWarps * BPW;   // lanes per key, bundles per warp and per block
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
    const int l_vis = max(0, min(sq.l_len, sq.q_pos0 + q_first + nq - 1 - sq.l_pos0 + 1));
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
    struct Batch { Codes<W> k[U], v[U]; uint32_t ks[U], vs[U]; int pos[U]; };
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
                t.k[u] = load_codes<W>(q4_0 + at * (DH / 4));
                t.v[u] = load_codes<W>(q4_0 + at * (DH / 4) + DH / 8);
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
    auto write_out = [&](int q2, int dim, float M, float L, float o) {
        const size_t orow = static_cast<size_t>(qrow0 + q2) * H + h;
        store_out(O + orow * DH + dim, L != 0.f ? o / L : 0.f);   // (a NaN sum stays one)
        if (lse != nullptr && dim == 0) lse[orow] = L != 0.f ? (M + log2f(L)) * 0.6931471805599453f : -INFINITY;
    };
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
            write_out(q2, dim, M, L, o);
        } else {
            float* pr = partials + (static_cast<size_t>(sq.part0) + (static_cast<size_t>(q_first + q2) * H + h) * nchunk + chunk) * RED;
            pr[dim] = o;
            if (dim == 0) { pr[DH] = M; pr[DH + 1] = L; }
        }
    }
    if (nchunk == 1) return;

    // ---- the last chunk to arrive merges the partials of its (query tile, head); nobody waits ----------------------------
    __threadfence();
    __syncthreads();
    if (tid == 0) {
        int* tk = tickets + sq.tick0 + qtile * H + h;
        const int t = atomicAdd(tk, 1);
        s_flag = (t == nchunk - 1);
        if (s_flag) *tk = 0;  // leave the counter clean for the next launch
    }
    __syncthreads();
    if (!s_flag) return;
    __threadfence();
    for (int i = tid; i < QT * DH; i += kThreads) {
        const int q2 = i / DH, dim = i % DH;
        if (q2 >= nq) continue;
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
        write_out(q2, dim, M, L, o);
    }
}

template <typename T, int DH, int QT, int FPL, int U>
int launch_t(dodo_ctx* ctx, int H, float sm_scale, const AttendGroup& g, const void* Q, const Q4Source& src,
             const int32_t* cache_pos, void* O, float* lse, float* partials, int* tickets, bool early, cudaStream_t st) {
    const int dtype = sizeof(T) == 4 ? DODO_F32 : DODO_BF16;
    const cudaError_t e = dodo_launch_dependent(attend_q4_kernel<T, DH, QT, FPL, U>, dim3(static_cast<unsigned>(g.cta0[g.nseq])), dim3(kThreads), 0,
                                                st, static_cast<const T*>(Q), src, g, cache_pos, H, sm_scale * 1.4426950408889634f,
                                                dodo_attend_tile_keys(dtype, DH), static_cast<T*>(O), lse, partials, tickets, early ? 1 : 0);
    return dodo_check_cuda(ctx, e, "4-bit attend launch");
}

template <typename T, int DH>
int launch_qt(dodo_ctx* ctx, int H, float sm_scale, int qt, const AttendGroup& g, const void* Q, const Q4Source& src,
              const int32_t* cache_pos, void* O, float* lse, float* partials, int* tickets, bool early, cudaStream_t st) {
    switch (qt) {
        case 1: return launch_t<T, DH, 1, 16, 4>(ctx, H, sm_scale, g, Q, src, cache_pos, O, lse, partials, tickets, early, st);
        case 2: return launch_t<T, DH, 2, 16, 2>(ctx, H, sm_scale, g, Q, src, cache_pos, O, lse, partials, tickets, early, st);
        case 4: return launch_t<T, DH, 4, 16, 2>(ctx, H, sm_scale, g, Q, src, cache_pos, O, lse, partials, tickets, early, st);
        default: break;
    }
    return dodo_fail(ctx, DODO_ERR_UNSUPPORTED, "4-bit attend: query tile %d is not built", qt);
}

}  // namespace

int dodo_launch_attend_q4(dodo_ctx* ctx, int dtype, int H, int dh, float sm_scale, const AttendPlan& plan,
                          const AttendGroup& g, const void* Q, const void* cache_q4, const uint32_t* cache_scale,
                          const int32_t* cache_pos, const void* locK, const void* locV, void* O, float* lse,
                          float* partials, int* tickets, bool early_cache, cudaStream_t st) {
    if (g.cta0[g.nseq] == 0) return DODO_OK;
    const Q4Source src = {static_cast<const uint32_t*>(cache_q4), cache_scale, locK, locV};
    if (dtype == DODO_BF16 && dh == 128)
        return launch_qt<__nv_bfloat16, 128>(ctx, H, sm_scale, plan.qt, g, Q, src, cache_pos, O, lse, partials, tickets, early_cache, st);
    if (dtype == DODO_BF16 && dh == 64)
        return launch_qt<__nv_bfloat16, 64>(ctx, H, sm_scale, plan.qt, g, Q, src, cache_pos, O, lse, partials, tickets, early_cache, st);
    if (dtype == DODO_F32 && dh == 128)
        return launch_qt<float, 128>(ctx, H, sm_scale, plan.qt, g, Q, src, cache_pos, O, lse, partials, tickets, early_cache, st);
    if (dtype == DODO_F32 && dh == 64)
        return launch_qt<float, 64>(ctx, H, sm_scale, plan.qt, g, Q, src, cache_pos, O, lse, partials, tickets, early_cache, st);
    return dodo_fail(ctx, DODO_ERR_UNSUPPORTED, "4-bit attend: dtype %d with head size %d", dtype, dh);
}
