// Nugget cache held in 4 bits: the gather (Eq. 5) that quantises the selected K/V rows on the way into it, and the
// expansion of its rows back to a floating type.
//
// Format.  A row of one head is cut into groups of 32 features.  With lo and hi the group's least and largest value,
//   m = the largest bf16 number <= lo,   s = the least bf16 number with 15 s >= hi - m,
//   c_i = (x_i - m) / s rounded to the nearest whole number, ties to even (0 where s = 0),
// and feature i stands for m + c_i s.  Both roundings go outwards, so every x_i lies in [m, m + 15 s], no code is
// clamped and the error is at most s / 2 for every feature.  The codes are defined on real numbers; the kernel finds
// them in fp32 and decides the few that lie next to a border exactly (see code_of).  A group that holds a NaN or an
// infinity, or whose span overflows, is stored as NaN: all of its features read back as NaN.
// Storage: a (row, head) owns dh bytes of codes, K's dh / 2 then V's (feature 2i in the low half of byte i), which is
// one 128-byte line at head size 128, and 2 dh / 32 words, K's then V's, with s in the low and m in the high 16 bits.
#include "dodo_internal.cuh"

namespace {

constexpr int kThreads = 128;
constexpr int kGroup = DODO_Q4_GROUP;
constexpr int kOctet = 8;                       // features per thread and step: one word of codes
constexpr float kFinite = 3.4028234663852886e38f;

__device__ __forceinline__ float cut_bf16(float x) { return __uint_as_float(__float_as_uint(x) & 0xffff0000u); }   // towards 0
__device__ __forceinline__ float bf16_down(float x) {
    const uint32_t b = __float_as_uint(x), c = b & 0xffff0000u;
    return __uint_as_float(c != b && (b >> 31) != 0u ? c + 0x10000u : c);
}
// a - b as an unevaluated sum t + e, exactly (two-sum)
__device__ __forceinline__ void two_diff(float a, float b, float& t, float& e) {
    t = __fsub_rn(a, b);
    const float z = __fsub_rn(t, a);
    e = __fadd_rn(__fsub_rn(a, __fsub_rn(t, z)), __fsub_rn(-b, z));
}
// Least bf16 s with 15 s >= t + e.  The quotient is off by at most a few units of fp32, so its bf16 cut is s or one
// or two steps below; 15 s is exact (8 + 4 bits).
__device__ __forceinline__ float step_of(float t, float e) {
    float s = cut_bf16(__fdiv_rn(t, 15.f));
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const float p = __fmul_rn(15.f, s);
        if (p < t || (p == t && e > 0.f)) s = __uint_as_float(__float_as_uint(s) + 0x10000u);
    }
    return s;
}
// The code of x, decided exactly: a first guess, then the borders (c -+ 1/2) s, which are exact in fp32 (5 + 8 bits),
// against the exact difference t + e.
__device__ __noinline__ int code_of(float x, float m, float s) {
    float t, e;
    two_diff(x, m, t, e);
    int c = static_cast<int>(fminf(fmaxf(rintf(__fdiv_rn(t, s)), 0.f), 15.f));
    const float up = __fmul_rn(static_cast<float>(c) + 0.5f, s), down = __fmul_rn(static_cast<float>(c) - 0.5f, s);
    const bool odd = (c & 1) != 0;
    if (t > up || (t == up && (e > 0.f || (e == 0.f && odd)))) ++c;
    else if (t < down || (t == down && (e < 0.f || (e == 0.f && odd)))) --c;
    return min(max(c, 0), 15);
}

template <typename T> __device__ __forceinline__ void load_octet(const unsigned char* p, uint4* v);
template <> __device__ __forceinline__ void load_octet<__nv_bfloat16>(const unsigned char* p, uint4* v) { v[0] = ld_stream16(p); }
template <> __device__ __forceinline__ void load_octet<float>(const unsigned char* p, uint4* v) {
    v[0] = ld_stream16(p);
    v[1] = ld_stream16(p + 16);
}

// Quantise one octet; the four lanes of a quad hold one group.  All lanes of the warp take part.
__device__ __forceinline__ uint32_t quantise(const float* x, uint32_t& word) {
    float lo = x[0], hi = x[0];
    bool fine = fabsf(x[0]) <= kFinite;
#pragma unroll
    for (int i = 1; i < kOctet; ++i) {
        lo = fminf(lo, x[i]);
        hi = fmaxf(hi, x[i]);
        fine = fine && fabsf(x[i]) <= kFinite;
    }
    if (!fine) hi = INFINITY;   // poisons the span
#pragma unroll
    for (int o = 1; o < 4; o <<= 1) {
        lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, o));
        hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, o));
    }
    const float m = bf16_down(lo);
    float t, e;
    two_diff(hi, m, t, e);
    if (!(t <= kFinite)) {
        word = 0x00007fc0u;     // step NaN
        return 0u;
    }
    const float s = step_of(t, e);
    word = (__float_as_uint(s) >> 16) | (__float_as_uint(m) & 0xffff0000u);
    if (s == 0.f) return 0u;
    // Codes by a reciprocal: f = (x - m) / s comes out within 3e-6 of the true quotient (at most 15), so k = round(f - 1/2) is
    // the whole number below it or one of its two neighbours' border lies within 3e-6; either way the code is k or k + 1, by
    // which side of the border (k + 1/2) s the difference lies on.  The border is exact in fp32 (5 + 8 bits); where the
    // difference equals it, what its rounding lost decides, or the even code if nothing was (bf16 rows, whose values lie on
    // a coarse grid, meet that in about one octet in fifty).  Steps whose reciprocal overflows go through code_of.
    const float inv = __fdiv_rn(1.f, s), half = 0.5f * s;
    constexpr float kMagic = 12582912.f;    // 1.5 * 2^23: adding it rounds to whole numbers, in the low mantissa bits
    uint32_t codes = 0u;
#pragma unroll
    for (int i = 0; i < kOctet; ++i) {
        const float d = __fsub_rn(x[i], m);
        const float r = __fadd_rn(__fmaf_rn(d, inv, -0.5f), kMagic);
        const float border = __fmaf_rn(__fsub_rn(r, kMagic), s, half);
        bool up = d > border;
        if (d == border) {
            float t2, e2;
            two_diff(x[i], m, t2, e2);
            up = e2 > 0.f || (e2 == 0.f && (__float_as_uint(r) & 1u) != 0u);
        }
        codes |= ((__float_as_uint(r) & 15u) + (up ? 1u : 0u)) << (4 * i);
    }
    if (s < 1e-36f) {
        codes = 0u;
#pragma unroll 1
        for (int i = 0; i < kOctet; ++i) codes |= static_cast<uint32_t>(code_of(x[i], m, s)) << (4 * i);
    }
    return codes;
}

// One block per nugget: 8 features a thread and step, kUnroll steps' loads of both rows in flight.  Bound by HBM: it reads
// the two rows and writes 80 (dh 128) of their 256 bytes a head.
template <typename T>
__global__ void __launch_bounds__(kThreads)
gather_q4_kernel(const unsigned char* __restrict__ K, const unsigned char* __restrict__ V, int H, int dh,
                 const int32_t* __restrict__ idx, const __grid_constant__ GatherGroup g, unsigned char* __restrict__ cache_q4,
                 uint32_t* __restrict__ cache_scale, int32_t* __restrict__ cache_pos, int* __restrict__ dev_status) {
    constexpr int kVecs = kOctet / Vec16<T>::kElems;    // 16-byte loads per octet
    constexpr int kUnroll = 4 / kVecs;
    const int j = g.idx0[0] + static_cast<int>(blockIdx.x);
    int lo = 0, hi = g.nseq;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (g.idx0[mid] <= j) lo = mid; else hi = mid;
    }
    const int b = lo;
    dodo_grid_dependency_sync();   // the indices come from the kernel before
    const int token = __ldg(idx + j);
    if (static_cast<unsigned>(token) >= static_cast<unsigned>(g.n[b])) {
        if (threadIdx.x == 0) atomicOr(dev_status, DODO_DEV_BAD_INDEX);
        return;
    }
    const int octets = H * dh / kOctet, per_head = dh / kOctet;
    const size_t src = (static_cast<size_t>(g.src_row0[b]) + static_cast<size_t>(token)) * static_cast<size_t>(H) * dh * sizeof(T);
    const int dst_row = g.dst_row0[b] + (j - g.idx0[b]);
    uint32_t* const q4 = reinterpret_cast<uint32_t*>(cache_q4 + static_cast<size_t>(dst_row) * H * dh);
    uint32_t* const sc = cache_scale + static_cast<size_t>(dst_row) * H * (2 * dh / kGroup);
    if (threadIdx.x == 0) cache_pos[dst_row] = g.pos_base[b] + token;

    for (int c0 = 0; c0 < octets; c0 += kUnroll * kThreads) {
        uint4 raw[2][kUnroll][kVecs];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int c = c0 + u * kThreads + static_cast<int>(threadIdx.x);
#pragma unroll
            for (int e = 0; e < kVecs; ++e) raw[0][u][e] = raw[1][u][e] = make_uint4(0, 0, 0, 0);
            if (c < octets) {
                const size_t at = src + static_cast<size_t>(c) * kOctet * sizeof(T);
                load_octet<T>(K + at, raw[0][u]);
                load_octet<T>(V + at, raw[1][u]);
            }
        }
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int c = c0 + u * kThreads + static_cast<int>(threadIdx.x);
            const int h = c / per_head, w = c - h * per_head;   // head and word within the head's K (or V) codes
#pragma unroll
            for (int kv = 0; kv < 2; ++kv) {
                float x[kOctet];
#pragma unroll
                for (int e = 0; e < kVecs; ++e) Vec16<T>::unpack(raw[kv][u][e], x + e * Vec16<T>::kElems);
                uint32_t word;
                const uint32_t codes = quantise(x, word);
                if (c < octets) {
                    q4[h * (dh / 4) + kv * (dh / 8) + w] = codes;
                    if ((w & 3) == 0) sc[(h * 2 + kv) * (dh / kGroup) + w / 4] = word;
                }
            }
        }
    }
}

template <typename T> __device__ __forceinline__ void store_octet(T* p, const float* x);
template <> __device__ __forceinline__ void store_octet<float>(float* p, const float* x) {
    reinterpret_cast<float4*>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
}
template <> __device__ __forceinline__ void store_octet<__nv_bfloat16>(__nv_bfloat16* p, const float* x) {
    uint32_t v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
        v[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    *reinterpret_cast<uint4*>(p) = make_uint4(v[0], v[1], v[2], v[3]);
}

// One block per cache row in use: a thread reads one word of codes and its group's word and writes 8 features; m + c s is
// rounded once to fp32 (c s is exact) and, for bf16, once more.  Bound by the HBM writes.
template <typename T>
__global__ void __launch_bounds__(kThreads)
expand_q4_kernel(const unsigned char* __restrict__ cache_q4, const uint32_t* __restrict__ cache_scale, int H, int dh,
                 const __grid_constant__ ExpandGroup g, T* __restrict__ K, T* __restrict__ V) {
    constexpr int kUnroll = 4;
    const int j = static_cast<int>(blockIdx.x);
    int lo = 0, hi = g.nseq;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (g.out0[mid] <= j) lo = mid; else hi = mid;
    }
    const size_t row = static_cast<size_t>(g.row0[lo]) + static_cast<size_t>(j - g.out0[lo]);
    const uint32_t* const q4 = reinterpret_cast<const uint32_t*>(cache_q4 + row * H * dh);
    const uint32_t* const sc = cache_scale + row * H * (2 * dh / kGroup);
    const int words = H * dh / 4, per_kv = dh / 8;     // words of codes of the row: [head][K, V][dh / 8]
    dodo_grid_dependency_sync();
    for (int c0 = 0; c0 < words; c0 += kUnroll * kThreads) {
        uint32_t codes[kUnroll], meta[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int c = c0 + u * kThreads + static_cast<int>(threadIdx.x);
            codes[u] = meta[u] = 0u;
            if (c < words) {
                codes[u] = __ldg(q4 + c);
                meta[u] = __ldg(sc + c / 4);
            }
        }
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
            const int c = c0 + u * kThreads + static_cast<int>(threadIdx.x);
            if (c >= words) break;
            const float s = __uint_as_float(meta[u] << 16), m = __uint_as_float(meta[u] & 0xffff0000u);
            float x[kOctet];
#pragma unroll
            for (int i = 0; i < kOctet; ++i) x[i] = fmaf(static_cast<float>((codes[u] >> (4 * i)) & 15u), s, m);
            const int hk = c / per_kv, w = c - hk * per_kv;   // hk = 2 head + (0 for K, 1 for V)
            T* const out = (hk & 1) != 0 ? V : K;
            store_octet<T>(out + row * H * dh + static_cast<size_t>(hk >> 1) * dh + w * kOctet, x);
        }
    }
}

}  // namespace

int dodo_launch_gather_q4(dodo_ctx* ctx, const void* K, const void* V, int dtype, int H, int dh, const int32_t* idx,
                          const GatherGroup& g, void* cache_q4, uint32_t* cache_scale, int32_t* cache_pos, int* dev_status,
                          cudaStream_t st) {
    const int total = g.idx0[g.nseq] - g.idx0[0];
    if (total == 0) return DODO_OK;
    const unsigned char* k = static_cast<const unsigned char*>(K);
    const unsigned char* v = static_cast<const unsigned char*>(V);
    unsigned char* q4 = static_cast<unsigned char*>(cache_q4);
    const dim3 grid(static_cast<unsigned>(total)), block(kThreads);
    const cudaError_t e = dtype == DODO_BF16
        ? dodo_launch_dependent(gather_q4_kernel<__nv_bfloat16>, grid, block, 0, st, k, v, H, dh, idx, g, q4, cache_scale, cache_pos, dev_status)
        : dodo_launch_dependent(gather_q4_kernel<float>, grid, block, 0, st, k, v, H, dh, idx, g, q4, cache_scale, cache_pos, dev_status);
    return dodo_check_cuda(ctx, e, "4-bit gather launch");
}

int dodo_launch_expand_q4(dodo_ctx* ctx, const void* cache_q4, const uint32_t* cache_scale, int H, int dh, int dtype,
                          const ExpandGroup& g, void* K, void* V, cudaStream_t st) {
    const int total = g.out0[g.nseq];
    if (total == 0) return DODO_OK;
    const unsigned char* q4 = static_cast<const unsigned char*>(cache_q4);
    const dim3 grid(static_cast<unsigned>(total)), block(kThreads);
    const cudaError_t e = dtype == DODO_BF16
        ? dodo_launch_dependent(expand_q4_kernel<__nv_bfloat16>, grid, block, 0, st, q4, cache_scale, H, dh, g,
                                static_cast<__nv_bfloat16*>(K), static_cast<__nv_bfloat16*>(V))
        : dodo_launch_dependent(expand_q4_kernel<float>, grid, block, 0, st, q4, cache_scale, H, dh, g, static_cast<float*>(K),
                                static_cast<float*>(V));
    return dodo_check_cuda(ctx, e, "4-bit expansion launch");
}
