// Nugget cache held in 4 bits: the gather (Eq. 5) that quantises the selected K/V rows on the way into it, and the
// expansion of its rows back to a floating type.
//
// Format.  A row of one head is cut into groups of 32 features.  With lo and hi the group's least and largest value,
//   m = the largest bf16 number <= lo,   s = the least bf16 number with 15 s >= hi - m,
//   c_i = (x_i - m) / s rounded to the nearest whole number, ties to even (0 where s = 0),
// and feature i stands for m + c_i s.  Both roundings go outwards, so every x_i lies in [m, m + 15 s], no code is
// clamped and the error is at most s / 2 for every feature.  The codes are defined on real numbers; the kernel finds
// them in fp32 and decides the few that lie on a border exactly (see quantise).  A group that holds a NaN or an
// infinity, or whose span overflows, is stored as NaN: all of its features read back as NaN.
// Storage: a (row, head) owns dh bytes of codes, K's dh / 2 then V's (feature 2i in the low half of byte i), which is
// one 128-byte line at head size 128, and 2 dh / 32 words, K's then V's, with s in the low and m in the high 16 bits.
#include "dodo_internal.cuh"

namespace {

constexpr int kThreads = 128;
constexpr int kGatherThreads = 64;              // small blocks leave the last wave fuller (4 x 600 fp32 rows of 12 x 64: 9.5 us at 256, 8.2 at 64)
constexpr int kGroup = DODO_Q4_GROUP;
constexpr int kOctet = 8;                       // features per word of codes
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
// Least bf16 s with 15 s >= t + e.  The quotient is off by a few units of fp32, so its bf16 cut is s or one or two steps
// below; 15 s is exact (8 + 4 bits).
__device__ __forceinline__ float step_of(float t, float e) {
    float s = cut_bf16(__fmul_rn(t, 1.f / 15.f));
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

__device__ __forceinline__ float min3(float a, float b, float c) {   // (a NaN stays one)
    float d;
    asm("min.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
    float d;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
__device__ __forceinline__ float rcp_approx(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// 32 bytes, streaming; kWhole: p is a multiple of 32, else of 16
template <bool kWhole>
__device__ __forceinline__ void load32(const unsigned char* p, uint32_t* v) {
    if constexpr (!kWhole) {
        const uint4 a = ld_stream16(p), b = ld_stream16(p + 16);
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
        v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
        return;
    }
    asm volatile("ld.global.nc.L1::no_allocate.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]) : "l"(p));
}
// the storage words of a group as floats
template <typename T> __device__ __forceinline__ void widen(const uint32_t* raw, float* x);
template <> __device__ __forceinline__ void widen<float>(const uint32_t* raw, float* x) {
#pragma unroll
    for (int i = 0; i < kGroup; ++i) x[i] = __uint_as_float(raw[i]);
}
template <> __device__ __forceinline__ void widen<__nv_bfloat16>(const uint32_t* raw, float* x) {
#pragma unroll
    for (int i = 0; i < kGroup / 2; ++i) {
        x[2 * i] = __uint_as_float(raw[i] << 16);
        x[2 * i + 1] = __uint_as_float(raw[i] & 0xffff0000u);
    }
}

// Codes (four words) and group word of 32 features; kWide: they have more than the 8 significant bits of bf16.
template <bool kWide>
__device__ __forceinline__ uint32_t quantise(const float* x, uint32_t* codes) {
    float lo = min3(x[0], x[0], x[1]), hi = max3(x[0], x[0], x[1]);
#pragma unroll
    for (int i = 2; i < kGroup; i += 2) {
        lo = min3(lo, x[i], x[i + 1]);
        hi = max3(hi, x[i], x[i + 1]);
    }
    const float m = bf16_down(lo);
    float t, e;
    two_diff(hi, m, t, e);
#pragma unroll
    for (int w = 0; w < 4; ++w) codes[w] = 0u;
    if (!(t <= kFinite)) return 0x00007fc0u;     // NaN, an infinity or too wide a span: step NaN
    const float s = step_of(t, e);
    const uint32_t word = (__float_as_uint(s) >> 16) | (__float_as_uint(m) & 0xffff0000u);
    // Codes by a reciprocal.  k = round((x - m) / s - 1/2), off by far less than one half, so the code is k or k + 1, by the
    // side of the border (k + 1/2) s that d = x - m lies on; the border is exact in fp32 (5 + 8 bits).  At the border the even
    // code wins: there d >= border is asked for odd k, which on the bits of non-negative floats is d + 1 > border.  k sits in
    // the low bits of r = k + 1.5 * 2^23; the words are summed with those bits' constant part and freed of it at the end.
    const float inv = rcp_approx(s), half = 0.5f * s;
    constexpr float kMagic = 12582912.f;
    constexpr uint32_t kMagicBits = 0x4b400000u;
    const float2 m2 = make_float2(-m, -m), inv2 = make_float2(inv, inv), s2 = make_float2(s, s), half2 = make_float2(half, half);
    const float2 low2 = make_float2(-0.5f, -0.5f), magic2 = make_float2(kMagic, kMagic), back2 = make_float2(-kMagic, -kMagic);
    bool met = false;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        uint32_t c = 0u - kMagicBits * 0x11111111u;
#pragma unroll
        for (int i = 0; i < kOctet; i += 2) {        // two features per instruction
            const float2 d = __fadd2_rn(make_float2(x[w * kOctet + i], x[w * kOctet + i + 1]), m2);
            const float2 r = __fadd2_rn(__ffma2_rn(d, inv2, low2), magic2);
            const float2 border = __ffma2_rn(__fadd2_rn(r, back2), s2, half2);
            const uint32_t r0 = __float_as_uint(r.x), r1 = __float_as_uint(r.y);
            c += r0 << (4 * i);
            c += r1 << (4 * i + 4);
            if (__float_as_uint(d.x) + (r0 & 1u) > __float_as_uint(border.x)) c += 1u << (4 * i);
            if (__float_as_uint(d.y) + (r1 & 1u) > __float_as_uint(border.y)) c += 1u << (4 * i + 4);
            if (kWide) met = met || d.x == border.x || d.y == border.y;
        }
        codes[w] = c;
    }
    // What rounding took from d matters only at a border.  bf16 values of exponents at most 15 apart subtract exactly, so for
    // bf16 rows d is inexact only where |x| < 2^-14 |m|, when d is within 2^-14 of -m and a border has to be as near, or where
    // |m| < 2^-14 |x| (1.3e-4 is above 2 * 2^-14).  fp32 rows look at every feature.  Such groups, and steps without a reciprocal in range, go through code_of.
    const float z = -m * inv, zk = z - floorf(z) - 0.5f;
    bool exactly = s < 1e-36f || (kWide ? met : m != 0.f && fabsf(m) < 1.3e-4f * fabsf(hi));
    if (!kWide && fabsf(zk) < 2e-3f) {
        const float small = 1.3e-4f * fabsf(m);
#pragma unroll
        for (int i = 0; i < kGroup; ++i) exactly = exactly || (fabsf(x[i]) < small && x[i] != 0.f);
    }
    if (exactly) {
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            codes[w] = 0u;
            if (s > 0.f) {       // (s = 0: a constant group)
#pragma unroll
                for (int i = 0; i < kOctet; ++i) codes[w] |= static_cast<uint32_t>(code_of(x[w * kOctet + i], m, s)) << (4 * i);
            }
        }
    }
    return word;
}

// A thread takes one group of 32 features of one nugget's K or V row (bf16: 64 bytes in two 32-byte loads), so a group's
// extremes, step and reciprocal cost it no exchange and are found once; the groups of all nuggets are laid end to end over the
// threads, whatever a row's length.  It reads two rows and writes 80 (dh 128) of their 256 bytes a head, about 16 instructions
// per feature.  8 x 205 nuggets of 32 heads of 128, bf16: 15.8 us (17.1 with one feature per instruction, 24 with an octet per
// thread; dodo_gather_kv takes 10.1 to copy the same rows), bound by issue and by the load's latency, which a thread's single
// group does not cover.
template <typename T, bool kWhole>
__global__ void __launch_bounds__(kGatherThreads, 16)
gather_q4_kernel(const unsigned char* __restrict__ K, const unsigned char* __restrict__ V, int H, int dh,
                 const int32_t* __restrict__ idx, const __grid_constant__ GatherGroup g, unsigned char* __restrict__ cache_q4,
                 uint32_t* __restrict__ cache_scale, int32_t* __restrict__ cache_pos, int* __restrict__ dev_status) {
    constexpr int kWords = kGroup * static_cast<int>(sizeof(T)) / 4;    // storage words of a group
    const int per_head = dh / kGroup, groups = H * per_head;            // of K; as many of V
    const long long item = static_cast<long long>(blockIdx.x) * kGatherThreads + threadIdx.x;
    const int slot = static_cast<int>(item / (2 * groups)), i = static_cast<int>(item - static_cast<long long>(slot) * (2 * groups));
    const int j = g.idx0[0] + slot;
    if (j >= g.idx0[g.nseq]) return;
    int lo = 0, hi = g.nseq;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (g.idx0[mid] <= j) lo = mid; else hi = mid;
    }
    const int b = lo;
    dodo_grid_dependency_sync();   // the indices come from the kernel before
    const int token = __ldg(idx + j);
    if (static_cast<unsigned>(token) >= static_cast<unsigned>(g.n[b])) {
        if (i == 0) atomicOr(dev_status, DODO_DEV_BAD_INDEX);
        return;
    }
    const int kv = i < groups ? 0 : 1, c = i - kv * groups, h = c / per_head;
    const size_t src = ((static_cast<size_t>(g.src_row0[b]) + static_cast<size_t>(token)) * groups + c) * (kWords * 4);
    uint32_t raw[kWords];
#pragma unroll
    for (int w = 0; w < kWords; w += 8) load32<kWhole>((kv == 0 ? K : V) + src + 4 * w, raw + w);
    const int dst_row = g.dst_row0[b] + (j - g.idx0[b]);
    if (i == 0) cache_pos[dst_row] = g.pos_base[b] + token;
    float x[kGroup];
    widen<T>(raw, x);
    uint32_t codes[4];
    const uint32_t word = quantise<sizeof(T) == 4>(x, codes);
    const size_t at = static_cast<size_t>(dst_row) * (2 * groups) + (h * 2 + kv) * per_head + (c - h * per_head);
    reinterpret_cast<uint4*>(cache_q4)[at] = make_uint4(codes[0], codes[1], codes[2], codes[3]);
    cache_scale[at] = word;
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
    const long long items = static_cast<long long>(total) * 2 * H * (dh / kGroup);
    const dim3 grid(static_cast<unsigned>((items + kGatherThreads - 1) / kGatherThreads)), block(kGatherThreads);
    const bool whole = ((reinterpret_cast<uintptr_t>(K) | reinterpret_cast<uintptr_t>(V)) & 31u) == 0u;      // (rows are multiples of 128 bytes)
    auto kern = dtype == DODO_BF16 ? (whole ? gather_q4_kernel<__nv_bfloat16, true> : gather_q4_kernel<__nv_bfloat16, false>)
                                   : (whole ? gather_q4_kernel<float, true> : gather_q4_kernel<float, false>);
    const cudaError_t e = dodo_launch_dependent(kern, grid, block, 0, st, k, v, H, dh, idx, g, q4, cache_scale, cache_pos, dev_status);
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
