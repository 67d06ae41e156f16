// Rotary positions: the device side shared by the rotation of whole arrays and by the paged append.
//
// The angle of a pair at a position is kept as a fraction of a turn in 64 bits: position x turn[i] modulo 2^64 is one integer
// product that loses nothing but what the frequency's rounding to 64 bits did (two's complement covers negative positions), where a float angle
// has lost 17 bits at 100,000 tokens.  Rounded to 32 bits (2^-33 turns) it gives the quarter turn and a remainder within an eighth of a turn,
// whose sine and cosine are their Taylor series (degrees 9 and 10 on [-pi/4, pi/4]: 2e-9 off, below fp32's rounding).
#pragma once

#include "dodo_internal.cuh"

namespace dodo_rotary {

struct Rotation {
    int half;               // pairs that are turned
    float scale;            // with the sign of the angle in `sign`: -1 turns back (the gradient)
    float sign;
    unsigned long long turn[DODO_ROPE_MAX / 2];
};

// (cos, sin) of the angle of pair i at a position, times the scale
__device__ __forceinline__ float2 cos_sin(const Rotation& p, int i, int pos) {
    const unsigned long long phase = static_cast<unsigned long long>(static_cast<long long>(pos)) * p.turn[i];
    const uint32_t t = static_cast<uint32_t>((phase + 0x80000000ull) >> 32), q = (t + 0x20000000u) >> 30;      // rounded; a whole turn is none
    const float a = static_cast<float>(static_cast<int>(t - (q << 30))) * 1.46291807926715968e-9f;    // 2 pi / 2^32
    const float b = a * a;
    const float s = fmaf(a * b, fmaf(b, fmaf(b, fmaf(b, 1.f / 362880.f, -1.f / 5040.f), 1.f / 120.f), -1.f / 6.f), a);
    const float c = fmaf(b, fmaf(b, fmaf(b, fmaf(b, fmaf(b, -1.f / 3628800.f, 1.f / 40320.f), -1.f / 720.f), 1.f / 24.f), -0.5f), 1.f);
    float co = (q & 1u) ? s : c, si = (q & 1u) ? c : s;
    if (((q + 1u) & 2u) != 0u) co = -co;      // quarters 1 and 2
    if ((q & 2u) != 0u) si = -si;             // quarters 2 and 3
    return make_float2(co * p.scale, si * (p.scale * p.sign));
}

// VEC elements of T as floats; 16 bytes at once, or one by one where alignment allows no more
template <typename T, int VEC>
struct Piece {
    static constexpr bool kWide = VEC * sizeof(T) == 16;
    uint4 raw;
    T one[kWide ? 1 : VEC];
    __device__ __forceinline__ void load(const T* p) {
        if constexpr (kWide) {
            // (not the read-only path: a rotation may work in place)
            asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(raw.x), "=r"(raw.y), "=r"(raw.z), "=r"(raw.w) : "l"(p) : "memory");
        } else {
#pragma unroll
            for (int e = 0; e < VEC; ++e) one[e] = p[e];
        }
    }
    __device__ __forceinline__ void floats(float* f) const {
        if constexpr (kWide) {
            Vec16<T>::unpack(raw, f);
        } else {
#pragma unroll
            for (int e = 0; e < VEC; ++e) f[e] = static_cast<float>(one[e]);
        }
    }
    static __device__ __forceinline__ void store(T* p, const float* f) {
        if constexpr (kWide && sizeof(T) == 4) {
            *reinterpret_cast<float4*>(p) = make_float4(f[0], f[1], f[2], f[3]);
        } else if constexpr (kWide) {
            uint32_t w[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const __nv_bfloat162 v = __floats2bfloat162_rn(f[2 * e], f[2 * e + 1]);
                w[e] = *reinterpret_cast<const uint32_t*>(&v);
            }
            *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
        } else {
#pragma unroll
            for (int e = 0; e < VEC; ++e) p[e] = static_cast<T>(f[e]);
        }
    }
    __device__ __forceinline__ void copy_to(T* p) const {
        if constexpr (kWide) {
            *reinterpret_cast<uint4*>(p) = raw;
        } else {
#pragma unroll
            for (int e = 0; e < VEC; ++e) p[e] = one[e];
        }
    }
};

// A head is cut into slots, one thread's work: in the half layout VEC pairs (two pieces half a rotation apart), then pieces that
// are only copied; in the interleaved one pieces of neighbouring pairs.
template <int VEC, bool INTER>
__host__ __device__ inline int slots_of(int dh, int half) { return INTER ? dh / VEC : half / VEC + (dh - 2 * half) / VEC; }

template <typename T, int VEC, bool INTER>
struct Slot {
    Piece<T, VEC> a, b;
    __device__ __forceinline__ void load(const T* head, int slot, int half) {
        if constexpr (INTER) {
            a.load(head + slot * VEC);
        } else {
            const int pairs = half / VEC;
            if (slot < pairs) {
                a.load(head + slot * VEC);
                b.load(head + half + slot * VEC);
            } else {
                a.load(head + 2 * half + (slot - pairs) * VEC);
            }
        }
    }
    // cs: cosines and sines of the token's pairs, in shared memory
    __device__ __forceinline__ void store(T* head, int slot, int half, const float2* cs) const {
        if constexpr (INTER) {
            const int p0 = slot * (VEC / 2);
            if (p0 >= half) { a.copy_to(head + slot * VEC); return; }
            float x[VEC], y[VEC];
            a.floats(x);
#pragma unroll
            for (int e = 0; e < VEC / 2; ++e) {
                const bool in = p0 + e < half;
                const float2 r = in ? cs[p0 + e] : make_float2(1.f, 0.f);
                y[2 * e] = in ? fmaf(x[2 * e], r.x, -x[2 * e + 1] * r.y) : x[2 * e];
                y[2 * e + 1] = in ? fmaf(x[2 * e], r.y, x[2 * e + 1] * r.x) : x[2 * e + 1];
            }
            Piece<T, VEC>::store(head + slot * VEC, y);
        } else {
            const int pairs = half / VEC;
            if (slot >= pairs) { a.copy_to(head + 2 * half + (slot - pairs) * VEC); return; }
            float x[VEC], y[VEC], u[VEC], v[VEC];
            a.floats(x);
            b.floats(y);
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                const float2 r = cs[slot * VEC + e];
                u[e] = fmaf(x[e], r.x, -y[e] * r.y);
                v[e] = fmaf(x[e], r.y, y[e] * r.x);
            }
            Piece<T, VEC>::store(head + slot * VEC, u);
            Piece<T, VEC>::store(head + half + slot * VEC, v);
        }
    }
};

// Whether pieces of 16 bytes fit a head of this size and rotation (addresses and strides are the caller's to check)
inline bool wide_fits(int dtype, int layout, int dh, int rot) {
    const int vec = dtype == DODO_F32 ? 4 : 8;
    return dh % vec == 0 && (layout == DODO_ROPE_INTERLEAVED || ((rot / 2) % vec == 0 && rot % vec == 0));
}

}  // namespace dodo_rotary

int dodo_check_paged(dodo_ctx* ctx, const dodo_paged_cache* c, const int32_t* page_off, const int32_t* cache_len, int B, bool rows);
int dodo_check_rope(dodo_ctx* ctx, const dodo_rope_spec* rope, int dh);
dodo_rotary::Rotation dodo_rotation(const dodo_rope_spec* rope, bool back);
