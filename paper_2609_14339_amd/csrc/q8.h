// Device code that the norm, the linear layers and the checkpoints share:
// eight-column accesses, activation functions, and the 8-bit checkpoint's
// coding of one group.
#pragma once

#include "common.h"

#include <algorithm>

namespace acsc {

constexpr int kGroup = ACSC_Q8_GROUP;

// The checkpoint descriptor as kernels take it (codes == nullptr: none).
struct Q8 {
    int8_t *codes;
    float *scales;
    int64_t ldc, lds;
};

inline Q8 q8_of(const q8_tensor *q)
{
    return q ? Q8{q->codes, q->scales, q->ld_codes, q->ld_scales} : Q8{nullptr, nullptr, 0, 0};
}

// Host checks of a checkpoint of a [rows, H] tensor.
inline int check_q8(const q8_tensor *q, int64_t rows, int H)
{
    ACSC_CHECK_ARG(rows == 0 || (q->codes && q->scales), ACSC_EINVAL, "null pointer in the checkpoint");
    ACSC_CHECK_ARG(q->ld_codes >= H, ACSC_EINVAL, "ld_codes=%lld < H=%d", (long long)q->ld_codes, H);
    ACSC_CHECK_ARG(q->ld_scales >= (H + kGroup - 1) / kGroup, ACSC_EINVAL, "ld_scales=%lld < %d groups",
                   (long long)q->ld_scales, (H + kGroup - 1) / kGroup);
    ACSC_CHECK_ARG(aligned(q->scales, 4), ACSC_EALIGN, "scales not 4-byte aligned");
    return ACSC_OK;
}

inline int check_act(int act)
{
    ACSC_CHECK_ARG(act >= ACSC_ACT_NONE && act <= ACSC_ACT_SILU, ACSC_EINVAL, "unknown activation %d", act);
    return ACSC_OK;
}

struct __attribute__((packed, aligned(1))) C8Any {
    uint32_t w[2];
};

// Eight consecutive elements as floats; only the first nv are read (the rest
// become 0).  Whole chunks are 16-byte accesses at any element's alignment.
__device__ __forceinline__ void load8(const uint16_t *p, int nv, float (&v)[8])
{
    if (nv >= 8) {
        const Bf8Any c = *reinterpret_cast<const Bf8Any *>(p);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float(c.w[i] << 16);
            v[2 * i + 1] = __uint_as_float(c.w[i] & 0xffff0000u);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            v[i] = i < nv ? bf16_to_f32(p[i]) : 0.f;
    }
}
// (Both ways end in the same two values: stores to v in each left v in memory,
// and layer norms of fp32 rows at 1.9 TB/s.)
__device__ __forceinline__ void load8(const float *p, int nv, float (&v)[8])
{
    F4Any a = {}, b = {};
    if (nv >= 8) {
        a = *reinterpret_cast<const F4Any *>(p);
        b = *reinterpret_cast<const F4Any *>(p + 4);
    } else if (nv > 0) {
        // taken as new, so that no loop keeps its eight comparisons at hand
        asm volatile("" : "+v"(nv));
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            a.v[i] = i < nv ? p[i] : 0.f;
            b.v[i] = i + 4 < nv ? p[i + 4] : 0.f;
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[i] = a.v[i];
        v[4 + i] = b.v[i];
    }
}
__device__ __forceinline__ void store8(uint16_t *p, int nv, const float (&v)[8])
{
    if (nv >= 8) {
        Bf8Any c;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            c.w[i] = f32x2_to_bf16x2(v[2 * i], v[2 * i + 1]);
        *reinterpret_cast<Bf8Any *>(p) = c;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < nv)
                p[i] = f32_to_bf16(v[i]);
    }
}
__device__ __forceinline__ void store8(float *p, int nv, const float (&v)[8])
{
    if (nv >= 8) {
        F4Any a, b;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            a.v[i] = v[i];
            b.v[i] = v[4 + i];
        }
        *reinterpret_cast<F4Any *>(p) = a;
        *reinterpret_cast<F4Any *>(p + 4) = b;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < nv)
                p[i] = v[i];
    }
}

// A code's value, rounded once as the format asks: not contracted into what
// it is added to.
__device__ __forceinline__ float code_value(float code, float scale)
{
#pragma clang fp contract(off)
    return code * scale;
}

// Eight consecutive elements or codes as they are stored; those past the
// first nv are 0.
template <typename T>
struct Raw8;
template <>
struct Raw8<uint16_t> {
    uint32_t w[4];
    __device__ __forceinline__ float at(int i) const
    {
        return __uint_as_float(i & 1 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
    }
};
template <>
struct Raw8<float> {
    float w[8];
    __device__ __forceinline__ float at(int i) const { return w[i]; }
};
struct Codes8 {
    uint32_t w[2];
    __device__ __forceinline__ float at(int i) const
    {
        return static_cast<float>(static_cast<int8_t>(w[i / 4] >> (8 * (i % 4))));
    }
};
__device__ __forceinline__ void load_raw(const uint16_t *p, int nv, Raw8<uint16_t> &r)
{
    if (nv >= 8) {
        const Bf8Any c = *reinterpret_cast<const Bf8Any *>(p);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            r.w[i] = c.w[i];
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            r.w[i] = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < nv)
                r.w[i / 2] |= static_cast<uint32_t>(p[i]) << (16 * (i & 1));
    }
}
__device__ __forceinline__ void load_raw(const float *p, int nv, Raw8<float> &r) { load8(p, nv, r.w); }
__device__ __forceinline__ void load_raw(const int8_t *p, int nv, Codes8 &r)
{
    if (nv >= 8) {
        const C8Any c = *reinterpret_cast<const C8Any *>(p);
        r.w[0] = c.w[0];
        r.w[1] = c.w[1];
    } else {
        r.w[0] = r.w[1] = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < nv)
                r.w[i / 4] |= (static_cast<uint32_t>(p[i]) & 0xffu) << (8 * (i % 4));
    }
}

// Values of eight consecutive codes under one scale.
__device__ __forceinline__ void load_codes(const int8_t *p, int nv, float scale, float (&v)[8])
{
    if (nv >= 8) {
        const C8Any c = *reinterpret_cast<const C8Any *>(p);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            v[i] = code_value(static_cast<float>(static_cast<int8_t>(c.w[i / 4] >> (8 * (i % 4)))), scale);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            v[i] = i < nv ? code_value(static_cast<float>(p[i]), scale) : 0.f;
    }
}

// A group's largest magnitude is found as the maximum of its values' bits
// without the sign: that order puts NaN above infinity above every number.
__device__ __forceinline__ uint32_t mag(float x) { return __float_as_uint(x) & 0x7fffffffu; }

// scale = a / 127 and inv = 127 / a of a group whose largest magnitude has the
// bits a.  A group below 2^-120 (127 / a would leave fp32's range not far
// below) is kept as zeros; one with an infinity or NaN reads as NaN.
__device__ __forceinline__ void group_scale(uint32_t a, float &scale, float &inv)
{
    if (a >= 0x7f800000u) {
        scale = __uint_as_float(0x7fc00000u);
        inv = 0.f;
    } else if (a < 0x03800000u) {   // 2^-120
        scale = inv = 0.f;
    } else {
        const float f = __uint_as_float(a);
        if (a - 0x0d800000u < 0x64000000u) {   // 2^-100 <= a < 2^100: nothing under- or overflows
            // Quotients by one residual step from a reciprocal: rounded as the
            // divisions below are, for every 24-bit significand of a (checked
            // over all 2^23 of them, with the hardware's reciprocal one unit
            // off either way).
            constexpr float r127 = 1.f / 127.f;
            scale = f * r127;
            scale = __builtin_fmaf(__builtin_fmaf(-127.f, scale, f), r127, scale);
            float y = __builtin_amdgcn_rcpf(f);
            y = __builtin_fmaf(__builtin_fmaf(-f, y, 1.f), y, y);
            inv = 127.f * y;
            inv = __builtin_fmaf(__builtin_fmaf(-f, inv, 127.f), y, inv);
        } else {
            scale = f / 127.f;
            inv = 127.f / f;
        }
    }
}

// Codes of eight values: rint(x * inv), in -127 .. 127 because |x| <= a makes
// |x * inv| round to at most 127 (1 + 2^-23).  Adding 1.5 * 2^23 rounds to a
// whole number, ties to even, whose low byte is the code; the product is
// rounded before that, as the format asks (no contraction).  inv = 0 gives
// zeros, for the non-finite values of a NaN group too.
__device__ __forceinline__ void store_codes(int8_t *p, int nv, float inv, const float (&v)[8])
{
#pragma clang fp contract(off)
    uint32_t w[2];
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        uint32_t b[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float t = v[4 * q + i] * inv;
            b[i] = __float_as_uint(t + 12582912.f);
        }
        const uint32_t lo = __builtin_amdgcn_perm(b[1], b[0], 0x0c0c0400), hi = __builtin_amdgcn_perm(b[3], b[2], 0x04000c0c);
        w[q] = inv == 0.f ? 0u : lo | hi;
    }
    if (nv >= 8) {
        *reinterpret_cast<C8Any *>(p) = C8Any{{w[0], w[1]}};
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < nv)
                p[i] = static_cast<int8_t>(w[i / 4] >> (8 * (i % 4)));
    }
}

// Maximum over the 16 lanes of a row of the wave, in every lane (row_ror).
__device__ __forceinline__ uint32_t max16(uint32_t x)
{
#define ACSC_ROR(n) x = max(x, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(x), 0x120 + n, 0xF, 0xF, false)))
    ACSC_ROR(8);
    ACSC_ROR(4);
    ACSC_ROR(2);
    ACSC_ROR(1);
#undef ACSC_ROR
    return x;
}

// act(z) and act'(z).  gelu(z) = z Phi(z), gelu'(z) = Phi(z) + z phi(z);
// silu(z) = z s, silu'(z) = s (1 + z (1 - s)), s = 1 / (1 + exp(-z)), with
// s and 1 - s both from exp(-|z|), so that neither is a difference.
//
// T is the type that the result is rounded to.  Phi is formed from its tail
// q = Phi(-|z|), as q or 1 - q, so that it keeps its relative accuracy where it
// is small.
//
// bf16 (half a unit: 2^-8): q = (a1 t + .. + a5 t^5) exp(-z^2 / 2) / 2,
// t = 1 / (1 + p |z| / sqrt 2) (Abramowitz & Stegun, Handbook of Mathematical
// Functions, 7.1.26: within 0.75e-7), and exponentials and reciprocals are the
// hardware's (one unit of 2^-23): a dozen instructions in epilogues that
// nothing hides (see the forward product's figures).
//
// fp32: q = p(t) exp(-z^2 / 2) / (|z| + 4), t = (|z| - 4) / (|z| + 4), p the
// polynomial of degree 9 that interpolates (x + 4) Phi(-x) exp(x^2 / 2) at the
// Chebyshev points of t in -1 .. 1 (within 4e-8 of it, relative): q within 7 +
// 1.2 z^2 units of 2^-24 of itself, 3 of 1 near 0; 0 from about -13.2 on, where
// it leaves the normal range.  Decoding 8192 x 28672 through gelu takes 356 us;
// by the library's erfc, as accurate, 435; by 1 + erf, which has lost 4% of Phi
// at -5 and all of it at -6, 352.
template <typename T>
__device__ __forceinline__ float normal_tail(float z, float &e)
{
    if (sizeof(T) == 4) {
        const float x = fminf(fabsf(z), 64.f), d = x + 4.f;
        float r = __builtin_amdgcn_rcpf(d);
        r = __builtin_fmaf(__builtin_fmaf(-d, r, 1.f), r, r);
        const float t = __builtin_fmaf(-8.f, r, 1.f);
        e = __builtin_amdgcn_exp2f(-0.72134752044448170f * x * x);
        float q = -0.000162616314f;
        q = __builtin_fmaf(q, t, 0.000129340129f);
        q = __builtin_fmaf(q, t, 0.00157575205f);
        q = __builtin_fmaf(q, t, -0.00347619643f);
        q = __builtin_fmaf(q, t, -0.00752125541f);
        q = __builtin_fmaf(q, t, 0.0603953153f);
        q = __builtin_fmaf(q, t, -0.186524183f);
        q = __builtin_fmaf(q, t, 0.387137562f);
        q = __builtin_fmaf(q, t, -0.607896566f);
        q = __builtin_fmaf(q, t, 0.755285144f);
        return q * r * e;
    }
    const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.3275911f * 0.70710678118654752f, fabsf(z), 1.f));
    e = __builtin_amdgcn_exp2f(-0.72134752044448170f * z * z);
    float q = 0.5f * 1.061405429f;
    q = __builtin_fmaf(q, t, 0.5f * -1.453152027f);
    q = __builtin_fmaf(q, t, 0.5f * 1.421413741f);
    q = __builtin_fmaf(q, t, 0.5f * -0.284496736f);
    q = __builtin_fmaf(q, t, 0.5f * 0.254829592f);
    return q * (t * e);
}
// s and 1 - s
template <typename T>
__device__ __forceinline__ void sigmoid(float z, float &s, float &c)
{
    const float e = sizeof(T) == 4 ? expf(-fabsf(z)) : __builtin_amdgcn_exp2f(-1.4426950408889634f * fabsf(z));
    const float r = sizeof(T) == 4 ? 1.f / (1.f + e) : __builtin_amdgcn_rcpf(1.f + e);
    s = z < 0.f ? e * r : r;
    c = z < 0.f ? r : e * r;
}
template <typename T>
__device__ __forceinline__ float act_value(float z, int act)
{
    if (act == ACSC_ACT_RELU)
        return z > 0.f ? z : (z != z ? z : 0.f);
    if (act == ACSC_ACT_GELU) {
        float e;
        const float q = normal_tail<T>(z, e);
        // past 64 q is 0, and infinity times it would be NaN
        return __builtin_fmaf(-fabsf(z > 64.f ? 64.f : z), q, z < 0.f ? 0.f : z);
    }
    if (act == ACSC_ACT_SILU) {
        float s, c;
        sigmoid<T>(z, s, c);
        return z * s;
    }
    return z;
}
template <typename T>
__device__ __forceinline__ float act_slope(float z, int act)
{
    if (act == ACSC_ACT_RELU)
        return z > 0.f ? 1.f : (z != z ? z : 0.f);
    if (act == ACSC_ACT_GELU) {
        float e;
        const float q = normal_tail<T>(z, e);
        return __builtin_fmaf(z * 0.39894228040143268f, e, z < 0.f ? q : 1.f - q);
    }
    if (act == ACSC_ACT_SILU) {
        float s, c;
        sigmoid<T>(z, s, c);
        return s * __builtin_fmaf(z, c, 1.f);
    }
    return 1.f;
}

// Eight values at a time: one branch on the function, not one a value.
template <typename T>
__device__ __forceinline__ void apply_act(float (&v)[8], int act)
{
    const auto each = [&](int a) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            v[i] = act_value<T>(v[i], a);
    };
    if (act == ACSC_ACT_GELU)
        each(ACSC_ACT_GELU);
    else if (act == ACSC_ACT_SILU)
        each(ACSC_ACT_SILU);
    else if (act == ACSC_ACT_RELU)
        each(ACSC_ACT_RELU);
}
template <typename T>
__device__ __forceinline__ void apply_slope(float (&v)[8], const float (&z)[8], int act)
{
    const auto each = [&](int a) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            v[i] *= act_slope<T>(z[i], a);
    };
    if (act == ACSC_ACT_GELU)
        each(ACSC_ACT_GELU);
    else if (act == ACSC_ACT_SILU)
        each(ACSC_ACT_SILU);
    else if (act == ACSC_ACT_RELU)
        each(ACSC_ACT_RELU);
}

}  // namespace acsc
