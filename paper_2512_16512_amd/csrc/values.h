// Element types of the normalisation and 8-bit kernels: groups of eight
// consecutive values as floats, from and to rows at any element boundary, and
// the conversion to e4m3.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace xtc {

struct Bf16 {
    unsigned short bits;
};

__device__ __forceinline__ float widen(Bf16 v) { return __uint_as_float((unsigned)v.bits << 16); }
__device__ __forceinline__ float widen(float v) { return v; }
// round to nearest even; a NaN stays one
__device__ __forceinline__ void narrow(float v, Bf16 *p) {
    p->bits = __builtin_bit_cast(unsigned short, (__bf16)v);
}
__device__ __forceinline__ void narrow(float v, float *p) { *p = v; }

// Eight consecutive values as they lie in memory.
template <typename T>
struct Raw8 {
    T v[8];
    __device__ __forceinline__ float at(int i) const { return widen(v[i]); }
};
// Whole groups are read with 16-byte loads, which the memory pipeline takes at
// any address; of one that ends inside, or past the row's end, zeros stand for
// the rest.
template <typename T>
__device__ __forceinline__ Raw8<T> raw8(const T *p, int valid) {
    Raw8<T> r;
    if (valid >= 8) {
        __builtin_memcpy(r.v, p, sizeof(r.v));
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            r.v[i] = T{};
            if (i < valid) r.v[i] = p[i];
        }
    }
    return r;
}

// Values p[0 .. 7], zeros from `valid` on.  Whole groups are read with 16-byte
// loads, which the memory pipeline takes at any address.
template <typename T>
__device__ __forceinline__ void load8(const T *p, int valid, float (&v)[8]) {
    T t[8];
    if (valid >= 8) {
        __builtin_memcpy(t, p, sizeof(t));
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = widen(t[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < valid ? widen(p[i]) : 0.f;
    }
}

template <typename T>
__device__ __forceinline__ void store8(T *p, int valid, const float (&v)[8]) {
    T t[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) narrow(v[i], &t[i]);
    if (valid >= 8) {
        __builtin_memcpy(p, t, sizeof(t));
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < valid) p[i] = t[i];
    }
}

// store8 and raw8 of values that nothing reads (or read) soon: past the caches.
template <typename T>
__device__ __forceinline__ void store8_past(T *p, int valid, const float (&v)[8]) {
    typedef unsigned u32x4s __attribute__((ext_vector_type(4), aligned(2)));
    T t[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) narrow(v[i], &t[i]);
    if (valid >= 8) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(t) / 16; ++i) {
            u32x4s q;
            __builtin_memcpy(&q, reinterpret_cast<unsigned char *>(t) + 16 * i, 16);
            __builtin_nontemporal_store(q, reinterpret_cast<u32x4s *>(p) + i);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < valid) p[i] = t[i];
    }
}
// Whether rows begin at 16 bytes: whole lines leave past the caches, pieces of lines had better meet there.
inline bool whole_lines(const void *p, int64_t ld, int64_t bytes) {
    return (reinterpret_cast<uintptr_t>(p) & 15) == 0 && ld * bytes % 16 == 0;
}
template <typename T>
__device__ __forceinline__ void store8_to(T *p, int valid, const float (&v)[8], int past) {
    if (past) store8_past(p, valid, v);
    else store8(p, valid, v);
}
template <typename T>
__device__ __forceinline__ Raw8<T> raw8_once(const T *p, int valid) {
    typedef unsigned u32x4s __attribute__((ext_vector_type(4), aligned(2)));
    Raw8<T> r;
    if (valid >= 8) {
#pragma unroll
        for (int i = 0; i < (int)sizeof(r.v) / 16; ++i) {
            const u32x4s q = __builtin_nontemporal_load(reinterpret_cast<const u32x4s *>(p) + i);
            __builtin_memcpy(reinterpret_cast<unsigned char *>(r.v) + 16 * i, &q, 16);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            r.v[i] = T{};
            if (i < valid) r.v[i] = p[i];
        }
    }
    return r;
}

constexpr float kFp8Most = 448.f;                 // largest e4m3 value
constexpr float kFp8Tiny = 1.17549435e-38f;       // least scale: 2^-126, whose reciprocal is finite

__device__ __forceinline__ float finite_abs(float v) {
    const float a = __builtin_fabsf(v);
    return a < __builtin_inff() ? a : 0.f;        // (a NaN compares false)
}

// Scale of a block whose largest finite magnitude is `amax`.  A true division: the product with 1/448
// would round twice.
__device__ __forceinline__ float fp8_scale(float amax) {
    const float s = amax / kFp8Most;
    return s > kFp8Tiny ? s : kFp8Tiny;
}

// Eight e4m3 values v / scale in memory order (round to nearest even; what is not finite becomes NaN).
// The quotient is the true one: a product with 1/scale, corrected by its remainder, since bf16 values
// meet ties between e4m3 values often (by the product alone one value in a hundred went the other way).
// |v| / scale is at most 448 up to a rounding, far below 464, from where it would no longer round to 448.
__device__ __forceinline__ uint2 to_fp8(const float (&v)[8], float scale) {
    const float inv = 1.f / scale;
    float t[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float q = v[i] * inv;
        const float exact = __builtin_fmaf(__builtin_fmaf(-q, scale, v[i]), inv, q);
        t[i] = __builtin_fabsf(v[i]) < __builtin_inff() ? exact : __builtin_nanf("");
    }
    int lo = __builtin_amdgcn_cvt_pk_fp8_f32(t[0], t[1], 0, false);
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(t[2], t[3], lo, true);
    int hi = __builtin_amdgcn_cvt_pk_fp8_f32(t[4], t[5], 0, false);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(t[6], t[7], hi, true);
    return make_uint2((unsigned)lo, (unsigned)hi);
}

__device__ __forceinline__ void store_fp8(uint8_t *p, int valid, uint2 q) {
    if (valid >= 8) {
        __builtin_memcpy(p, &q, 8);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < valid) p[i] = (uint8_t)((i < 4 ? q.x : q.y) >> (8 * (i & 3)));
    }
}

// Largest and sum over the 2^n neighbouring lanes `span` counts, in all of them.
template <int SPAN>
__device__ __forceinline__ float lanes_max(float v) {
#pragma unroll
    for (int d = 1; d < SPAN; d *= 2) v = fmaxf(v, __shfl_xor(v, d, 64));
    return v;
}
template <int SPAN>
__device__ __forceinline__ float lanes_sum(float v) {
#pragma unroll
    for (int d = 1; d < SPAN; d *= 2) v += __shfl_xor(v, d, 64);
    return v;
}

}  // namespace xtc
