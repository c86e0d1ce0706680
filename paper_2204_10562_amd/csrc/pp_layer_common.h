// What the layer operators (include/pp_layer.h) share: types, loads and stores of eight values,
// blocks of 32 and their scales.
#pragma once

#include "pp_common.h"
#include "pp_layer.h"

#define PP_BLOCK 32
#define PP_GROUP 128
#define PP_GROUP_CODES8 128  // bytes of a group's codes
#define PP_GROUP_CODES4 64

static inline int64_t pp_groups(int64_t cols) { return (cols + PP_GROUP - 1) / PP_GROUP; }
static inline int pp_type_size(int type) { return type == PP_TYPE_F32 ? 4 : 2; }

// Host checks: a matrix operand and a packed one (nothing of theirs is read where there are no rows).
static inline bool pp_bad_matrix(const void *p, int type, int64_t rows, int64_t cols, int64_t ld) {
    return rows && (!p || ((uintptr_t)p & (pp_type_size(type) - 1)) || (rows > 1 && ld < cols));
}
static inline bool pp_bad_packed(const void *codes, const void *scales, int64_t rows) {
    return rows && (!codes || !scales || ((uintptr_t)codes & 15) || ((uintptr_t)scales & 15));
}
static inline bool pp_bad_sizes(int type, int64_t rows, int64_t cols) {
    return type < PP_TYPE_F32 || type > PP_TYPE_BF16 || rows < 0 || rows > PP_LAYER_MAX_ROWS || cols < 1 ||
           cols > PP_LAYER_MAX_COLS;
}

typedef __bf16 pp_bf2 __attribute__((ext_vector_type(2)));
typedef float pp_f2 __attribute__((ext_vector_type(2)));
typedef float pp_f4 __attribute__((ext_vector_type(4)));
typedef int pp_i4 __attribute__((ext_vector_type(4)));
typedef unsigned pp_u2 __attribute__((ext_vector_type(2)));
typedef unsigned pp_u4 __attribute__((ext_vector_type(4)));
typedef unsigned short pp_us2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ float pp_bits(unsigned u) { return __builtin_bit_cast(float, u); }
__device__ __forceinline__ unsigned pp_bits(float f) { return __builtin_bit_cast(unsigned, f); }

// 16 bytes at an address that is a multiple of A only (the hardware takes any)
template <int A> struct pp_any16 { pp_u4 v __attribute__((packed, aligned(A))); };

struct PpF32 {
    typedef float T;
    static __device__ __forceinline__ float get(T x) { return x; }
    static __device__ __forceinline__ T put(float x) { return x; }
};
struct PpF16 {
    typedef _Float16 T;
    static __device__ __forceinline__ float get(T x) { return (float)x; }
    static __device__ __forceinline__ T put(float x) { return (T)x; }
};
struct PpBF16 {
    typedef __bf16 T;
    static __device__ __forceinline__ float get(T x) { return (float)x; }
    static __device__ __forceinline__ T put(float x) { return (T)x; }
};

// Eight neighbours as they lie in memory: 16 bytes of a 16-bit type, 32 of float.
template <class Y> struct PpRaw {
    static const int W = sizeof(typename Y::T) / 2;
    pp_u4 w[W];
};

// n (at most 8) values from p on, zeros behind them
template <class Y> __device__ __forceinline__ PpRaw<Y> pp_load8(const typename Y::T *p, long long n) {
    typedef typename Y::T T;
    PpRaw<Y> r;
    if (n >= 8) {
#pragma unroll
        for (int i = 0; i < PpRaw<Y>::W; ++i) r.w[i] = ((const pp_any16<sizeof(T)> *)p)[i].v;
    } else {
        T t[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) t[i] = i < n ? p[i] : (T)0.0f;
        __builtin_memcpy(&r, t, sizeof(r));
    }
    return r;
}

template <class Y> __device__ __forceinline__ void pp_values(const PpRaw<Y> &r, float *v) {
    typename Y::T t[8];
    __builtin_memcpy(t, &r, sizeof(r));
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = Y::get(t[i]);
}

// max |v| of eight values as the bits of a float: NaN above infinity above the numbers
template <class Y> __device__ __forceinline__ unsigned pp_absmax(const PpRaw<Y> &r, const float *v) {
    unsigned m = 0;
    if constexpr (sizeof(typename Y::T) == 2) {  // two at a time: 16-bit floats order like whole numbers too
        pp_us2 a = __builtin_bit_cast(pp_us2, r.w[0][0] & 0x7fff7fffu);
#pragma unroll
        for (int i = 1; i < 4; ++i) a = __builtin_elementwise_max(a, __builtin_bit_cast(pp_us2, r.w[0][i] & 0x7fff7fffu));
        const unsigned short b = a[0] > a[1] ? a[0] : a[1];
        m = pp_bits(Y::get(__builtin_bit_cast(typename Y::T, b)));
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const unsigned b = pp_bits(v[i]) & 0x7fffffffu;
            m = b > m ? b : m;
        }
    }
    return m;
}

template <class Y> __device__ __forceinline__ void pp_store8(typename Y::T *p, long long n, const float *v) {
    typedef typename Y::T T;
    T t[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) t[i] = Y::put(v[i]);
    if (n >= 8) {
        PpRaw<Y> r;
        __builtin_memcpy(&r, t, sizeof(r));
#pragma unroll
        for (int i = 0; i < PpRaw<Y>::W; ++i) ((pp_any16<sizeof(T)> *)p)[i].v = r.w[i];
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) p[i] = t[i];
    }
}

// the largest of the four lanes of a quad
__device__ __forceinline__ unsigned pp_quad_max(unsigned m) {
    const unsigned a = __builtin_amdgcn_update_dpp(0, m, 0xB1, 0xf, 0xf, true);  // lanes 1 0 3 2
    m = a > m ? a : m;
    const unsigned b = __builtin_amdgcn_update_dpp(0, m, 0x4E, 0xf, 0xf, true);  // lanes 2 3 0 1
    return b > m ? b : m;
}

// 2^(byte - 133): what an 8-bit code of 1 stands for; 255: NaN
__device__ __forceinline__ float pp_unit8(unsigned byte) {
    const unsigned b = byte >= 7 ? (byte - 6) << 23 : 1u << (byte + 16);
    return pp_bits(byte == 255 ? 0x7fc00000u : b);
}
// 2^(byte - 127): the scale of a 4-bit block; 255: NaN
__device__ __forceinline__ float pp_unit4(unsigned byte) {
    const unsigned b = byte ? byte << 23 : 0x00400000u;
    return pp_bits(byte == 255 ? 0x7fc00000u : b);
}

// Eight 8-bit codes of a block whose largest value has the bits m; returns the scale byte.
// 64 v / 2^e is an exact product (a power of two), and adding 1.5 * 2^23 rounds it to the nearest
// whole number, ties to even, in the low bits of the sum.
__device__ __forceinline__ unsigned pp_codes8(const float *v, unsigned m, pp_u2 &codes) {
    const unsigned e = m >> 23;
    float pre = 1.0f;
    unsigned f = e;
    if (e < 6) { pre = 0x1p64f; f = e + 64; }  // 2^(133 - e) is no float: in two steps
    const float s = pp_bits((260 - f) << 23), magic = 0x1.8p23f;
    unsigned b[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float t = __builtin_fmaf(v[i] * pre, s, magic);
        b[i] = pp_bits(__builtin_amdgcn_fmed3f(t, magic - 127.0f, magic + 127.0f));
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const unsigned lo = __builtin_amdgcn_perm(b[4 * h + 1], b[4 * h], 0x0c0c0400);
        const unsigned hi = __builtin_amdgcn_perm(b[4 * h + 3], b[4 * h + 2], 0x0c0c0400);
        codes[h] = e == 255 ? 0 : (lo | hi << 16);
    }
    return e;
}

// Eight 4-bit codes, by the conversion of the hardware (to the nearest, ties to even, 6 beyond 6).
__device__ __forceinline__ unsigned pp_codes4(const float *v, unsigned m, unsigned &codes) {
    const unsigned e = m >> 23;
    const unsigned byte = e == 255 ? 255 : e >= 2 ? e - 2 : 0;
    const float s = pp_unit4(e == 255 ? 0 : byte);
    unsigned c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[0], v[1], s, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[2], v[3], s, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[4], v[5], s, 2);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[6], v[7], s, 3);
    codes = e == 255 ? 0 : c;
    return byte;
}

// the values of eight 8-bit codes in units of `unit`
__device__ __forceinline__ void pp_values8(pp_u2 codes, float unit, float *v) {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (float)(signed char)(codes[i >> 2] >> (8 * (i & 3))) * unit;
}

__device__ __forceinline__ void pp_values4(unsigned codes, unsigned byte, float *v) {
    const float s = pp_unit4(byte == 255 ? 0 : byte);
    pp_f2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, s, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, s, 1);
    pp_f2 c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, s, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, s, 3);
    v[0] = a[0]; v[1] = a[1]; v[2] = b[0]; v[3] = b[1];
    v[4] = c[0]; v[5] = c[1]; v[6] = d[0]; v[7] = d[1];
    if (byte == 255)
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = pp_bits(0x7fc00000u);
}

// Calls f with the tag of a type.
template <class F> static inline int pp_by_type(int type, F f) {
    if (type == PP_TYPE_F32) return f(PpF32());
    if (type == PP_TYPE_F16) return f(PpF16());
    return f(PpBF16());
}
