// How the losses (pp_logprob.hip, pp_distill.hip) divide rows of logits, and what they share.
//
// With k = log2(e) / T and m = max x, a segment of a row has s = sum 2^((x - m) k).  The difference comes first: k x - k m in one
// multiply-add would be an instruction less, and nothing where m k passes 2^31, as in rows masked with a type's lowest value.
#pragma once

#include "pp_rows.h"

#define LS_THREADS 256
#define LS_STEP (LS_THREADS * 8)  // logits that a workgroup reads at a time
#define LS_MAX_GRID (1 << 22)
#define LS_ENOUGH 1024           // workgroups that fill the chip
#define LS_CAP 1024               // candidates of a segment that are kept: what fewer threads than PP_TOP_MAX have at least

// Rows of `cols` in `segs` segments of `size` (the last shorter), `held` chunks of eight to a thread.
struct ls_plan {
    int held;
    int segs;
    long long size;
};

// Most chunks that a thread holds: a 16-bit type's `most`, half of that in float
static inline int ls_held(int type, int most) { return type == PP_TYPE_F32 ? most / 2 : most; }

// The size of segments that are about equally long, at multiples of 128 bytes or more
static inline long long ls_even(int64_t cols, int segs) { return ((cols + segs - 1) / segs + 63) & ~63ll; }

// The largest segments, for their fewer partial results; smaller ones where those are as few, and to spread few rows over the chip.
static inline ls_plan ls_divide(int type, int64_t rows, int64_t cols, int most) {
    const int sizes[3] = {ls_held(type, most), most > 8 ? 4 : ls_held(type, most) / 2, 1};
    ls_plan p = {};
    for (int i = 0;; ++i) {
        p.held = sizes[i];
        p.size = (long long)sizes[i] * LS_STEP;
        p.segs = (int)((cols + p.size - 1) / p.size);
        const int64_t next = i < 2 ? (cols + (int64_t)sizes[i + 1] * LS_STEP - 1) / ((int64_t)sizes[i + 1] * LS_STEP) : 0;
        if (i == 2 || (next > p.segs && (next > 64 || rows * p.segs >= LS_ENOUGH))) break;
    }
    p.size = ls_even(cols, p.segs);
    return p;
}

// No more segments than this of any number of rows up to `rows` (those that are not the largest are less than LS_ENOUGH
// segments of the size before, of at most four each).
static inline int64_t ls_most(int type, int64_t rows, int64_t cols, int most) {
    const int64_t size = (int64_t)ls_held(type, most) * LS_STEP, all = rows * ((cols + size - 1) / size);
    return all > 4 * LS_ENOUGH ? all : 4 * LS_ENOUGH;
}

// Eight logits as floats, -infinity behind the n-th
template <class Y> __device__ __forceinline__ PpRaw<Y> ls_load(const typename Y::T *p, long long n) {
    typedef typename Y::T T;
    PpRaw<Y> r;
    if (n >= 8) {
#pragma unroll
        for (int i = 0; i < PpRaw<Y>::W; ++i) r.w[i] = ((const pp_any16<sizeof(T)> *)p)[i].v;
    } else {
        T t[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) t[i] = i < n ? p[i] : (T)-__builtin_inff();
        __builtin_memcpy(&r, t, sizeof(r));
    }
    return r;
}

// A thread's chunks of a segment x[0 .. n), -infinity behind it; of a whole one without a branch, so that all loads are on their way
// together
template <class Y, int HELD> __device__ __forceinline__ void ls_load_all(PpRaw<Y> (&raw)[HELD], const typename Y::T *x, long long n) {
    const unsigned lane = threadIdx.x * (unsigned)(8 * sizeof(typename Y::T));
    if (n >= (long long)HELD * LS_STEP) {
#pragma unroll
        for (int i = 0; i < HELD; ++i)
#pragma unroll
            for (int j = 0; j < PpRaw<Y>::W; ++j) raw[i].w[j] = ((const pp_any16<sizeof(typename Y::T)> *)((const char *)(x + i * LS_STEP) + lane))[j].v;
    } else {
#pragma unroll
        for (int i = 0; i < HELD; ++i) raw[i] = ls_load<Y>((const typename Y::T *)((const char *)(x + i * LS_STEP) + lane), (int)n - 8 * (int)threadIdx.x - i * LS_STEP);
    }
}

// Makes the compiler convert held values again where they are used again: kept as floats they would take twice the registers.
template <class Y, int N> __device__ __forceinline__ void ls_hold(PpRaw<Y> (&raw)[N]) {
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int j = 0; j < PpRaw<Y>::W; ++j) asm volatile("" : "+v"(raw[i].w[j]));
}

// (The compiler's fmax quiets each operand first, which is an instruction to a logit.  A NaN may be passed over or not: a row that has
// one has a sum that is none.)
__device__ __forceinline__ float ls_max3(float a, float b, float c) {
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}
__device__ __forceinline__ float ls_max8(const float *v) {
    return ls_max3(ls_max3(ls_max3(v[0], v[1], v[2]), v[3], v[4]), ls_max3(v[5], v[6], v[7]), v[7]);
}

// Calls f with the chunks that a thread holds in a division with this `most` as a constant.
template <class Y, int MOST, class F> static inline void ls_by_held(int held, F f) {
    constexpr int LARGE = sizeof(typename Y::T) == 4 ? MOST / 2 : MOST, MIDDLE = MOST > 8 ? 4 : LARGE / 2;
    if (held == LARGE) f(std::integral_constant<int, LARGE>());
    else if (held == MIDDLE) f(std::integral_constant<int, MIDDLE>());
    else f(std::integral_constant<int, 1>());
}
static inline unsigned ls_grid(int64_t items) { return (unsigned)(items < LS_MAX_GRID ? items : LS_MAX_GRID); }

// What a maximum is subtracted as: 0 where there is nothing but -infinity (then every term is 0)
__device__ __forceinline__ float ls_base(float m) { return m == -__builtin_inff() ? 0.0f : m; }

template <int WAVES> __device__ __forceinline__ float ls_group_max(float v, float *room) {
    v = pp_wave_max(v);
    if (!(threadIdx.x & (PP_WAVE - 1))) room[threadIdx.x / PP_WAVE] = v;
    __syncthreads();
    v = room[0];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) v = __builtin_fmaxf(v, room[w]);
    return v;
}

// Numbers in the order of their keys; -0 as 0.  -infinity: key 0, which stands for none.
__device__ __forceinline__ unsigned ls_key(float x) {
    if (x == -__builtin_inff()) return 0;
    const unsigned b = pp_bits(x + 0.0f);
    return b ^ ((unsigned)((int)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float ls_value(unsigned key) { return pp_bits(key ^ (key & 0x80000000u ? 0x80000000u : 0xffffffffu)); }
