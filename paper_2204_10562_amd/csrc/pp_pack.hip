// pp_pack, pp_unpack, pp_act_forward, pp_act_backward: one pass over rows of values and of
// packed blocks.
//
// A thread takes eight neighbours (16 bytes of a 16-bit type), the four threads of a quad make a
// block of 32 and find its largest value by two moves between lanes; nothing goes through LDS.
// Each byte is read and written once, and bytes bound all four at a size: gated silu of 8192 x 16384 bf16
// with both checkpoints (1.08 GB) takes 185 us forward and as long backward, 5.8 TB/s where a copy of 1 GiB
// reaches 5.2, gated gelu the same; without a gate (0.68 GB) silu 104 to 107 us forward, 6.4 TB/s, and 122 backward, gelu
// 124 to 134 either way, where its instructions show; float32 5003 x 4099 into 4 bits 14 us, 6.6 TB/s (its rows start at
// no multiple of 16 bytes; loads and stores of 16 bytes are made all the same); small ones a launch,
// 1.5 to 2 us.  Four rows to a thread, their loads in flight together, were slower but for packing alone
// (8 %, and 2 % the other way): a chip full of threads has enough in flight.
// Values are scaled and rounded in 32 bits, once for each result.
#include "pp_layer_common.h"

#define PK_THREADS 256

// What a launch covers: rows of `chunks` chunks of eight columns (those of whole groups), a thread to each.
struct pk_shape {
    long long cols;
    unsigned chunks, magic;  // t / chunks = t * magic >> 32 + shift
    int shift;
    unsigned items;  // chunks of all rows
};

static pk_shape pk_plan(int64_t rows, int64_t cols) {
    pk_shape s;
    s.cols = cols;
    s.chunks = (unsigned)(pp_groups(cols) * (PP_GROUP / 8));
    s.shift = 0;
    while ((2ull << s.shift) < s.chunks) ++s.shift;  // (t < 2^31: 32 bits of the reciprocal are enough)
    s.magic = (unsigned)(((1ull << (32 + s.shift)) + s.chunks - 1) / s.chunks);
    const int64_t most = (((int64_t)1 << 31) - 1) / s.chunks;
    s.items = (unsigned)(rows < most ? rows : most) * s.chunks;
    return s;
}

// In a kernel of shape `s`: `at` the thread's chunk of all, q that of its row r.  The lanes of a quad have
// one row and four neighbouring chunks (chunks is a multiple of 16), and go together.
#define PK_THREAD(s)                                                              \
    const unsigned at = blockIdx.x * PK_THREADS + threadIdx.x;                    \
    if (at >= (s).items) return;                                                  \
    const unsigned run = __umulhi(at, (s).magic) >> (s).shift;                    \
    const unsigned q = at - run * (s).chunks;                                     \
    const long long r = run;                                                      \
    const long long left = (s).cols - 8ll * q; /* columns from the chunk's first on, maybe <= 0 */

// Runs launch(part, grid, first row) for as many launches as the rows take.
template <class F> static int pk_launch(int64_t rows, int64_t cols, F launch) {
    for (int64_t r = 0; r < rows;) {
        const pk_shape s = pk_plan(rows - r, cols);
        launch(s, (s.items + PK_THREADS - 1) / PK_THREADS, r);
        if (hipGetLastError() != hipSuccess) return PP_ERR_HIP;
        r += s.items / s.chunks;
    }
    return PP_OK;
}

__device__ __forceinline__ void put_codes8(unsigned at, unsigned m, const float *v, uint8_t *codes, uint8_t *scales) {
    pp_u2 c;
    const unsigned byte = pp_codes8(v, m, c);
    *(pp_u2 *)(codes + at * 8ll) = c;
    if (!(at & 3)) scales[at >> 2] = (uint8_t)byte;
}
__device__ __forceinline__ void put_codes4(unsigned at, unsigned m, const float *v, uint8_t *codes, uint8_t *scales) {
    unsigned c;
    const unsigned byte = pp_codes4(v, m, c);
    *(unsigned *)(codes + at * 4ll) = c;
    if (!(at & 3)) scales[at >> 2] = (uint8_t)byte;
}

// FMT, or both formats at once (PK_BOTH)
#define PK_BOTH 2
template <int FMT, class Y>
__global__ __launch_bounds__(PK_THREADS) void k_pack(pk_shape s, const typename Y::T *__restrict__ src, long long ld, uint8_t *__restrict__ codes,
                                                     uint8_t *__restrict__ scales, uint8_t *__restrict__ codes8, uint8_t *__restrict__ scales8) {
    PK_THREAD(s)
    const PpRaw<Y> raw = pp_load8<Y>(src + r * ld + 8 * q, left);
    float v[8];
    pp_values<Y>(raw, v);
    const unsigned m = pp_quad_max(pp_absmax<Y>(raw, v));
    if constexpr (FMT == PP_PACK_INT8) {
        put_codes8(at, m, v, codes, scales);
    } else {
        put_codes4(at, m, v, codes, scales);
        if constexpr (FMT == PK_BOTH) put_codes8(at, m, v, codes8, scales8);
    }
}

template <int FMT, class Y>
__global__ __launch_bounds__(PK_THREADS) void k_unpack(pk_shape s, const uint8_t *__restrict__ codes, const uint8_t *__restrict__ scales,
                                                       typename Y::T *__restrict__ dst, long long ld) {
    PK_THREAD(s)
    if (left <= 0) return;
    float v[8];
    if constexpr (FMT == PP_PACK_INT8) pp_values8(*(const pp_u2 *)(codes + at * 8ll), pp_unit8(scales[at >> 2]), v);
    else pp_values4(*(const unsigned *)(codes + at * 4ll), scales[at >> 2], v);
    pp_store8<Y>(dst + r * ld + 8 * q, left, v);
}

// f and f'.  exp2 and the reciprocal are the hardware's (a unit or two of the last place), which give zero for what is no normal
// number.  sigmoid(z) is taken from h = exp(-|z| / 2) and hr = h / (1 + h^2): h hr for z < 0, else 1 - h hr, whose rounding is
// the last place's alone; its derivative is hr^2, without a difference of which nothing is left where sigmoid is near 1.  (x h) hr
// loses nothing while it is a normal number.  tanh is 2 sigmoid(2 z) - 1, which loses nothing where it is near -1.
struct pk_sigmoid {
    float h, hr;
    bool low;
    __device__ __forceinline__ pk_sigmoid(float z) : low(z < 0.0f) {
        h = __builtin_amdgcn_exp2f(-0.72134752f * __builtin_fabsf(z));
        hr = h * __builtin_amdgcn_rcpf(__builtin_fmaf(h, h, 1.0f));
    }
    __device__ __forceinline__ float value() const { return low ? h * hr : __builtin_fmaf(-h, hr, 1.0f); }
    __device__ __forceinline__ float times(float x) const { return low ? x * h * hr : x * __builtin_fmaf(-h, hr, 1.0f); }
};

// e = exp(-x^2 / 2), and Phi(x) = erfc(-x / sqrt 2) / 2 from it: Phi(-|x|) / e falls from 1/2 as slowly as 1 / |x|, which
// 1/2 - v Q(v) with v = p |x| / (1 + p |x|) follows to 2^-26 of itself (Q's coefficients by least squares of the relative
// error over |x| <= 14.5, weighted until it was even; beyond, nothing is left).  So what is left far on the negative
// side keeps its digits, to (8 + 1.2 x^2) 2^-24 of itself down to the last normal numbers, where 1 + erf has none at -6.
__device__ __forceinline__ float gauss(float x, float &e) {
    const float h = __builtin_amdgcn_exp2f(-0.36067376f * (x * x));  // (of half the exponent: exp2 gives no subnormal numbers)
    e = h * h;
    const float m = __builtin_amdgcn_fmed3f(0.33f * __builtin_fabsf(x), 0.0f, 0x1p30f), v = m * __builtin_amdgcn_rcpf(1.0f + m);
    const float c[] = {1.20891619f, -1.08676934f, 0.317839444f, 0.154287234f, -0.0652996749f, -0.0222513955f, -0.0651500002f, 0.0843002498f, -0.0258791298f};
    float q = c[8];
#pragma unroll
    for (int k = 7; k >= 0; --k) q = __builtin_fmaf(q, v, c[k]);
    const float g = e * __builtin_fmaf(-v, q, 0.5f);
    return x < 0.0f ? g : 1.0f - g;
}

template <int KIND> __device__ __forceinline__ float act(float x) {
    if constexpr (KIND == PP_ACT_SILU) return pk_sigmoid(x).times(x);
    if constexpr (KIND == PP_ACT_GELU_TANH) return pk_sigmoid(1.5957691216057308f * (x + 0.044715f * x * x * x)).times(x);
    float e;
    return x * gauss(x, e);
}

// f(x) and f'(x)
template <int KIND> __device__ __forceinline__ void act_both(float x, float &f, float &d) {
    if constexpr (KIND == PP_ACT_GELU) {
        float e;
        const float g = gauss(x, e);
        f = x * g;
        d = __builtin_fmaf(x * e, 0.39894228040143268f, g);
    } else {
        const float c = KIND == PP_ACT_SILU ? x : __builtin_amdgcn_fmed3f(x, -32.0f, 32.0f);  // beyond, f is x or 0 and f' 1 or 0
        const float z = KIND == PP_ACT_SILU ? x : 1.5957691216057308f * (c + 0.044715f * c * c * c);
        const float dz = KIND == PP_ACT_SILU ? 1.0f : 1.5957691216057308f * (1.0f + 3.0f * 0.044715f * c * c);
        const pk_sigmoid s(z);
        f = s.times(x);
        d = __builtin_fmaf(c * dz, s.hr * s.hr, s.value());
        if (KIND == PP_ACT_GELU_TANH) d = x != x ? x : d;
    }
}

template <int KIND, class Y, bool GATED>
__global__ __launch_bounds__(PK_THREADS) void k_act_forward(pk_shape s, const typename Y::T *__restrict__ x, long long ld_x,
                                                            const typename Y::T *__restrict__ u, long long ld_u,
                                                            typename Y::T *__restrict__ y, long long ld_y, uint8_t *__restrict__ xc,
                                                            uint8_t *__restrict__ xs, uint8_t *__restrict__ uc, uint8_t *__restrict__ us) {
    PK_THREAD(s)
    const PpRaw<Y> rx = pp_load8<Y>(x + r * ld_x + 8 * q, left);
    PpRaw<Y> ru;
    if constexpr (GATED) ru = pp_load8<Y>(u + r * ld_u + 8 * q, left);
    float v[8], w[8], t[8];
    pp_values<Y>(rx, v);
    if (xc) put_codes8(at, pp_quad_max(pp_absmax<Y>(rx, v)), v, xc, xs);
#pragma unroll
    for (int j = 0; j < 8; ++j) t[j] = act<KIND>(v[j]);
    if constexpr (GATED) {
        pp_values<Y>(ru, w);
        if (uc) put_codes8(at, pp_quad_max(pp_absmax<Y>(ru, w)), w, uc, us);
#pragma unroll
        for (int j = 0; j < 8; ++j) t[j] *= w[j];
    }
    if (left > 0) pp_store8<Y>(y + r * ld_y + 8 * q, left, t);
}

// dy and dx may be one matrix: a thread reads its values before it writes them
template <int KIND, class Y, bool GATED>
__global__ __launch_bounds__(PK_THREADS) void k_act_backward(pk_shape s, const typename Y::T *dy, long long ld_dy,
                                                             const uint8_t *__restrict__ xc, const uint8_t *__restrict__ xs,
                                                             const uint8_t *__restrict__ uc, const uint8_t *__restrict__ us,
                                                             typename Y::T *dx, long long ld_dx, typename Y::T *__restrict__ du, long long ld_du) {
    PK_THREAD(s)
    if (left <= 0) return;
    const PpRaw<Y> rd = pp_load8<Y>(dy + r * ld_dy + 8 * q, left);
    float g[8], v[8], w[8], a[8];
    pp_values8(*(const pp_u2 *)(xc + at * 8ll), pp_unit8(xs[at >> 2]), v);
    if constexpr (GATED) pp_values8(*(const pp_u2 *)(uc + at * 8ll), pp_unit8(us[at >> 2]), w);
    pp_values<Y>(rd, g);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        float f, d;
        act_both<KIND>(v[j], f, d);
        a[j] = g[j] * f;
        v[j] = g[j] * d;
        if constexpr (GATED) v[j] *= w[j];
    }
    pp_store8<Y>(dx + r * ld_dx + 8 * q, left, v);
    if constexpr (GATED) pp_store8<Y>(du + r * ld_du + 8 * q, left, a);
}

// `p` moved on by so many bytes; NULL stays.
static uint8_t *on(void *p, int64_t bytes) { return p ? (uint8_t *)p + bytes : NULL; }
static const uint8_t *on(const void *p, int64_t bytes) { return p ? (const uint8_t *)p + bytes : NULL; }

template <int FMT> static int launch_pack(int type, int64_t rows, int64_t cols, const void *src, int64_t ld, void *codes, void *scales, void *codes8,
                                          void *scales8, hipStream_t st) {
    const int64_t g = pp_groups(cols), width = FMT == PP_PACK_INT8 ? PP_GROUP_CODES8 : PP_GROUP_CODES4;
    return pp_by_type(type, [&](auto y) {
        typedef decltype(y) Y;
        typedef typename Y::T T;
        return pk_launch(rows, cols, [&](const pk_shape &s, unsigned grid, int64_t r) {
            k_pack<FMT, Y><<<grid, PK_THREADS, 0, st>>>(s, (const T *)src + r * ld, ld, on(codes, r * g * width), on(scales, r * g * 4),
                                                                            on(codes8, r * g * PP_GROUP_CODES8), on(scales8, r * g * 4));
        });
    });
}

int pp_launch_pack_both(int type, int64_t rows, int64_t cols, const void *src, int64_t ld, void *codes4, void *scales4, void *codes8, void *scales8,
                        hipStream_t st) {
    if (codes8) return launch_pack<PK_BOTH>(type, rows, cols, src, ld, codes4, scales4, codes8, scales8, st);
    return launch_pack<PP_PACK_FP4>(type, rows, cols, src, ld, codes4, scales4, NULL, NULL, st);
}

extern "C" int pp_pack(int format, int type, int64_t rows, int64_t cols, const void *src, int64_t ld_src, void *codes, void *scales,
                       void *stream) {
    if (pp_bad_sizes(type, rows, cols) || (format != PP_PACK_INT8 && format != PP_PACK_FP4)) return PP_ERR_INVALID_ARG;
    if (pp_bad_matrix(src, type, rows, cols, ld_src) || pp_bad_packed(codes, scales, rows)) return PP_ERR_INVALID_ARG;
    if (format == PP_PACK_INT8) return launch_pack<PP_PACK_INT8>(type, rows, cols, src, ld_src, codes, scales, NULL, NULL, (hipStream_t)stream);
    return launch_pack<PP_PACK_FP4>(type, rows, cols, src, ld_src, codes, scales, NULL, NULL, (hipStream_t)stream);
}

extern "C" int pp_unpack(int format, int type, int64_t rows, int64_t cols, const void *codes, const void *scales, void *dst,
                         int64_t ld_dst, void *stream) {
    if (pp_bad_sizes(type, rows, cols) || (format != PP_PACK_INT8 && format != PP_PACK_FP4)) return PP_ERR_INVALID_ARG;
    if (pp_bad_matrix(dst, type, rows, cols, ld_dst) || pp_bad_packed(codes, scales, rows)) return PP_ERR_INVALID_ARG;
    const int64_t g = pp_groups(cols);
    hipStream_t st = (hipStream_t)stream;
    return pp_by_type(type, [&](auto y) {
        typedef decltype(y) Y;
        typedef typename Y::T T;
        return pk_launch(rows, cols, [&](const pk_shape &s, unsigned grid, int64_t r) {
            if (format == PP_PACK_INT8)
                k_unpack<PP_PACK_INT8, Y><<<grid, PK_THREADS, 0, st>>>(s, on(codes, r * g * PP_GROUP_CODES8), on(scales, r * g * 4), (T *)dst + r * ld_dst, ld_dst);
            else
                k_unpack<PP_PACK_FP4, Y><<<grid, PK_THREADS, 0, st>>>(s, on(codes, r * g * PP_GROUP_CODES4), on(scales, r * g * 4), (T *)dst + r * ld_dst, ld_dst);
        });
    });
}

// Calls f with the kind as a constant.
template <class F> static int by_kind(int kind, F f) {
    if (kind == PP_ACT_GELU) return f(std::integral_constant<int, PP_ACT_GELU>());
    if (kind == PP_ACT_GELU_TANH) return f(std::integral_constant<int, PP_ACT_GELU_TANH>());
    return f(std::integral_constant<int, PP_ACT_SILU>());
}

extern "C" int pp_act_forward(int kind, int type, int64_t rows, int64_t cols, const void *x, int64_t ld_x, const void *u, int64_t ld_u,
                              void *y, int64_t ld_y, void *x_codes, void *x_scales, void *u_codes, void *u_scales, void *stream) {
    if (pp_bad_sizes(type, rows, cols) || kind < PP_ACT_GELU || kind > PP_ACT_SILU) return PP_ERR_INVALID_ARG;
    if (pp_bad_matrix(x, type, rows, cols, ld_x) || pp_bad_matrix(y, type, rows, cols, ld_y)) return PP_ERR_INVALID_ARG;
    if (u && pp_bad_matrix(u, type, rows, cols, ld_u)) return PP_ERR_INVALID_ARG;
    if ((x_codes || x_scales) && pp_bad_packed(x_codes, x_scales, rows)) return PP_ERR_INVALID_ARG;
    if ((u_codes || u_scales) && (pp_bad_packed(u_codes, u_scales, rows) || (rows && !u))) return PP_ERR_INVALID_ARG;
    const int64_t g = pp_groups(cols);
    hipStream_t st = (hipStream_t)stream;
    return pp_by_type(type, [&](auto t) {
        typedef decltype(t) Y;
        typedef typename Y::T T;
        return by_kind(kind, [&](auto k) {
            constexpr int K = decltype(k)::value;
            return pk_launch(rows, cols, [&](const pk_shape &s, unsigned grid, int64_t r) {
                uint8_t *xc = on(x_codes, r * g * PP_GROUP_CODES8), *xs = on(x_scales, r * g * 4);
                uint8_t *uc = on(u_codes, r * g * PP_GROUP_CODES8), *us = on(u_scales, r * g * 4);
                if (u)
                    k_act_forward<K, Y, true><<<grid, PK_THREADS, 0, st>>>(s, (const T *)x + r * ld_x, ld_x, (const T *)u + r * ld_u, ld_u, (T *)y + r * ld_y,
                                                                              ld_y, xc, xs, uc, us);
                else
                    k_act_forward<K, Y, false><<<grid, PK_THREADS, 0, st>>>(s, (const T *)x + r * ld_x, ld_x, (const T *)NULL, 0, (T *)y + r * ld_y, ld_y, xc, xs,
                                                                               (uint8_t *)NULL, (uint8_t *)NULL);
            });
        });
    });
}

extern "C" int pp_act_backward(int kind, int type, int64_t rows, int64_t cols, const void *dy, int64_t ld_dy, const void *x_codes,
                               const void *x_scales, const void *u_codes, const void *u_scales, void *dx, int64_t ld_dx, void *du,
                               int64_t ld_du, void *stream) {
    if (pp_bad_sizes(type, rows, cols) || kind < PP_ACT_GELU || kind > PP_ACT_SILU) return PP_ERR_INVALID_ARG;
    if (pp_bad_matrix(dy, type, rows, cols, ld_dy) || pp_bad_matrix(dx, type, rows, cols, ld_dx)) return PP_ERR_INVALID_ARG;
    if (pp_bad_packed(x_codes, x_scales, rows)) return PP_ERR_INVALID_ARG;
    const bool gated = u_codes || u_scales || du;
    if (gated && (pp_bad_packed(u_codes, u_scales, rows) || pp_bad_matrix(du, type, rows, cols, ld_du))) return PP_ERR_INVALID_ARG;
    const int64_t g = pp_groups(cols);
    hipStream_t st = (hipStream_t)stream;
    return pp_by_type(type, [&](auto t) {
        typedef decltype(t) Y;
        typedef typename Y::T T;
        return by_kind(kind, [&](auto k) {
            constexpr int K = decltype(k)::value;
            return pk_launch(rows, cols, [&](const pk_shape &s, unsigned grid, int64_t r) {
                const uint8_t *xc = on(x_codes, r * g * PP_GROUP_CODES8), *xs = on(x_scales, r * g * 4);
                const uint8_t *uc = on(u_codes, r * g * PP_GROUP_CODES8), *us = on(u_scales, r * g * 4);
                if (gated)
                    k_act_backward<K, Y, true><<<grid, PK_THREADS, 0, st>>>(s, (const T *)dy + r * ld_dy, ld_dy, xc, xs, uc, us, (T *)dx + r * ld_dx, ld_dx,
                                                                               (T *)du + r * ld_du, ld_du);
                else
                    k_act_backward<K, Y, false><<<grid, PK_THREADS, 0, st>>>(s, (const T *)dy + r * ld_dy, ld_dy, xc, xs, uc, us, (T *)dx + r * ld_dx, ld_dx,
                                                                                (T *)NULL, 0);
            });
        });
    });
}
