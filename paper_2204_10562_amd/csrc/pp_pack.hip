// pp_pack, pp_unpack, pp_act_forward, pp_act_backward: one pass over rows of values and of
// packed blocks.
//
// A thread takes eight neighbours (16 bytes of a 16-bit type), the four threads of a quad make a
// block of 32 and find its largest value by two moves between lanes; nothing goes through LDS.
// All four operators are bound by the bytes they move.
#include "pp_layer_common.h"

#define PK_THREADS 256
#define PK_ROWS 4  // rows whose loads a thread has in flight

// What a launch covers: blocks of 2^cx8 chunks of eight columns by ry * PK_ROWS rows.
struct pk_shape {
    long long rows, cols;
    int chunks;  // of eight columns in a row of whole groups
    int cx_log;  // chunks side by side in a workgroup
    unsigned gx, gy;
};

static pk_shape pk_plan(int64_t rows, int64_t cols) {
    pk_shape s;
    s.rows = rows;
    s.cols = cols;
    s.chunks = (int)(pp_groups(cols) * (PP_GROUP / 8));
    s.cx_log = 4;
    while (s.cx_log < 8 && (1 << s.cx_log) < s.chunks) ++s.cx_log;
    const int ry = PK_THREADS >> s.cx_log;
    s.gx = (unsigned)((s.chunks + (1 << s.cx_log) - 1) >> s.cx_log);
    // at most 2^31 threads to a launch; the rows beyond are taken in further turns
    const int64_t want = (rows + ry * PK_ROWS - 1) / (ry * PK_ROWS), most = ((int64_t)1 << 23) / s.gx;
    s.gy = (unsigned)(want < most ? want : most);
    return s;
}

// Runs body(r, q) for PK_ROWS rows at a time: body gets the row numbers (valid ones first) and the
// thread's chunk.  The four lanes of a quad always take part together.
#define PK_LOOP(s)                                                                                   \
    const int cx = 1 << (s).cx_log, ry = PK_THREADS >> (s).cx_log;                                   \
    const unsigned bx = blockIdx.x % (s).gx, by = blockIdx.x / (s).gx;                               \
    const int q = (int)(bx << (s).cx_log) + ((int)threadIdx.x & (cx - 1));                           \
    if (q >= (s).chunks) return;                                                                     \
    const long long left = (s).cols - 8ll * q; /* columns from the chunk's first on, maybe <= 0 */   \
    for (long long r0 = (long long)by * ry * PK_ROWS + ((int)threadIdx.x >> (s).cx_log); r0 < (s).rows; \
         r0 += (long long)(s).gy * ry * PK_ROWS)

__device__ __forceinline__ void put_codes8(long long r, int q, int chunks, unsigned m, const float *v, uint8_t *codes, uint8_t *scales) {
    pp_u2 c;
    const unsigned byte = pp_codes8(v, pp_quad_max(m), c);
    *(pp_u2 *)(codes + (r * chunks + q) * 8) = c;
    if (!(q & 3)) scales[(r * chunks + q) >> 2] = (uint8_t)byte;
}

template <int FMT, class Y>
__global__ __launch_bounds__(PK_THREADS) void k_pack(pk_shape s, const typename Y::T *__restrict__ src, long long ld,
                                                     uint8_t *__restrict__ codes, uint8_t *__restrict__ scales) {
    PK_LOOP(s) {
        PpRaw<Y> raw[PK_ROWS];
#pragma unroll
        for (int i = 0; i < PK_ROWS; ++i) {
            const long long r = r0 + (long long)i * ry;
            raw[i] = pp_load8<Y>(src + r * ld + 8 * q, r < s.rows ? left : 0);
        }
#pragma unroll
        for (int i = 0; i < PK_ROWS; ++i) {
            const long long r = r0 + (long long)i * ry;
            if (r >= s.rows) break;
            float v[8];
            pp_values<Y>(raw[i], v);
            const unsigned m = pp_absmax<Y>(raw[i], v);
            if constexpr (FMT == PP_PACK_INT8) {
                put_codes8(r, q, s.chunks, m, v, codes, scales);
            } else {
                unsigned c;
                const unsigned byte = pp_codes4(v, pp_quad_max(m), c);
                *(unsigned *)(codes + (r * s.chunks + q) * 4) = c;
                if (!(q & 3)) scales[(r * s.chunks + q) >> 2] = (uint8_t)byte;
            }
        }
    }
}

template <int FMT, class Y>
__global__ __launch_bounds__(PK_THREADS) void k_unpack(pk_shape s, const uint8_t *__restrict__ codes, const uint8_t *__restrict__ scales,
                                                       typename Y::T *__restrict__ dst, long long ld) {
    PK_LOOP(s) {
        if (left <= 0) return;
#pragma unroll
        for (int i = 0; i < PK_ROWS; ++i) {
            const long long r = r0 + (long long)i * ry;
            if (r >= s.rows) break;
            const unsigned byte = scales[(r * s.chunks + q) >> 2];
            float v[8];
            if constexpr (FMT == PP_PACK_INT8)
                pp_values8(*(const pp_u2 *)(codes + (r * s.chunks + q) * 8), pp_unit8(byte), v);
            else
                pp_values4(*(const unsigned *)(codes + (r * s.chunks + q) * 4), byte, v);
            pp_store8<Y>(dst + r * ld + 8 * q, left, v);
        }
    }
}

// f and f'.  exp2 and the reciprocal are the hardware's (a unit or two of the last place), which
// give zero for what is no normal number: x sigmoid(z) is taken from exp(-|z|), for z < 0 held 2^16
// times as large until x has been multiplied in.  tanh is 2 sigmoid(2 z) - 1, which loses nothing
// where it is near -1.
__device__ __forceinline__ float times_sigmoid(float x, float z) {
    const float t = __builtin_amdgcn_exp2f(__builtin_fmaf(-1.4426950408889634f, __builtin_fabsf(z), 16.0f));
    const float r = __builtin_amdgcn_rcpf(__builtin_fmaf(t, 0x1p-16f, 1.0f));
    return z < 0.0f ? x * t * r * 0x1p-16f : x * r;
}

template <int KIND> __device__ __forceinline__ float act(float x) {
    if constexpr (KIND == PP_ACT_SILU) return times_sigmoid(x, x);
    if constexpr (KIND == PP_ACT_GELU_TANH) return times_sigmoid(x, 1.5957691216057308f * (x + 0.044715f * x * x * x));
    return 0.5f * x * (1.0f + erff(0.70710678118654752f * x));
}

// f(x) and f'(x)
template <int KIND> __device__ __forceinline__ void act_both(float x, float &f, float &d) {
    if constexpr (KIND == PP_ACT_GELU) {
        const float g = 0.5f * (1.0f + erff(0.70710678118654752f * x));
        f = x * g;
        d = g + x * __expf(-0.5f * x * x) * 0.39894228040143268f;
    } else {
        f = act<KIND>(x);
        const float c = KIND == PP_ACT_SILU ? x : __builtin_amdgcn_fmed3f(x, -32.0f, 32.0f);  // beyond, g is 0 or 1 and the second term 0
        const float z = KIND == PP_ACT_SILU ? x : 1.5957691216057308f * (c + 0.044715f * c * c * c);
        const float dz = KIND == PP_ACT_SILU ? 1.0f : 1.5957691216057308f * (1.0f + 3.0f * 0.044715f * c * c);
        const float g = times_sigmoid(1.0f, z);
        d = g + c * g * (1.0f - g) * dz;
        if (KIND == PP_ACT_GELU_TANH) d = x != x ? x : d;
    }
}

template <int KIND, class Y, bool GATED>
__global__ __launch_bounds__(PK_THREADS) void k_act_forward(pk_shape s, const typename Y::T *__restrict__ x, long long ld_x,
                                                            const typename Y::T *__restrict__ u, long long ld_u,
                                                            typename Y::T *__restrict__ y, long long ld_y, uint8_t *__restrict__ xc,
                                                            uint8_t *__restrict__ xs, uint8_t *__restrict__ uc, uint8_t *__restrict__ us) {
    PK_LOOP(s) {
        PpRaw<Y> rx[PK_ROWS], ru[PK_ROWS];
#pragma unroll
        for (int i = 0; i < PK_ROWS; ++i) {
            const long long r = r0 + (long long)i * ry, n = r < s.rows ? left : 0;
            rx[i] = pp_load8<Y>(x + r * ld_x + 8 * q, n);
            if constexpr (GATED) ru[i] = pp_load8<Y>(u + r * ld_u + 8 * q, n);
        }
#pragma unroll
        for (int i = 0; i < PK_ROWS; ++i) {
            const long long r = r0 + (long long)i * ry;
            if (r >= s.rows) break;
            float v[8], w[8], t[8];
            pp_values<Y>(rx[i], v);
            if (xc) put_codes8(r, q, s.chunks, pp_absmax<Y>(rx[i], v), v, xc, xs);
#pragma unroll
            for (int j = 0; j < 8; ++j) t[j] = act<KIND>(v[j]);
            if constexpr (GATED) {
                pp_values<Y>(ru[i], w);
                if (uc) put_codes8(r, q, s.chunks, pp_absmax<Y>(ru[i], w), w, uc, us);
#pragma unroll
                for (int j = 0; j < 8; ++j) t[j] *= w[j];
            }
            if (left > 0) pp_store8<Y>(y + r * ld_y + 8 * q, left, t);
        }
    }
}

// dy and dx may be one matrix: a thread reads its eight values before it writes them
template <int KIND, class Y, bool GATED>
__global__ __launch_bounds__(PK_THREADS) void k_act_backward(pk_shape s, const typename Y::T *dy, long long ld_dy,
                                                             const uint8_t *__restrict__ xc, const uint8_t *__restrict__ xs,
                                                             const uint8_t *__restrict__ uc, const uint8_t *__restrict__ us,
                                                             typename Y::T *dx, long long ld_dx, typename Y::T *__restrict__ du, long long ld_du) {
    PK_LOOP(s) {
        if (left <= 0) return;
        PpRaw<Y> rd[PK_ROWS];
        pp_u2 cx8[PK_ROWS], cu8[PK_ROWS];
        unsigned bx8[PK_ROWS], bu8[PK_ROWS];
#pragma unroll
        for (int i = 0; i < PK_ROWS; ++i) {
            const long long r = r0 + (long long)i * ry;
            if (r >= s.rows) break;
            rd[i] = pp_load8<Y>(dy + r * ld_dy + 8 * q, left);
            cx8[i] = *(const pp_u2 *)(xc + (r * s.chunks + q) * 8);
            bx8[i] = xs[(r * s.chunks + q) >> 2];
            if constexpr (GATED) {
                cu8[i] = *(const pp_u2 *)(uc + (r * s.chunks + q) * 8);
                bu8[i] = us[(r * s.chunks + q) >> 2];
            }
        }
#pragma unroll
        for (int i = 0; i < PK_ROWS; ++i) {
            const long long r = r0 + (long long)i * ry;
            if (r >= s.rows) break;
            float g[8], v[8], w[8], a[8];
            pp_values<Y>(rd[i], g);
            pp_values8(cx8[i], pp_unit8(bx8[i]), v);
            if constexpr (GATED) pp_values8(cu8[i], pp_unit8(bu8[i]), w);
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
    }
}

static int launched() { return hipGetLastError() == hipSuccess ? PP_OK : PP_ERR_HIP; }

int pp_launch_pack(int format, int type, int64_t rows, int64_t cols, const void *src, int64_t ld, void *codes, void *scales,
                   hipStream_t st) {
    const pk_shape s = pk_plan(rows, cols);
    return pp_by_type(type, [&](auto y) {
        typedef decltype(y) Y;
        if (format == PP_PACK_INT8)
            k_pack<PP_PACK_INT8, Y><<<s.gx * s.gy, PK_THREADS, 0, st>>>(s, (const typename Y::T *)src, ld, (uint8_t *)codes, (uint8_t *)scales);
        else
            k_pack<PP_PACK_FP4, Y><<<s.gx * s.gy, PK_THREADS, 0, st>>>(s, (const typename Y::T *)src, ld, (uint8_t *)codes, (uint8_t *)scales);
        return launched();
    });
}

extern "C" int pp_pack(int format, int type, int64_t rows, int64_t cols, const void *src, int64_t ld_src, void *codes, void *scales,
                       void *stream) {
    if (pp_bad_sizes(type, rows, cols) || (format != PP_PACK_INT8 && format != PP_PACK_FP4)) return PP_ERR_INVALID_ARG;
    if (pp_bad_matrix(src, type, rows, cols, ld_src) || pp_bad_packed(codes, scales, rows)) return PP_ERR_INVALID_ARG;
    if (!rows) return PP_OK;
    return pp_launch_pack(format, type, rows, cols, src, ld_src, codes, scales, (hipStream_t)stream);
}

extern "C" int pp_unpack(int format, int type, int64_t rows, int64_t cols, const void *codes, const void *scales, void *dst,
                         int64_t ld_dst, void *stream) {
    if (pp_bad_sizes(type, rows, cols) || (format != PP_PACK_INT8 && format != PP_PACK_FP4)) return PP_ERR_INVALID_ARG;
    if (pp_bad_matrix(dst, type, rows, cols, ld_dst) || pp_bad_packed(codes, scales, rows)) return PP_ERR_INVALID_ARG;
    if (!rows) return PP_OK;
    const pk_shape s = pk_plan(rows, cols);
    hipStream_t st = (hipStream_t)stream;
    return pp_by_type(type, [&](auto y) {
        typedef decltype(y) Y;
        if (format == PP_PACK_INT8)
            k_unpack<PP_PACK_INT8, Y><<<s.gx * s.gy, PK_THREADS, 0, st>>>(s, (const uint8_t *)codes, (const uint8_t *)scales, (typename Y::T *)dst, ld_dst);
        else
            k_unpack<PP_PACK_FP4, Y><<<s.gx * s.gy, PK_THREADS, 0, st>>>(s, (const uint8_t *)codes, (const uint8_t *)scales, (typename Y::T *)dst, ld_dst);
        return launched();
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
    if (!rows) return PP_OK;
    const pk_shape s = pk_plan(rows, cols);
    hipStream_t st = (hipStream_t)stream;
    return pp_by_type(type, [&](auto t) {
        typedef decltype(t) Y;
        typedef typename Y::T T;
        return by_kind(kind, [&](auto k) {
            constexpr int K = decltype(k)::value;
            if (u)
                k_act_forward<K, Y, true><<<s.gx * s.gy, PK_THREADS, 0, st>>>(s, (const T *)x, ld_x, (const T *)u, ld_u, (T *)y, ld_y, (uint8_t *)x_codes,
                                                                            (uint8_t *)x_scales, (uint8_t *)u_codes, (uint8_t *)u_scales);
            else
                k_act_forward<K, Y, false><<<s.gx * s.gy, PK_THREADS, 0, st>>>(s, (const T *)x, ld_x, (const T *)NULL, 0, (T *)y, ld_y, (uint8_t *)x_codes,
                                                                             (uint8_t *)x_scales, (uint8_t *)NULL, (uint8_t *)NULL);
            return launched();
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
    if (!rows) return PP_OK;
    const pk_shape s = pk_plan(rows, cols);
    hipStream_t st = (hipStream_t)stream;
    return pp_by_type(type, [&](auto t) {
        typedef decltype(t) Y;
        typedef typename Y::T T;
        return by_kind(kind, [&](auto k) {
            constexpr int K = decltype(k)::value;
            const uint8_t *xc = (const uint8_t *)x_codes, *xs = (const uint8_t *)x_scales, *uc = (const uint8_t *)u_codes, *us = (const uint8_t *)u_scales;
            if (gated)
                k_act_backward<K, Y, true><<<s.gx * s.gy, PK_THREADS, 0, st>>>(s, (const T *)dy, ld_dy, xc, xs, uc, us, (T *)dx, ld_dx, (T *)du, ld_du);
            else
                k_act_backward<K, Y, false><<<s.gx * s.gy, PK_THREADS, 0, st>>>(s, (const T *)dy, ld_dy, xc, xs, uc, us, (T *)dx, ld_dx, (T *)NULL, 0);
            return launched();
        });
    });
}
