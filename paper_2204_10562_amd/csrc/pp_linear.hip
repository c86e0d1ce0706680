// pp_linear_forward, pp_linear_backward_input, pp_linear_backward_weight: products with a packed
// operand.
//
// One kernel for all: tiles of 64 by 64 results, both operands read back to floats on their way
// into LDS, 16 results to a thread.
#include "pp_layer_common.h"

int pp_launch_pack(int format, int type, int64_t rows, int64_t cols, const void *src, int64_t ld, void *codes, void *scales, hipStream_t st);

// Operand elements by (index along the result, index along the sum).
struct FromFp4 {
    const uint8_t *codes, *scales;
    long long groups;
    __device__ float at(long long r, long long c) const {
        const unsigned byte = scales[r * groups * 4 + c / PP_BLOCK];
        const unsigned n = codes[r * groups * PP_GROUP_CODES4 + c / 2] >> (4 * (c & 1)) & 15;
        const unsigned e = n >> 1 & 3;
        const float m = e ? pp_bits((126 + e) << 23 | (n & 1) << 22) : 0.5f * (n & 1);
        return (n & 8 ? -m : m) * pp_unit4(byte);
    }
};
struct FromInt8 {
    const uint8_t *codes, *scales;
    long long groups;
    __device__ float at(long long r, long long c) const {
        return (float)((const int8_t *)codes)[r * groups * PP_GROUP + c] * pp_unit8(scales[r * groups * 4 + c / PP_BLOCK]);
    }
};
template <class Y> struct FromMatrix {
    const typename Y::T *p;
    long long ld;
    __device__ float at(long long r, long long c) const { return Y::get(p[r * ld + c]); }
};
template <class P> struct Flip {
    P p;
    __device__ float at(long long r, long long c) const { return p.at(c, r); }
};

template <class Y> struct ToMatrix {
    typename Y::T *p;
    long long ld;
    const float *add;
    long long add_ld;  // 0: one row for all
    __device__ void put(long long i, long long j, float v) const { p[i * ld + j] = Y::put(add ? v + add[i * add_ld + j] : v); }
};

template <class A, class B, class C>
__global__ __launch_bounds__(256) void k_product(long long rows, long long cols, long long len, unsigned gx, A a, B b, C c) {
    __shared__ float sa[16][65], sb[16][65];
    const long long i0 = (long long)(blockIdx.x / gx) * 64, j0 = (long long)(blockIdx.x % gx) * 64;
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    float acc[4][4] = {};
    for (long long k0 = 0; k0 < len; k0 += 16) {
        for (int t = threadIdx.x; t < 1024; t += 256) {
            const int k = t & 15, i = t >> 4;
            sa[k][i] = i0 + i < rows && k0 + k < len ? a.at(i0 + i, k0 + k) : 0.0f;
            sb[k][i] = j0 + i < cols && k0 + k < len ? b.at(j0 + i, k0 + k) : 0.0f;
        }
        __syncthreads();
        for (int k = 0; k < 16; ++k)
#pragma unroll
            for (int u = 0; u < 4; ++u)
#pragma unroll
                for (int v = 0; v < 4; ++v) acc[u][v] += sa[k][ty + 16 * u] * sb[k][tx + 16 * v];
        __syncthreads();
    }
    for (int u = 0; u < 4; ++u)
        for (int v = 0; v < 4; ++v)
            if (i0 + ty + 16 * u < rows && j0 + tx + 16 * v < cols) c.put(i0 + ty + 16 * u, j0 + tx + 16 * v, acc[u][v]);
}

template <class A, class B, class C>
static int product(long long rows, long long cols, long long len, const A &a, const B &b, const C &c, hipStream_t st) {
    const unsigned gx = (unsigned)((cols + 63) / 64), gy = (unsigned)((rows + 63) / 64);
    k_product<<<gx * gy, 256, 0, st>>>(rows, cols, len, gx, a, b, c);
    return hipGetLastError() == hipSuccess ? PP_OK : PP_ERR_HIP;
}

template <class Y>
__global__ void k_column_sums(long long rows, long long cols, const typename Y::T *__restrict__ p, long long ld, float *__restrict__ out) {
    const long long c = (long long)blockIdx.x * 64 + (threadIdx.x & 63);
    __shared__ float part[4][64];
    float s = 0;
    if (c < cols)
        for (long long r = threadIdx.x >> 6; r < rows; r += 4) s += Y::get(p[r * ld + c]);
    part[threadIdx.x >> 6][threadIdx.x & 63] = s;
    __syncthreads();
    if (threadIdx.x < 64 && c < cols) out[c] = part[0][threadIdx.x] + part[1][threadIdx.x] + part[2][threadIdx.x] + part[3][threadIdx.x];
}

static bool bad_layer(int type, int64_t rows, int64_t n_in, int64_t n_out) {
    return pp_bad_sizes(type, rows, n_in) || n_out < 1 || n_out > PP_LAYER_MAX_COLS;
}

extern "C" size_t pp_linear_workspace_bytes(int call, int type, int64_t rows, int64_t n_in, int64_t n_out) {
    if (call < PP_LINEAR_FORWARD || call > PP_LINEAR_BACKWARD_WEIGHT || bad_layer(type, rows, n_in, n_out)) return 0;
    if (call != PP_LINEAR_FORWARD) return 256;
    return 256 + pp_align256((size_t)rows * pp_groups(n_in) * PP_GROUP_CODES4) + pp_align256((size_t)rows * pp_groups(n_in) * 4);
}

static int bad_workspace(int call, int type, int64_t rows, int64_t n_in, int64_t n_out, const void *ws, size_t bytes) {
    return !ws || ((uintptr_t)ws & 255) || bytes < pp_linear_workspace_bytes(call, type, rows, n_in, n_out) ? PP_ERR_WORKSPACE : PP_OK;
}

extern "C" int pp_linear_forward(int type, int64_t rows, int64_t n_in, int64_t n_out, const void *x, int64_t ld_x, const void *w_codes,
                                 const void *w_scales, const float *bias, void *y, int64_t ld_y, void *x_codes, void *x_scales,
                                 void *workspace, size_t workspace_bytes, void *stream) {
    if (bad_layer(type, rows, n_in, n_out)) return PP_ERR_INVALID_ARG;
    if (pp_bad_matrix(x, type, rows, n_in, ld_x) || pp_bad_matrix(y, type, rows, n_out, ld_y)) return PP_ERR_INVALID_ARG;
    if (pp_bad_packed(w_codes, w_scales, n_out) || ((uintptr_t)bias & 3)) return PP_ERR_INVALID_ARG;
    if ((x_codes || x_scales) && pp_bad_packed(x_codes, x_scales, rows)) return PP_ERR_INVALID_ARG;
    if (int rc = bad_workspace(PP_LINEAR_FORWARD, type, rows, n_in, n_out, workspace, workspace_bytes)) return rc;
    if (!rows) return PP_OK;
    hipStream_t st = (hipStream_t)stream;
    uint8_t *codes = (uint8_t *)workspace, *scales = codes + pp_align256((size_t)rows * pp_groups(n_in) * PP_GROUP_CODES4);
    if (x_codes)
        if (int rc = pp_launch_pack(PP_PACK_INT8, type, rows, n_in, x, ld_x, x_codes, x_scales, st)) return rc;
    if (int rc = pp_launch_pack(PP_PACK_FP4, type, rows, n_in, x, ld_x, codes, scales, st)) return rc;
    const long long g = pp_groups(n_in);
    return pp_by_type(type, [&](auto t) {
        typedef decltype(t) Y;
        return product(rows, n_out, n_in, FromFp4{codes, scales, g}, FromFp4{(const uint8_t *)w_codes, (const uint8_t *)w_scales, g},
                       ToMatrix<Y>{(typename Y::T *)y, ld_y, bias, 0}, st);
    });
}

extern "C" int pp_linear_backward_input(int type, int64_t rows, int64_t n_in, int64_t n_out, const void *dy, int64_t ld_dy,
                                        const void *w_codes, const void *w_scales, void *dx, int64_t ld_dx, void *workspace,
                                        size_t workspace_bytes, void *stream) {
    if (bad_layer(type, rows, n_in, n_out)) return PP_ERR_INVALID_ARG;
    if (pp_bad_matrix(dy, type, rows, n_out, ld_dy) || pp_bad_matrix(dx, type, rows, n_in, ld_dx)) return PP_ERR_INVALID_ARG;
    if (pp_bad_packed(w_codes, w_scales, n_out)) return PP_ERR_INVALID_ARG;
    if (int rc = bad_workspace(PP_LINEAR_BACKWARD_INPUT, type, rows, n_in, n_out, workspace, workspace_bytes)) return rc;
    if (!rows) return PP_OK;
    return pp_by_type(type, [&](auto t) {
        typedef decltype(t) Y;
        return product(rows, n_in, n_out, FromMatrix<Y>{(const typename Y::T *)dy, ld_dy},
                       Flip<FromFp4>{{(const uint8_t *)w_codes, (const uint8_t *)w_scales, pp_groups(n_in)}},
                       ToMatrix<Y>{(typename Y::T *)dx, ld_dx, NULL, 0}, (hipStream_t)stream);
    });
}

extern "C" int pp_linear_backward_weight(int type, int64_t rows, int64_t n_in, int64_t n_out, const void *dy, int64_t ld_dy,
                                         const void *x_codes, const void *x_scales, const float *dw_in, float *dw, int64_t ld_dw,
                                         float *db, void *workspace, size_t workspace_bytes, void *stream) {
    if (bad_layer(type, rows, n_in, n_out)) return PP_ERR_INVALID_ARG;
    if (pp_bad_matrix(dy, type, rows, n_out, ld_dy) || pp_bad_packed(x_codes, x_scales, rows)) return PP_ERR_INVALID_ARG;
    if (pp_bad_matrix(dw, PP_TYPE_F32, n_out, n_in, ld_dw) || ((uintptr_t)dw_in & 3) || ((uintptr_t)db & 3)) return PP_ERR_INVALID_ARG;
    if (int rc = bad_workspace(PP_LINEAR_BACKWARD_WEIGHT, type, rows, n_in, n_out, workspace, workspace_bytes)) return rc;
    hipStream_t st = (hipStream_t)stream;
    return pp_by_type(type, [&](auto t) {
        typedef decltype(t) Y;
        typedef typename Y::T T;
        if (db) {
            k_column_sums<Y><<<(unsigned)((n_out + 63) / 64), 256, 0, st>>>(rows, n_out, (const T *)dy, ld_dy, db);
            if (hipGetLastError() != hipSuccess) return PP_ERR_HIP;
        }
        return product(n_out, n_in, rows, Flip<FromMatrix<Y>>{{(const T *)dy, ld_dy}},
                       Flip<FromInt8>{{(const uint8_t *)x_codes, (const uint8_t *)x_scales, pp_groups(n_in)}},
                       ToMatrix<PpF32>{dw, ld_dw, dw_in, ld_dw}, st);
    });
}
