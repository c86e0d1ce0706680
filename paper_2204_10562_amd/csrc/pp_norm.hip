// pp_norm_forward, pp_norm_backward: root-mean-square norm of rows with the residual's addition.
//
// forward   s = x + res, inv = 1 / sqrt(mean s^2 + eps), y = s inv g
// backward  with z = s inv:  dx = inv (g dy - z mean(g dy z)) + dtotal,  dg = dg_in + sum over the rows of dy z
//
// A row stays in the registers of the threads that read it (a wave, or workgroups of up to 16) between its sum and its results, so
// every byte is read and written once; rows of more than 32768 columns forward, 16384 backward, are read twice.  A thread takes
// eight neighbours at a time, a quad a block of 32, as in packing.
//
// Bytes bound both passes.  8192 x 4096 bf16, where a copy of 1 GiB reaches 5.1 to 5.2 TB/s: forward 50 us (268 MB, 5.3 TB/s), with s and y in
// 8 bits as well 62 to 66 (338 MB, 5.3); backward 52 (268 MB, 5.2), from s in 8 bits 53 to 58 (236 MB, 4.2) of which 4.7 are the second
// kernel, which adds the parts of dg.  Small ones are launches: one row of 4096 3.1 us.  Rows below 512 columns have a wave each all the same, and leave
// most of its lanes idle: 262144 x 128 bf16 139 and 152 us (52 by bytes), x 64 113 and 143 (26).  The backward pass of float32 rows of 8193 to 16384
// columns from 8 bits wants 7 registers more than there are.
// Waves to a row, by eight chunks of columns: with more chunks to a thread and fewer waves less is on its way, 2048 x 16384 bf16 forward 77 us with
// four waves and 57 with eight, 4096 x 8192 with copies 86 and 71; sixteen 59 and 74; 8192 x 6144 with four
// 89, with twelve 79.  (Backward twelve instead of sixteen give nothing.)
#include "pp_rows.h"

#define NM_MAX_GRID (1 << 20)
// Most waves of a backward pass (16 to a unit); each workgroup has its own part of dg.  Half as many take 74 us for the 53 of 8192 x 4096 bf16 from
// 8 bits, half as many again 48, but 62 for 50 of 4096 x 8192 and 43 for 36 of 32768 x 512.
#define NM_PART_WAVES 4096
#define NM_WIDE 2048         // most chunks of a row in the backward pass that holds it (16384 columns)
#define NM_WIDE_GROUPS 2048  // workgroups of one that does not

// A row's values: a matrix of type Y, or what PP_PACK_INT8 left of one.
template <class Y> struct nm_matrix {
    const typename Y::T *p;
    long long ld;
};
struct nm_packed {
    uint8_t *codes, *scales;
};

struct nm_forward {
    long long rows, cols;
    float eps;
    const float *gain;
    float *inv;
    nm_packed y8, s8;  // codes NULL: not wanted
};

__device__ __forceinline__ void load_gain(const float *gain, long long c, long long left, float *g) {
    if (gain) {
        const PpRaw<PpF32> raw = pp_load8<PpF32>(gain + c, left);
        pp_values<PpF32>(raw, g);
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) g[j] = 1.0f;
    }
}

// s of chunk q of a row, zeros beyond the last column
template <class Y> __device__ __forceinline__ void load_sum(nm_matrix<Y> x, nm_matrix<Y> res, long long row, long long q, long long left, float *s) {
    pp_values<Y>(pp_load8<Y>(x.p + row * x.ld + 8 * q, left), s);
    if (res.p) {
        float r[8];
        pp_values<Y>(pp_load8<Y>(res.p + row * res.ld + 8 * q, left), r);
#pragma unroll
        for (int j = 0; j < 8; ++j) s[j] += r[j];
    }
}

template <class Y>
__device__ __forceinline__ void put_forward(const nm_forward &f, typename Y::T *total, long long ld_total, typename Y::T *y, long long ld_y,
                                            long long row, long long q, long long chunks, long long left, float inv, const float *s, const float *g) {
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = left > j ? s[j] * inv * g[j] : 0.0f;
    if (total && left > 0) pp_store8<Y>(total + row * ld_total + 8 * q, left, s);
    if (f.s8.codes) pp_put_codes8(row * chunks + q, s, f.s8.codes, f.s8.scales);
    if (y && left > 0) pp_store8<Y>(y + row * ld_y + 8 * q, left, v);
    if (f.y8.codes) pp_put_codes8(row * chunks + q, v, f.y8.codes, f.y8.scales);
}

// WAVES waves to a row, CH chunks to a thread; CH = 0: the row is read twice, whatever its length.
// total may be res or x: a thread writes a chunk after its last read of it.
template <class Y, int WAVES, int CH>
__global__ __launch_bounds__(WAVES == 1 ? 256 : WAVES * PP_WAVE) void k_norm_forward(nm_forward f, nm_matrix<Y> x, nm_matrix<Y> res, typename Y::T *total,
                                                                                      long long ld_total, typename Y::T *y, long long ld_y) {
    __shared__ float room[2][WAVES];
    const int t = WAVES == 1 ? threadIdx.x & (PP_WAVE - 1) : threadIdx.x;
    const long long chunks = (f.cols + PP_GROUP - 1) / PP_GROUP * (PP_GROUP / 8);
    const long long per = WAVES == 1 ? 256 / PP_WAVE : 1;
    int turn = 0;
    for (long long row = blockIdx.x * per + (WAVES == 1 ? threadIdx.x / PP_WAVE : 0); row < f.rows; row += gridDim.x * per) {
        float s[CH ? CH : 1][8], g[CH ? CH : 1][8], sum = 0.0f;
        if constexpr (CH > 0) {
#pragma unroll
            for (int i = 0; i < CH; ++i) {
                const long long q = t + i * WAVES * PP_WAVE;
                load_sum<Y>(x, res, row, q, f.cols - 8 * q, s[i]);
            }
#pragma unroll
            for (int i = 0; i < CH; ++i) {
                const long long q = t + i * WAVES * PP_WAVE;
                load_gain(f.gain, 8 * q, f.cols - 8 * q, g[i]);
            }
#pragma unroll
            for (int i = 0; i < CH; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) sum = __builtin_fmaf(s[i][j], s[i][j], sum);
        } else {
            for (long long q = t; q < chunks; q += WAVES * PP_WAVE) {
                load_sum<Y>(x, res, row, q, f.cols - 8 * q, s[0]);
                float part = 0.0f;
#pragma unroll
                for (int j = 0; j < 8; ++j) part = __builtin_fmaf(s[0][j], s[0][j], part);
                sum += part;
            }
        }
        sum = pp_group_sum<WAVES>(sum, room[turn]);
        turn ^= 1;
        const float inv = __builtin_amdgcn_rsqf(sum / (float)f.cols + f.eps);
        if (f.inv && !t) f.inv[row] = inv;
        if constexpr (CH > 0) {
#pragma unroll
            for (int i = 0; i < CH; ++i) {
                const long long q = t + i * WAVES * PP_WAVE;
                if (q < chunks) put_forward<Y>(f, total, ld_total, y, ld_y, row, q, chunks, f.cols - 8 * q, inv, s[i], g[i]);
            }
        } else {
            for (long long q = t; q < chunks; q += WAVES * PP_WAVE) {
                load_sum<Y>(x, res, row, q, f.cols - 8 * q, s[0]);
                load_gain(f.gain, 8 * q, f.cols - 8 * q, g[0]);
                put_forward<Y>(f, total, ld_total, y, ld_y, row, q, chunks, f.cols - 8 * q, inv, s[0], g[0]);
            }
        }
    }
}

static int64_t nm_chunks(int64_t cols) { return pp_groups(cols) * (PP_GROUP / 8); }

template <class Y, int WAVES, int CH>
static void forward(hipStream_t st, const nm_forward &f, nm_matrix<Y> x, nm_matrix<Y> res, typename Y::T *total, int64_t ld_total, typename Y::T *y,
                    int64_t ld_y) {
    const int64_t per = WAVES == 1 ? 256 / PP_WAVE : 1, want = (f.rows + per - 1) / per;
    k_norm_forward<Y, WAVES, CH><<<(unsigned)(want < NM_MAX_GRID ? want : NM_MAX_GRID), WAVES == 1 ? 256 : WAVES * PP_WAVE, 0, st>>>(
        f, x, res, total, ld_total, y, ld_y);
}

static bool nm_bad_pair(const void *codes, const void *scales, int64_t rows) { return (codes || scales) && pp_bad_packed(codes, scales, rows); }
static bool nm_bad_floats(const void *p) { return ((uintptr_t)p & 3) != 0; }

extern "C" int pp_norm_forward(int type, int64_t rows, int64_t cols, const void *x, int64_t ld_x, const void *res, int64_t ld_res, const float *gain,
                               float eps, void *total, int64_t ld_total, void *y, int64_t ld_y, void *y_codes, void *y_scales, void *total_codes,
                               void *total_scales, float *inv, void *stream) {
    if (pp_bad_sizes(type, rows, cols) || !(eps >= 0x1p-126f) || eps > 0x1p126f) return PP_ERR_INVALID_ARG;
    if (pp_bad_matrix(x, type, rows, cols, ld_x) || (res && pp_bad_matrix(res, type, rows, cols, ld_res))) return PP_ERR_INVALID_ARG;
    if ((total && pp_bad_matrix(total, type, rows, cols, ld_total)) || (y && pp_bad_matrix(y, type, rows, cols, ld_y))) return PP_ERR_INVALID_ARG;
    if (nm_bad_pair(y_codes, y_scales, rows) || nm_bad_pair(total_codes, total_scales, rows)) return PP_ERR_INVALID_ARG;
    if (rows && !y && !y_codes) return PP_ERR_INVALID_ARG;
    if (nm_bad_floats(gain) || nm_bad_floats(inv)) return PP_ERR_INVALID_ARG;
    if (!rows) return PP_OK;
    const int64_t chunks = nm_chunks(cols);
    hipStream_t st = (hipStream_t)stream;
    return pp_by_type(type, [&](auto tag) {
        typedef decltype(tag) Y;
        typedef typename Y::T T;
        const nm_forward f = {rows, cols, eps, gain, inv, {(uint8_t *)y_codes, (uint8_t *)y_scales}, {(uint8_t *)total_codes, (uint8_t *)total_scales}};
        const nm_matrix<Y> mx = {(const T *)x, ld_x}, mr = {(const T *)res, ld_res};
        auto go = [&](auto waves, auto ch) {
            forward<Y, decltype(waves)::value, decltype(ch)::value>(st, f, mx, mr, (T *)total, ld_total, (T *)y, ld_y);
        };
#define I(n) std::integral_constant<int, n>()
        if (chunks <= 64) go(I(1), I(1));
        else if (chunks <= 128 && rows >= 1024) go(I(1), I(2));
        else if (chunks <= 256 && rows >= 1024) go(I(1), I(4));
        else if (chunks <= 256) go(I(4), I(1));
        else if (chunks <= 512) go(I(8), I(1));
        else if (chunks <= 768) go(I(12), I(1));
        else if (chunks <= 1024) go(I(8), I(2));
        else if (chunks <= 1536) go(I(8), I(3));
        else if (chunks <= 2048) go(I(8), I(4));
        else if (chunks <= 4096) go(I(16), I(4));
        else go(I(16), I(0));
        return hipGetLastError() == hipSuccess ? PP_OK : PP_ERR_HIP;
    });
}

// ---------------------------------------------------------------- backward

struct nm_backward {
    long long rows, cols;
    const float *inv, *gain;
    float *part;  // [parts][cols] of dg, or NULL: not wanted
    nm_packed s8; // the kept sum; codes NULL: a matrix
};

// A chunk of a row as it was loaded
template <class Y, bool PACKED> struct nm_chunk {
    PpRaw<Y> dy, more, s[PACKED ? 0 : 1];
    pp_u2 codes;
    unsigned char scale;
};
template <class Y, bool PACKED>
__device__ __forceinline__ nm_chunk<Y, PACKED> load_chunk(const nm_backward &b, nm_matrix<Y> dy, nm_matrix<Y> s, nm_matrix<Y> dtotal, long long row, long long q,
                                                          long long chunks) {
    nm_chunk<Y, PACKED> c = {};
    const long long left = b.cols - 8 * q;
    c.dy = pp_load8<Y>(dy.p + row * dy.ld + 8 * q, left);
    if constexpr (!PACKED) c.s[0] = pp_load8<Y>(s.p + row * s.ld + 8 * q, left);
    else if (left > 0) {
        c.codes = *(const pp_u2 *)(b.s8.codes + (row * chunks + q) * 8);
        c.scale = b.s8.scales[(row * chunks + q) >> 2];
    }
    if (dtotal.p) c.more = pp_load8<Y>(dtotal.p + row * dtotal.ld + 8 * q, left);
    return c;
}

// With one chunk to a thread the next row is on its way while a row's sum is made (with more the registers for it cost more than
// it gives).  dx may be dy or dtotal: their values of a row have been read before it is written.
template <class Y, int WAVES, int CH, bool PACKED>
__global__ __launch_bounds__(WAVES *PP_WAVE) void k_norm_backward(nm_backward b, nm_matrix<Y> dy, nm_matrix<Y> s, nm_matrix<Y> dtotal, typename Y::T *dx,
                                                                   long long ld_dx) {
    __shared__ float room[2][WAVES];
    const int t = threadIdx.x;
    const long long chunks = (b.cols + PP_GROUP - 1) / PP_GROUP * (PP_GROUP / 8);
    float dg[CH][8] = {}, g[CH][8];
    nm_chunk<Y, PACKED> c[CH];
    int turn = 0;
#pragma unroll
    for (int i = 0; i < CH; ++i) {
        const long long q = t + i * WAVES * PP_WAVE;
        if constexpr (CH == 1) c[i] = load_chunk<Y, PACKED>(b, dy, s, dtotal, blockIdx.x, q, chunks);
        load_gain(b.gain, 8 * q, b.cols - 8 * q, g[i]);
    }
    for (long long row = blockIdx.x; row < b.rows; row += gridDim.x) {
        const float inv = b.inv[row];
        float d[CH][8], z[CH][8], dot = 0.0f;
        if constexpr (CH > 1)
#pragma unroll
            for (int i = 0; i < CH; ++i) c[i] = load_chunk<Y, PACKED>(b, dy, s, dtotal, row, t + i * WAVES * PP_WAVE, chunks);
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            const long long left = b.cols - 8ll * (t + i * WAVES * PP_WAVE);
            pp_values<Y>(c[i].dy, d[i]);
            if constexpr (PACKED) pp_values8(c[i].codes, pp_unit8(c[i].scale), z[i]);
            else pp_values<Y>(c[i].s[0], z[i]);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                z[i][j] = left > j ? z[i][j] * inv : 0.0f;
                dg[i][j] = __builtin_fmaf(d[i][j], z[i][j], dg[i][j]);
                d[i][j] *= g[i][j];
                dot = __builtin_fmaf(d[i][j], z[i][j], dot);
            }
        }
        PpRaw<Y> extra[CH];
#pragma unroll
        for (int i = 0; i < CH; ++i) extra[i] = c[i].more;
        if (CH == 1 && row + gridDim.x < b.rows) c[0] = load_chunk<Y, PACKED>(b, dy, s, dtotal, row + gridDim.x, t, chunks);
        const float mean = pp_group_sum<WAVES>(dot, room[turn]) / (float)b.cols;
        turn ^= 1;
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            const long long q = t + i * WAVES * PP_WAVE, left = b.cols - 8 * q;
            float more[8];
            pp_values<Y>(extra[i], more);
#pragma unroll
            for (int j = 0; j < 8; ++j) d[i][j] = __builtin_fmaf(inv, __builtin_fmaf(-z[i][j], mean, d[i][j]), more[j]);
            if (left > 0) pp_store8<Y>(dx + row * ld_dx + 8 * q, left, d[i]);
        }
    }
    if (b.part)
#pragma unroll
        for (int i = 0; i < CH; ++i) {
            const long long q = t + i * WAVES * PP_WAVE, left = b.cols - 8 * q;
            if (left > 0) pp_store8<PpF32>(b.part + blockIdx.x * b.cols + 8 * q, left, dg[i]);
        }
}

// Rows too long to be held: their mean(g dy z) first, then a workgroup to 2048 columns of some rows.
template <class Y> __global__ __launch_bounds__(1024) void k_norm_dot(nm_backward b, nm_matrix<Y> dy, nm_matrix<Y> s, float *means) {
    __shared__ float room[2][16];
    const long long chunks = (b.cols + PP_GROUP - 1) / PP_GROUP * (PP_GROUP / 8);
    int turn = 0;
    for (long long row = blockIdx.x; row < b.rows; row += gridDim.x) {
        const float inv = b.inv[row];
        float dot = 0.0f;
        for (long long q = threadIdx.x; 8 * q < b.cols; q += 1024) {
            const long long left = b.cols - 8 * q;
            float d[8], z[8], g[8], part = 0.0f;
            pp_values<Y>(pp_load8<Y>(dy.p + row * dy.ld + 8 * q, left), d);
            if (b.s8.codes) pp_get_codes8(row * chunks + q, b.s8.codes, b.s8.scales, z);
            else pp_values<Y>(pp_load8<Y>(s.p + row * s.ld + 8 * q, left), z);
            load_gain(b.gain, 8 * q, left, g);
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (left > j) part = __builtin_fmaf(d[j] * g[j], z[j] * inv, part);
            dot += part;
        }
        dot = pp_group_sum<16>(dot, room[turn]);
        turn ^= 1;
        if (!threadIdx.x) means[row] = dot / (float)b.cols;
    }
}

template <class Y>
__global__ __launch_bounds__(256) void k_norm_wide(nm_backward b, const float *means, nm_matrix<Y> dy, nm_matrix<Y> s, nm_matrix<Y> dtotal,
                                                   typename Y::T *dx, long long ld_dx) {
    const long long chunks = (b.cols + PP_GROUP - 1) / PP_GROUP * (PP_GROUP / 8), q = blockIdx.x * 256ll + threadIdx.x, left = b.cols - 8 * q;
    if (left <= 0) return;
    float dg[8] = {}, g[8];
    load_gain(b.gain, 8 * q, left, g);
    for (long long row = blockIdx.y; row < b.rows; row += gridDim.y) {
        const float inv = b.inv[row], mean = means[row];
        float d[8], z[8], more[8] = {};
        pp_values<Y>(pp_load8<Y>(dy.p + row * dy.ld + 8 * q, left), d);
        if (b.s8.codes) pp_get_codes8(row * chunks + q, b.s8.codes, b.s8.scales, z);
        else pp_values<Y>(pp_load8<Y>(s.p + row * s.ld + 8 * q, left), z);
        if (dtotal.p) pp_values<Y>(pp_load8<Y>(dtotal.p + row * dtotal.ld + 8 * q, left), more);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            z[j] *= inv;
            dg[j] = __builtin_fmaf(d[j], z[j], dg[j]);
            d[j] = __builtin_fmaf(inv, __builtin_fmaf(-z[j], mean, d[j] * g[j]), more[j]);
        }
        pp_store8<Y>(dx + row * ld_dx + 8 * q, left, d);
    }
    if (b.part) pp_store8<PpF32>(b.part + blockIdx.y * b.cols + 8 * q, left, dg);
}

// dg = dg_in + the parts: a workgroup to 32 columns, eight threads to four columns each by 32 groups of parts
__global__ __launch_bounds__(256) void k_norm_gain(long long cols, int parts, const float *__restrict__ part, const float *dg_in, float *dg) {
    __shared__ float room[32][33];
    const int t = threadIdx.x & 7, w = threadIdx.x >> 3;
    const long long c = blockIdx.x * 32ll + 4 * t;
    // The last columns' four end with the last one, and some are added by two threads: one by one they took 60 us of 11953 x 394.  (Of fewer than
    // four columns a part is read with what lies behind it in the workspace.)
    const long long from = c + 4 <= cols || cols < 4 ? c : cols - 4;
    float sum[4] = {};
    if (c < cols) {
#pragma unroll 8
        for (int p = w; p < parts; p += 32) {
            const pp_u4 v = ((const pp_any16<4> *)(part + p * cols + from))->v;
#pragma unroll
            for (int k = 0; k < 4; ++k) sum[k] += pp_bits(v[k]);
        }
    }
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if (from + k >= c) room[w][from + k - blockIdx.x * 32ll] = sum[k];
    __syncthreads();
    const long long col = blockIdx.x * 32ll + threadIdx.x;
    if (threadIdx.x >= 32 || col >= cols) return;
    float all = 0.0f;
#pragma unroll
    for (int k = 0; k < 32; ++k) all += room[k][threadIdx.x];
    dg[col] = dg_in ? dg_in[col] + all : all;
}

// Waves to a row of the backward pass that holds it, and workgroups that have parts of dg
static int nm_waves(int64_t chunks) { return chunks <= 64 ? 1 : chunks <= 128 ? 2 : chunks <= 256 ? 4 : chunks <= 512 ? 8 : 16; }
static int64_t nm_parts(int64_t rows, int64_t cols) {
    const int64_t chunks = nm_chunks(cols), columns = (chunks + 255) / 256;  // (of workgroups beside each other, for rows that are not held)
    const int64_t wide = columns >= NM_WIDE_GROUPS ? 1 : columns * 256 <= NM_WIDE_GROUPS ? 256 : NM_WIDE_GROUPS / columns;
    const int64_t most = chunks > NM_WIDE ? wide : NM_PART_WAVES / nm_waves(chunks);
    return rows < most ? rows : most;
}

extern "C" size_t pp_norm_workspace_bytes(int type, int64_t rows, int64_t cols) {
    if (pp_bad_sizes(type, rows, cols)) return 0;
    return pp_align256((size_t)nm_parts(rows, cols) * cols * 4) + pp_align256((size_t)rows * 4) + 256;
}

extern "C" int pp_norm_backward(int type, int64_t rows, int64_t cols, const void *dy, int64_t ld_dy, const void *total, int64_t ld_total,
                                const void *total_codes, const void *total_scales, const float *inv, const float *gain, const void *dtotal,
                                int64_t ld_dtotal, void *dx, int64_t ld_dx, const float *dgain_in, float *dgain, void *workspace, size_t workspace_bytes,
                                void *stream) {
    if (pp_bad_sizes(type, rows, cols) || nm_bad_floats(inv) || nm_bad_floats(gain) || nm_bad_floats(dgain) || nm_bad_floats(dgain_in)) return PP_ERR_INVALID_ARG;
    if (pp_bad_matrix(dy, type, rows, cols, ld_dy) || pp_bad_matrix(dx, type, rows, cols, ld_dx)) return PP_ERR_INVALID_ARG;
    if (dtotal && pp_bad_matrix(dtotal, type, rows, cols, ld_dtotal)) return PP_ERR_INVALID_ARG;
    if (nm_bad_pair(total_codes, total_scales, rows) || (dgain_in && !dgain) || (rows && !inv)) return PP_ERR_INVALID_ARG;
    if (rows && (total_codes ? total != NULL : pp_bad_matrix(total, type, rows, cols, ld_total))) return PP_ERR_INVALID_ARG;
    const bool wide = nm_chunks(cols) > NM_WIDE;
    if (dgain || wide)
        if (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < pp_norm_workspace_bytes(type, rows, cols)) return PP_ERR_WORKSPACE;
    hipStream_t st = (hipStream_t)stream;
    const int64_t parts = nm_parts(rows, cols), chunks = nm_chunks(cols);
    float *part = (float *)workspace, *means = (float *)((char *)workspace + pp_align256((size_t)parts * cols * 4));
    int rc = PP_OK;
    if (rows)
        rc = pp_by_type(type, [&](auto tag) {
            typedef decltype(tag) Y;
            typedef typename Y::T T;
            const nm_backward b = {rows, cols, inv, gain, dgain ? part : NULL, {(uint8_t *)total_codes, (uint8_t *)total_scales}};
            const nm_matrix<Y> md = {(const T *)dy, ld_dy}, ms = {(const T *)total, ld_total}, mt = {(const T *)dtotal, ld_dtotal};
            auto go = [&](auto waves, auto ch) {
                constexpr int W = decltype(waves)::value, C = decltype(ch)::value;
                if (total_codes) k_norm_backward<Y, W, C, true><<<(unsigned)parts, W * PP_WAVE, 0, st>>>(b, md, ms, mt, (T *)dx, ld_dx);
                else k_norm_backward<Y, W, C, false><<<(unsigned)parts, W * PP_WAVE, 0, st>>>(b, md, ms, mt, (T *)dx, ld_dx);
            };
            if (wide) {
                k_norm_dot<Y><<<(unsigned)(rows < NM_MAX_GRID ? rows : NM_MAX_GRID), 1024, 0, st>>>(b, md, ms, means);
                if (hipGetLastError() != hipSuccess) return PP_ERR_HIP;
                k_norm_wide<Y><<<dim3((unsigned)((chunks + 255) / 256), (unsigned)parts), 256, 0, st>>>(b, means, md, ms, mt, (T *)dx, ld_dx);
            } else if (chunks <= 64) go(I(1), I(1));
            else if (chunks <= 128) go(I(2), I(1));
            else if (chunks <= 256) go(I(4), I(1));
            else if (chunks <= 512) go(I(8), I(1));
            else if (chunks <= 1024) go(I(16), I(1));
            else go(I(16), I(2));
            return hipGetLastError() == hipSuccess ? PP_OK : PP_ERR_HIP;
        });
    if (rc != PP_OK || !dgain) return rc;
    k_norm_gain<<<(unsigned)((cols + 31) / 32), 256, 0, st>>>(cols, (int)parts, part, dgain_in, dgain);
    return hipGetLastError() == hipSuccess ? PP_OK : PP_ERR_HIP;
}
