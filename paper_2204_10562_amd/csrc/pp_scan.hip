// pp_scan_forward, pp_scan_backward, pp_scan_step: the gated linear recurrence h_t = a_t h_(t-1) + (1 - a_t) v_t, a = sigmoid(gate).
#include "pp_rows.h"

#define SC_CHUNK 32  // tokens between kept states
#define SC_MAX_SEQS (1 << 30)

// A token's gate.  s = sigmoid(-|gate|) is the smaller of a and 1 - a; the state moves by it from the nearer end, so that one that
// is kept for thousands of tokens does not lose the digits of 1 - a.
struct sc_gate {
    float s;
    bool keeps;
    __device__ __forceinline__ sc_gate(float f) : keeps(f >= 0.0f) {
        const float e = __builtin_amdgcn_exp2f(-1.44269504f * __builtin_fabsf(f));
        s = e * __builtin_amdgcn_rcpf(1.0f + e);
    }
    __device__ __forceinline__ float next(float h, float v) const {
        const float from = keeps ? h : v, to = keeps ? v : h;
        return __builtin_fmaf(s, to - from, from);
    }
    __device__ __forceinline__ float take(float g) const { return keeps ? s * g : __builtin_fmaf(-s, g, g); }  // (1 - a) g
    __device__ __forceinline__ float keep(float g) const { return keeps ? __builtin_fmaf(-s, g, g) : s * g; }  // a g
    __device__ __forceinline__ float slope() const { return __builtin_fmaf(-s, s, s); }                        // a (1 - a)
};

struct sc_args {
    long long rows, cols, seqs;
    const int *starts;
    const float *h0;
    float *kept;
};

// Rows lo .. hi - 1 of sequence n
__device__ __forceinline__ void sc_bounds(const sc_args &a, long long n, long long &lo, long long &hi) {
    lo = a.starts ? a.starts[n] : 0;
    hi = a.starts ? a.starts[n + 1] : a.rows;
    lo = lo < 0 ? 0 : lo > a.rows ? a.rows : lo;
    hi = hi < lo ? lo : hi > a.rows ? a.rows : hi;
}

template <class Y>
__global__ __launch_bounds__(64) void k_scan_forward(sc_args a, const typename Y::T *__restrict__ gate, long long ld_gate, const typename Y::T *__restrict__ v,
                                                     long long ld_v, typename Y::T *__restrict__ h, long long ld_h, float *__restrict__ h_last) {
    const long long c = blockIdx.x * 64ll + threadIdx.x;
    if (c >= a.cols) return;
    for (long long n = blockIdx.y; n < a.seqs; n += gridDim.y) {
        long long lo, hi;
        sc_bounds(a, n, lo, hi);
        float s = a.h0 ? a.h0[n * a.cols + c] : 0.0f;
        for (long long t = lo; t < hi; ++t) {
            if (a.kept && !(t % SC_CHUNK)) a.kept[t / SC_CHUNK * a.cols + c] = s;
            s = sc_gate(Y::get(gate[t * ld_gate + c])).next(s, Y::get(v[t * ld_v + c]));
            h[t * ld_h + c] = Y::put(s);
        }
        if (h_last) h_last[n * a.cols + c] = s;
    }
}

template <class Y>
__global__ __launch_bounds__(64) void k_scan_backward(sc_args a, const typename Y::T *__restrict__ dh, long long ld_dh, const typename Y::T *__restrict__ gate,
                                                      long long ld_gate, const typename Y::T *__restrict__ v, long long ld_v,
                                                      const float *__restrict__ dh_last, typename Y::T *__restrict__ dgate, long long ld_dgate,
                                                      typename Y::T *__restrict__ dv, long long ld_dv, float *__restrict__ dh0) {
    __shared__ float before[SC_CHUNK][64];
    const long long c = blockIdx.x * 64ll + threadIdx.x;
    if (c >= a.cols) return;
    for (long long n = blockIdx.y; n < a.seqs; n += gridDim.y) {
        long long lo, hi;
        sc_bounds(a, n, lo, hi);
        float g = dh_last ? dh_last[n * a.cols + c] : 0.0f;  // a_(t+1) g_(t+1)
        for (long long end = hi; end > lo;) {
            const long long chunk = (end - 1) / SC_CHUNK, begin = chunk * SC_CHUNK > lo ? chunk * SC_CHUNK : lo;
            float s = begin > lo ? a.kept[chunk * a.cols + c] : a.h0 ? a.h0[n * a.cols + c] : 0.0f;
            for (long long t = begin; t < end; ++t) {
                before[t - begin][threadIdx.x] = s;
                s = sc_gate(Y::get(gate[t * ld_gate + c])).next(s, Y::get(v[t * ld_v + c]));
            }
            for (long long t = end - 1; t >= begin; --t) {
                const sc_gate p(Y::get(gate[t * ld_gate + c]));
                g += Y::get(dh[t * ld_dh + c]);
                dv[t * ld_dv + c] = Y::put(p.take(g));
                dgate[t * ld_dgate + c] = Y::put(p.slope() * (before[t - begin][threadIdx.x] - Y::get(v[t * ld_v + c])) * g);
                g = p.keep(g);
            }
            end = begin;
        }
        if (dh0) dh0[n * a.cols + c] = g;
    }
}

// A thread to eight channels of a row.
template <class Y>
__global__ __launch_bounds__(256) void k_scan_step(long long rows, long long cols, long long chunks, long long n_slots, const int *__restrict__ slots,
                                                   const typename Y::T *__restrict__ gate, long long ld_gate, const typename Y::T *__restrict__ v,
                                                   long long ld_v, float *__restrict__ state, typename Y::T *__restrict__ h, long long ld_h) {
    for (long long at = blockIdx.x * 256ll + threadIdx.x; at < rows * chunks; at += gridDim.x * 256ll) {
        const long long row = at / chunks, c = 8 * (at - row * chunks), left = cols - c, slot = slots ? slots[row] : row;
        if (slot < 0 || slot >= n_slots) continue;
        float f[8], x[8], s[8];
        const PpRaw<Y> rf = pp_load8<Y>(gate + row * ld_gate + c, left), rv = pp_load8<Y>(v + row * ld_v + c, left);
        const PpRaw<PpF32> rs = pp_load8<PpF32>(state + slot * cols + c, left);
        pp_values<Y>(rf, f);
        pp_values<Y>(rv, x);
        pp_values<PpF32>(rs, s);
#pragma unroll
        for (int j = 0; j < 8; ++j) s[j] = sc_gate(f[j]).next(s[j], x[j]);
        pp_store8<PpF32>(state + slot * cols + c, left, s);
        pp_store8<Y>(h + row * ld_h + c, left, s);
    }
}

static bool sc_bad(int type, int64_t rows, int64_t cols, int64_t seqs, const int32_t *starts, const float *h0, const float *kept, const float *x,
                   const float *y) {
    if (pp_bad_sizes(type, rows, cols) || seqs < 0 || seqs > SC_MAX_SEQS || (!starts && seqs != 1)) return true;
    for (const void *p : {(const void *)starts, (const void *)h0, (const void *)kept, (const void *)x, (const void *)y})
        if ((uintptr_t)p & 3) return true;
    return false;
}

extern "C" size_t pp_scan_workspace_bytes(int call, int type, int64_t rows, int64_t cols) {
    if (pp_bad_sizes(type, rows, cols) || (call != PP_SCAN_FORWARD && call != PP_SCAN_BACKWARD)) return 0;
    return 256;
}

extern "C" int64_t pp_scan_kept_rows(int type, int64_t rows, int64_t cols) {
    return pp_bad_sizes(type, rows, cols) ? -1 : (rows + SC_CHUNK - 1) / SC_CHUNK;
}

static dim3 sc_grid(int64_t cols, int64_t seqs) { return dim3((unsigned)((cols + 63) / 64), (unsigned)(seqs < 4096 ? seqs : 4096)); }

extern "C" int pp_scan_forward(int type, int64_t rows, int64_t cols, const void *gate, int64_t ld_gate, const void *v, int64_t ld_v, int64_t seqs,
                               const int32_t *starts, const float *h0, void *h, int64_t ld_h, float *h_last, float *kept, void *workspace,
                               size_t workspace_bytes, void *stream) {
    if (sc_bad(type, rows, cols, seqs, starts, h0, kept, h_last, NULL)) return PP_ERR_INVALID_ARG;
    if (pp_bad_matrix(gate, type, rows, cols, ld_gate) || pp_bad_matrix(v, type, rows, cols, ld_v) || pp_bad_matrix(h, type, rows, cols, ld_h))
        return PP_ERR_INVALID_ARG;
    if (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < pp_scan_workspace_bytes(PP_SCAN_FORWARD, type, rows, cols)) return PP_ERR_WORKSPACE;
    if (!seqs) return PP_OK;
    const sc_args a = {rows, cols, seqs, starts, h0, kept};
    return pp_by_type(type, [&](auto tag) {
        typedef decltype(tag) Y;
        typedef typename Y::T T;
        k_scan_forward<Y><<<sc_grid(cols, seqs), 64, 0, (hipStream_t)stream>>>(a, (const T *)gate, ld_gate, (const T *)v, ld_v, (T *)h, ld_h, h_last);
        return hipGetLastError() == hipSuccess ? PP_OK : PP_ERR_HIP;
    });
}

extern "C" int pp_scan_backward(int type, int64_t rows, int64_t cols, const void *dh, int64_t ld_dh, const void *gate, int64_t ld_gate, const void *v,
                                int64_t ld_v, int64_t seqs, const int32_t *starts, const float *h0, const float *kept, const float *dh_last, void *dgate,
                                int64_t ld_dgate, void *dv, int64_t ld_dv, float *dh0, void *workspace, size_t workspace_bytes, void *stream) {
    if (sc_bad(type, rows, cols, seqs, starts, h0, kept, dh_last, dh0) || (rows && !kept)) return PP_ERR_INVALID_ARG;
    if (pp_bad_matrix(dh, type, rows, cols, ld_dh) || pp_bad_matrix(gate, type, rows, cols, ld_gate) || pp_bad_matrix(v, type, rows, cols, ld_v) ||
        pp_bad_matrix(dgate, type, rows, cols, ld_dgate) || pp_bad_matrix(dv, type, rows, cols, ld_dv))
        return PP_ERR_INVALID_ARG;
    if (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < pp_scan_workspace_bytes(PP_SCAN_BACKWARD, type, rows, cols)) return PP_ERR_WORKSPACE;
    if (!seqs) return PP_OK;
    const sc_args a = {rows, cols, seqs, starts, h0, (float *)kept};
    return pp_by_type(type, [&](auto tag) {
        typedef decltype(tag) Y;
        typedef typename Y::T T;
        k_scan_backward<Y><<<sc_grid(cols, seqs), 64, 0, (hipStream_t)stream>>>(a, (const T *)dh, ld_dh, (const T *)gate, ld_gate, (const T *)v, ld_v, dh_last,
                                                                                (T *)dgate, ld_dgate, (T *)dv, ld_dv, dh0);
        return hipGetLastError() == hipSuccess ? PP_OK : PP_ERR_HIP;
    });
}

extern "C" int pp_scan_step(int type, int64_t rows, int64_t cols, const void *gate, int64_t ld_gate, const void *v, int64_t ld_v, int64_t n_slots,
                            const int32_t *slots, float *state, void *h, int64_t ld_h, void *stream) {
    if (pp_bad_sizes(type, rows, cols) || n_slots < 0 || n_slots > PP_LAYER_MAX_ROWS || ((uintptr_t)slots & 3) || ((uintptr_t)state & 3)) return PP_ERR_INVALID_ARG;
    if (pp_bad_matrix(gate, type, rows, cols, ld_gate) || pp_bad_matrix(v, type, rows, cols, ld_v) || pp_bad_matrix(h, type, rows, cols, ld_h))
        return PP_ERR_INVALID_ARG;
    if (rows && (!state || (!slots && rows > n_slots))) return PP_ERR_INVALID_ARG;
    if (!rows) return PP_OK;
    const int64_t chunks = (cols + 7) / 8, groups = (rows * chunks + 255) / 256;
    return pp_by_type(type, [&](auto tag) {
        typedef decltype(tag) Y;
        typedef typename Y::T T;
        k_scan_step<Y><<<(unsigned)(groups < (1 << 20) ? groups : 1 << 20), 256, 0, (hipStream_t)stream>>>(rows, cols, chunks, n_slots, slots, (const T *)gate, ld_gate,
                                                                                                         (const T *)v, ld_v, state, (T *)h, ld_h);
        return hipGetLastError() == hipSuccess ? PP_OK : PP_ERR_HIP;
    });
}
