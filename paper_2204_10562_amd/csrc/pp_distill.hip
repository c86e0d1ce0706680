// pp_distill_loss: the divergence of a student's rows of logits from a teacher of whom the top entries are known, and its gradient.
//
// With p = softmax(x / T) and q the listed entries' probabilities (PP_DISTILL_TOP: softmax(value / T); PP_DISTILL_REST: exp(value), and
// r = 1 - sum q for all others):
//   loss = w (sum q (ln q - ln p) + r (ln r - ln p_rest)),  dx_j = (w / T) (p_j - q_j), and beside the list (w / T) p_j (1 - r / p_rest)
// p_rest is the sum over what is not listed and not 1 less what is: a student that is nearly sure of the listed entries keeps the
// digits of the rest.  So the pass over a row leaves the listed entries out (a bit each in LDS), and they are added afterwards.
//
// Three kernels: the sums of segments; a wave to a row for the list; the gradient.
#include "pp_loss.h"

struct ds_args {
    long long rows, cols, size, ld, ld_d;
    int segs, top, rest;
    float k;
    double inv_t;
    const int *index;
    const float *value, *weight;
    float *loss;
    pp_f2 *sums;   // [rows][segs]: m, s of what is not listed
    pp_f2 *tail;   // [rows]: dx beside the list is [1] 2^((x - [0]) k)
    float *listed; // [rows][top]: dx of the listed
};

// Bits of the listed columns of a segment: byte i of thread t for its chunk i.
template <int HELD> __device__ __forceinline__ void mark_listed(const ds_args &a, long long row, long long first, unsigned *marks) {
    const int t = threadIdx.x, words = (HELD + 3) / 4;
    for (int i = 0; i < words; ++i) marks[t * words + i] = 0;
    __syncthreads();
    for (int e = t; e < a.top; e += LS_THREADS) {
        const long long at = a.index[row * a.top + e] - first;
        if (at >= 0 && at < a.size && at + first < a.cols) {
            const int c = (int)(at >> 3), i = c / LS_THREADS;
            atomicOr(&marks[c % LS_THREADS * words + i / 4], 1u << (8 * (i & 3) + (int)(at & 7)));
        }
    }
    __syncthreads();
}

template <class Y, int HELD> __global__ __launch_bounds__(LS_THREADS, 4) void k_distill_sums(ds_args a, const typename Y::T *__restrict__ logits) {
    const int t = threadIdx.x, words = (HELD + 3) / 4;
    __shared__ unsigned marks[LS_THREADS * ((HELD + 3) / 4)];
    __shared__ float room[8];
    for (long long item = blockIdx.x; item < a.rows * a.segs; item += gridDim.x) {
        const long long row = item / a.segs, first = (item - row * a.segs) * a.size;
        if (a.weight && a.weight[row] == 0.0f) continue;
        const typename Y::T *x = logits + row * a.ld + first;
        const long long n = a.cols - first < a.size ? a.cols - first : a.size;
        PpRaw<Y> raw[HELD];
        ls_load_all<Y, HELD>(raw, x, n);
        mark_listed<HELD>(a, row, first, marks);
        float v[8], m = -__builtin_inff();
#pragma unroll
        for (int i = 0; i < HELD; ++i) {
            const unsigned mark = marks[t * words + i / 4] >> (8 * (i & 3)) & 255;
            if (mark) {
                typename Y::T u[8];
                __builtin_memcpy(u, &raw[i], sizeof(u));
#pragma unroll
                for (int j = 0; j < 8; ++j) u[j] = mark >> j & 1 ? (typename Y::T)-__builtin_inff() : u[j];
                __builtin_memcpy(&raw[i], u, sizeof(u));
            }
            pp_values<Y>(raw[i], v);
            m = __builtin_fmaxf(m, ls_max8(v));
        }
        const float base = ls_base(ls_group_max<4>(m, room));
        float s = 0.0f;
        ls_hold<Y>(raw);
#pragma unroll
        for (int i = 0; i < HELD; ++i) {
            pp_values<Y>(raw[i], v);
#pragma unroll
            for (int j = 0; j < 8; ++j) s += __builtin_amdgcn_exp2f((v[j] - base) * a.k);
        }
        s = pp_group_sum<4>(s, room + 4);
        if (!t) a.sums[item] = pp_f2{base, s};
        __syncthreads();
    }
}

__device__ __forceinline__ double wave_sum(double v) {
    for (int d = 1; d < PP_WAVE; d <<= 1) v += __shfl_xor(v, d);
    return v;
}
__device__ __forceinline__ double wave_max(double v) {
    for (int d = 1; d < PP_WAVE; d <<= 1) v = __builtin_fmax(v, __shfl_xor(v, d));
    return v;
}

// A row's list: in 64 bits, since 1 less the listed probabilities has nothing left in 32 where the teacher is sure, and a
// divergence is a small difference of large terms.
#define DS_PER (PP_TOP_MAX / PP_WAVE)
template <class Y> __global__ __launch_bounds__(PP_WAVE) void k_distill_list(ds_args a, const typename Y::T *logits) {
    __shared__ int index[PP_TOP_MAX];
    __shared__ double q_of[PP_TOP_MAX];
    const int t = threadIdx.x;
    const double inf = __builtin_inf(), kd = a.inv_t;
    for (long long row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const float weight = a.weight ? a.weight[row] : 1.0f;
        __syncthreads();
        if (weight == 0.0f) {
            if (!t) {
                a.loss[row] = 0.0f;
                a.tail[row] = pp_f2{0.0f, 0.0f};
            }
            for (int e = t; e < a.top; e += PP_WAVE) a.listed[row * a.top + e] = 0.0f;
            continue;
        }
        // what is not listed
        double m = -inf, s = 0.0;
        for (int i = t; i < a.segs; i += PP_WAVE) {
            const pp_f2 p = a.sums[row * a.segs + i];
            if (p[1] != 0.0f) m = __builtin_fmax(m, (double)p[0]);
        }
        m = wave_max(m);
        if (m == -inf) m = 0.0;
        for (int i = t; i < a.segs; i += PP_WAVE) {
            const pp_f2 p = a.sums[row * a.segs + i];
            if (p[1] != 0.0f) s += (double)p[1] * exp(((double)p[0] - m) * kd);
        }
        s = wave_sum(s);
        // the list: entries without a column or with a value of -infinity say nothing (a column of theirs is listed all the same)
        double z[DS_PER], lq[DS_PER], most = -inf, sum_q = 0.0, top_x = s > 0.0 ? m : -inf;
        int at[DS_PER];
#pragma unroll
        for (int i = 0; i < DS_PER; ++i) {
            const int e = t + i * PP_WAVE;
            at[i] = e < a.top ? a.index[row * a.top + e] : -1;
            if (at[i] >= a.cols) at[i] = -1;
            lq[i] = at[i] >= 0 ? (double)a.value[row * a.top + e] * (a.rest ? 1.0 : kd) : -inf;
            z[i] = at[i] >= 0 ? (double)Y::get(logits[row * a.ld + at[i]]) : -inf;
            if (e < a.top) index[e] = at[i];
            top_x = __builtin_fmax(top_x, z[i]);
            most = __builtin_fmax(most, lq[i]);
        }
        // exponents from the row's largest logit on: beside the type's lowest value, as a mask, a logarithm has no digits left
        top_x = wave_max(top_x);
        const bool empty = top_x == -inf && s == 0.0;
        const double base = top_x == -inf ? 0.0 : top_x, zm = (m - base) * kd;
#pragma unroll
        for (int i = 0; i < DS_PER; ++i) z[i] = (z[i] - base) * kd;
        double r = 0.0;
        if (a.rest) {
#pragma unroll
            for (int i = 0; i < DS_PER; ++i) sum_q += exp(lq[i]);
            r = 1.0 - wave_sum(sum_q);
            if (r < 0x1p-20) r = 0.0;
        } else {
            most = wave_max(most);
            if (most == -inf) most = 0.0;
#pragma unroll
            for (int i = 0; i < DS_PER; ++i) sum_q += exp(lq[i] - most);
            sum_q = wave_sum(sum_q);
            const double shift = most + log(sum_q);
#pragma unroll
            for (int i = 0; i < DS_PER; ++i) lq[i] = sum_q > 0.0 ? lq[i] - shift : -inf;
        }
        const bool none = !a.rest && sum_q == 0.0;  // no teacher
#pragma unroll
        for (int i = 0; i < DS_PER; ++i)
            if (t + i * PP_WAVE < a.top) q_of[t + i * PP_WAVE] = exp(lq[i]);
        __syncthreads();
        // columns that are listed more than once: the first of them has the student's p, each of them the sum of their q
        double same_q[DS_PER];
        bool first[DS_PER];
#pragma unroll
        for (int i = 0; i < DS_PER; ++i) {
            first[i] = at[i] >= 0;
            same_q[i] = 0.0;
            for (int e = 0; e < a.top; ++e)
                if (index[e] == at[i]) {
                    same_q[i] += q_of[e];
                    first[i] = first[i] && e >= t + i * PP_WAVE;
                }
        }
        double all = 0.0;
#pragma unroll
        for (int i = 0; i < DS_PER; ++i) all += first[i] ? exp(z[i]) : 0.0;
        const double rest_e = s > 0.0 ? s * exp(zm) : s;  // (NaN stays)
        all = wave_sum(all) + rest_e;
        const double log_all = log(all);
        double loss = 0.0;
        const double scale = (double)weight * kd;
#pragma unroll
        for (int i = 0; i < DS_PER; ++i) {
            const double lp = z[i] - log_all, q = exp(lq[i]);
            if (at[i] >= 0 && !(q == 0.0)) loss += q * (lq[i] - lp);
            const int e = t + i * PP_WAVE;
            if (e < a.top) a.listed[row * a.top + e] = (float)(empty || none ? 0.0 : scale * (exp(lp) - same_q[i]));
        }
        loss = wave_sum(loss);
        const double log_rest = zm + log(s) - log_all;
        if (r > 0.0) loss += r * (log(r) - log_rest);
        if (all != all) loss = all;
        if (empty) loss = none || (a.rest && r == 1.0) ? 0.0 : inf;
        if (none) loss = 0.0;
        if (!t) {
            a.loss[row] = (float)(loss * (double)weight);
            // (w / T) (p_rest - r) 2^((x - m) k) / s
            const double c = none || empty || s == 0.0 ? 0.0 : scale * (exp(log_rest) - r) / s;
            a.tail[row] = pp_f2{(float)m, (float)(all != all && !none ? all : c)};
        }
    }
}

// logits and dlogits may be one matrix: a thread reads its values before it writes them, and what the list needs has been read
template <class Y, int HELD> __global__ __launch_bounds__(LS_THREADS) void k_distill_grad(ds_args a, const typename Y::T *logits, typename Y::T *dlogits) {
    for (long long item = blockIdx.x; item < a.rows * a.segs; item += gridDim.x) {
        const long long row = item / a.segs, first = (item - row * a.segs) * a.size;
        const pp_f2 tail = a.tail[row];
        const long long end = first + a.size < a.cols ? first + a.size : a.cols;
#pragma unroll
        for (int i = 0; i < HELD; ++i) {
            const long long c = first + 8ll * (threadIdx.x + i * LS_THREADS), left = end - c;
            if (left <= 0) break;
            float v[8];
            pp_values<Y>(ls_load<Y>(logits + row * a.ld + c, left), v);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = tail[1] == 0.0f ? 0.0f : tail[1] * __builtin_amdgcn_exp2f((v[j] - tail[0]) * a.k);
            pp_store8<Y>(dlogits + row * a.ld_d + c, left, v);
        }
        __syncthreads();  // the listed columns' values come after what was written there
        for (int e = threadIdx.x; e < a.top; e += LS_THREADS) {
            const long long at = a.index[row * a.top + e];
            if (at >= first && at < end) dlogits[row * a.ld_d + at] = Y::put(a.listed[row * a.top + e]);
        }
    }
}

template <class F> static void by_held(int held, F f) {
    if (held == 16) f(std::integral_constant<int, 16>());
    else if (held == 8) f(std::integral_constant<int, 8>());
    else if (held == 4) f(std::integral_constant<int, 4>());
    else f(std::integral_constant<int, 1>());
}

static unsigned grid_of(int64_t items) { return (unsigned)(items < LS_MAX_GRID ? items : LS_MAX_GRID); }

extern "C" size_t pp_distill_workspace_bytes(int type, int64_t rows, int64_t cols, int top) {
    if (pp_bad_sizes(type, rows, cols) || top < 1 || top > PP_TOP_MAX) return 0;
    return pp_align256((size_t)ls_most(type, rows, cols) * sizeof(pp_f2)) + pp_align256((size_t)rows * sizeof(pp_f2)) + pp_align256((size_t)rows * top * 4) + 256;
}

extern "C" int pp_distill_loss(int kind, int type, int64_t rows, int64_t cols, const void *logits, int64_t ld, float temperature, int top,
                               const int32_t *top_index, const float *top_value, const float *weight, float *loss, void *dlogits, int64_t ld_d,
                               void *workspace, size_t workspace_bytes, void *stream) {
    if (pp_bad_sizes(type, rows, cols) || pp_bad_matrix(logits, type, rows, cols, ld) || (kind != PP_DISTILL_TOP && kind != PP_DISTILL_REST)) return PP_ERR_INVALID_ARG;
    if (dlogits && pp_bad_matrix(dlogits, type, rows, cols, ld_d)) return PP_ERR_INVALID_ARG;
    if (top < 1 || top > PP_TOP_MAX || !(temperature >= 0x1p-20f && temperature <= 0x1p20f)) return PP_ERR_INVALID_ARG;
    for (const void *p : {(const void *)top_index, (const void *)top_value, (const void *)weight, (const void *)loss})
        if ((uintptr_t)p & 3) return PP_ERR_INVALID_ARG;
    if (rows && (!top_index || !top_value || !loss)) return PP_ERR_INVALID_ARG;
    if (!rows) return PP_OK;
    if (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < pp_distill_workspace_bytes(type, rows, cols, top)) return PP_ERR_WORKSPACE;
    const ls_plan p = ls_divide(type, rows, cols);
    char *ws = (char *)workspace;
    pp_f2 *sums = (pp_f2 *)ws, *tail = (pp_f2 *)(ws + pp_align256((size_t)rows * p.segs * sizeof(pp_f2)));
    float *listed = (float *)((char *)tail + pp_align256((size_t)rows * sizeof(pp_f2)));
    const ds_args a = {rows, cols, p.size, ld, ld_d, p.segs, top, kind == PP_DISTILL_REST, (float)(1.4426950408889634 / temperature), 1.0 / temperature, top_index,
                       top_value, weight, loss, sums, tail, listed};
    hipStream_t st = (hipStream_t)stream;
    return pp_by_type(type, [&](auto tag) {
        typedef decltype(tag) Y;
        typedef typename Y::T T;
        by_held(p.held, [&](auto h) {
            if constexpr (decltype(h)::value * sizeof(T) <= 32) k_distill_sums<Y, decltype(h)::value><<<grid_of(rows * p.segs), LS_THREADS, 0, st>>>(a, (const T *)logits);
        });
        if (hipGetLastError() != hipSuccess) return PP_ERR_HIP;
        k_distill_list<Y><<<grid_of(rows), PP_WAVE, 0, st>>>(a, (const T *)logits);
        if (hipGetLastError() != hipSuccess) return PP_ERR_HIP;
        if (dlogits)
            by_held(p.held, [&](auto h) {
                if constexpr (decltype(h)::value * sizeof(T) <= 32) k_distill_grad<Y, decltype(h)::value><<<grid_of(rows * p.segs), LS_THREADS, 0, st>>>(a, (const T *)logits, (T *)dlogits);
            });
        return hipGetLastError() == hipSuccess ? PP_OK : PP_ERR_HIP;
    });
}
