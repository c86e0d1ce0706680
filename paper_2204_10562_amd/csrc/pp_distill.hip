// pp_distill_loss: the divergence of a student's rows of logits from a teacher of whom the top entries are known, and its gradient.
//
// With p = softmax(x / T) and q the listed entries' probabilities (PP_DISTILL_TOP: softmax(value / T); PP_DISTILL_REST: exp(value), and
// r = 1 - sum q for all others):
//   loss = w (sum q (ln q - ln p) + r (ln r - ln p_rest)),  dx_j = (w / T) (p_j - q_j), and beside the list (w / T) p_j (1 - r / p_rest)
// p_rest is the sum over what is not listed and not 1 less what is: a student that is nearly sure of the listed entries keeps the
// digits of the rest.  So the pass over a row leaves the listed entries out (a bit each in LDS), and they are added afterwards.
//
// From 128 MiB of logits on workgroups hold a row's segments until they know each other's sums, so that logits are read once; else (and for rows
// of more than 524288 columns, 262144 in float32) three kernels: the sums of segments; a wave to a row for the list; the gradient.
//
// 2048 x 131072 bf16 with 64 entries: the loss alone 110 us (537 MB, 4.9 TB/s), with the gradient (1.07 GB) 246 us, 4.4 TB/s where a copy reaches 5.1 to 5.2, and 13 for the lists, which are exponentials in 64 bits and
// the way there and back; read twice 142 and 195 and the lists.  A workgroup to a whole row, in up to 16 waves' registers, took 369: nothing is read while
// it computes.  777 x 50001 fp16 with 20 entries 28, 8 and 34 us: logits and gradient, 155 MB, mostly in the last cache.
#include "pp_loss.h"

#define DS_MEET 16   // most segments of a row whose workgroups meet
#define DS_MEET_FROM (1ll << 27)  // bytes of logits from which on they are read once
#define DS_HELD 8    // chunks to a thread

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
    float *listed; // [rows][top]: dx of the listed, or their logits
    unsigned *ticket;
    unsigned long long *words;  // [rows][segs][2]: m and s of what is not listed and of what is, or DS_EMPTY
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

// -infinity in the place of the listed columns of chunk i
template <class Y, int HELD> __device__ __forceinline__ void leave_out(PpRaw<Y> &raw, const unsigned *marks, int i) {
    const unsigned mark = marks[threadIdx.x * ((HELD + 3) / 4) + i / 4] >> (8 * (i & 3)) & 255;
    if (!mark) return;
    typename Y::T u[8];
    __builtin_memcpy(u, &raw, sizeof(u));
#pragma unroll
    for (int j = 0; j < 8; ++j) u[j] = mark >> j & 1 ? (typename Y::T)-__builtin_inff() : u[j];
    __builtin_memcpy(&raw, u, sizeof(u));
}

template <class Y, int HELD> __global__ __launch_bounds__(LS_THREADS, 4) void k_distill_sums(ds_args a, const typename Y::T *__restrict__ logits) {
    const int t = threadIdx.x;
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
            leave_out<Y, HELD>(raw[i], marks, i);
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

// A row's list, in one wave, entries lane and lane + 64: in 64 bits, since 1 less the listed probabilities has nothing left in 32
// where the teacher is sure, and a divergence is a small difference of large terms.
#define DS_PER (PP_TOP_MAX / PP_WAVE)
struct ds_list {
    double z[PP_TOP_MAX], lq[PP_TOP_MAX], q[PP_TOP_MAX], same_q[PP_TOP_MAX];
    double r, weight, zm, s, all;
    int at[PP_TOP_MAX];     // column, -1: none
    int first[PP_TOP_MAX];  // whether it is the first entry of its column
    int none, empty;
};

// The entries of this lane (all lanes have as many: an exponential in 64 bits is a hundred instructions, whoever needs it)
#define DS_EACH(e) for (int e = threadIdx.x & (PP_WAVE - 1); e - (int)(threadIdx.x & (PP_WAVE - 1)) < a.top; e += PP_WAVE)

// The teacher's side, and the listed logits, logit(entry, column).  Entries without a column or with a value of -infinity have no q (a column of
// theirs is listed all the same).
template <class F> __device__ __forceinline__ void ds_teacher(const ds_args &a, ds_list &l, long long row, F logit) {
    const double inf = __builtin_inf(), weight = a.weight ? (double)a.weight[row] : 1.0;
    double most = -inf, sum = 0.0, lq[DS_PER], q[DS_PER], z[DS_PER], r = 0.0;
    int at[DS_PER];
    float value[DS_PER];
#pragma unroll
    for (int i = 0; i < DS_PER; ++i) {
        const int e = (threadIdx.x & (PP_WAVE - 1)) + i * PP_WAVE;
        at[i] = e < a.top ? a.index[row * a.top + e] : -1;
        value[i] = e < a.top ? a.value[row * a.top + e] : 0.0f;
        if (at[i] >= a.cols || at[i] < 0) at[i] = -1;
    }
#pragma unroll
    for (int i = 0; i < DS_PER; ++i) z[i] = at[i] >= 0 ? logit((threadIdx.x & (PP_WAVE - 1)) + i * PP_WAVE, at[i]) : -inf;
#pragma unroll
    for (int i = 0; i < DS_PER; ++i) {
        lq[i] = at[i] >= 0 ? (double)value[i] * (a.rest ? 1.0 : a.inv_t) : -inf;
        most = __builtin_fmax(most, lq[i]);
    }
    most = a.rest ? 0.0 : pp_wave_max(most);
    if (most == -inf) most = 0.0;
#pragma unroll
    for (int i = 0; i < DS_PER; ++i) {
        q[i] = i * PP_WAVE < a.top ? exp(lq[i] - most) : 0.0;
        sum += q[i];
    }
    sum = pp_wave_sum(sum);
    const bool none = !a.rest && sum == 0.0;  // no teacher
    if (a.rest) {
        r = 1.0 - sum;
        if (r < 0x1p-20) r = 0.0;
    } else if (!none) {
        const double shift = most + log(sum), over = 1.0 / sum;
#pragma unroll
        for (int i = 0; i < DS_PER; ++i) lq[i] -= shift, q[i] *= over;
    }
#pragma unroll
    for (int i = 0; i < DS_PER; ++i) {
        const int e = (threadIdx.x & (PP_WAVE - 1)) + i * PP_WAVE;
        l.at[e] = at[i];
        l.z[e] = z[i];
        l.lq[e] = lq[i];
        l.q[e] = l.same_q[e] = q[i];
        l.first[e] = at[i] >= 0;
    }
    if (!(threadIdx.x & (PP_WAVE - 1))) l.r = r, l.weight = weight, l.none = none || weight == 0.0;
    __builtin_amdgcn_wave_barrier();
    // columns that are listed more than once: the first of them has the student's p, each of them the sum of their q
    int same[DS_PER] = {};
    for (int e = 0; e < a.top; ++e)
#pragma unroll
        for (int i = 0; i < DS_PER; ++i) same[i] += l.at[e] == at[i];
    bool twice = false;
#pragma unroll
    for (int i = 0; i < DS_PER; ++i) twice = twice || (at[i] >= 0 && same[i] > 1);
    if (!__any(twice)) return;
    DS_EACH(own) {
        double sum_q = 0.0;
        int first = -1;
        for (int e = a.top - 1; e >= 0; --e)
            if (l.at[e] == l.at[own]) first = e;
        for (int e = 0; e < a.top; ++e)
            if (l.at[e] == l.at[own]) sum_q += l.q[e];
        l.same_q[own] = sum_q;
        l.first[own] = l.at[own] >= 0 && first == own;
    }
    __builtin_amdgcn_wave_barrier();
}

// The student's, with what is not listed (its largest logit m, s = sum exp((x - m) / T)): x becomes z = (x - base) / T from the row's
// largest logit on (beside the type's lowest value, as a mask, a logarithm of a sum has no digits left), `all` the sum over all.
// Returns what 2^((x - m) k) is multiplied by for dx beside the list, (w / T) (p_rest - r) / s.
__device__ __forceinline__ float ds_student(const ds_args &a, ds_list &l, double m, double s) {
    const double inf = __builtin_inf();
    double top_x = s > 0.0 ? m : -inf, all = 0.0;
    DS_EACH(e) top_x = __builtin_fmax(top_x, l.z[e]);
    top_x = pp_wave_max(top_x);
    const bool empty = top_x == -inf && s == 0.0;
    const double base = top_x == -inf ? 0.0 : top_x, zm = (m - base) * a.inv_t;
    DS_EACH(e) {
        const double z = (l.z[e] - base) * a.inv_t;
        l.z[e] = z;
        all += l.first[e] ? exp(z) : 0.0;
    }
    const double rest = s > 0.0 ? s * exp(zm) : s;  // (NaN stays)
    all = pp_wave_sum(all) + rest;
    if (!(threadIdx.x & (PP_WAVE - 1))) l.zm = zm, l.s = s, l.all = all, l.empty = empty;
    __builtin_amdgcn_wave_barrier();
    if (l.none) return 0.0f;
    if (all != all) return (float)all;
    return empty || s == 0.0 ? 0.0f : (float)(l.weight * a.inv_t * (rest / all - l.r) / s);
}

// The loss, and dx of the listed into put(entry, column, dx)
template <class F> __device__ __forceinline__ float ds_loss(const ds_args &a, const ds_list &l, F put) {
    const double log_all = log(l.all), scale = l.weight * a.inv_t;
    double sum = 0.0;
    DS_EACH(e) {
        const double lp = l.z[e] - log_all, q = l.q[e];
        if (l.at[e] >= 0 && !(q == 0.0)) sum += q * (l.lq[e] - lp);
        put(e, l.at[e], (float)(l.empty || l.none ? 0.0 : scale * (exp(lp) - l.same_q[e])));
    }
    sum = pp_wave_sum(sum);
    if (l.r > 0.0) sum += l.r * (log(l.r) - (l.zm + log(l.s) - log_all));
    if (l.all != l.all) sum = l.all;
    if (l.empty) sum = a.rest && l.r == 1.0 ? 0.0 : __builtin_inf();
    return l.none ? 0.0f : (float)(sum * l.weight);
}

// HELD_ROWS: behind k_distill_meet, which has put the listed logits aside in `listed` (dlogits may have been written over them);
// dx of the listed goes to dlogits.  Else to `listed`, for k_distill_grad.
template <class Y, bool HELD_ROWS> __global__ __launch_bounds__(PP_WAVE) void k_distill_list(ds_args a, const typename Y::T *logits, typename Y::T *dlogits) {
    __shared__ ds_list list;
    const int t = threadIdx.x;
    for (long long row = blockIdx.x; row < a.rows; row += gridDim.x) {
        double m = 0.0, s = 0.0;
        ds_teacher(a, list, row, [&](int e, int at) { return HELD_ROWS ? (double)a.listed[row * a.top + e] : (double)Y::get(logits[row * a.ld + at]); });
        if (!a.weight || a.weight[row] != 0.0f) {
            m = -__builtin_inf();
            for (int i = t; i < a.segs; i += PP_WAVE) {
                const pp_f2 p = a.sums[row * a.segs + i];
                if (p[1] != 0.0f) m = __builtin_fmax(m, (double)p[0]);
            }
            m = pp_wave_max(m);
            if (m == -__builtin_inf()) m = 0.0;
            for (int i = t; i < a.segs; i += PP_WAVE) {
                const pp_f2 p = a.sums[row * a.segs + i];
                if (p[1] != 0.0f) s += (double)p[1] * exp(((double)p[0] - m) * a.inv_t);
            }
            s = pp_wave_sum(s);
        }
        const float slope = ds_student(a, list, m, s);
        const float loss = ds_loss(a, list, [&](int e, int at, float dx) {
            if constexpr (HELD_ROWS) {
                if (at >= 0) dlogits[row * a.ld_d + at] = Y::put(dx);
            } else if (e < a.top) a.listed[row * a.top + e] = dx;
        });
        if (!t) {
            a.loss[row] = loss;
            if (!HELD_ROWS) a.tail[row] = pp_f2{(float)m, slope};
        }
        __builtin_amdgcn_wave_barrier();
    }
}

#define DS_EMPTY (~0ull)
__device__ __forceinline__ unsigned long long ds_word(float m, float s) {
    return (unsigned long long)(s != s ? 0x7fc00000u : pp_bits(s)) << 32 | pp_bits(m);
}

// From logits to the gradient beside the list in one reading: a workgroup holds a segment until the sums of all of the row's are known.
// The sums of what is listed and of what is not are made apart, so p_rest keeps its digits; of the teacher only r is needed, and
// whether there is one.  (p_rest - r is a
// difference in 32 bits here, and one in 64 in k_distill_list.)
//
// The workgroups of a row wait for one another, each after it has told its own sums.  Tickets are drawn at the start of a workgroup, so
// all below the highest one run or have ended, and only the row of the highest ticket, of at most DS_MEET workgroups, can wait for one
// that has not begun; the others go on and make room for it (a unit holds four at least, the chip 1024).  A word says by itself
// whether it is there, and every workgroup adds the row's words in the same order.
template <class Y, int HELD>
__global__ __launch_bounds__(LS_THREADS, 4) void k_distill_meet(ds_args a, const typename Y::T *logits, typename Y::T *dlogits) {
    constexpr int WORDS = (HELD + 3) / 4;
    __shared__ unsigned marks[LS_THREADS * WORDS];
    __shared__ float room[4][4], m_room, slope_room;
    __shared__ unsigned ticket;
    const int t = threadIdx.x;
    if (!t) ticket = atomicAdd(a.ticket, 1u);
    __syncthreads();
    const unsigned item = __builtin_amdgcn_readfirstlane(ticket), row32 = item / (unsigned)a.segs, seg = item - row32 * (unsigned)a.segs;
    const long long row = row32, first = seg * a.size;
    const typename Y::T *x = logits + row * a.ld + first;
    const int n = (int)(a.cols - first < a.size ? a.cols - first : a.size);
    PpRaw<Y> raw[HELD];
    ls_load_all<Y, HELD>(raw, x, n);
    mark_listed<HELD>(a, row, first, marks);
    const float weight = a.weight ? a.weight[row] : 1.0f;
    float r = 0.0f;
    if (t < PP_WAVE) {
        double sum = 0.0;
        bool any = false;
#pragma unroll 1
        for (int e = t; e < a.top; e += PP_WAVE) {
            const int at = a.index[row * a.top + e];
            if (at < 0 || at >= a.cols) continue;
            const float value = a.value[row * a.top + e];
            if (a.rest) sum += exp((double)value);
            any = any || !(value == -__builtin_inff());
            if (at >= first && at < first + n) a.listed[row * a.top + e] = Y::get(x[at - first]);
        }
        sum = pp_wave_sum(sum);
        r = !a.rest || 1.0 - sum < 0x1p-20 ? 0.0f : (float)(1.0 - sum);
        if ((!a.rest && !__any(any)) || weight == 0.0f) r = -1.0f;  // nothing to learn from the row
    }
    unsigned mark[WORDS];
#pragma unroll
    for (int i = 0; i < WORDS; ++i) mark[i] = marks[t * WORDS + i];
    float v[8], m = -__builtin_inff(), listed_m = -__builtin_inff(), s = 0.0f, listed_s = 0.0f;
#pragma unroll
    for (int i = 0; i < HELD; ++i) {
        pp_values<Y>(raw[i], v);
        const unsigned bits = mark[i / 4] >> (8 * (i & 3)) & 255;
        if (bits)
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (bits >> j & 1) listed_m = v[j] != v[j] ? __builtin_inff() : __builtin_fmaxf(listed_m, v[j]), v[j] = -__builtin_inff();
        m = __builtin_fmaxf(m, ls_max8(v));
        asm volatile("" : "+v"(m), "+v"(listed_m));  // (chunk by chunk: else values are put away until all are converted)
    }
    m = pp_wave_max(m);
    listed_m = pp_wave_max(listed_m);
    if (!(t & (PP_WAVE - 1))) room[0][t / PP_WAVE] = m, room[1][t / PP_WAVE] = listed_m;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 4; ++w) m = __builtin_fmaxf(m, room[0][w]), listed_m = __builtin_fmaxf(listed_m, room[1][w]);
    m = ls_base(m);
    listed_m = ls_base(listed_m);
    ls_hold<Y>(raw);
#pragma unroll
    for (int i = 0; i < HELD; ++i) {
        pp_values<Y>(raw[i], v);
        const unsigned bits = mark[i / 4] >> (8 * (i & 3)) & 255;
        if (bits)
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (bits >> j & 1) listed_s += __builtin_amdgcn_exp2f((v[j] - listed_m) * a.k), v[j] = -__builtin_inff();
#pragma unroll
        for (int j = 0; j < 8; ++j) s += __builtin_amdgcn_exp2f((v[j] - m) * a.k);
        asm volatile("" : "+v"(s), "+v"(listed_s));
    }
    s = pp_wave_sum(s);
    listed_s = pp_wave_sum(listed_s);
    if (!(t & (PP_WAVE - 1))) room[2][t / PP_WAVE] = s, room[3][t / PP_WAVE] = listed_s;
    __syncthreads();
    if (t < PP_WAVE) {
        s = room[2][0] + room[2][1] + room[2][2] + room[2][3];
        listed_s = room[3][0] + room[3][1] + room[3][2] + room[3][3];
        if (a.segs > 1) {
            unsigned long long *words = a.words + 2ll * row * a.segs;
            if (!t) {
                __hip_atomic_store(words + 2 * seg, ds_word(m, s), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                __hip_atomic_store(words + 2 * seg + 1, ds_word(listed_m, listed_s), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            }
            // lane i has the i-th segment's sums
            unsigned long long beside = 0, listed = 0;
            for (;;) {
                if (t < a.segs) {
                    beside = __hip_atomic_load(words + 2 * t, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                    listed = __hip_atomic_load(words + 2 * t + 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
                }
                if (!__any(beside == DS_EMPTY || listed == DS_EMPTY)) break;
                __builtin_amdgcn_s_sleep(2);
            }
            const float own_m = pp_bits((unsigned)beside), own_listed = pp_bits((unsigned)listed);
            s = pp_bits((unsigned)(beside >> 32));
            listed_s = pp_bits((unsigned)(listed >> 32));
            m = ls_base(pp_wave_max(s != 0.0f ? own_m : -__builtin_inff()));
            listed_m = ls_base(pp_wave_max(listed_s != 0.0f ? own_listed : -__builtin_inff()));
            s = pp_wave_sum(s != 0.0f ? s * __builtin_amdgcn_exp2f((own_m - m) * a.k) : 0.0f);
            listed_s = pp_wave_sum(listed_s != 0.0f ? listed_s * __builtin_amdgcn_exp2f((own_listed - listed_m) * a.k) : 0.0f);
        }
        // p_rest = s / (s + listed_s 2^((listed_m - m) k)), from whichever of the two exponentials is below 1
        const float d = s != 0.0f && listed_s != 0.0f ? (listed_m - m) * a.k : 0.0f, up = __builtin_amdgcn_exp2f(-__builtin_fabsf(d));
        const float own = d > 0.0f ? s * up : s, other = d > 0.0f ? listed_s : listed_s * up;
        float slope = weight * (float)a.inv_t * (own / (own + other) - r) / s;
        if (s == 0.0f) slope = listed_s != listed_s ? listed_s : 0.0f;  // nothing beside the list: 0 throughout, or NaN with what is listed
        if (r < 0.0f) slope = 0.0f;
        if (!t) {
            m_room = m;
            slope_room = slope;
            if (!seg) a.sums[row] = pp_f2{m, s};
        }
    }
    __syncthreads();
    m = m_room;
    const float slope = slope_room;
    ls_hold<Y>(raw);
#pragma unroll
    for (int i = 0; i < HELD; ++i) {
        const int left = n - 8 * (t + i * LS_THREADS);
        if (left <= 0) break;
        pp_values<Y>(raw[i], v);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = slope == 0.0f ? 0.0f : slope * __builtin_amdgcn_exp2f((v[j] - m) * a.k);
        pp_store8<Y>((typename Y::T *)((char *)(dlogits + row * a.ld_d + first + 8 * i * LS_THREADS) + t * (unsigned)(8 * sizeof(typename Y::T))), left, v);
    }
}

__global__ __launch_bounds__(256) void k_distill_clear(unsigned *ticket, unsigned long long *words, long long n) {
    if (blockIdx.x == 0 && !threadIdx.x) *ticket = 0;
    for (long long i = blockIdx.x * 256ll + threadIdx.x; i < n; i += gridDim.x * 256ll) words[i] = DS_EMPTY;
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

// Calls f with the chunks that a thread holds as a constant.
template <int HELD, class F> static void by_held(int held, F f) {
    if (held == HELD) f(std::integral_constant<int, HELD>());
    else if constexpr (HELD > 1) by_held<HELD - 1>(held, f);
}

// The segments of a row whose workgroups meet, about equally long; segs 0: rows are too long for it.  Few chunks to a
// thread, so that more workgroups than four are there to work while one waits.  What the last cache holds (256 MB, logits and
// gradient) is as well read twice: 777 x 50001 fp16 80 us in a meeting, 76 read twice, 4096 x 8000 bf16 87 and 63; but
// 1500 x 50001 fp16 117 and 132, 1024 x 131072 bf16 151 and 173.
static ls_plan ds_segments(int type, int64_t cols) {
    ls_plan p = {};
    const int most = ls_held(type, DS_HELD);
    for (int held = most; held <= 2 * most; held += most) {
        const int64_t segs = (cols + (int64_t)held * LS_STEP - 1) / ((int64_t)held * LS_STEP);
        if (segs > DS_MEET) continue;
        p.size = ls_even(cols, (int)segs);
        p.held = held > most ? held : (int)((p.size + LS_STEP - 1) / LS_STEP);
        p.segs = (int)((cols + p.size - 1) / p.size);
        break;
    }
    return p;
}
// (A launch has fewer than 2^32 threads: of 2^24 workgroups and more, rows are read twice, in loops.)
static bool ds_meets(int type, int64_t rows, int64_t cols, const ls_plan &p) {
    return p.segs && rows * cols * pp_type_size(type) >= DS_MEET_FROM && rows * p.segs < 1 << 24;
}

extern "C" size_t pp_distill_workspace_bytes(int type, int64_t rows, int64_t cols, int top) {
    if (pp_bad_sizes(type, rows, cols) || top < 1 || top > PP_TOP_MAX) return 0;
    return 256 + pp_align256((size_t)ls_most(type, rows, cols, DS_HELD) * sizeof(pp_f2)) + pp_align256((size_t)rows * sizeof(pp_f2)) + pp_align256((size_t)rows * top * 4) +
           pp_align256((size_t)rows * ds_segments(type, cols).segs * 16);
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
    const ls_plan p = ls_divide(type, rows, cols, DS_HELD);
    const ls_plan meet = ds_segments(type, cols);
    char *ws = (char *)workspace + 256;
    pp_f2 *sums = (pp_f2 *)ws, *tail = (pp_f2 *)(ws + pp_align256((size_t)ls_most(type, rows, cols, DS_HELD) * sizeof(pp_f2)));
    float *listed = (float *)((char *)tail + pp_align256((size_t)rows * sizeof(pp_f2)));
    unsigned long long *words = (unsigned long long *)((char *)listed + pp_align256((size_t)rows * top * 4));
    ds_args a = {rows, cols, p.size, ld, ld_d, p.segs, top, kind == PP_DISTILL_REST, (float)(1.4426950408889634 / temperature), 1.0 / temperature, top_index,
                 top_value, weight, loss, sums, tail, listed, (unsigned *)workspace, words};
    hipStream_t st = (hipStream_t)stream;
    return pp_by_type(type, [&](auto tag) {
        typedef decltype(tag) Y;
        typedef typename Y::T T;
        if (dlogits && ds_meets(type, rows, cols, meet)) {
            a.segs = meet.segs;
            a.size = meet.size;
            const int64_t items = rows * meet.segs, groups = (items * 2 + 1023) / 1024;
            k_distill_clear<<<(unsigned)(groups < 1024 ? groups : 1024), 256, 0, st>>>(a.ticket, a.words, items * 2);
            if (hipGetLastError() != hipSuccess) return PP_ERR_HIP;
            constexpr int MOST = sizeof(T) == 4 ? DS_HELD / 2 : DS_HELD;
            auto go = [&](auto h) { k_distill_meet<Y, decltype(h)::value><<<(unsigned)items, LS_THREADS, 0, st>>>(a, (const T *)logits, (T *)dlogits); };
            if (meet.held > MOST) go(std::integral_constant<int, 2 * MOST>());
            else by_held<MOST>(meet.held, go);
            if (hipGetLastError() != hipSuccess) return PP_ERR_HIP;
            a.segs = 1;  // (the list finds the row's sums in one place)
            k_distill_list<Y, true><<<ls_grid(rows), PP_WAVE, 0, st>>>(a, (const T *)logits, (T *)dlogits);
            return hipGetLastError() == hipSuccess ? PP_OK : PP_ERR_HIP;
        }
        ls_by_held<Y, DS_HELD>(p.held, [&](auto h) { k_distill_sums<Y, decltype(h)::value><<<ls_grid(rows * p.segs), LS_THREADS, 0, st>>>(a, (const T *)logits); });
        if (hipGetLastError() != hipSuccess) return PP_ERR_HIP;
        k_distill_list<Y, false><<<ls_grid(rows), PP_WAVE, 0, st>>>(a, (const T *)logits, (T *)dlogits);
        if (hipGetLastError() != hipSuccess) return PP_ERR_HIP;
        if (dlogits)
            ls_by_held<Y, DS_HELD>(p.held, [&](auto h) {
                k_distill_grad<Y, decltype(h)::value><<<ls_grid(rows * p.segs), LS_THREADS, 0, st>>>(a, (const T *)logits, (T *)dlogits);
            });
        return hipGetLastError() == hipSuccess ? PP_OK : PP_ERR_HIP;
    });
}
