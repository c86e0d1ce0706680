// pp_logprob_forward, pp_logprob_backward: log probabilities of given tokens, entropies and the top alternatives of rows of
// logits, and their gradient.
//
// With z = x / T, p = exp(z) / sum exp(z):  logp = ln p[token],  H = -sum p ln p,
//   dx = (dlogp ([j = token] - p_j) - dH p_j (ln p_j + H)) / T
// A workgroup holds a segment of a row in registers: its maximum, then its sums, then the alternatives; rows of more than one
// segment are joined by a second kernel.
//
// 2048 x 131072 bf16 (537 MB): 107 us without alternatives, 5.0 TB/s, where a copy reaches 5.1 to 5.2; with 20 of them 122, with 64 140, since a
// segment stays in its registers while its 64 are found (about 4 us) and nothing is read in its place.  333 x 50001 float32 25 us and 6 to join
// them; its gradient 22.7 (133 MB, 5.9 TB/s); that of 2048 x 131072 bf16 185 us, with the entropy's 189 to 199 (1.07 GB, 5.4 to 5.8).  One row of 131072 with 20 alternatives 6 us in 64 segments, and 6 more to join them.
//
// Alternatives: each thread knows its chunks' maxima.  The K-th largest of the 256 threads' maxima, found bit by bit by one wave,
// is at most the K-th largest logit, and the logits from there on lie in the chunks of at most K threads (or tie with them): they
// are read again, ranked by counting and written in order.  Where ties make them too many, the K-th largest pair of logit and
// column is found bit by bit by all threads, in 64 more readings of the segment: 2048 x 131072 bf16 with 64 takes 7.8 ms in place
// of 0.14 to 0.16 where half of every row is a mask of the lowest value, or all of it is one value (with a mask of -infinity 0.14); one row of them
// 71 us for 12.  Segments' lists are joined in the same way.
#include "pp_loss.h"

// Chunks to a thread: of half as many each has its alternatives found (2048 x 131072 bf16 with 64 164 us for 144, without 108 for 107).
#define LP_HELD 16

struct lp_args {
    long long rows, cols, size, ld;
    int segs, top;
    float k;
    const int *tokens;
    float *logp, *entropy, *norm, *top_logp;
    int *top_index;
    pp_f4 *sums;   // [rows][segs]: m, s, w
    unsigned long long *kept;  // [rows][segs][top]: lp_entry, in order
};

// What a row's sums say: s NaN: no numbers; s = 0: nothing but -infinity.
struct lp_row {
    float m, s, log2_s;
    __device__ __forceinline__ float logp(float x, float k) const { return 0.69314718f * ((x - m) * k - log2_s); }
};

template <class Y> __device__ __forceinline__ void put_row(const lp_args &a, long long row, const typename Y::T *x, float m, float s, float w) {
    const lp_row r = {m, s, __builtin_amdgcn_logf(s)};
    if (a.norm) {
        a.norm[2 * row] = m;
        a.norm[2 * row + 1] = s;
    }
    if (a.entropy) a.entropy[row] = s == 0.0f ? 0.0f : __builtin_fmaxf(0.0f, 0.69314718f * (r.log2_s - w / s)) + (s != s ? s : 0.0f);
    if (a.logp) {
        const int tok = a.tokens[row];
        float v = 0.0f;
        if (tok >= 0) v = tok >= a.cols ? __builtin_nanf("") : s == 0.0f ? -__builtin_inff() : r.logp(Y::get(x[tok]), a.k);
        a.logp[row] = v;
    }
}

// A logit and its column as one number that orders as the alternatives do: the larger logit first, then the lower column. 0: none.
typedef unsigned long long lp_entry;
__device__ __forceinline__ lp_entry lp_make(unsigned key, long long column) { return key ? (lp_entry)key << 32 | (0xffffffffu - (unsigned)column) : 0; }
__device__ __forceinline__ unsigned lp_key(lp_entry e) { return (unsigned)(e >> 32); }
__device__ __forceinline__ unsigned lp_column(lp_entry e) { return 0xffffffffu - (unsigned)e; }

__device__ __forceinline__ void put_top(const lp_args &a, long long row, int rank, lp_entry e, const lp_row &r) {
    const bool bad = r.s != r.s;
    a.top_index[row * a.top + rank] = e && !bad ? (int)lp_column(e) : -1;
    a.top_logp[row * a.top + rank] = bad ? r.s : e ? r.logp(ls_value(lp_key(e)), a.k) : -__builtin_inff();
}

struct lp_room {
    float wave[8];
    unsigned max[LS_THREADS];
    unsigned found, tau, count[4];
    lp_entry entry[LS_CAP + 32];
};

// The K-th largest of the 256 keys in room.max, by one wave.  0 if there are fewer.
template <class Y> __device__ __forceinline__ void find_threshold(lp_room &room, int top) {
    const int low = sizeof(typename Y::T) == 4 ? 0 : __is_same(Y, PpBF16) ? 16 : 13;  // (bits below are the same for all)
    if (threadIdx.x >= PP_WAVE) return;
    unsigned key[4], tau = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) key[i] = room.max[threadIdx.x + i * PP_WAVE];
    for (int bit = 31; bit >= low; --bit) {
        const unsigned to = tau | 1u << bit;
        int c = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) c += __popcll(__ballot(key[i] >= to));
        if (c >= top) tau = to;
        if (c == top) break;
    }
    if (!threadIdx.x) room.tau = tau, room.found = 0;
}

// Entries of this thread, `mine` of them wanted, into the room's list.
template <class F> __device__ __forceinline__ void append(lp_room &room, int mine, F each) {
    if (!mine) return;
    unsigned at = atomicAdd(&room.found, (unsigned)mine);
    each([&](lp_entry e) {
        if (at < LS_CAP) room.entry[at] = e;
        ++at;
    });
}

__device__ __forceinline__ unsigned group_count(unsigned c, unsigned *room) {
    for (int d = 1; d < PP_WAVE; d <<= 1) c += __shfl_xor(c, d);
    __syncthreads();
    if (!(threadIdx.x & (PP_WAVE - 1))) room[threadIdx.x / PP_WAVE] = c;
    __syncthreads();
    return room[0] + room[1] + room[2] + room[3];
}

// Where ties are too many for the list: the K-th largest entry bit by bit.  all(f) calls f for every entry of this thread.
template <class F> __device__ __forceinline__ void narrow(lp_room &room, int top, F all) {
    lp_entry tau = 0;
#pragma unroll 1
    for (int bit = 63; bit >= 0; --bit) {
        const lp_entry to = tau | 1ull << bit;
        unsigned c = 0;
        all([&](lp_entry e) { c += e >= to; });
        if (group_count(c, room.count) >= (unsigned)top) tau = to;
    }
    __syncthreads();
    if (!threadIdx.x) room.found = 0;
    __syncthreads();
    all([&](lp_entry e) {
        if (e && e >= tau) append(room, 1, [&](auto put) { put(e); });
    });
    __syncthreads();
}

// A long list once more: where fewer threads than `top` had anything, all of it is there.  Of four entries to a thread the
// maxima give a threshold as those of a segment do.
template <class Y> __device__ __forceinline__ void shorten(lp_room &room, int top) {
    const int t = threadIdx.x, found = (int)room.found;
    lp_entry mine[LS_CAP / LS_THREADS];
    unsigned most = 0;
#pragma unroll
    for (int i = 0; i < LS_CAP / LS_THREADS; ++i) {
        mine[i] = t + i * LS_THREADS < found ? room.entry[t + i * LS_THREADS] : 0;
        most = lp_key(mine[i]) > most ? lp_key(mine[i]) : most;
    }
    room.max[t] = most;
    __syncthreads();
    find_threshold<Y>(room, top);
    __syncthreads();
    const unsigned tau = room.tau > 1 ? room.tau : 1;
#pragma unroll
    for (int i = 0; i < LS_CAP / LS_THREADS; ++i) append(room, lp_key(mine[i]) >= tau, [&](auto put) { put(mine[i]); });
    __syncthreads();
}

// The list's first `top` entries in order into put(rank, entry), and none behind them.  Four lanes to an entry, each with a
// quarter of the others.
template <class Y, class F> __device__ __forceinline__ void rank_list(lp_room &room, int top, F put) {
    if (room.found > LS_THREADS) shorten<Y>(room, top);
    const int t = threadIdx.x, found = (int)room.found, ends = (found + 31) & ~31;
    if (t < ends - found) room.entry[found + t] = 0;
    __syncthreads();
    for (int i = t >> 2; i < ends; i += LS_THREADS / 4) {
        const lp_entry mine = room.entry[i];
        unsigned rank = 0;
        for (int o = t & 3; o < ends; o += 32)
#pragma unroll
            for (int k = 0; k < 8; ++k) rank += room.entry[o + 4 * k] > mine;
        rank += pp_moved<0xB1>(rank);
        rank += pp_moved<0x4E>(rank);
        if (!(t & 3) && mine && rank < (unsigned)top) put((int)rank, mine);
    }
    for (int rank = found + t; rank < top; rank += LS_THREADS) put(rank, (lp_entry)0);
}

// The top of a segment x[0 .. n) that starts at column `first`; x is read again.
template <class Y, int HELD, class F>
__device__ __forceinline__ void select_top(lp_room &room, const typename Y::T *x, long long n, long long first, int top, const float *chunk_max,
                                           float thread_max, F put) {
    const int t = threadIdx.x;
    room.max[t] = ls_key(thread_max);
    __syncthreads();
    find_threshold<Y>(room, top);
    __syncthreads();
    const unsigned low = 0x00800000u;  // the key of the lowest float
    const float tau = ls_value(room.tau > low ? room.tau : low);
    unsigned todo = 0;
#pragma unroll
    for (int i = 0; i < HELD; ++i) todo |= (chunk_max[i] >= tau ? 1u : 0u) << i;
    while (todo) {
        const int i = __builtin_ctz(todo);
        todo &= todo - 1;
        const long long c = 8ll * (t + i * LS_THREADS);
        float v[8];
        pp_values<Y>(ls_load<Y>(x + c, n - c), v);
        int mine = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) mine += v[j] >= tau;
        append(room, mine, [&](auto put_one) {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (v[j] >= tau) put_one(lp_make(ls_key(v[j]), first + c + j));
        });
    }
    __syncthreads();
    if (room.found > LS_CAP)
        narrow(room, top, [&](auto f) {
#pragma unroll 1
            for (int i = 0; i < HELD; ++i) {
                const long long c = 8ll * (t + i * LS_THREADS);
                float v[8];
                pp_values<Y>(ls_load<Y>(x + c, n - c), v);
                for (int j = 0; j < 8; ++j)
                    if (v[j] == v[j]) f(lp_make(ls_key(v[j]), first + c + j));
            }
        });
    rank_list<Y>(room, top, put);
}

template <class Y, int HELD> __global__ __launch_bounds__(LS_THREADS, 4) void k_logprob(lp_args a, const typename Y::T *__restrict__ logits) {
    __shared__ lp_room room;
    const int t = threadIdx.x;
    for (long long item = blockIdx.x; item < a.rows * a.segs; item += gridDim.x) {
        const long long row = a.segs == 1 ? item : item / a.segs, seg = item - row * a.segs, first = seg * a.size;
        const typename Y::T *x = logits + row * a.ld + first;
        const long long n = a.cols - first < a.size ? a.cols - first : a.size;
        PpRaw<Y> raw[HELD];
        float chunk_max[HELD], v[8], m = -__builtin_inff();
        ls_load_all<Y, HELD>(raw, x, n);
#pragma unroll
        for (int i = 0; i < HELD; ++i) {
            pp_values<Y>(raw[i], v);
            chunk_max[i] = ls_max8(v);
            m = __builtin_fmaxf(m, chunk_max[i]);
            __builtin_amdgcn_sched_barrier(0);  // (chunk by chunk: else all are converted first, and put away)
        }
        const float base = ls_base(ls_group_max<4>(m, room.wave));
        float s = 0.0f, w = 0.0f;
        ls_hold<Y>(raw);
#pragma unroll
        for (int i = 0; i < HELD; ++i) {
            pp_values<Y>(raw[i], v);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float d = (v[j] - base) * a.k, e = __builtin_amdgcn_exp2f(d);
                s += e;
                w = __builtin_fmaf(e, __builtin_fmaxf(d, -256.0f), w);  // (-infinity: 0)
            }
            asm volatile("" : "+v"(s), "+v"(w));  // (here and not behind the sums of s, with all that is added put away until then)
        }
        __syncthreads();
        s = pp_group_sum<4>(s, room.wave);
        w = pp_group_sum<4>(w, room.wave + 4);
        if (!t) {
            if (a.segs == 1) put_row<Y>(a, row, x, base, s, w);
            else a.sums[item] = pp_f4{base, s, w, 0.0f};
        }
        if (a.top) {
            const lp_row r = {base, s, __builtin_amdgcn_logf(s)};
            select_top<Y, HELD>(room, x, n, first, a.top, chunk_max, m, [&](int rank, lp_entry e) {
                if (a.segs == 1) put_top(a, row, rank, e, r);
                else a.kept[item * a.top + rank] = e;
            });
        }
        __syncthreads();
    }
}

// Sums of segments on the largest maximum: with d = (a segment's - the largest) k, its s and w are multiplied by 2^d, and d is added
// to every exponent of w.
template <class Y> __global__ __launch_bounds__(LS_THREADS) void k_logprob_join(lp_args a, const typename Y::T *__restrict__ logits) {
    __shared__ lp_room room;
    const int t = threadIdx.x;
    for (long long row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const pp_f4 *sums = a.sums + row * a.segs;
        float m = -__builtin_inff(), s = 0.0f, w = 0.0f;
        for (int i = t; i < a.segs; i += LS_THREADS)
            if (sums[i][1] != 0.0f) m = __builtin_fmaxf(m, sums[i][0]);
        m = ls_base(ls_group_max<4>(m, room.wave));
        for (int i = t; i < a.segs; i += LS_THREADS) {
            const pp_f4 p = sums[i];
            if (p[1] == 0.0f) continue;
            const float d = (p[0] - m) * a.k, e = __builtin_amdgcn_exp2f(d);
            s = __builtin_fmaf(e, p[1], s);
            w = __builtin_fmaf(e, __builtin_fmaf(p[1], __builtin_fmaxf(d, -256.0f), p[2]), w);
        }
        __syncthreads();
        s = pp_group_sum<4>(s, room.wave);
        w = pp_group_sum<4>(w, room.wave + 4);
        if (!t) put_row<Y>(a, row, logits + row * a.ld, m, s, w);
        if (a.top) {
            const lp_row r = {m, s, __builtin_amdgcn_logf(s)};
            const lp_entry *kept = a.kept + row * a.segs * a.top;
            const int n = a.segs * a.top;
            unsigned most = 0;
            for (int c = t; c < n; c += LS_THREADS) {
                const unsigned key = lp_key(kept[c]);
                most = key > most ? key : most;
            }
            room.max[t] = most;
            __syncthreads();
            find_threshold<Y>(room, a.top);
            __syncthreads();
            const unsigned tau = room.tau > 1 ? room.tau : 1;
            for (int c = t; c < n; c += LS_THREADS) {
                const lp_entry e = kept[c];
                append(room, lp_key(e) >= tau, [&](auto put_one) { put_one(e); });
            }
            __syncthreads();
            if (room.found > LS_CAP)
                narrow(room, a.top, [&](auto f) {
                    for (int c = t; c < n; c += LS_THREADS) f(kept[c]);
                });
            rank_list<Y>(room, a.top, [&](int rank, lp_entry e) { put_top(a, row, rank, e, r); });
        }
        __syncthreads();
    }
}

struct lp_back {
    long long rows, cols, size, ld, ld_d;
    int segs;
    float k, inv_t;
    const int *tokens;
    const float *norm, *dlogp, *entropy, *dentropy;
};

// logits and dlogits may be one matrix: a thread reads its values before it writes them
template <class Y, int HELD> __global__ __launch_bounds__(LS_THREADS) void k_logprob_back(lp_back a, const typename Y::T *logits, typename Y::T *dlogits) {
    for (long long item = blockIdx.x; item < a.rows * a.segs; item += gridDim.x) {
        const long long row = item / a.segs, first = (item - row * a.segs) * a.size;
        const float m = a.norm[2 * row], s = a.norm[2 * row + 1];
        const long long tok = a.tokens ? a.tokens[row] : -1;
        float g = a.dlogp && tok >= 0 ? a.dlogp[row] * a.inv_t : 0.0f;
        if (a.dlogp && tok >= a.cols) g = __builtin_nanf("");
        const float dh = a.dentropy ? a.dentropy[row] * a.inv_t : 0.0f, h = a.dentropy ? a.entropy[row] : 0.0f;
        // (of padding nothing is asked, and what it holds may be no numbers)
        const bool asked = (a.dlogp && tok >= 0) || dh != 0.0f;
        // p (-g - dh (ln p + H)), with ln p = ln 2 (d - log2 s)
        const float scale = s == 0.0f ? 0.0f : 1.0f / s, log2_s = __builtin_amdgcn_logf(s);
        const float slope = -dh * 0.69314718f * scale, level = s == 0.0f ? 0.0f : (-g - dh * (h - 0.69314718f * log2_s)) * scale;
        const long long end = first + a.size < a.cols ? first + a.size : a.cols;
#pragma unroll
        for (int i = 0; i < HELD; ++i) {
            const long long c = first + 8ll * (threadIdx.x + i * LS_THREADS), left = end - c;
            if (left <= 0) break;
            float v[8] = {};
            if (asked) {
                pp_values<Y>(ls_load<Y>(logits + row * a.ld + c, left), v);
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float d = (v[j] - m) * a.k, e = __builtin_amdgcn_exp2f(d);
                    v[j] = e * __builtin_fmaf(__builtin_fmaxf(d, -256.0f), slope, level);
                    if (c + j == tok && s != 0.0f) v[j] += g;
                }
            }
            pp_store8<Y>(dlogits + row * a.ld_d + c, left, v);
        }
    }
}

static bool bad_temperature(float t) { return !(t >= 0x1p-20f && t <= 0x1p20f); }
static bool bad4(const void *p) { return ((uintptr_t)p & 3) != 0; }

extern "C" size_t pp_logprob_workspace_bytes(int type, int64_t rows, int64_t cols, int top) {
    if (pp_bad_sizes(type, rows, cols) || top < 0 || top > PP_TOP_MAX) return 0;
    const size_t most = (size_t)ls_most(type, rows, cols, LP_HELD);
    return pp_align256(most * sizeof(pp_f4)) + pp_align256(most * top * sizeof(unsigned long long)) + 256;
}

extern "C" int pp_logprob_forward(int type, int64_t rows, int64_t cols, const void *logits, int64_t ld, float temperature, const int32_t *tokens,
                                  float *logp, float *entropy, float *norm, int top, int32_t *top_index, float *top_logp, void *workspace,
                                  size_t workspace_bytes, void *stream) {
    if (pp_bad_sizes(type, rows, cols) || pp_bad_matrix(logits, type, rows, cols, ld) || bad_temperature(temperature)) return PP_ERR_INVALID_ARG;
    if (bad4(tokens) || bad4(logp) || bad4(entropy) || ((uintptr_t)norm & 7) || bad4(top_index) || bad4(top_logp)) return PP_ERR_INVALID_ARG;
    if (top < 0 || top > PP_TOP_MAX || (rows && ((logp && !tokens) || (top && (!top_index || !top_logp))))) return PP_ERR_INVALID_ARG;
    if (!rows) return PP_OK;
    const ls_plan p = ls_divide(type, rows, cols, LP_HELD);
    if (p.segs > 1)
        if (!workspace || ((uintptr_t)workspace & 255) || workspace_bytes < pp_logprob_workspace_bytes(type, rows, cols, top)) return PP_ERR_WORKSPACE;
    pp_f4 *sums = (pp_f4 *)workspace;
    unsigned long long *kept = (unsigned long long *)((char *)workspace + pp_align256((size_t)rows * p.segs * sizeof(pp_f4)));
    const lp_args a = {rows, cols, p.size, ld, p.segs, top, (float)(1.4426950408889634 / temperature), tokens, logp, entropy, norm, top_logp, top_index, sums, kept};
    hipStream_t st = (hipStream_t)stream;
    return pp_by_type(type, [&](auto tag) {
        typedef decltype(tag) Y;
        typedef typename Y::T T;
        ls_by_held<Y, LP_HELD>(p.held, [&](auto h) { k_logprob<Y, decltype(h)::value><<<ls_grid(rows * p.segs), LS_THREADS, 0, st>>>(a, (const T *)logits); });
        if (hipGetLastError() != hipSuccess) return PP_ERR_HIP;
        if (p.segs > 1) k_logprob_join<Y><<<ls_grid(rows), LS_THREADS, 0, st>>>(a, (const T *)logits);
        return hipGetLastError() == hipSuccess ? PP_OK : PP_ERR_HIP;
    });
}

extern "C" int pp_logprob_backward(int type, int64_t rows, int64_t cols, const void *logits, int64_t ld, float temperature, const int32_t *tokens,
                                   const float *norm, const float *dlogp, const float *entropy, const float *dentropy, void *dlogits, int64_t ld_d,
                                   void *stream) {
    if (pp_bad_sizes(type, rows, cols) || pp_bad_matrix(logits, type, rows, cols, ld) || pp_bad_matrix(dlogits, type, rows, cols, ld_d)) return PP_ERR_INVALID_ARG;
    if (bad_temperature(temperature) || bad4(tokens) || ((uintptr_t)norm & 7) || bad4(dlogp) || bad4(entropy) || bad4(dentropy)) return PP_ERR_INVALID_ARG;
    if (rows && (!norm || (dlogp && !tokens) || (dentropy && !entropy))) return PP_ERR_INVALID_ARG;
    if (!rows) return PP_OK;
    const int held = type == PP_TYPE_F32 ? 2 : 4;
    const int64_t size = (int64_t)held * LS_STEP, segs = (cols + size - 1) / size;
    const lp_back a = {rows, cols, size, ld, ld_d, (int)segs, (float)(1.4426950408889634 / temperature), 1.0f / temperature, tokens, norm, dlogp, entropy, dentropy};
    hipStream_t st = (hipStream_t)stream;
    return pp_by_type(type, [&](auto tag) {
        typedef decltype(tag) Y;
        typedef typename Y::T T;
        k_logprob_back<Y, sizeof(T) == 4 ? 2 : 4><<<ls_grid(rows * segs), LS_THREADS, 0, st>>>(a, (const T *)logits, (T *)dlogits);
        return hipGetLastError() == hipSuccess ? PP_OK : PP_ERR_HIP;
    });
}
