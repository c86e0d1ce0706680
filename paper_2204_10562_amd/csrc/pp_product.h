// What the products of pp_linear.hip share: tiles, their order over the chip, loads from global
// memory straight into LDS, and the way results leave.
//
// A product is out[o][i] = sum_c outer[o][c] inner[i][c].  The inner index runs along a row of the
// result: the packed operand (W's rows forward, the columns of W or X8 in the backward products) is
// the matrix instruction's first operand, so that a lane ends up with neighbours of a row.
#pragma once

#include "pp_layer_common.h"

#define PR_THREADS 256
#define PR_STEP 64  // bytes of an operand row to a step: 128 values of 4 bits, 32 of 16

typedef int pr_i8 __attribute__((ext_vector_type(8)));
typedef __bf16 pr_bf8 __attribute__((ext_vector_type(8)));
typedef short pr_s4 __attribute__((ext_vector_type(4)));
#define PR_LDS __attribute__((address_space(3)))

// How a launch divides its results: ti x to tiles by `splits` pieces of the sum.  Pieces beyond one
// leave floats in `partial` [splits][outer][inner padded to 4], which k_join adds in their order.
struct pr_plan {
    long long inner, outer;
    int steps;   // of the whole sum
    int per;     // of a piece
    int splits;
    unsigned ni, no;  // tiles
    float *partial;
    long long partial_ld;
};

// Where results go: rows of `type`, a row added to all (bias) or a matrix (add).
template <class Y> struct pr_out {
    typename Y::T *p;
    long long ld;
    const float *bias, *add;
    long long add_ld;
};

// Tile of a workgroup.  Workgroups go to the eight dies in turn, and each die has an L2 of its own:
// a die gets a run of neighbouring tiles, and within it patches of eight outer tiles by as many inner
// ones as fit, so that what is in flight shares operands.
__device__ __forceinline__ void pr_tile(const pr_plan &p, unsigned b, unsigned &ti, unsigned &to) {
    const unsigned n = p.ni * p.no, die = b & 7, at = b >> 3, per = n >> 3, more = n & 7;
    const unsigned t = die * per + (die < more ? die : more) + at;
    const unsigned strip = t / (8 * p.ni), in = t - strip * 8 * p.ni, o0 = strip * 8;
    const unsigned high = p.no - o0 < 8 ? p.no - o0 : 8;
    to = o0 + in % high;
    ti = in / high;
}

// A buffer descriptor: loads at or beyond `bytes` give zeros.  Uniform over the wave.
__device__ __forceinline__ pp_i4 pr_buffer(const void *base, long long bytes) {
    const unsigned long long a = (unsigned long long)base;
    const unsigned n = bytes < 0 ? 0 : bytes > 0xffffffffll ? 0xffffffffu : (unsigned)bytes;
    pp_i4 r;
    r[0] = __builtin_amdgcn_readfirstlane((int)a);
    r[1] = __builtin_amdgcn_readfirstlane((int)(a >> 32) & 0xffff);
    r[2] = __builtin_amdgcn_readfirstlane((int)n);
    r[3] = 0x00027000;
    return r;
}
// The same for loads into registers.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t pr_resource(const void *base, long long bytes) {
    return __builtin_amdgcn_make_buffer_rsrc((void *)base, 0, bytes < 0 ? 0 : bytes > 0xffffffffll ? -1 : (int)bytes, 0x00027000);
}
#define PR_BEYOND 0xfffffff0u  // an offset that no buffer reaches

// 16 bytes per lane from base + voff + soff to LDS byte `lds` + 16 * lane, in the background: the
// compiler does not know of it, waits are PR_WAIT's.
__device__ __forceinline__ void pr_to_lds(pp_i4 buf, unsigned voff, unsigned soff, unsigned lds) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds"
                 ::"s"(__builtin_amdgcn_readfirstlane(lds)), "v"(voff), "s"(buf), "s"(__builtin_amdgcn_readfirstlane(soff)) : "memory");
}
#define PR_WAIT(n) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(n) : "memory")

// A barrier that leaves loads in flight: what a wave has read from LDS has arrived.
__device__ __forceinline__ void pr_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

__device__ __forceinline__ unsigned pr_lds_of(const void *p) { return (unsigned)(uintptr_t)(PR_LDS const void *)p; }

// Row of the inner operand that lane row `i` (0..15) of fragment f takes: a lane's results of two
// fragments are eight neighbours, 16 bytes of a 16-bit type.
__device__ __forceinline__ int pr_inner_row(int f, int i) { return 32 * (f >> 1) + 8 * (i >> 2) + 4 * (f & 1) + (i & 3); }

// Eight results of a lane, inner index i on, row o.
template <class Y> __device__ __forceinline__ void pr_put8(const pr_plan &p, const pr_out<Y> &out, long long o, long long i, int piece, float *v) {
    if (o >= p.outer || i >= p.inner) return;
    const long long n = p.inner - i;
    if (p.splits > 1) {
        float *q = p.partial + ((long long)piece * p.outer + o) * p.partial_ld + i;  // rows padded to 8
        *(pp_f4 *)q = *(pp_f4 *)v;
        *(pp_f4 *)(q + 4) = *(pp_f4 *)(v + 4);
        return;
    }
    if (out.bias || out.add) {
        const float *a = out.bias ? out.bias + i : out.add + o * out.add_ld + i;
        const PpRaw<PpF32> r = pp_load8<PpF32>(a, n);
        float w[8];
        pp_values<PpF32>(r, w);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] += w[j];
    }
    pp_store8<Y>(out.p + o * out.ld + i, n, v);
}

// acc[j] += a b[j] for N fragments of the outer operand, 16 x 16 x 32 in bf16.  Written as one block
// because the results have to stay in their registers: where the compiler chooses, it gives every
// product new ones and moves sums about.  What the compiler then does not see is waited for here: two
// wait states from a register's writing to its use as an operand, and pr_settle before a sum is read.
template <int N> __device__ __forceinline__ void pr_multiply(pp_f4 *acc, pr_bf8 a, const pr_bf8 *b) {
    if constexpr (N == 4)
        asm volatile("s_nop 1\n\t"
                     "v_mfma_f32_16x16x32_bf16 %0, %4, %5, %0\n\t"
                     "v_mfma_f32_16x16x32_bf16 %1, %4, %6, %1\n\t"
                     "v_mfma_f32_16x16x32_bf16 %2, %4, %7, %2\n\t"
                     "v_mfma_f32_16x16x32_bf16 %3, %4, %8, %3"
                     : "+a"(acc[0]), "+a"(acc[1]), "+a"(acc[2]), "+a"(acc[3]) : "v"(a), "v"(b[0]), "v"(b[1]), "v"(b[2]), "v"(b[3]));
    else
#pragma unroll
        for (int j = 0; j < N; ++j) asm volatile("s_nop 1\n\tv_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+a"(acc[j]) : "v"(a), "v"(b[j]));
}

// Behind a loop's last products (where s == end): the matrix units have written their results.  The
// branch around the two waits is in here so that it stays within the loop, before any use of a sum.
__device__ __forceinline__ void pr_settle(int s, int end) {
    asm volatile("s_cmp_lg_u32 %0, %1\n\ts_cbranch_scc1 2\n\ts_nop 15\n\ts_nop 15" ::"s"(s), "s"(end) : "scc", "memory");
}

