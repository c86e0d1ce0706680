// What the products of pp_linear.hip share: tiles, their order over the chip, loads from global
// memory straight into LDS, and the way results leave.
//
// A product is out[o][i] = sum_c outer[o][c] inner[i][c].  The inner index runs along a row of the
// result: the packed operand (W's rows forward, the columns of W or X8 in the backward products) is
// the matrix instruction's first operand, so that a lane ends up with neighbours of a row.
#pragma once

#include "pp_layer_common.h"
#include "pp_linear_plan.h"

#define PR_PIN __builtin_amdgcn_sched_barrier(0)  // instructions stay on their side
#define PR_STEP 64  // bytes of a row of 4-bit values to a step: 128 of them

typedef int pr_i8 __attribute__((ext_vector_type(8)));
typedef __bf16 pr_bf8 __attribute__((ext_vector_type(8)));
typedef short pr_s4 __attribute__((ext_vector_type(4)));
#define PR_LDS __attribute__((address_space(3)))

// Where results go: rows of `type`, a row added to all (bias) or a matrix (add).
template <class Y> struct pr_out {
    typename Y::T *p;
    long long ld;
    const float *bias, *add;
    long long add_ld;
};

// Tile and piece of a workgroup.  Workgroups go to the eight dies in turn, and each die has an L2 of its own:
// a die gets a run of neighbouring tiles, and within it patches of eight outer tiles by as many inner ones as
// fit, so that what is in flight shares operands.  Its run is of each piece's tiles, or of all the pieces' one
// after the other (by_piece), where a die reads little beside its own part of the sum.
__device__ __forceinline__ void pr_tile(const pr_plan &p, unsigned b, unsigned &ti, unsigned &to, int &piece) {
    const unsigned tiles = p.ni * p.no, z = p.by_piece ? 0 : b / tiles, n = p.by_piece ? tiles * p.splits : tiles;
    b -= z * tiles;
    const unsigned die = b & 7, at = b >> 3, per = n >> 3, more = n & 7;
    const unsigned all = die * per + (die < more ? die : more) + at, y = all / tiles, t = all - y * tiles;
    const unsigned strip = t / (8 * p.ni), in = t - strip * 8 * p.ni, o0 = strip * 8;
    const unsigned high = p.no - o0 < 8 ? p.no - o0 : 8;
    piece = (int)(z + y);
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
// The same in two halves, for between products: where to, and (an instruction later) the load.
__device__ __forceinline__ void pr_aim(unsigned lds, int offset) {
    asm volatile("s_add_u32 m0, %0, %1" ::"s"(__builtin_amdgcn_readfirstlane(lds)), "n"(offset) : "scc");
}
__device__ __forceinline__ void pr_fire(pp_i4 buf, unsigned voff, unsigned soff) {
    asm volatile("buffer_load_dwordx4 %0, %1, %2 offen lds" ::"v"(voff), "s"(buf), "s"(__builtin_amdgcn_readfirstlane(soff)) : "memory");
}
#define PR_WAIT(n) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(n) : "memory")

// A barrier that leaves loads in flight: what a wave has read from LDS has arrived.
__device__ __forceinline__ void pr_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

__device__ __forceinline__ unsigned pr_lds_of(const void *p) { return (unsigned)(uintptr_t)(PR_LDS const void *)p; }

// The matrix instructions here are those of 32 x 32 results: lane l holds column l % 32 of the outer
// operand and, of the inner one's 32 rows, 8 q + 4 (l / 32) + 0..3 for q = 0..3.  Row i of a fragment
// is therefore read from row pr_inner_row(i) of the tile (bits 2 and 3 exchanged), which makes a lane's
// results two runs of eight neighbours, 16 bytes of a 16-bit type each.
__device__ __forceinline__ int pr_inner_row(int i) { return (i & ~12) | (i & 4) << 1 | (i & 8) >> 1; }
typedef float pr_f16 __attribute__((ext_vector_type(16)));

// How results leave.  A lane holds runs of eight neighbours of a row, a wave's fragments 32 rows of
// 32 WI of them: stored as they are, a wave would write 32 bytes here and there, which costs four times
// what whole lines do.  So a wave turns its fragments round in LDS (16-byte units exchanged by the row,
// an exclusive or, so that neighbouring rows fall on different banks) and writes rows of them.
// `room` is the wave's own, 32 rows of 32 WI results in 32 bits; no other wave reads there any more.
template <class Y, int WI> struct PrRows {
    static const int SIZE = sizeof(typename Y::T), UNITS = 32 * WI * SIZE / 16, VALUES = 16 / SIZE;
    static const int ROWS = 64 / UNITS;  // that 64 lanes take at once
    static __device__ __forceinline__ int at(int row, int unit) { return (row * UNITS + (unit ^ (row & (UNITS - 1)))) * 16; }
    static __device__ __forceinline__ void put(uint8_t *room, int row, int col, const float *v) {
        typename Y::T t[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) t[i] = Y::put(v[i]);
        PpRaw<Y> r;
        __builtin_memcpy(&r, t, sizeof(r));
#pragma unroll
        for (int i = 0; i < PpRaw<Y>::W; ++i) *(pp_u4 *)(room + at(row, col / VALUES + i)) = r.w[i];
    }
    static const int TURNS = 32 / ROWS / 2;  // of half the rows
    // What is added to 16 rows from o0 on, where Y is float: asked for before those in front of them are written.
    // (What a row's end leaves over is not used.  Offsets are within 32 bits: add_ld <= 2^24.)
    static __device__ __forceinline__ void fetch(pp_u4 *d, int lane, long long o0, long long outer, long long i0, long long inner, const float *add,
                                                 long long add_ld) {
        const auto b = pr_resource(add + o0 * add_ld + i0, o0 < outer ? (((outer - o0 < 16 ? outer - o0 : 16) - 1) * add_ld + inner - i0) * 4 : 0);
#pragma unroll
        for (int t = 0; t < TURNS; ++t)
            d[t] = __builtin_bit_cast(pp_u4, __builtin_amdgcn_raw_buffer_load_b128(b, (unsigned)((t * ROWS + lane / UNITS) * add_ld + lane % UNITS * 4) * 4, 0, 0));
    }
    // half h of the 32 rows in `room`, the result's rows o0.., columns i0..
    static __device__ __forceinline__ void store(const uint8_t *room, int h, int lane, typename Y::T *p, long long ld, long long o0, long long outer,
                                                 long long i0, long long inner, const pp_u4 *d) {
        const long long i = i0 + lane % UNITS * VALUES;
        typename Y::T *q = p + (o0 + lane / UNITS) * ld + i;
        const bool all = o0 + 16 <= outer && i0 + 32 * WI <= inner;
#pragma unroll
        for (int t = 0; t < TURNS; ++t) {
            const int row = t * ROWS + lane / UNITS;
            pp_u4 w = *(const pp_u4 *)(room + at(16 * h + row, lane % UNITS));
            if constexpr (SIZE == 4)
                if (d) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) w[j] = pp_bits(pp_bits(w[j]) + pp_bits(d[t][j]));
                }
            if (all || (o0 + row < outer && i + VALUES <= inner)) {
                ((pp_any16<SIZE> *)(q + t * ROWS * ld))->v = w;
            } else if (o0 + row < outer) {
                typename Y::T v[VALUES];
                __builtin_memcpy(v, &w, 16);
#pragma unroll
                for (int j = 0; j < VALUES; ++j)
                    if (i + j < inner) q[t * ROWS * ld + j] = v[j];
            }
        }
    }
};

// A wave's results: columns i0.., rows o0...  What is known at run time alone (whole or partial, a bias, a matrix to add, ends) is
// decided for every fragment, and the largest tiles have no registers left for it: 256 x 256 puts 48 of them away (float: 192)
// in the 4-bit product and 32 (114) in the gradients', here, behind the loops, which hold none.
template <class Y, int WI, int WO, class ACC>
__device__ __forceinline__ void pr_leave(const pr_plan &p, const pr_out<Y> &out, ACC &acc, uint8_t *room, int lane, long long i0, long long o0, int piece) {
    const int r = lane & 31, g = lane >> 5;
    const bool whole = p.splits == 1;
    typedef PrRows<Y, WI> Rows;
    typedef PrRows<PpF32, WI> Part;
    const bool adding = Rows::SIZE == 4 && whole && out.add;
    pp_u4 d[2][Rows::SIZE == 4 ? Rows::TURNS : 1];
    if (adding) Rows::fetch(d[0], lane, o0, p.outer, i0, p.inner, out.add, out.add_ld);
#pragma unroll
    for (int q = 0; q < 2 * WO; ++q) {
        const int j = q >> 1, h = q & 1;
        if (h == 0)
#pragma unroll
            for (int i = 0; i < WI; ++i) {
                float v[16];
                *(pr_f16 *)v = acc[i][j];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int col = 32 * i + 16 * e + 8 * g;
                    if (!whole) {
                        Part::put(room, r, col, v + 8 * e);
                        continue;
                    }
                    if (out.bias) {
                        const PpRaw<PpF32> b = pp_load8<PpF32>(out.bias + i0 + col, p.inner - i0 - col);
                        float w[8];
                        pp_values<PpF32>(b, w);
#pragma unroll
                        for (int k = 0; k < 8; ++k) v[8 * e + k] += w[k];
                    }
                    Rows::put(room, r, col, v + 8 * e);
                }
                PR_PIN;
            }
        // (loads wait for the stores before them: what is added next is asked for first)
        if (adding && q + 1 < 2 * WO) Rows::fetch(d[(q + 1) & 1], lane, o0 + 16 * (q + 1), p.outer, i0, p.inner, out.add, out.add_ld);
        if (whole) Rows::store(room, h, lane, out.p, out.ld, o0 + 16 * q, p.outer, i0, p.inner, adding ? d[q & 1] : NULL);
        else Part::store(room, h, lane, p.partial + (long long)piece * p.outer * p.partial_ld, p.partial_ld, o0 + 16 * q, p.outer, i0, p.inner, NULL);
        PR_PIN;
    }
}

// Sums start at zero, in their registers and settled there before the first product.
template <int WI, int WO> __device__ __forceinline__ void pr_clear(pr_f16 (&acc)[WI][WO]) {
#pragma unroll
    for (int i = 0; i < WI; ++i)
#pragma unroll
        for (int j = 0; j < WO; ++j) {
            acc[i][j] = pr_f16{};
            asm volatile("" : "+a"(acc[i][j]));
        }
    asm volatile("s_nop 7" ::: "memory");
}

// Products are written in assembly because their results have to stay in their registers: where the
// compiler chooses, it gives every product new ones and moves sums about.  They stand one by one, with
// what else there is to do between them: a wave has a matrix unit to itself and issues in order, so
// a product's 32 cycles leave room for seven other instructions, and what comes in a heap leaves the
// unit idle.  What the compiler does not see has to be right as it stands: operands come from loads
// (which it waits for), never from an instruction less than three ahead, and sums are read behind
// pr_settle.
__device__ __forceinline__ void pr_multiply(pr_f16 &acc, pr_bf8 a, pr_bf8 b) {
    asm volatile("v_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+a"(acc) : "v"(a), "v"(b));
}
// Behind a loop's last products (where s == end): the matrix units have written their results.  The
// branch around the waits is in here so that it stays within the loop, before any use of a sum.
__device__ __forceinline__ void pr_settle(int s, int end) {
    asm volatile("s_cmp_lg_u32 %0, %1\n\ts_cbranch_scc1 2\n\ts_nop 15\n\ts_nop 15" ::"s"(s), "s"(end) : "scc", "memory");
}
