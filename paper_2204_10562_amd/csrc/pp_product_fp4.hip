// Products of two matrices in blocks of 4 bits: y = X4 W4^T on the scaled matrix instructions, which
// take 128 values of either operand and a power of two for every 32 at once.
//
// k_product4: both operands go from global memory straight to LDS, 64 bytes (128 values) of a row to
// a step, three steps deep; a wave reads the fragments of the next step while the matrix units work
// on this one.  The 16-byte pieces of a row are rotated by the row (swapped by an exclusive or), so
// that the 16 rows of a fragment fall on different banks.
#include "pp_product.h"
#include "pp_product_fp4.h"

// Four bytes from any address of LDS: the scale is the low one, the others are not looked at.  (A
// byte load would do, but the compiler clears the upper bytes again where a value goes round a loop.)
struct p4_any4 { int v __attribute__((packed, aligned(1))); };

// pr_multiply for 128 values of 4 bits and their scales.
template <int N> __device__ __forceinline__ void p4_multiply(pp_f4 *acc, pp_i4 a, int ca, const pp_i4 *b, const int *cb) {
    if constexpr (N == 4)
        asm volatile("s_nop 1\n\t"
                     "v_mfma_scale_f32_16x16x128_f8f6f4 %0, %4, %6, %0, %5, %7 op_sel_hi:[0,0,0] cbsz:4 blgp:4\n\t"
                     "v_mfma_scale_f32_16x16x128_f8f6f4 %1, %4, %8, %1, %5, %9 op_sel_hi:[0,0,0] cbsz:4 blgp:4\n\t"
                     "v_mfma_scale_f32_16x16x128_f8f6f4 %2, %4, %10, %2, %5, %11 op_sel_hi:[0,0,0] cbsz:4 blgp:4\n\t"
                     "v_mfma_scale_f32_16x16x128_f8f6f4 %3, %4, %12, %3, %5, %13 op_sel_hi:[0,0,0] cbsz:4 blgp:4"
                     : "+a"(acc[0]), "+a"(acc[1]), "+a"(acc[2]), "+a"(acc[3])
                     : "v"(a), "v"(ca), "v"(b[0]), "v"(cb[0]), "v"(b[1]), "v"(cb[1]), "v"(b[2]), "v"(cb[2]),
                       "v"(b[3]), "v"(cb[3]));
    else
#pragma unroll
        for (int j = 0; j < N; ++j)
            asm volatile("s_nop 1\n\tv_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %3, %0, %2, %4 op_sel_hi:[0,0,0] cbsz:4 blgp:4"
                         : "+a"(acc[j]) : "v"(a), "v"(ca), "v"(b[j]), "v"(cb[j]));
}
template <int WI, int WO, int NI, int NO> struct P4Tile {
    static const int TI = 16 * WI * NI, TO = 16 * WO * NO;
    static const int SI = TI * PR_STEP, SO = TO * PR_STEP;           // bytes of a stage
    static const int CI = TI * 16, CO = (TO < 64 ? 64 : TO) * 16;    // bytes of four steps' scales
    static const int LDS = 3 * (SI + SO) + 2 * (CI + CO) + 16;  // a scale is read with what follows it
    static const int LI = TI / 64, LO = TO < 64 ? 1 : TO / 64;       // loads of a wave to a step
};

template <int WI, int WO, int NI, int NO, class Y>
__global__ __launch_bounds__(PR_THREADS, 1) void k_product4(pr_plan p, p4_operands q, pr_out<Y> out) {
    typedef P4Tile<WI, WO, NI, NO> L;
    constexpr int H = WO / 2, P = H ? H : WO;
    extern __shared__ uint8_t sm[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    unsigned ti, to;
    pr_tile(p, blockIdx.x, ti, to);
    const int piece = blockIdx.y, s0 = piece * p.per;
    const int steps = p.steps - s0 < p.per ? p.steps - s0 : p.per;
    const long long i0 = (long long)ti * L::TI, o0 = (long long)to * L::TO;
    const long long pitch = (long long)p.steps * PP_GROUP_CODES4, spitch = (long long)p.steps * 4;
    const long long ri = p.inner - i0 < L::TI ? p.inner - i0 : L::TI, ro = p.outer - o0 < L::TO ? p.outer - o0 : L::TO;
    const pp_i4 bi = pr_buffer(q.inner_codes + i0 * pitch, ri * pitch), bo = pr_buffer(q.outer_codes + o0 * pitch, ro * pitch);
    const pp_i4 ci = pr_buffer(q.inner_scales + i0 * spitch, ri * spitch), co = pr_buffer(q.outer_scales + o0 * spitch, ro * spitch);
    const unsigned base = pr_lds_of(sm), scales = base + 3 * (L::SI + L::SO);

    // where this lane's pieces come from: 16 rows of four pieces to a load.  Inner rows differ in
    // bits 3 and 4 within a fragment, outer ones in bits 2 and 3.
    unsigned vi[L::LI], vo[L::LO];
    int li[L::LI], lo[L::LO];
#pragma unroll
    for (int j = 0; j < L::LI; ++j) {
        const int chunk = wave * L::LI + j, row = 16 * chunk + (lane >> 2);
        vi[j] = (unsigned)(row * pitch) + 16 * ((lane & 3) ^ ((row >> 3) & 3));
        li[j] = chunk * 1024;
    }
#pragma unroll
    for (int j = 0; j < L::LO; ++j) {
        const int chunk = (wave * L::LO + j) % (L::TO / 16), row = 16 * chunk + (lane >> 2);
        vo[j] = (unsigned)(row * pitch) + 16 * ((lane & 3) ^ ((row >> 2) & 3));
        lo[j] = chunk * 1024;
    }
    const int wi64 = wave % (L::TI / 64), wo64 = wave % (L::TO < 64 ? 1 : L::TO / 64);
    const unsigned vci = (unsigned)((64 * wi64 + lane) * spitch);
    const unsigned vco = L::TO < 64 && lane >= L::TO ? 0xfffffff0u : (unsigned)((64 * wo64 + lane) * spitch);

    auto load = [&](int s, unsigned buf) {  // step s of this piece into stage `buf`
        if (!(s & 3)) {
            const unsigned c = scales + ((s >> 2) & 1) * (L::CI + L::CO);
            pr_to_lds(ci, vci, (unsigned)(s0 + s) * 4, c + wi64 * 1024);
            pr_to_lds(co, vco, (unsigned)(s0 + s) * 4, c + L::CI + wo64 * 1024);
        }
        const unsigned b = base + buf * (L::SI + L::SO), at = (unsigned)(s0 + s) * PR_STEP;
#pragma unroll
        for (int j = 0; j < L::LI; ++j) pr_to_lds(bi, vi[j], at, b + li[j]);
#pragma unroll
        for (int j = 0; j < L::LO; ++j) pr_to_lds(bo, vo[j], at, b + L::SI + lo[j]);
    };

    const int wi = wave % NI, wo = wave / NI, r = lane & 15, g = lane >> 4;
    const int ir = 8 * (r >> 2) + (r & 3);
    const int fi = (wi * WI * 16 + ir) * PR_STEP + 16 * (g ^ (ir >> 3));                    // + 4 rows for odd fragments, 32 for pairs
    const int fo = L::SI + (wo * WO * 16 + r) * PR_STEP + 16 * (g ^ (r >> 2));
    const int si = (wi * WI * 16 + ir) * 16 + g, so = L::CI + (wo * WO * 16 + r) * 16 + g;  // + 4 bytes to a step

    // The fragments of a step: the inner ones, the first half of the outer ones and the second.
    // What is read for the next step takes the place of what has just been used.
    pp_i4 in[WI], first[P], late[H ? H : 1];
    int in_c[WI], first_c[P], late_c[H ? H : 1];
    auto codes_at = [&](int buf) { return sm + buf * (L::SI + L::SO); };
    auto scales_at = [&](int s) { return sm + 3 * (L::SI + L::SO) + ((s >> 2) & 1) * (L::CI + L::CO) + (s & 3) * 4; };
    auto read_i = [&](int j, const uint8_t *b, const uint8_t *c) {
        in[j] = *(const pp_i4 *)(b + fi + (32 * (j >> 1) + 4 * (j & 1)) * PR_STEP);
        in_c[j] = ((const p4_any4 *)(c + si + (32 * (j >> 1) + 4 * (j & 1)) * 16))->v;
    };
    auto read_o = [&](pp_i4 *f, int *fc, int j0, int n, const uint8_t *b, const uint8_t *c) {
#pragma unroll
        for (int j = 0; j < n; ++j) {
            f[j] = *(const pp_i4 *)(b + fo + (j0 + j) * 16 * PR_STEP);
            fc[j] = ((const p4_any4 *)(c + so + (j0 + j) * 256))->v;
        }
    };
    pp_f4 acc[WI][WO] = {};

    load(0, 0);
    if (steps > 1) load(1, 1);
    if (steps > 2) load(2, 2);
    PR_WAIT(0);
    pr_barrier();
#pragma unroll
    for (int j = 0; j < WI; ++j) read_i(j, codes_at(0), scales_at(0));
    read_o(first, first_c, 0, P, codes_at(0), scales_at(0));
    __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0): the compiler need not wait for these within the loop
    int b0 = 0, b1 = 1, b2 = 2;  // the stages of steps s, s + 1 and s + 2
    for (int s = 0; s < steps; ++s) {
        if constexpr (H > 0) {
            read_o(late, late_c, H, H, codes_at(b0), scales_at(s));
#pragma unroll
            for (int i = 0; i < WI; ++i) p4_multiply<H>(acc[i], in[i], in_c[i], first, first_c);
        }
        // stage s + 1 has arrived for every wave, and every wave has read all of stage s
        if (s + 2 < steps) PR_WAIT(L::LI + L::LO);
        else PR_WAIT(0);
        pr_barrier();
        if (s + 3 < steps) load(s + 3, b0);
        const uint8_t *b = codes_at(b1), *c = scales_at(s + 1);  // after the last step: what lies there, for nothing
        if constexpr (H > 0) read_o(first, first_c, 0, H, b, c);
#pragma unroll
        for (int i = 0; i < WI; ++i) {
            if constexpr (H > 0) p4_multiply<H>(acc[i] + H, in[i], in_c[i], late, late_c);
            else p4_multiply<WO>(acc[i], in[i], in_c[i], first, first_c);
            read_i(i, b, c);
        }
        if constexpr (H == 0) read_o(first, first_c, 0, P, b, c);
        const int t = b0;
        b0 = b1;
        b1 = b2;
        b2 = t;
        pr_settle(s + 1, steps);
    }
#pragma unroll
    for (int j = 0; j < WO; ++j)
#pragma unroll
        for (int i = 0; i < WI; i += 2) {
            float v[8];
            *(pp_f4 *)v = acc[i][j];
            *(pp_f4 *)(v + 4) = acc[i + 1][j];
            pr_put8<Y>(p, out, o0 + (wo * WO + j) * 16 + r, i0 + wi * WI * 16 + 16 * i + 8 * g, piece, v);
        }
}

template <int WI, int WO, int NI, int NO> static int launch4(int type, pr_plan p, const p4_operands &q, void *y, long long ld, const float *bias, hipStream_t st) {
    typedef P4Tile<WI, WO, NI, NO> L;
    return pp_by_type(type, [&](auto t) {
        typedef decltype(t) Y;
        auto *k = k_product4<WI, WO, NI, NO, Y>;
        if (hipFuncSetAttribute((const void *)k, hipFuncAttributeMaxDynamicSharedMemorySize, L::LDS) != hipSuccess) return PP_ERR_HIP;
        k<<<dim3(p.ni * p.no, p.splits), PR_THREADS, L::LDS, st>>>(p, q, pr_out<Y>{(typename Y::T *)y, ld, bias, NULL, 0});
        return hipGetLastError() == hipSuccess ? PP_OK : PP_ERR_HIP;
    });
}

int p4_launch(int shape, int type, const pr_plan &p, const p4_operands &q, void *y, long long ld, const float *bias, hipStream_t st) {
    if (shape == 0) return launch4<8, 8, 2, 2>(type, p, q, y, ld, bias, st);
    if (shape == 1) return launch4<4, 4, 2, 2>(type, p, q, y, ld, bias, st);
    return launch4<4, 2, 4, 1>(type, p, q, y, ld, bias, st);
}
