// Products of a matrix of gradients with a packed operand whose rows the sum runs over: dx = dy W4
// and dw = dy^T X8, on the 16-bit matrix instructions with sums in 32 bits.
//
// Both operands lie in LDS as bf16, 64 rows of the sum to a step.  Gradients go there straight from
// global memory; packed values are read into registers, turned into bf16 (which holds every one of
// them: seven bits of code and a power of two) and written.  Operands that lie with the sum across
// their rows are read transposed (four values of a column to a lane, two reads to a fragment).
#include "pp_product_grad.h"

template <int WI, int WO, int NI, int NO> struct PgTile {
    static const int TI = 16 * WI * NI, TO = 16 * WO * NO;
    static const int SI = TI * 128, SO = TO * 128;  // bytes of a stage: 64 values of the sum
    static const int LDS = 2 * (SI + SO);
};

// 32-byte units of a row of the sum are swapped by this (an exclusive or), so that the 16 rows which
// the lanes of a transposed read take fall on different banks.
__device__ __forceinline__ int pg_turn(int row) { return (row & 3) | ((row >> 3) & 1) << 2; }

__device__ __forceinline__ pr_bf8 pg_read_t(const uint8_t *p, int second) {  // rows c..c+3 and c+4..c+7
    typedef PR_LDS pr_s4 *L4;
    const pr_s4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((L4)p), b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((L4)(p + second));
    return __builtin_bit_cast(pr_bf8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
}

// Sixteen packed values as bf16: exact, NaN where the block is.
template <int FMT> __device__ __forceinline__ void pg_convert(pp_u4 raw, unsigned byte, pp_u4 *out) {
    if constexpr (FMT == PP_PACK_INT8) {
        const float unit = pp_unit8(byte);
#pragma unroll
        for (int w = 0; w < 8; ++w) {
            const unsigned c = raw[w >> 1] >> (16 * (w & 1));
            const pp_bf2 v = {(__bf16)((float)(signed char)c * unit), (__bf16)((float)(signed char)(c >> 8) * unit)};
            out[w >> 2][w & 3] = __builtin_bit_cast(unsigned, v);
        }
    } else {
        const float unit = pp_unit4(byte == 255 ? 0 : byte);
        const unsigned nan = byte == 255 ? 0x7fc07fc0u : 0;
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            out[w][0] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(raw[w], unit, 0)) | nan;
            out[w][1] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(raw[w], unit, 1)) | nan;
            out[w][2] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(raw[w], unit, 2)) | nan;
            out[w][3] = __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(raw[w], unit, 3)) | nan;
        }
    }
}

template <int FMT, bool ALONG, int WI, int WO, int NI, int NO, class Y, bool SUMS>
__global__ __launch_bounds__(PR_THREADS, 1) void k_product_grad(pr_plan p, pg_inner x, pg_outer y, pr_out<Y> out, float *sums) {
    typedef PgTile<WI, WO, NI, NO> L;
    constexpr int H = WO / 2, P = H ? H : WO;
    constexpr int CB = FMT == PP_PACK_INT8 ? 16 : 8;  // bytes of sixteen codes
    constexpr int PER_ROW = L::TI / 16, ROWS = PR_THREADS / PER_ROW, PIECES = 64 / ROWS;  // sixteen codes to a thread, PIECES times
    constexpr int RI = L::TI * 2, RO = L::TO * 2;     // bytes of a row of the sum
    constexpr int LO = L::SO / 4096 ? L::SO / 4096 : 1;  // loads of a wave for the outer operand
    constexpr int TURN_O = L::TO / 16 < 8 ? L::TO / 16 - 1 : 7;
    extern __shared__ uint8_t sm[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    unsigned ti, to;
    pr_tile(p, blockIdx.x, ti, to);
    const int piece = blockIdx.y, s0 = piece * p.per;
    const int steps = p.steps - s0 < p.per ? p.steps - s0 : p.per, per_plane = p.steps / y.planes;
    const long long i0 = (long long)ti * L::TI, o0 = (long long)to * L::TO;
    const unsigned base = pr_lds_of(sm);

    // the packed operand: this thread's sixteen codes of rows xr, xr + ROWS, ...
    const int xr = tid / PER_ROW, xc = tid % PER_ROW;
    const long long xpitch = x.groups * (FMT == PP_PACK_INT8 ? PP_GROUP_CODES8 : PP_GROUP_CODES4), spitch = x.groups * 4;
    const long long xcol = i0 / 16 + xc;
    const bool inside = xcol < x.groups * 8;
    unsigned vx[PIECES], vs[PIECES];  // whole offsets: what lies beyond the operand's last row is seen by them
#pragma unroll
    for (int j = 0; j < PIECES; ++j) {
        vx[j] = inside ? (unsigned)((xr + j * ROWS) * xpitch + xcol * CB) : PR_BEYOND;
        vs[j] = inside ? (unsigned)((xr + j * ROWS) * spitch + (xcol >> 1)) : PR_BEYOND;
    }
    pp_u4 raw[PIECES];
    unsigned char scale[PIECES];
    auto load_inner = [&](int s) {
        const long long c0 = (long long)((s0 + s) % per_plane) * 64;
        const auto b = pr_resource(x.codes + c0 * xpitch, (x.rows - c0) * xpitch), sc = pr_resource(x.scales + c0 * spitch, (x.rows - c0) * spitch);
#pragma unroll
        for (int j = 0; j < PIECES; ++j) {
            if constexpr (FMT == PP_PACK_INT8) {
                raw[j] = __builtin_bit_cast(pp_u4, __builtin_amdgcn_raw_buffer_load_b128(b, vx[j], 0, 0));
            } else {
                const pp_u2 t = __builtin_bit_cast(pp_u2, __builtin_amdgcn_raw_buffer_load_b64(b, vx[j], 0, 0));
                raw[j] = pp_u4{t[0], t[1], 0, 0};
            }
            scale[j] = __builtin_amdgcn_raw_buffer_load_b8(sc, vs[j], 0, 0);
        }
    };
    int wx[PIECES];
#pragma unroll
    for (int j = 0; j < PIECES; ++j) wx[j] = (xr + j * ROWS) * RI + 32 * (xc ^ pg_turn(xr + j * ROWS));
    auto store_inner = [&](int j, int s) {
        pp_u4 v[2];
        pg_convert<FMT>(raw[j], scale[j], v);
        uint8_t *q = sm + (s & 1) * (L::SI + L::SO) + wx[j];
        *(pp_u4 *)q = v[0];
        *(pp_u4 *)(q + 16) = v[1];
    };

    // the gradients: 1024 bytes of a stage to a load of a wave
    unsigned vo[LO];
    int lo[LO], col_o[LO];
#pragma unroll
    for (int j = 0; j < LO; ++j) {
        const int at = ((wave * LO + j) * 1024) % L::SO, b = at + lane * 16;  // byte of the stage
        lo[j] = at;
        if constexpr (ALONG) {
            const int row = b >> 7, unit = ((b >> 4) & 7) ^ ((row >> 1) & 7);
            col_o[j] = unit * 8;
            vo[j] = (unsigned)(row * y.ld * 2) + unit * 16;
        } else {
            const int row = b / RO, unit = (b % RO / 32) ^ (pg_turn(row) & TURN_O);
            col_o[j] = 0;
            vo[j] = (unsigned)(row * y.ld * 2) + unit * 32 + (b & 16);
        }
    }
    auto load_outer = [&](int s) {
        const int plane = (s0 + s) / per_plane;
        const long long c0 = (long long)(s0 + s - plane * per_plane) * 64;
        const uint8_t *q = y.p + plane * y.plane * 2;
        pp_i4 b;
        long long left = 1 << 30;
        if constexpr (ALONG) {
            const long long rows = y.rows - o0 < L::TO ? y.rows - o0 : L::TO;
            left = y.cols - c0;
            b = pr_buffer(q + (o0 * y.ld + c0) * 2, s < steps ? ((rows - 1) * y.ld + left) * 2 : 0);
        } else {
            // up to the end of the last value's four bytes: less than four count as beyond the buffer
            b = pr_buffer(q + (c0 * y.ld + o0) * 2, s < steps && c0 < y.rows ? (((y.rows - c0 - 1) * y.ld + y.cols - o0) * 2 + 3) & ~3ll : 0);
        }
#pragma unroll
        for (int j = 0; j < LO; ++j)
            pr_to_lds(b, ALONG && col_o[j] >= left ? PR_BEYOND : vo[j], 0, base + (s & 1) * (L::SI + L::SO) + L::SI + lo[j]);
    };

    // fragments: inner ones transposed, outer ones where the sum runs across their rows
    const int wi = wave % NI, wo = wave / NI, r = lane & 15, g = lane >> 4;
    const int row_t = 8 * g + (r >> 2), turn = pg_turn(row_t);
    int ai[WI / 2], ao[ALONG ? 1 : WO];
#pragma unroll
    for (int j = 0; j < WI / 2; ++j) ai[j] = row_t * RI + 32 * ((wi * WI + 2 * j + ((r & 3) >> 1)) ^ turn) + 16 * (r & 1);
    if constexpr (ALONG) {
        ao[0] = L::SI + (wo * WO * 16 + r) * 128;
    } else {
#pragma unroll
        for (int j = 0; j < WO; ++j) ao[j] = L::SI + row_t * RO + 32 * ((wo * WO + j) ^ (turn & TURN_O)) + 8 * (r & 3);
    }
    pr_bf8 in[WI], first[P], late[H ? H : 1];
    auto read_i = [&](int j, const uint8_t *b, int h) { in[j] = pg_read_t(b + ai[j >> 1] + 8 * (j & 1) + h * 32 * RI, 4 * RI); };
    auto read_o = [&](pr_bf8 *f, int j0, int n, const uint8_t *b, int h) {
#pragma unroll
        for (int j = 0; j < n; ++j) {
            if constexpr (ALONG) f[j] = *(const pr_bf8 *)(b + ao[0] + (j0 + j) * 2048 + 16 * ((4 * h + g) ^ (r >> 1)));
            else f[j] = pg_read_t(b + ao[j0 + j] + h * 32 * RO, 4 * RO);
        }
    };
    pp_f4 acc[WI][WO] = {}, acc_s[WO] = {};
    const bool summing = SUMS && ti == 0 && wi == 0;
    const pr_bf8 ones = {(__bf16)1.0f, (__bf16)1.0f, (__bf16)1.0f, (__bf16)1.0f, (__bf16)1.0f, (__bf16)1.0f, (__bf16)1.0f, (__bf16)1.0f};
    // The columns' sums, a product with ones: in ordinary registers (the others are full), and waited
    // for at once, as what only some waves do may be moved about behind it.
    auto add_up = [&](const pr_bf8 *f, int j0, int n) {
#pragma unroll
        for (int j = 0; j < n; ++j)
            asm volatile("s_nop 1\n\tv_mfma_f32_16x16x32_bf16 %0, %1, %2, %0" : "+v"(acc_s[j0 + j]) : "v"(ones), "v"(f[j]));
        asm volatile("s_nop 15" : "+v"(acc_s[j0]));
#pragma unroll
        for (int j = 1; j < n; ++j) asm volatile("" : "+v"(acc_s[j0 + j]));
    };

    load_outer(0);
    load_inner(0);
#pragma unroll
    for (int j = 0; j < PIECES; ++j) store_inner(j, 0);
    PR_WAIT(0);
    pr_barrier();
    load_outer(1);
    load_inner(1);
#pragma unroll
    for (int j = 0; j < WI; ++j) read_i(j, sm, 0);
    read_o(first, 0, P, sm, 0);
    __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0): the compiler need not wait for these within the loop
    for (int s = 0; s < steps; ++s) {
        const uint8_t *now = sm + (s & 1) * (L::SI + L::SO), *next = sm + ((s + 1) & 1) * (L::SI + L::SO);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            if constexpr (H > 0) {
                read_o(late, H, H, now, h);
                if (SUMS && summing) add_up(first, 0, H);
            }
#pragma unroll
            for (int i = 0; i < WI; ++i) {
                if constexpr (H > 0) pr_multiply<H>(acc[i], in[i], first);
                if (h == 1) {  // step s + 1's packed values, which were asked for a step ago
#pragma unroll
                    for (int j = i * PIECES / WI; j < (i + 1) * PIECES / WI; ++j) store_inner(j, s + 1);
                }
            }
            if (h == 1) {
                PR_WAIT(0);  // and its gradients
                pr_barrier();
                load_outer(s + 2);
                load_inner(s + 2);
            }
            const uint8_t *b = h == 0 ? now : next;  // after the last step: what lies there, for nothing
            if constexpr (H > 0) read_o(first, 0, H, b, 1 - h);
#pragma unroll
            for (int i = 0; i < WI; ++i) {
                if constexpr (H > 0) pr_multiply<H>(acc[i] + H, in[i], late);
                else pr_multiply<WO>(acc[i], in[i], first);
                read_i(i, b, 1 - h);
            }
            if constexpr (H > 0) {
                if (SUMS && summing) add_up(late, H, H);
            } else {
                if (SUMS && summing) add_up(first, 0, WO);
                read_o(first, 0, P, b, 1 - h);
            }
        }
        pr_settle(s + 1, steps);
    }
    PR_WAIT(0);  // nothing is on its way to LDS when the workgroup ends
#pragma unroll
    for (int j = 0; j < WO; ++j) {
        const long long o = o0 + (wo * WO + j) * 16 + r;
#pragma unroll
        for (int i = 0; i < WI; i += 2) {
            float v[8];
            *(pp_f4 *)v = acc[i][j];
            *(pp_f4 *)(v + 4) = acc[i + 1][j];
            pr_put8<Y>(p, out, o, i0 + wi * WI * 16 + 16 * i + 8 * g, piece, v);
        }
        if constexpr (SUMS)
            if (summing && g == 0 && o < p.outer) sums[piece * p.outer + o] = acc_s[j][0];
        __builtin_amdgcn_sched_barrier(0);
    }
}

template <int FMT, bool ALONG, int WI, int WO, int NI, int NO, class Y, bool SUMS>
static int launch_one(const pr_plan &p, const pg_inner &x, const pg_outer &y, const pr_out<Y> &out, float *sums, hipStream_t st) {
    typedef PgTile<WI, WO, NI, NO> L;
    auto *k = k_product_grad<FMT, ALONG, WI, WO, NI, NO, Y, SUMS>;
    if (hipFuncSetAttribute((const void *)k, hipFuncAttributeMaxDynamicSharedMemorySize, L::LDS) != hipSuccess) return PP_ERR_HIP;
    k<<<dim3(p.ni * p.no, p.splits), PR_THREADS, L::LDS, st>>>(p, x, y, out, sums);
    return hipGetLastError() == hipSuccess ? PP_OK : PP_ERR_HIP;
}

template <int WI, int WO, int NI, int NO>
static int launch_input(int type, const pr_plan &p, const pg_inner &x, const pg_outer &y, void *out, long long ld, hipStream_t st) {
    return pp_by_type(type, [&](auto t) {
        typedef decltype(t) Y;
        return launch_one<PP_PACK_FP4, true, WI, WO, NI, NO, Y, false>(p, x, y, pr_out<Y>{(typename Y::T *)out, ld, NULL, NULL, 0}, NULL, st);
    });
}
template <int WI, int WO, int NI, int NO>
static int launch_weight(const pr_plan &p, const pg_inner &x, const pg_outer &y, float *out, long long ld, const float *add, float *sums, hipStream_t st) {
    const pr_out<PpF32> o{out, ld, NULL, add, ld};
    if (sums) return launch_one<PP_PACK_INT8, false, WI, WO, NI, NO, PpF32, true>(p, x, y, o, sums, st);
    return launch_one<PP_PACK_INT8, false, WI, WO, NI, NO, PpF32, false>(p, x, y, o, sums, st);
}

int pg_launch_input(int shape, int type, const pr_plan &p, const pg_inner &w, const pg_outer &dy, void *dx, long long ld, hipStream_t st) {
    if (shape == 0) return launch_input<8, 8, 2, 2>(type, p, w, dy, dx, ld, st);
    if (shape == 1) return launch_input<4, 4, 2, 2>(type, p, w, dy, dx, ld, st);
    return launch_input<4, 2, 4, 1>(type, p, w, dy, dx, ld, st);
}

int pg_launch_weight(int shape, const pr_plan &p, const pg_inner &x, const pg_outer &dy, float *dw, long long ld, const float *add, float *sums, hipStream_t st) {
    if (shape == 0) return launch_weight<8, 8, 2, 2>(p, x, dy, dw, ld, add, sums, st);
    return launch_weight<4, 4, 2, 2>(p, x, dy, dw, ld, add, sums, st);
}
