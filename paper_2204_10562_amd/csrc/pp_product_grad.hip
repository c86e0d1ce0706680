// Products of a matrix of gradients with a packed operand whose rows the sum runs over: dx = dy W4
// and dw = dy^T X8, on the 16-bit matrix instructions with sums in 32 bits.
//
// Both operands lie in LDS as bf16, 64 rows of the sum to a step.  Gradients go there straight from
// global memory; packed values are read into registers, turned into bf16 (which holds every one of
// them: seven bits of code and a power of two) and written.  Operands that lie with the sum across
// their rows are read transposed (four values of a column to a lane, two reads to a fragment).
// A packed operand's blocks lie across the sum here, so no scaled instruction can take them as they are.
// Nothing is rounded on the way: products are exact in 32 bits, sums are held there.
//
// What bounds it.  Tiles of 256 x 256, eight waves with eight fragments each: 8192 rows, 16384 -> 4096
// (1.1 TFLOP) take 830 to 930 us for dx, 1.2 to 1.3 PFLOP/s (the library's product of two bf16 matrices of 8192 reaches
// 1.2 to 1.4), and 1060 to 1160 us for dw, whose 0.8 GB of results and of what they are added to come on top; of zeros
// 730 and 920: power first, with the clock at 1.5 GHz (zeros 2.1) and the matrix units at work in 73 % of the cycles for dx; for dw in
// 56 %, the rest the way out.  (Four waves with sixteen fragments each have no registers left for
// what is on its way.)  Smaller tiles are bound by instruction issue: 16 products to 170 or 190 other instructions
// (250 of 8 bits) a step and wave.  256 x 128 for dx, eight waves, turns a packed value for twice as many products as
// 128 x 128 with two workgroups to a compute unit, which wastes less where there are few: 333 rows, 5000 -> 4100 from
// fp16, two planes, in five pieces 40 us (44).  For dw the same (128 x 256) is 5 % faster where the operands are in
// cache and 8 % slower where they come from memory, with one workgroup to wait for them, so it is left out; dw and db
// of 32771 rows, 520 -> 1000, take 62 to 66 us in twelve pieces, 0.53 PFLOP/s.  256 x 32 is for few rows of dy: 16 rows,
// 16384 -> 4096 takes 16 us.
#include "pp_product_grad.h"

// WI x WO fragments of 32 x 32 to a wave, NI x NO waves
template <int WI, int WO, int NI, int NO> struct PgTile {
    static const int TI = 32 * WI * NI, TO = 32 * WO * NO, WAVES = NI * NO;
    static const int SI = TI * 128, SO = TO * 128;  // bytes of a stage: 64 values of the sum
    static const int LDS = 2 * (SI + SO) > WAVES * 4096 * WI ? 2 * (SI + SO) : WAVES * 4096 * WI;
};

// 32-byte units of a row of the sum are swapped by this (an exclusive or), so that the 16 rows which
// the lanes of a transposed read take are spread over the banks.  (Not all of them: what is counted of two lengths of the sum, 96
// of a wave's 224 LDS cycles a step for dx and 128 of 256 for dw, fits two cycles more than two for each such read, and eight
// more than eight for each write of turned values.  LDS is busy 55 to 65 % of the time.)
__device__ __forceinline__ int pg_turn(int row) { return (row & 3) | ((row >> 3) & 1) << 2; }

__device__ __forceinline__ pr_bf8 pg_read_t(const uint8_t *p, int second) {  // rows c..c+3 and c+4..c+7
    typedef PR_LDS pr_s4 *L4;
    const pr_s4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((L4)p), b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((L4)(p + second));
    return __builtin_bit_cast(pr_bf8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
}

// Two packed values, the w-th of a piece of sixteen, as bf16: exact, and NaN where the block is (products
// with a unit that is NaN are, and so are conversions of 4 bits).
template <int FMT> struct PgUnit {
    float unit;
    __device__ __forceinline__ void set(unsigned byte) {
        unit = __builtin_amdgcn_ldexpf(1.0f, (int)byte - (FMT == PP_PACK_INT8 ? 133 : 127));
        unit = byte == 255 ? pp_bits(0x7fc00000u) : unit;
    }
    __device__ __forceinline__ unsigned two(pp_u4 raw, int w) const {
        if constexpr (FMT == PP_PACK_INT8) {
            const unsigned c = raw[w >> 1] >> (16 * (w & 1));
            const pp_bf2 v = {(__bf16)((float)(signed char)c * unit), (__bf16)((float)(signed char)(c >> 8) * unit)};
            return __builtin_bit_cast(unsigned, v);
        }
        const unsigned c = raw[w >> 2];
        pp_bf2 v;
        if ((w & 3) == 0) v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, unit, 0);
        else if ((w & 3) == 1) v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, unit, 1);
        else if ((w & 3) == 2) v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, unit, 2);
        else v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, unit, 3);
        return __builtin_bit_cast(unsigned, v);
    }
};

template <int FMT, bool ALONG, int WI, int WO, int NI, int NO, class Y, bool SUMS>
__global__ __launch_bounds__(64 * NI * NO, 1) void k_product_grad(pr_plan p, pg_inner x, pg_outer y, pr_out<Y> out, float *sums) {
    typedef PgTile<WI, WO, NI, NO> L;
    constexpr int CB = FMT == PP_PACK_INT8 ? 16 : 8;  // bytes of sixteen codes
    constexpr int PER_ROW = L::TI / 16, ROWS = 64 * L::WAVES / PER_ROW, PIECES = 64 / ROWS;  // sixteen codes to a thread, PIECES times
    constexpr int RI = L::TI * 2, RO = L::TO * 2;     // bytes of a row of the sum
    constexpr int LO = L::SO / 1024 / L::WAVES ? L::SO / 1024 / L::WAVES : 1;  // loads of a wave for the outer operand
    constexpr int TURN_O = L::TO / 16 < 8 ? L::TO / 16 - 1 : 7;
    extern __shared__ uint8_t sm[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    unsigned ti, to;
    int piece;
    pr_tile(p, blockIdx.x, ti, to, piece);
    const int s0 = piece * p.per;
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
    // The rows of the step that is loaded next; behind the last step loads find nothing.  (64 rows are less
    // than 2^29 bytes.)
    __amdgpu_buffer_rsrc_t xb, xsb;
    int xi = s0 % per_plane, xleft = (int)x.rows - xi * 64;  // its number in its plane, the rows from there on
    const uint8_t *xat = x.codes + (long long)xi * 64 * xpitch, *xsat = x.scales + (long long)xi * 64 * spitch;
    auto next_inner = [&](bool some) {
        // (a scalar, which the compiler has to be told: it would load in a loop over the lanes' buffers)
        const int n = __builtin_amdgcn_readfirstlane(!some || xleft < 0 ? 0 : xleft < 64 ? xleft : 64);
        xb = __builtin_amdgcn_make_buffer_rsrc((void *)xat, 0, n * (int)xpitch, 0x00027000);
        xsb = __builtin_amdgcn_make_buffer_rsrc((void *)xsat, 0, n * (int)spitch, 0x00027000);
        const bool wrap = ++xi == per_plane;
        xi = wrap ? 0 : xi;
        xat = wrap ? x.codes : xat + 64 * xpitch;
        xsat = wrap ? x.scales : xsat + 64 * spitch;
        xleft = wrap ? (int)x.rows : xleft - 64;
    };
    auto load_inner = [&](int j) {
        if constexpr (FMT == PP_PACK_INT8) {
            raw[j] = __builtin_bit_cast(pp_u4, __builtin_amdgcn_raw_buffer_load_b128(xb, vx[j], 0, 0));
        } else {
            const pp_u2 t = __builtin_bit_cast(pp_u2, __builtin_amdgcn_raw_buffer_load_b64(xb, vx[j], 0, 0));
            raw[j][0] = t[0];
            raw[j][1] = t[1];
        }
        scale[j] = __builtin_amdgcn_raw_buffer_load_b8(xsb, vs[j], 0, 0);
    };
    int wx[PIECES];
#pragma unroll
    for (int j = 0; j < PIECES; ++j) wx[j] = (xr + j * ROWS) * RI + 32 * (xc ^ pg_turn(xr + j * ROWS));
    PgUnit<FMT> unit;
    pp_u4 half;
    // Part t of turning step s's packed values into bf16: two of them, the eighth part of a piece.
    auto turn_inner = [&](int t, int s) {
        const int j = t >> 3, w = t & 7;
        if (w == 0) unit.set(scale[j]);
        half[w & 3] = unit.two(raw[j], w);
        if ((w & 3) == 3) *(pp_u4 *)(sm + (s & 1) * (L::SI + L::SO) + wx[j] + 16 * (w >> 2)) = half;
    };

    // the gradients: 1024 bytes of a stage to a load of a wave
    unsigned vo[LO];
    int col_o[LO];
    const int chunk = (wave * LO) % (L::SO / 1024);
#pragma unroll
    for (int j = 0; j < LO; ++j) {
        const int b = (chunk + j) * 1024 + lane * 16;  // byte of the stage
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
    const unsigned to_o = base + L::SI + chunk * 1024;
    // From the step on that is loaded next: address, and bytes that it may use (less than 2^32, and whole words: less than
    // four bytes count as beyond the buffer).
    const int per_step = ALONG ? 128 : (int)(y.ld * 128);
    const int orows = y.rows - o0 < L::TO ? (int)(y.rows - o0) : L::TO, row_bytes = (int)(y.cols - (ALONG ? 0 : o0)) * 2;
    const uint8_t *oplane = y.p + (ALONG ? o0 * y.ld : o0) * 2 + (s0 / per_plane) * y.plane * 2;
    int oi = s0 % per_plane;
    const uint8_t *oat = oplane + (long long)oi * per_step;
    pp_i4 ob;
    int ocols;
    auto next_outer = [&](bool some) {
        unsigned bytes;
        if constexpr (ALONG) {
            ocols = (int)y.cols - 64 * oi;
            bytes = (unsigned)((orows - 1) * (int)y.ld) * 2 + ocols * 2;
        } else {
            const int left = (int)y.rows - 64 * oi, n = left < 64 ? left : 64;
            bytes = n <= 0 ? 0 : ((unsigned)(n - 1) * (unsigned)y.ld) * 2 + row_bytes;
        }
        const unsigned long long at = (unsigned long long)oat;
        ob[0] = __builtin_amdgcn_readfirstlane((int)at);
        ob[1] = __builtin_amdgcn_readfirstlane((int)(at >> 32) & 0xffff);
        ob[2] = __builtin_amdgcn_readfirstlane(some ? (int)bytes : 0);
        ob[3] = 0x00027000;
        const bool wrap = ++oi == per_plane;
        oi = wrap ? 0 : oi;
        oplane = wrap ? oplane + y.plane * 2 : oplane;
        oat = wrap ? oplane : oat + per_step;
    };
    auto aim = [&](int j, int s) { pr_aim(to_o + (s & 1) * (L::SI + L::SO), j * 1024); };
    auto fire = [&](int j) { pr_fire(ob, ALONG && col_o[j] >= ocols ? PR_BEYOND : vo[j], 0); };

    // fragments: inner ones transposed, outer ones where the sum runs across their rows.  A quarter of
    // a step is 16 values of the sum, eight to a half of the lanes.
    const int wi = wave % NI, wo = wave / NI, r = lane & 31, g = lane >> 5, h = (lane >> 4) & 1, u = lane & 15;
    const int row_t = 8 * g + (u >> 2), turn = pg_turn(row_t);
    int ai[WI], ao[ALONG ? 4 : WO];
#pragma unroll
    for (int j = 0; j < WI; ++j)  // chunk u % 4 of four columns, bits exchanged as by pr_inner_row
        ai[j] = row_t * RI + 32 * ((2 * (wi * WI + j) + h) ^ turn) + 16 * (u & 1) + 4 * (u & 2);
    if constexpr (ALONG) {
#pragma unroll
        for (int k = 0; k < 4; ++k) ao[k] = L::SI + (wo * WO * 32 + r) * 128 + 16 * ((2 * k + g) ^ ((r >> 1) & 7));
    } else {
#pragma unroll
        for (int j = 0; j < WO; ++j) ao[j] = L::SI + row_t * RO + 32 * ((2 * (wo * WO + j) + h) ^ (turn & TURN_O)) + 8 * (u & 3);
    }
    auto read_i = [&](const uint8_t *b, int k, int j) { return pg_read_t(b + ai[j] + k * 16 * RI, 4 * RI); };
    auto read_o = [&](const uint8_t *b, int k, int j) {
        if constexpr (ALONG) return *(const pr_bf8 *)(b + ao[k] + j * 4096);
        else return pg_read_t(b + ao[j] + k * 16 * RO, 4 * RO);
    };
    // Fragments.  The middle tile has room for a whole step's, read two quarters ahead (2 % faster than the other way);
    // otherwise the inner are replaced as they have been used, and the outer of odd quarters have places of their own
    // (4 % faster for the flat tile, whose quarters are two products).
    constexpr int N = WI * WO;  // products of a quarter step
    constexpr bool DEEP = N == 4;
    pr_bf8 in[DEEP ? 4 : 1][WI], outer[DEEP ? 4 : 2][WO];
    pr_f16 acc[WI][WO];
    // The columns' sums: a lane's eight rows by pairs, in 32 bits.  In one piece the first tile of a row of tiles adds
    // them all up, in several pieces its tiles take the steps in turn (what one of them adds keeps the others waiting:
    // dw of 32771 rows, 520 -> 1000, 73 us with the first alone, 69 in turn), and k_join adds what they found.
    const bool in_turn = p.splits > 1;
    int until = wi ? 0x7fffffff : in_turn || ti == 0 ? (int)ti : 0x7fffffff;  // steps until this wave's next
    float total[SUMS ? WO : 1] = {};
    auto add_up = [&](const pr_bf8 *f) {
#pragma unroll
        for (int j = 0; j < (SUMS ? WO : 0); ++j) {
            const pp_bf2 one = {(__bf16)1.0f, (__bf16)1.0f};
            float v = __builtin_amdgcn_fdot2_f32_bf16(__builtin_shufflevector(f[j], f[j], 0, 1), one, 0.0f, false);
            v = __builtin_amdgcn_fdot2_f32_bf16(__builtin_shufflevector(f[j], f[j], 2, 3), one, v, false);
            v = __builtin_amdgcn_fdot2_f32_bf16(__builtin_shufflevector(f[j], f[j], 4, 5), one, v, false);
            total[j] += __builtin_amdgcn_fdot2_f32_bf16(__builtin_shufflevector(f[j], f[j], 6, 7), one, v, false);
        }
    };

    // The waves meet in front of product MEET: step s + 1 is there then, and every wave has read all of step s.
    constexpr int MEET = DEEP ? 2 * N + N / 2 : 3 * N + WO;
    constexpr int PARTS = 8 * PIECES;
    // Step s + 2's gradients are asked for in the SLOTS products behind a meeting; step s + 1's packed values
    // turned from product TURN to TURN_END of a step on.  (Waiting for a packed value the compiler, which does
    // not know of the gradients, waits for those of them that were asked for later too: they have to be old.)
    constexpr int SLOTS = 4 * N - MEET, TURN = DEEP ? N : 2 * N, TURN_END = DEEP ? MEET : 3 * N;
    next_inner(true);
#pragma unroll
    for (int j = 0; j < PIECES; ++j) load_inner(j);
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        next_outer(t < steps);
#pragma unroll
        for (int j = 0; j < LO; ++j) {
            aim(j, t);
            asm volatile("s_nop 0");
            fire(j);
        }
    }
#pragma unroll
    for (int t = 0; t < PARTS; ++t) turn_inner(t, 0);
    next_inner(steps > 1);
#pragma unroll
    for (int j = 0; j < PIECES; ++j) load_inner(j);
    PR_WAIT(2 * PIECES);
    pr_barrier();
#pragma unroll
    for (int k = 0; k < (DEEP ? 2 : 1); ++k) {
#pragma unroll
        for (int j = 0; j < WI; ++j) in[k][j] = read_i(sm, k, j);
#pragma unroll
        for (int j = 0; j < WO; ++j) outer[k][j] = read_o(sm, k, j);
    }
    pr_clear(acc);
    __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0): the compiler need not wait for these within the loop
    auto behind = [&](int m, int stage) {  // what goes out behind product m from a meeting on
#pragma unroll
        for (int j = m * LO / SLOTS; j < (m + 1) * LO / SLOTS; ++j) {
            if (j > m * LO / SLOTS) asm volatile("s_nop 0");
            fire(j);
            if (j + 1 < LO) aim(j + 1, stage);
        }
    };
    for (int s = 0; s < steps; ++s) {
        const uint8_t *now = sm + (s & 1) * (L::SI + L::SO), *next = sm + ((s + 1) & 1) * (L::SI + L::SO);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const pr_bf8 *f = in[DEEP ? k : 0], *o = outer[DEEP ? k : k & 1];
            const int ahead = DEEP ? (k + 2) & 3 : (k + 1) & 3;  // the quarter read meanwhile
            const uint8_t *b = k < (DEEP ? 2 : 3) ? now : next;  // after the last step: what lies there, for nothing
            if (SUMS && until == 0) add_up(o);
            if (k == TURN / N) next_inner(s + 2 < steps);
#pragma unroll
            for (int m = 0; m < N; ++m) {
                const int i = m / WO, j = m % WO, at = k * N + m;
                if (at == MEET) {
                    PR_WAIT(2 * PIECES);  // (but for the packed values of the step after it)
                    pr_barrier();
                    next_outer(s + 2 < steps);
                    aim(0, s);
                }
                pr_multiply(acc[i][j], f[i], o[j]);
                const int from = k == MEET / N ? MEET % N : 0, n = m - from;  // the quarter's reads start here
                if (n >= 0) {
                    constexpr int TO = DEEP ? 4 : 2;
                    pr_bf8 *fa = in[DEEP ? ahead : 0], *oa = outer[ahead % TO];
                    if (n < WO) oa[n] = read_o(b, ahead, n);
                    if (!DEEP && from && n == 0) fa[0] = read_i(b, ahead, 0);  // (used up before the meeting)
                    if (!DEEP && j == WO - 1) fa[i] = read_i(b, ahead, i);
                    if (DEEP)
#pragma unroll
                        for (int q = n * WI / (N - from); q < (n + 1) * WI / (N - from); ++q) fa[q] = read_i(b, ahead, q);
                }
                if (at >= TURN && at < TURN_END) {
                    const int slot = at - TURN;
#pragma unroll
                    for (int t = slot * PARTS / (TURN_END - TURN); t < (slot + 1) * PARTS / (TURN_END - TURN); ++t) {
                        turn_inner(t, s + 1);
                        if ((t & 7) == 7) load_inner(t >> 3);  // step s + 2's: a whole step ahead
                    }
                }
                if (at >= MEET) behind(at - MEET, s);
                PR_PIN;
            }
        }
        if (SUMS) until = until ? until - 1 : in_turn ? (int)p.ni - 1 : 0;
        pr_settle(s + 1, steps);
    }
    PR_WAIT(0);  // nothing is on its way to LDS any more
    pr_barrier();
    if constexpr (SUMS)
        if (wi == 0 && (in_turn || ti == 0)) {
            float *part = sums + (in_turn ? ((long long)piece * p.ni + ti) * p.outer : 0);
#pragma unroll
            for (int j = 0; j < WO; ++j) {
                const float v = total[j] + __shfl_xor(total[j], 32);
                const long long o = o0 + (wo * WO + j) * 32 + r;
                if (g == 0 && o < p.outer) part[o] = v;
            }
        }
    pr_leave<Y, WI, WO>(p, out, acc, sm + wave * (32 * 32 * WI * 4), lane, i0 + wi * WI * 32, o0 + wo * WO * 32, piece);
}

template <int FMT, bool ALONG, int WI, int WO, int NI, int NO, class Y, bool SUMS>
static int launch_one(const pr_plan &p, const pg_inner &x, const pg_outer &y, const pr_out<Y> &out, float *sums, hipStream_t st) {
    typedef PgTile<WI, WO, NI, NO> L;
    auto *k = k_product_grad<FMT, ALONG, WI, WO, NI, NO, Y, SUMS>;
    k<<<p.ni * p.no * p.splits, 64 * L::WAVES, L::LDS, st>>>(p, x, y, out, sums);
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
    if (shape == 0) return launch_input<4, 2, 2, 4>(type, p, w, dy, dx, ld, st);
    if (shape == 1) return launch_input<2, 2, 2, 2>(type, p, w, dy, dx, ld, st);
    if (shape == 2) return launch_input<2, 1, 4, 1>(type, p, w, dy, dx, ld, st);
    return launch_input<2, 2, 4, 2>(type, p, w, dy, dx, ld, st);
}

int pg_launch_weight(int shape, const pr_plan &p, const pg_inner &x, const pg_outer &dy, float *dw, long long ld, const float *add, float *sums, hipStream_t st) {
    if (shape == 0) return launch_weight<4, 2, 2, 4>(p, x, dy, dw, ld, add, sums, st);
    return launch_weight<2, 2, 2, 2>(p, x, dy, dw, ld, add, sums, st);
}
