// Products of two matrices in blocks of 4 bits: y = X4 W4^T on the scaled matrix instructions, which
// take 64 values of either operand and a power of two for every 32 at once.
//
// k_product4: both operands go from global memory straight to LDS, 64 bytes (128 values) of a row to
// a step, three or four steps deep; a wave reads the fragments of the next half step while the matrix units
// work on this one.  Blocks of 32 lie along the sum in both operands, which is what the instructions' scales
// are for: a product of blocks is exact, and sums are in 32 bits.
//
// What bounds it.  Tiles of 256 x 256 with 16 fragments of 32 x 32 to a wave read each byte from LDS once
// for 128 results, which leaves LDS idle for four cycles of five; 8192 rows, 4096 -> 16384 (1.1 TFLOP) take 390 to 440 us, 2.5 to
// 2.8 PFLOP/s, by how warm the card is.  The matrix units work in 39 % of the cycles: of a tile's 40 us 12 are the
// start and the way out, with nothing beside them, and waves wait 28 % of their time (with buffers of no
// bytes, so that loads find nothing, a step takes a fifth less).  Then comes power: the clock is 1.7 GHz, and
// 2.2 with zeros (335 us).  The matrix instructions by themselves, on random values in
// registers, reach 5.1 PFLOP/s, on zeros 9.  Where 256 x 256 does not fill the chip, 128 x 128 with two
// workgroups to a compute unit does, and 256 x 32 for a few dozen rows: both wait for LDS and each other
// between short runs of products.  333 rows, 4100 -> 5000 (fp16): 18 to 20 us, 0.7 PFLOP/s, 120 tiles on 256 units.
#include "pp_product_fp4.h"

// Of the four scales of a row's step, the lane's own of either half become the bytes 0 and 2.  Three
// wait states have to lie between this and a product that takes it.
__device__ __forceinline__ int p4_own(int scales, int shift) {
    int v;
    asm volatile("v_lshrrev_b32 %0, %1, %2" : "=v"(v) : "v"(shift), "v"(scales));
    return v;
}

template <int HALF> __device__ __forceinline__ void p4_multiply(pr_f16 &acc, pp_i4 a, int ca, pp_i4 b, int cb) {
    if constexpr (HALF == 0)
        asm volatile("v_mfma_scale_f32_32x32x64_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel_hi:[0,0,0] cbsz:4 blgp:4" : "+a"(acc) : "v"(a), "v"(b), "v"(ca), "v"(cb));
    else
        asm volatile("v_mfma_scale_f32_32x32x64_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel_hi:[1,1,0] cbsz:4 blgp:4" : "+a"(acc) : "v"(a), "v"(b), "v"(ca), "v"(cb));
}

// The 16-byte pieces of a row lie exchanged by this (an exclusive or): LDS serves 64 lanes of 16 bytes
// in four turns of 16, whose rows (0-3, 12-15, 20-23 and 24-27, and so on) then fall on different banks.  (The
// conflicts that are counted, 48 of the 128 LDS cycles of a wave's step, fit the reads of scales, from rows 16 bytes apart.)
__device__ __forceinline__ int p4_turn(int row) { return (row >> 2) & 3; }

// WI x WO fragments of 32 x 32 to a wave, NI x NO waves
// (AHEAD steps in LDS)
template <int WI, int WO, int NI, int NO, int AHEAD> struct P4Tile {
    static const int TI = 32 * WI * NI, TO = 32 * WO * NO, WAVES = NI * NO;
    static const int SI = TI * PR_STEP, SO = TO * PR_STEP;           // bytes of a stage
    static const int CI = TI * 16, CO = (TO < 64 ? 64 : TO) * 16;    // bytes of four steps' scales
    static const int SCALES = AHEAD * (SI + SO), ALL = SCALES + 2 * (CI + CO);
    static const int LDS = ALL > WAVES * 4096 * WI ? ALL : WAVES * 4096 * WI;
    static const int LI = TI / 16 / WAVES, LO = TO / 16 < WAVES ? 1 : TO / 16 / WAVES, LL = LI + LO;  // loads of a wave to a step
};

template <int WI, int WO, int NI, int NO, int AHEAD, class Y>
__global__ __launch_bounds__(64 * NI * NO, 1) void k_product4(pr_plan p, p4_operands q, pr_out<Y> out) {
    typedef P4Tile<WI, WO, NI, NO, AHEAD> L;
    extern __shared__ uint8_t sm[];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    unsigned ti, to;
    int piece;
    pr_tile(p, blockIdx.x, ti, to, piece);
    const int s0 = piece * p.per;
    const int steps = p.steps - s0 < p.per ? p.steps - s0 : p.per;
    const long long i0 = (long long)ti * L::TI, o0 = (long long)to * L::TO;
    const long long pitch = (long long)p.steps * PP_GROUP_CODES4, spitch = (long long)p.steps * 4;
    const long long ri = p.inner - i0 < L::TI ? p.inner - i0 : L::TI, ro = p.outer - o0 < L::TO ? p.outer - o0 : L::TO;
    const pp_i4 bi = pr_buffer(q.inner_codes + i0 * pitch, ri * pitch), bo = pr_buffer(q.outer_codes + o0 * pitch, ro * pitch);
    const pp_i4 ci = pr_buffer(q.inner_scales + i0 * spitch, ri * spitch), co = pr_buffer(q.outer_scales + o0 * spitch, ro * spitch);
    const unsigned base = pr_lds_of(sm), scales = base + L::SCALES;

    // where this lane's pieces come from: 16 rows of four pieces to a load, a wave's loads 1024 bytes of LDS apart
    unsigned vi[L::LI], vo[L::LO];
#pragma unroll
    for (int j = 0; j < L::LI; ++j) {
        const int row = 16 * (wave * L::LI + j) + (lane >> 2);
        vi[j] = (unsigned)(row * pitch) + 16 * ((lane & 3) ^ p4_turn(row));
    }
    const int ochunk = wave * L::LO % (L::TO / 16);
#pragma unroll
    for (int j = 0; j < L::LO; ++j) {
        const int row = 16 * (ochunk + j) + (lane >> 2);
        vo[j] = (unsigned)(row * pitch) + 16 * ((lane & 3) ^ p4_turn(row));
    }
    const unsigned to_i = base + wave * L::LI * 1024, to_o = base + L::SI + ochunk * 1024;
    const int wi64 = wave % (L::TI / 64), wo64 = wave % (L::TO < 64 ? 1 : L::TO / 64);
    const unsigned vci = (unsigned)((64 * wi64 + lane) * spitch);
    const unsigned vco = L::TO < 64 && lane >= L::TO ? PR_BEYOND : (unsigned)((64 * wo64 + lane) * spitch);

    // The loads of a step of this piece into stage `buf`, in their order: at every fourth step the scales
    // of four, then load k of the codes.  Behind the last step they find nothing (buffers of no bytes), so
    // that there are always as many.  They go out one by one between the products: a wave whose loads
    // come all at once waits for room in their queue.
    auto load_scales = [&](int s) {
        if (!(s & 3) && s < steps) {
            const unsigned c = scales + ((s >> 2) & 1) * (L::CI + L::CO);
            pr_to_lds(ci, vci, (unsigned)(s0 + s) * 4, c + wi64 * 1024);
            pr_to_lds(co, vco, (unsigned)(s0 + s) * 4, c + L::CI + wo64 * 1024);
        }
    };
    auto aim = [&](int k, unsigned at) {
        if (k < L::LI) pr_aim(to_i + at, k * 1024);
        else pr_aim(to_o + at, (k - L::LI) * 1024);
    };
    pp_i4 ni = bi, no = bo;
    auto open = [&](int s) {
        ni[2] = s < steps ? bi[2] : 0;
        no[2] = s < steps ? bo[2] : 0;
    };
    auto fire = [&](int k, int s) {
        if (k < L::LI) pr_fire(ni, vi[k], (unsigned)(s0 + s) * PR_STEP);
        else pr_fire(no, vo[k - L::LI], (unsigned)(s0 + s) * PR_STEP);
    };

    const int wi = wave % NI, wo = wave / NI, r = lane & 31, g = lane >> 5;
    const int ir = wi * WI * 32 + pr_inner_row(r), rr = wo * WO * 32 + r, shift = 8 * g;
    const int fi0 = ir * PR_STEP + 16 * (g ^ p4_turn(ir)), fi1 = ir * PR_STEP + 16 * ((2 + g) ^ p4_turn(ir));
    const int fo0 = L::SI + rr * PR_STEP + 16 * (g ^ p4_turn(rr)), fo1 = L::SI + rr * PR_STEP + 16 * ((2 + g) ^ p4_turn(rr));
    const int si = ir * 16, so = L::CI + rr * 16;  // + 4 bytes to a step

    // Fragments: the inner ones of a half step are replaced as they have been used, the outer ones of
    // the two halves have a place each.  Scales are those of a whole step.
    pp_i4 in[WI], first[WO], late[WO];
    int in_raw[WI], out_raw[WO], in_c[WI], out_c[WO];
    auto codes_at = [&](int buf) { return sm + buf * (L::SI + L::SO); };
    auto scales_at = [&](int s) { return sm + L::SCALES + ((s >> 2) & 1) * (L::CI + L::CO) + (s & 3) * 4; };
    auto read = [&](const uint8_t *b, int at, int j) { return *(const pp_i4 *)(b + at + j * 32 * PR_STEP); };
    auto read_scales = [&](const uint8_t *c) {
#pragma unroll
        for (int j = 0; j < WI; ++j) in_raw[j] = *(const int *)(c + si + j * 512);
#pragma unroll
        for (int j = 0; j < WO; ++j) out_raw[j] = *(const int *)(c + so + j * 512);
    };
    pr_f16 acc[WI][WO];

#pragma unroll
    for (int t = 0; t < AHEAD; ++t) {
        load_scales(t);
        open(t);
#pragma unroll
        for (int k = 0; k < L::LL; ++k) {
            aim(k, t * (L::SI + L::SO));
            asm volatile("s_nop 0");
            fire(k, t);
        }
    }
    PR_WAIT(0);
    pr_barrier();
#pragma unroll
    for (int j = 0; j < WI; ++j) in[j] = read(codes_at(0), fi0, j);
#pragma unroll
    for (int j = 0; j < WO; ++j) first[j] = read(codes_at(0), fo0, j);
    read_scales(scales_at(0));
    pr_clear(acc);
    __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0): the compiler need not wait for these within the loop
    constexpr int N = WI * WO, MEET = WO;  // products of a half step; those of the second one before the waves meet
    constexpr int SLOTS = 2 * N - MEET;    // products from one meeting to the next: step s + AHEAD's loads go out behind them, into step s's stage
    int b0 = 0, b1 = 1;                    // the stages of steps s and s + 1
    int sent = AHEAD - 1;                  // the last step whose loads went out or are going out
    unsigned sent_at = sent * (L::SI + L::SO);
    for (int s = 0; s < steps; ++s) {
        const uint8_t *now = codes_at(b0), *next = codes_at(b1);  // after the last step: what lies there, for nothing
        // what follows product m, counted from the meeting of the step before
        auto behind = [&](int m) {
#pragma unroll
            for (int k = m * L::LL / SLOTS; k < (m + 1) * L::LL / SLOTS; ++k) {
                if (k > m * L::LL / SLOTS) asm volatile("s_nop 0");
                fire(k, sent);
                if (k + 1 < L::LL) aim(k + 1, sent_at);
            }
        };
        in_c[0] = p4_own(in_raw[0], shift);
        out_c[0] = p4_own(out_raw[0], shift);
        asm volatile("s_nop 3");
#pragma unroll
        for (int m = 0; m < N; ++m) {
            const int i = m / WO, j = m % WO;
            p4_multiply<0>(acc[i][j], in[i], in_c[i], first[j], out_c[j]);
            if (i == 0 && j + 1 < WO) out_c[j + 1] = p4_own(out_raw[j + 1], shift);
            if (j == WO - 1 && i + 1 < WI) in_c[i + 1] = p4_own(in_raw[i + 1], shift);
            if (i == 0) late[j] = read(now, fo1, j);
            if (j == WO - 1) in[i] = read(now, fi1, i);
            if (s > 0) behind(N - MEET + m);
            if (i == 0 || j == WO - 1) asm volatile("s_nop 2");
            PR_PIN;
        }
#pragma unroll
        for (int m = 0; m < N; ++m) {
            const int i = m / WO, j = m % WO;
            if (m == MEET) {  // step s + 1 has arrived for every wave, and every wave has read all of step s
                PR_WAIT((AHEAD - 2) * L::LL);
                pr_barrier();
                sent = s + AHEAD;
                sent_at = b0 * (L::SI + L::SO);
                open(sent);
                load_scales(sent);
                aim(0, sent_at);
            }
            p4_multiply<1>(acc[i][j], in[i], in_c[i], late[j], out_c[j]);
            if (m >= MEET) {
                if (m - MEET < WO) first[m - MEET] = read(next, fo0, m - MEET);
                if (m == MEET) in[0] = read(next, fi0, 0);
                if (m == (MEET + N) / 2) read_scales(scales_at(s + 1));
                if (j == WO - 1) in[i] = read(next, fi0, i);
                behind(m - MEET);
            }
            PR_PIN;
        }
        b0 = b1;
        b1 = b1 == AHEAD - 1 ? 0 : b1 + 1;
        pr_settle(s + 1, steps);
    }
    PR_WAIT(0);  // nothing is on its way to LDS any more
    pr_barrier();
    pr_leave<Y, WI, WO>(p, out, acc, sm + wave * (32 * 32 * WI * 4), lane, i0 + wi * WI * 32, o0 + wo * WO * 32, piece);
}

// k_rows4: few rows of x (16 NB at most), bound by the weight's bytes: a row, 4096 -> 16384 (36 MB), takes 9 to 10 us,
// 3.6 to 4 TB/s, of which 2 are the launch; 32 rows, 4096 -> 4096 8.0 us.  The weight is read once, straight into registers, by waves
// that divide the sum among them: a wave takes 16 rows of W and up to eight groups at a time, and what
// the waves of a workgroup have found is added in LDS.  With FUSED the workgroup also packs x itself
// (rows of it are little beside 16 rows of W) and, for pp_linear_backward_weight, a part of x in 8 bits.
#define R4_MAX_WAVES(NB) ((NB) == 1 ? 16 : 8)  // 128 registers to a thread, or 256
struct r4_x {  // FUSED: the matrix; else its codes and scales
    const void *x;
    long long ld, cols;
    uint8_t *kept_codes, *kept_scales;  // or NULL
    const uint8_t *codes, *scales;
};

template <int NB, bool FUSED, class Y>
__global__ __launch_bounds__(64 * R4_MAX_WAVES(NB)) void k_rows4(int rows, long long inner, int groups, const uint8_t *__restrict__ w_codes,
                                                             const uint8_t *__restrict__ w_scales, r4_x x, pr_out<Y> out) {
    typedef typename Y::T T;
    extern __shared__ uint8_t sm[];  // sums of the waves [NB][waves][64] of 16 bytes; FUSED: x's codes, then its scales
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, waves = blockDim.x >> 6;
    const int r = lane & 15, g = lane >> 4;
    const long long n0 = (long long)blockIdx.x * 16;
    const int per = (groups + waves - 1) / waves, k0 = wave * per, k1 = k0 + per < groups ? k0 + per : groups;
    uint8_t *xc = sm + NB * waves * 1024, *xs = xc + rows * groups * PP_GROUP_CODES4;
    const long long n = n0 + r < inner ? n0 + r : inner - 1;
    const uint8_t *wc = w_codes + n * groups * PP_GROUP_CODES4 + 16 * g, *ws = w_scales + n * groups * 4;

    // Up to eight groups of a row from p (16 bytes of each) and their scales from q on, none beyond k1.
    auto load = [&](int k, const uint8_t *p, const uint8_t *q, pp_u4 *c, pp_u4 *s4) {
#pragma unroll
        for (int t = 0; t < 8; ++t)
            if (k + t < k1) c[t] = *(const pp_u4 *)(p + (long long)(k + t) * PP_GROUP_CODES4);
#pragma unroll
        for (int h = 0; h < 2; ++h) {  // four groups' scales; one by one where fewer are left
            if (k + 4 * h + 4 <= k1) s4[h] = ((const pp_any16<4> *)(q + 4ll * (k + 4 * h)))->v;
            else
#pragma unroll
                for (int t = 0; t < 4; ++t)
                    if (k + 4 * h + t < k1) s4[h][t] = *(const unsigned *)(q + 4ll * (k + 4 * h + t));
        }
    };
    pp_u4 w[8], w4[2];
    if constexpr (FUSED) {
        const int row_chunks = groups * 16, chunks = rows * row_chunks, threads = blockDim.x;
        const T *src = (const T *)x.x;
        auto fetch = [&](int q) {
            const int row = q / row_chunks, c = q - row * row_chunks;
            return pp_load8<Y>(src + row * x.ld + 8 * c, q < chunks ? x.cols - 8ll * c : 0);
        };
        PpRaw<Y> raw = fetch(tid);  // before the weight's: what is waited for first is asked for first
        load(k0, wc, ws, w, w4);
        for (int q = tid; q < chunks; q += threads) {
            const PpRaw<Y> now = raw;
            if (q + threads < chunks) raw = fetch(q + threads);
            float v[8];
            pp_values<Y>(now, v);
            const unsigned m = pp_quad_max(pp_absmax<Y>(now, v));
            unsigned c;
            const unsigned byte = pp_codes4(v, m, c);
            *(unsigned *)(xc + q * 4) = c;
            if (!(q & 3)) xs[q >> 2] = (uint8_t)byte;
            if (x.kept_codes && (unsigned)(q / threads) % gridDim.x == blockIdx.x) {
                pp_u2 c8;
                const unsigned byte8 = pp_codes8(v, m, c8);
                *(pp_u2 *)(x.kept_codes + q * 8ll) = c8;
                if (!(q & 3)) x.kept_scales[q >> 2] = (uint8_t)byte8;
            }
        }
        __syncthreads();
    } else {
        load(k0, wc, ws, w, w4);
    }
    pp_f4 acc[NB] = {};
    for (int k = k0; k < k1; k += 8) {
        if (k > k0) load(k, wc, ws, w, w4);
        // x's, from memory all at once; from LDS as they are needed.  Lanes beyond the last row take it again, for
        // results that are not written.
        pp_u4 c[NB][8], c4[NB][2];
        long long m[NB];
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            m[b] = (long long)(16 * b + r < rows ? 16 * b + r : rows - 1) * groups;
            if constexpr (!FUSED) load(k, x.codes + m[b] * PP_GROUP_CODES4 + 16 * g, x.scales + m[b] * 4, c[b], c4[b]);
        }
#pragma unroll
        for (int t = 0; t < 8; ++t) {
            if (k + t >= k1) break;
            const pr_i8 a = {(int)w[t][0], (int)w[t][1], (int)w[t][2], (int)w[t][3]};
            const int ca = w4[t >> 2][t & 3] >> (8 * g);
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                int cb;
                if constexpr (FUSED) {
                    c[b][t] = *(const pp_u4 *)(xc + (m[b] + k + t) * PP_GROUP_CODES4 + 16 * g);
                    cb = xs[(m[b] + k + t) * 4 + g];
                } else {
                    cb = c4[b][t >> 2][t & 3] >> (8 * g);
                }
                const pr_i8 d = {(int)c[b][t][0], (int)c[b][t][1], (int)c[b][t][2], (int)c[b][t][3]};
                acc[b] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, d, acc[b], 4, 4, 0, ca, 0, cb);
            }
        }
    }
#pragma unroll
    for (int b = 0; b < NB; ++b) ((pp_f4 *)sm)[(b * waves + wave) * 64 + lane] = acc[b];
    __syncthreads();
    if (wave < NB) {
        pp_f4 v = {0, 0, 0, 0};
        for (int t = 0; t < waves; ++t) v += ((const pp_f4 *)sm)[(wave * waves + t) * 64 + lane];
        const int m = 16 * wave + r;
        if (m < rows)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const long long i = n0 + 4 * g + j;
                if (i < inner) out.p[m * out.ld + i] = Y::put(out.bias ? v[j] + out.bias[i] : v[j]);
            }
    }
}

// Waves to a workgroup: four where the rows of W alone fill the chip, more (down to two groups each)
// where they do not.
static int r4_waves(int nb, long long inner, long long groups) {
    int n = 4;
    while (n < R4_MAX_WAVES(nb) && (inner + 15) / 16 * n < 4096 && 2 * n * 2 <= groups) n *= 2;
    return n;
}
static size_t r4_lds(int nb, int waves, int64_t rows, long long groups, bool fused) {
    return (size_t)nb * waves * 1024 + (fused ? rows * groups * (PP_GROUP_CODES4 + 4) : 0);
}

// Whether few rows go this way.  Up to 16 they do; up to 32 where the weight is small: 4096 -> 4096 takes 8 us (12 in
// tiles of 256 x 32), 4096 -> 16384 19 us (17).  (16 rows: 15 us, and 15.)
bool r4_takes(int64_t rows, int64_t n_in, int64_t n_out) { return rows <= 16 || (rows <= 32 && n_in * n_out <= 1 << 25); }

// Whether a workgroup packs x itself, which saves a launch and costs every workgroup the same work: up to 64 groups
// of 128 values.  4096 -> 16384: a row 9.1 us (10.7 in two launches), four rows 13.4 us (11.7).
bool r4_fuses(int64_t rows, int64_t n_in) { return rows <= 16 && rows * pp_groups(n_in) <= 64; }

int r4_launch(int type, int64_t rows, int64_t n_in, int64_t n_out, const void *x, int64_t ld_x, uint8_t *kept_codes, uint8_t *kept_scales,
              const p4_operands &q, void *y, int64_t ld_y, const float *bias, hipStream_t st) {
    const long long groups = pp_groups(n_in);
    const int nb = rows > 16 ? 2 : 1, waves = r4_waves(nb, n_out, groups);
    const bool fused = r4_fuses(rows, n_in);
    const r4_x a = {x, ld_x, n_in, kept_codes, kept_scales, q.outer_codes, q.outer_scales};
    const size_t lds = r4_lds(nb, waves, rows, groups, fused);
    const unsigned grid = (unsigned)((n_out + 15) / 16);
    return pp_by_type(type, [&](auto t) {
        typedef decltype(t) Y;
        const pr_out<Y> o = {(typename Y::T *)y, ld_y, bias, NULL, 0};
        if (fused) k_rows4<1, true, Y><<<grid, 64 * waves, lds, st>>>((int)rows, n_out, (int)groups, q.inner_codes, q.inner_scales, a, o);
        else if (nb == 1) k_rows4<1, false, Y><<<grid, 64 * waves, lds, st>>>((int)rows, n_out, (int)groups, q.inner_codes, q.inner_scales, a, o);
        else k_rows4<2, false, Y><<<grid, 64 * waves, lds, st>>>((int)rows, n_out, (int)groups, q.inner_codes, q.inner_scales, a, o);
        return hipGetLastError() == hipSuccess ? PP_OK : PP_ERR_HIP;
    });
}

template <int WI, int WO, int NI, int NO, int AHEAD> static int launch4(int type, pr_plan p, const p4_operands &q, void *y, long long ld, const float *bias, hipStream_t st) {
    typedef P4Tile<WI, WO, NI, NO, AHEAD> L;
    return pp_by_type(type, [&](auto t) {
        typedef decltype(t) Y;
        auto *k = k_product4<WI, WO, NI, NO, AHEAD, Y>;
        k<<<p.ni * p.no * p.splits, 64 * L::WAVES, L::LDS, st>>>(p, q, pr_out<Y>{(typename Y::T *)y, ld, bias, NULL, 0});
        return hipGetLastError() == hipSuccess ? PP_OK : PP_ERR_HIP;
    });
}

int p4_launch(int shape, int type, const pr_plan &p, const p4_operands &q, void *y, long long ld, const float *bias, hipStream_t st) {
    if (shape == 0) return launch4<4, 4, 2, 2, 3>(type, p, q, y, ld, bias, st);
    if (shape == 1) return launch4<2, 2, 2, 2, 4>(type, p, q, y, ld, bias, st);
    return launch4<2, 1, 4, 1, 3>(type, p, q, y, ld, bias, st);
}
