// pp_linear_forward, pp_linear_backward_input, pp_linear_backward_weight: what is checked, how the
// work is divided, and the passes around the products of pp_product_fp4.hip and pp_product_grad.hip.
#include "pp_product_fp4.h"
#include "pp_product_grad.h"

// x in 4 bits, and in 8 where codes8 is given, in one pass (pp_pack.hip)
int pp_launch_pack_both(int type, int64_t rows, int64_t cols, const void *src, int64_t ld, void *codes4, void *scales4, void *codes8, void *scales8,
                        hipStream_t st);

// ---- gradients as bf16 planes

// dy in a form the product can load as it is: rows at multiples of 16 bytes, in bf16.  A type with
// more bits becomes two (f16) or three (float) planes that add up to it (but for what a float has below 2^-133,
// bf16's smallest value), each the leading
// eight bits of what the ones before leave; products with all of them are summed.  Bound by its bytes and the
// launch: 333 x 5000 fp16 (10 MB) 4.5 us.  (fp16 products would need the packed values in fp16, which does not
// hold all of their scales.)
template <class Y, int PLANES>
__global__ __launch_bounds__(256) void k_planes(long long row0, long long rows, long long cols, const typename Y::T *__restrict__ src, long long ld,
                                                uint16_t *__restrict__ dst, long long ld_dst) {
    const unsigned chunks = (unsigned)(ld_dst / 8), t = blockIdx.x * 256 + threadIdx.x, r_ = t / chunks;
    const long long r = row0 + r_, c = (t - r_ * chunks) * 8ll;
    if (r >= rows) return;
    const PpRaw<Y> raw = pp_load8<Y>(src + r * ld + c, cols - c);
    float v[8];
    pp_values<Y>(raw, v);
#pragma unroll
    for (int k = 0; k < PLANES; ++k) {
        unsigned h[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const unsigned b = pp_bits(v[j]);
            const bool finite = (b & 0x7f800000u) != 0x7f800000u;
            h[j] = (b >> 16) | ((b & 0x7fffffffu) > 0x7f800000u ? 0x40u : 0u);  // a NaN stays one
            v[j] = finite ? v[j] - pp_bits(b & 0xffff0000u) : 0.0f;
        }
        *(pp_u4 *)(dst + (k * rows + r) * ld_dst + c) = pp_u4{h[0] | h[1] << 16, h[2] | h[3] << 16, h[4] | h[5] << 16, h[6] | h[7] << 16};
    }
}

static int launch_planes(int type, int64_t rows, int64_t cols, const void *src, int64_t ld, void *dst, int64_t ld_dst, hipStream_t st) {
    const int64_t chunks = ld_dst / 8, most = ((int64_t)1 << 31) / chunks;  // rows of a launch
    for (int64_t r = 0; r < rows; r += most) {
        const int64_t n = rows - r < most ? rows - r : most;
        const unsigned grid = (unsigned)((n * chunks + 255) / 256);
        if (type == PP_TYPE_BF16) k_planes<PpBF16, 1><<<grid, 256, 0, st>>>(r, rows, cols, (const __bf16 *)src, ld, (uint16_t *)dst, ld_dst);
        else if (type == PP_TYPE_F16) k_planes<PpF16, 2><<<grid, 256, 0, st>>>(r, rows, cols, (const _Float16 *)src, ld, (uint16_t *)dst, ld_dst);
        else k_planes<PpF32, 3><<<grid, 256, 0, st>>>(r, rows, cols, (const float *)src, ld, (uint16_t *)dst, ld_dst);
        if (hipGetLastError() != hipSuccess) return PP_ERR_HIP;
    }
    return PP_OK;
}

// ---- pieces of a sum, added in their order

// Bound by the partial sums' bytes: 333 x 4100 in five pieces 6 us (27 MB, 4.5 TB/s).
// The first `sum_blocks` workgroups add the columns' sums.
template <class Y>
__global__ __launch_bounds__(256) void k_join(pr_plan p, pr_out<Y> out, const float *__restrict__ part_sums, float *__restrict__ sums, unsigned sum_blocks) {
    if (blockIdx.x < sum_blocks) {  // 32 sums, their parts by eight threads each
        __shared__ float found[8][32];
        const int lane = threadIdx.x & 31, eighth = threadIdx.x >> 5, parts = p.splits * (int)p.ni;
        const long long o = blockIdx.x * 32ll + lane;
        float v = 0;
        if (o < p.outer)
#pragma unroll 4
            for (int s = eighth; s < parts; s += 8) v += part_sums[s * p.outer + o];
        found[eighth][lane] = v;
        __syncthreads();
        if (eighth == 0 && o < p.outer) {
            for (int k = 1; k < 8; ++k) v += found[k][lane];
            sums[o] = v;
        }
        return;
    }
    // (Results of a divided sum are few: 512 tiles at most.)
    const unsigned chunks = (unsigned)(p.partial_ld / 8), n = (unsigned)p.outer * chunks;
    for (unsigned t = (blockIdx.x - sum_blocks) * 256 + threadIdx.x; t < n; t += (gridDim.x - sum_blocks) * 256) {
        const unsigned row = t / chunks;
        const long long o = row, i = (t - row * chunks) * 8ll;
        const float *q = p.partial + o * p.partial_ld + i;
        pp_f4 a = {0, 0, 0, 0}, b = a;
        int s = 0;
        for (; s + 4 <= p.splits; s += 4) {  // four pieces' loads in flight, added in their order
            pp_f4 u[4], w[4];
#pragma unroll
            for (int k = 0; k < 4; ++k, q += p.outer * p.partial_ld) {
                u[k] = *(const pp_f4 *)q;
                w[k] = *(const pp_f4 *)(q + 4);
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                a += u[k];
                b += w[k];
            }
        }
        for (; s < p.splits; ++s, q += p.outer * p.partial_ld) {
            a += *(const pp_f4 *)q;
            b += *(const pp_f4 *)(q + 4);
        }
        float v[8];
        *(pp_f4 *)v = a;
        *(pp_f4 *)(v + 4) = b;
        if (out.bias || out.add) {
            const PpRaw<PpF32> r = pp_load8<PpF32>(out.bias ? out.bias + i : out.add + o * out.add_ld + i, p.inner - i);
            float w[8];
            pp_values<PpF32>(r, w);
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] += w[j];
        }
        pp_store8<Y>(out.p + o * out.ld + i, p.inner - i, v);
    }
}

static int launch_join(int type, const pr_plan &p, void *out, long long ld, const float *bias, const float *add, const float *part_sums, float *sums,
                       hipStream_t st) {
    const long long blocks = (p.outer * (p.partial_ld / 8) + 255) / 256;
    const unsigned sum_blocks = sums ? (unsigned)((p.outer + 31) / 32) : 0;
    return pp_by_type(type, [&](auto t) {
        typedef decltype(t) Y;
        k_join<Y><<<sum_blocks + (unsigned)(blocks < 4096 ? blocks : 4096), 256, 0, st>>>(p, pr_out<Y>{(typename Y::T *)out, ld, bias, add, ld}, part_sums, sums, sum_blocks);
        return hipGetLastError() == hipSuccess ? PP_OK : PP_ERR_HIP;
    });
}

// ---- launches and workspaces

// Runs launch(part, first outer index) over the outer index in launches of at most 2^20 tiles.
template <class F> static int in_turns(const pr_plan &p, int to, F launch) {
    const long long most = ((1ll << 20) / p.ni < 1 ? 1 : (1ll << 20) / p.ni) * to;
    for (long long o = 0; o < p.outer; o += most) {
        pr_plan q = p;
        q.outer = p.outer - o < most ? p.outer - o : most;
        q.no = (unsigned)((q.outer + to - 1) / to);
        if (int rc = launch(q, o)) return rc;
    }
    return PP_OK;
}

// ---- entry points

static bool bad_layer(int type, int64_t rows, int64_t n_in, int64_t n_out) {
    return pp_bad_sizes(type, rows, n_in) || n_out < 1 || n_out > PP_LAYER_MAX_COLS;
}

static int64_t planes_ld(int64_t n_out) { return (n_out + 7) & ~(int64_t)7; }
static size_t planes_bytes(int type, int64_t rows, int64_t n_out) { return pp_align256((size_t)planes_of(type) * rows * planes_ld(n_out) * 2); }

// What a call keeps in its workspace: first x packed in 4 bits, or dy's planes, whose bytes grow with the rows; behind
// them, where the sum is divided, the partial sums and the columns'.
static size_t codes_bytes(int64_t rows, int64_t n_in) { return pp_align256((size_t)rows * pp_groups(n_in) * PP_GROUP_CODES4); }
static size_t packed_bytes(int64_t rows, int64_t n_in) { return codes_bytes(rows, n_in) + pp_align256((size_t)rows * pp_groups(n_in) * 4); }
static size_t total_bytes(size_t first, const pr_plan &p, bool sums) {
    return 256 + first + partial_bytes(p.splits, p.inner, p.outer) + (sums ? sums_bytes(p.splits, p.ni, p.outer) : 0);
}

extern "C" size_t pp_linear_workspace_bytes(int call, int type, int64_t rows, int64_t n_in, int64_t n_out) {
    if (call < PP_LINEAR_FORWARD || call > PP_LINEAR_BACKWARD_WEIGHT || bad_layer(type, rows, n_in, n_out)) return 0;
    int shape;
    if (call == PP_LINEAR_FORWARD) {
        if (r4_takes(rows, n_in, n_out)) return 256 + packed_bytes(rows, n_in);
        return total_bytes(packed_bytes(rows, n_in), plan_forward(rows, n_in, n_out, PR_ANY_ROOM, &shape), false);
    }
    // what the types of as many bits or fewer need: the work may be divided otherwise for them
    size_t most = 0;
    for (int t = type; t <= PP_TYPE_BF16; ++t) {
        const bool weight = call == PP_LINEAR_BACKWARD_WEIGHT;
        const pr_plan p = weight ? plan_weight(t, rows, n_in, n_out, PR_ANY_ROOM, &shape) : plan_input(t, rows, n_in, n_out, PR_ANY_ROOM, &shape);
        const size_t n = total_bytes(planes_bytes(t, rows, n_out), p, weight);
        most = n > most ? n : most;
    }
    return most;
}

static bool bad_workspace(const void *ws, size_t bytes, size_t first) { return !ws || ((uintptr_t)ws & 255) || bytes < 256 + first; }

extern "C" int pp_linear_forward(int type, int64_t rows, int64_t n_in, int64_t n_out, const void *x, int64_t ld_x, const void *w_codes,
                                 const void *w_scales, const float *bias, void *y, int64_t ld_y, void *x_codes, void *x_scales,
                                 void *workspace, size_t workspace_bytes, void *stream) {
    if (bad_layer(type, rows, n_in, n_out)) return PP_ERR_INVALID_ARG;
    if (pp_bad_matrix(x, type, rows, n_in, ld_x) || pp_bad_matrix(y, type, rows, n_out, ld_y)) return PP_ERR_INVALID_ARG;
    if (pp_bad_packed(w_codes, w_scales, n_out) || ((uintptr_t)bias & 3)) return PP_ERR_INVALID_ARG;
    if ((x_codes || x_scales) && pp_bad_packed(x_codes, x_scales, rows)) return PP_ERR_INVALID_ARG;
    hipStream_t st = (hipStream_t)stream;
    const bool few = r4_takes(rows, n_in, n_out);
    const size_t packed = packed_bytes(rows, n_in);
    if (bad_workspace(workspace, workspace_bytes, packed)) return PP_ERR_WORKSPACE;
    if (!rows) return PP_OK;
    if (rows == 1) ld_x = n_in;
    int shape;
    pr_plan p = {};
    if (!few) p = plan_forward(rows, n_in, n_out, workspace_bytes - 256 - packed, &shape);
    const long long g = pp_groups(n_in);
    uint8_t *codes = (uint8_t *)workspace, *scales = codes + codes_bytes(rows, n_in);
    const p4_operands all = {(const uint8_t *)w_codes, (const uint8_t *)w_scales, codes, scales};
    if (few && r4_fuses(rows, n_in))
        return r4_launch(type, rows, n_in, n_out, x, ld_x, (uint8_t *)x_codes, (uint8_t *)x_scales, all, y, ld_y, bias, st);
    if (int rc = pp_launch_pack_both(type, rows, n_in, x, ld_x, codes, scales, x_codes, x_scales, st)) return rc;
    if (few) return r4_launch(type, rows, n_in, n_out, x, ld_x, NULL, NULL, all, y, ld_y, bias, st);
    p.partial = (float *)((uint8_t *)workspace + packed);
    const int rc = in_turns(p, FORWARD[shape].to, [&](const pr_plan &q, long long o) {
        return p4_launch(shape, type, q, p4_operands{all.inner_codes, all.inner_scales, codes + o * g * PP_GROUP_CODES4, scales + o * g * 4},
                         (uint8_t *)y + o * ld_y * pp_type_size(type), ld_y, bias, st);
    });
    if (rc || p.splits == 1) return rc;
    return launch_join(type, p, y, ld_y, bias, NULL, NULL, NULL, st);
}

// dy as the products take it: as it is where it can be loaded so, else copied into `room`.  (As it is: bf16,
// rows at multiples of 16 bytes, and so near each other that 256 of them are within the reach of 32-bit offsets; along the sum
// whole 16 bytes of it, across it whole words: the last word of an odd row would reach two bytes behind the matrix; the copy takes
// 15 of 271 us at 8192 rows, 4096 -> 4095, and 19 of 87 at 32771 rows, 520 -> 1001.)
static int outer_of(int type, bool along_sum, int64_t rows, int64_t cols, const void *dy, int64_t ld, void *room, pg_outer *out, hipStream_t st) {
    if (rows < 2) ld = cols;
    if (type == PP_TYPE_BF16 && !((uintptr_t)dy & 15) && (rows < 2 || (!(ld & 7) && ld <= PP_LAYER_MAX_COLS)) && !(cols & (along_sum ? 7 : 1))) {
        *out = pg_outer{(const uint8_t *)dy, rows, cols, ld, 0, 1};
        return PP_OK;
    }
    const int64_t n = planes_ld(cols);
    *out = pg_outer{(const uint8_t *)room, rows, n, n, rows * n, planes_of(type)};
    return rows ? launch_planes(type, rows, cols, dy, ld, room, n, st) : PP_OK;
}

extern "C" int pp_linear_backward_input(int type, int64_t rows, int64_t n_in, int64_t n_out, const void *dy, int64_t ld_dy,
                                        const void *w_codes, const void *w_scales, void *dx, int64_t ld_dx, void *workspace,
                                        size_t workspace_bytes, void *stream) {
    if (bad_layer(type, rows, n_in, n_out)) return PP_ERR_INVALID_ARG;
    if (pp_bad_matrix(dy, type, rows, n_out, ld_dy) || pp_bad_matrix(dx, type, rows, n_in, ld_dx)) return PP_ERR_INVALID_ARG;
    if (pp_bad_packed(w_codes, w_scales, n_out)) return PP_ERR_INVALID_ARG;
    const size_t planes = planes_bytes(type, rows, n_out);
    if (bad_workspace(workspace, workspace_bytes, planes)) return PP_ERR_WORKSPACE;
    if (!rows) return PP_OK;
    int shape;
    pr_plan p = plan_input(type, rows, n_in, n_out, workspace_bytes - 256 - planes, &shape);
    hipStream_t st = (hipStream_t)stream;
    pg_outer y;
    if (int rc = outer_of(type, true, rows, n_out, dy, ld_dy, workspace, &y, st)) return rc;
    p.partial = (float *)((uint8_t *)workspace + planes);
    const pg_inner w = {(const uint8_t *)w_codes, (const uint8_t *)w_scales, n_out, pp_groups(n_in)};
    const int rc = in_turns(p, INPUT[shape].to, [&](const pr_plan &q, long long o) {
        pg_outer part = y;
        part.p += o * y.ld * 2;
        part.rows = q.outer;
        return pg_launch_input(shape, type, q, w, part, (uint8_t *)dx + o * ld_dx * pp_type_size(type), ld_dx, st);
    });
    if (rc || p.splits == 1) return rc;
    return launch_join(type, p, dx, ld_dx, NULL, NULL, NULL, NULL, st);
}

extern "C" int pp_linear_backward_weight(int type, int64_t rows, int64_t n_in, int64_t n_out, const void *dy, int64_t ld_dy,
                                         const void *x_codes, const void *x_scales, const float *dw_in, float *dw, int64_t ld_dw,
                                         float *db, void *workspace, size_t workspace_bytes, void *stream) {
    if (bad_layer(type, rows, n_in, n_out)) return PP_ERR_INVALID_ARG;
    if (pp_bad_matrix(dy, type, rows, n_out, ld_dy) || pp_bad_packed(x_codes, x_scales, rows)) return PP_ERR_INVALID_ARG;
    if (pp_bad_matrix(dw, PP_TYPE_F32, n_out, n_in, ld_dw) || ((uintptr_t)dw_in & 3) || ((uintptr_t)db & 3)) return PP_ERR_INVALID_ARG;
    if (dw_in && n_out > 1 && ld_dw > PP_LAYER_MAX_LD_DW) return PP_ERR_INVALID_ARG;
    if (n_out == 1) ld_dw = n_in;
    const size_t planes = planes_bytes(type, rows, n_out);
    if (bad_workspace(workspace, workspace_bytes, planes)) return PP_ERR_WORKSPACE;
    int shape;
    pr_plan p = plan_weight(type, rows, n_in, n_out, workspace_bytes - 256 - planes, &shape);
    hipStream_t st = (hipStream_t)stream;
    pg_outer y;
    if (int rc = outer_of(type, false, rows, n_out, dy, ld_dy, workspace, &y, st)) return rc;
    p.partial = (float *)((uint8_t *)workspace + planes);
    float *part_sums = (float *)((uint8_t *)p.partial + partial_bytes(p.splits, p.inner, p.outer));
    const pg_inner x = {(const uint8_t *)x_codes, (const uint8_t *)x_scales, rows, pp_groups(n_in)};
    const int rc = in_turns(p, WEIGHT[shape].to, [&](const pr_plan &q, long long o) {
        pg_outer part = y;
        part.p += o * 2;
        part.cols -= o;
        return pg_launch_weight(shape, q, x, part, dw + o * ld_dw, ld_dw, dw_in ? dw_in + o * ld_dw : NULL,
                                !db ? NULL : p.splits > 1 ? part_sums : db + o, st);
    });
    if (rc || p.splits == 1) return rc;
    return launch_join(PP_TYPE_F32, p, dw, ld_dw, NULL, dw_in, part_sums, db, st);
}
