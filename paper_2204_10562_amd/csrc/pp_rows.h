// What the operators that reduce rows share (norms, losses): sums and maxima of a wave and of a workgroup, in one
// order whatever the timing, and rows of chunks of eight columns.
#pragma once

#include "pp_layer_common.h"

#define PP_WAVE 64

template <int CTRL> __device__ __forceinline__ float pp_moved(float v) {
    return pp_bits((unsigned)__builtin_amdgcn_update_dpp(0, (int)pp_bits(v), CTRL, 0xf, 0xf, true));
}
template <int CTRL> __device__ __forceinline__ unsigned pp_moved(unsigned v) {
    return (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, true);
}
__device__ __forceinline__ float pp_lane(float v, int lane) { return pp_bits((unsigned)__builtin_amdgcn_readlane((int)pp_bits(v), lane)); }

// op over the 64 lanes, the same in all of them: within 16 lanes by moves (lanes 1 0 3 2, 2 3 0 1, the half row and the
// row mirrored), the four rows as scalars
template <class F> __device__ __forceinline__ float pp_wave_all(float v, F op) {
    v = op(v, pp_moved<0xB1>(v));
    v = op(v, pp_moved<0x4E>(v));
    v = op(v, pp_moved<0x141>(v));
    v = op(v, pp_moved<0x140>(v));
    return op(op(pp_lane(v, 0), pp_lane(v, 16)), op(pp_lane(v, 32), pp_lane(v, 48)));
}
__device__ __forceinline__ float pp_wave_sum(float v) {
    return pp_wave_all(v, [](float a, float b) { return a + b; });
}
__device__ __forceinline__ float pp_wave_max(float v) {
    return pp_wave_all(v, [](float a, float b) { return __builtin_fmaxf(a, b); });
}

template <int CTRL> __device__ __forceinline__ double pp_moved(double v) {
    const pp_u2 u = __builtin_bit_cast(pp_u2, v);
    return __builtin_bit_cast(double, pp_u2{pp_moved<CTRL>(u[0]), pp_moved<CTRL>(u[1])});
}
__device__ __forceinline__ double pp_lane(double v, int lane) {
    const pp_u2 u = __builtin_bit_cast(pp_u2, v);
    return __builtin_bit_cast(double, pp_u2{(unsigned)__builtin_amdgcn_readlane((int)u[0], lane), (unsigned)__builtin_amdgcn_readlane((int)u[1], lane)});
}
template <class F> __device__ __forceinline__ double pp_wave_all(double v, F op) {
    v = op(v, pp_moved<0xB1>(v));
    v = op(v, pp_moved<0x4E>(v));
    v = op(v, pp_moved<0x141>(v));
    v = op(v, pp_moved<0x140>(v));
    return op(op(pp_lane(v, 0), pp_lane(v, 16)), op(pp_lane(v, 32), pp_lane(v, 48)));
}
__device__ __forceinline__ double pp_wave_sum(double v) {
    return pp_wave_all(v, [](double a, double b) { return a + b; });
}
__device__ __forceinline__ double pp_wave_max(double v) {
    return pp_wave_all(v, [](double a, double b) { return __builtin_fmax(a, b); });
}

// The sum over a workgroup of WAVES waves.  `room` holds WAVES floats; whoever calls this again on the same room passes a
// barrier in between.
template <int WAVES> __device__ __forceinline__ float pp_group_sum(float v, float *room) {
    v = pp_wave_sum(v);
    if constexpr (WAVES > 1) {
        if (!(threadIdx.x & (PP_WAVE - 1))) room[threadIdx.x / PP_WAVE] = v;
        __syncthreads();
        v = room[0];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) v += room[w];
    }
    return v;
}

// max |v| of eight floats as the bits of a float: NaN above infinity above the numbers
__device__ __forceinline__ unsigned pp_absmax8(const float *v) {
    unsigned m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const unsigned b = pp_bits(v[i]) & 0x7fffffffu;
        m = b > m ? b : m;
    }
    return m;
}

// Eight values as 8-bit codes at chunk `at` of all; the four lanes of a quad have the four chunks of a block.
__device__ __forceinline__ void pp_put_codes8(long long at, const float *v, uint8_t *codes, uint8_t *scales) {
    pp_u2 c;
    const unsigned byte = pp_codes8(v, pp_quad_max(pp_absmax8(v)), c);
    *(pp_u2 *)(codes + at * 8) = c;
    if (!(at & 3)) scales[at >> 2] = (uint8_t)byte;
}

__device__ __forceinline__ void pp_get_codes8(long long at, const uint8_t *codes, const uint8_t *scales, float *v) {
    pp_values8(*(const pp_u2 *)(codes + at * 8), pp_unit8(scales[at >> 2]), v);
}
