// Activations kept in 8 bits between the forward and the backward pass.
//
// 32 columns of a row share the exponent k = the smallest integer, -126 at least, with amax <= M 2^k (M = 448 for e4m3, 127
// for int8); a code is x 2^-k, rounded to the nearest even one.  Scaling by a power of two is exact, so the code's is the
// only rounding: |x - x~| <= 2^-4 |x| from 2^(k-6) on and 2^(k-10) below (e4m3), 2^(k-1) (int8).  A scale that is no power
// of two would spare int8 up to one of its seven bits, but round twice and depend on how the quotient is formed.

#include <algorithm>

#include "columns.cuh"
#include "common.cuh"
#include "kernels.h"

namespace turnopd {
namespace {

constexpr int kWarps = 8;
constexpr int kChunk = 256;  // columns of a row that a warp takes at once, eight groups
constexpr int kUnits = 4;    // chunks of a row that it has in flight
constexpr int kStrip = kChunk * kUnits;

// The exponent byte of a group from the bits of its largest magnitude; 255 where that is infinite or NaN.
__device__ __forceinline__ uint32_t exponent_byte(uint32_t amax, bool e4m3)
{
    if (amax >= 0x7f800000u)
        return 255u;
    // amax = m 2^p with 1 <= m < 2; 448 = 1.75 2^8, 127 = 1.984375 2^6
    const int e = (int)(amax >> 23) - (e4m3 ? 8 : 6) + ((amax & 0x7fffffu) > (e4m3 ? 0x600000u : 0x7e0000u));
    return (uint32_t)max(e, 1);
}

// 2^-k for that byte (0 for a group that is not finite: its codes are zeros)
__device__ __forceinline__ float inverse_scale(uint32_t e)
{
    return e == 255u ? 0.f : __uint_as_float((254u - e) << 23);
}

__device__ __forceinline__ uint32_t encode2(float a, float b, bool e4m3)
{
    if (e4m3)
        return __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
    return ((uint32_t)__float2int_rn(a) & 0xffu) | ((uint32_t)__float2int_rn(b) & 0xffu) << 8;
}

__device__ __forceinline__ uint32_t magnitude(float x) { return __float_as_uint(x) & 0x7fffffffu; }

// A warp takes strips of four chunks of a row; a block's strips begin at one column (no division tells a row from its columns:
// with one for each chunk 32,768 x 4,096 bf16 took 132 us).  VEC (rows of x on 16-byte boundaries, of codes on 8-byte ones):
// eight columns to a lane, four lanes to a group.  Else a group at a time, a column to a lane.
template <typename TX, bool VEC> __global__ void __launch_bounds__(32 * kWarps, 4) k_act8_store(Act8Call c)
{
    const int lane = threadIdx.x & 31;
    const int64_t d = c.d, groups = (d + kActGroup - 1) / kActGroup;
    const bool e4m3 = c.code_dtype == TURNOPD_E4M3;
    for (int64_t strip = (int64_t)blockIdx.y * kStrip; strip < d; strip += (int64_t)gridDim.y * kStrip)
        for (int64_t row = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5); row < c.T; row += (int64_t)gridDim.x * kWarps) {
            const bool on = !c.mask || c.mask[row];
            float v[kUnits][8];
#pragma unroll
            for (int q = 0; q < kUnits; ++q) {
                const TX *x = static_cast<const TX *>(c.x) + row * c.ldx;
                const int64_t j = (strip + q * kChunk) + (VEC ? lane * 8 : lane);
                if (VEC && on && j + 8 <= d) {
                    load8(x + j, v[q]);
                } else {
#pragma unroll
                    for (int k = 0; k < 8; ++k)
                        v[q][k] = on && j + (VEC ? k : k * kActGroup) < d ? to_float(x[j + (VEC ? k : k * kActGroup)]) : 0.f;
                }
            }
#pragma unroll
            for (int q = 0; q < kUnits; ++q) {
                uint8_t *codes = static_cast<uint8_t *>(c.codes) + row * c.ldc, *exps = c.exps + row * groups;
                if constexpr (VEC) {
                    const int64_t j = (strip + q * kChunk) + lane * 8;
                    uint32_t amax = 0;
#pragma unroll
                    for (int k = 0; k < 8; ++k)
                        amax = max(amax, magnitude(v[q][k]));
                    amax = max(amax, __shfl_xor_sync(~0u, amax, 1));
                    amax = max(amax, __shfl_xor_sync(~0u, amax, 2));
                    const uint32_t e = on ? exponent_byte(amax, e4m3) : 0u;
                    const float s = inverse_scale(e);
                    if (e == 255u) {
#pragma unroll
                        for (int k = 0; k < 8; ++k)
                            v[q][k] = 0.f;
                    }
                    uint2 w;
                    w.x = encode2(v[q][0] * s, v[q][1] * s, e4m3) | encode2(v[q][2] * s, v[q][3] * s, e4m3) << 16;
                    w.y = encode2(v[q][4] * s, v[q][5] * s, e4m3) | encode2(v[q][6] * s, v[q][7] * s, e4m3) << 16;
                    if (j + 8 <= d) {
                        __stcs(reinterpret_cast<uint2 *>(codes + j), w);
                    } else {
#pragma unroll
                        for (int k = 0; k < 8; ++k)
                            if (j + k < d)
                                codes[j + k] = (uint8_t)((k < 4 ? w.x : w.y) >> (8 * (k & 3)));
                    }
                    if ((lane & 3) == 0 && j < d) {
                        exps[j / kActGroup] = (uint8_t)e;
                        if (e == 255u)
                            set_status(c.status, TURNOPD_ERR_NONFINITE);
                    }
                } else {
#pragma unroll
                    for (int g = 0; g < 8; ++g) {
                        const int64_t j = (strip + q * kChunk) + g * kActGroup + lane;
                        const uint32_t amax = __reduce_max_sync(~0u, magnitude(v[q][g]));
                        const uint32_t e = on ? exponent_byte(amax, e4m3) : 0u;
                        const float t = e == 255u ? 0.f : v[q][g] * inverse_scale(e);
                        if (j < d)
                            codes[j] = (uint8_t)encode2(t, 0.f, e4m3);
                        if (lane == 0 && j < d) {
                            exps[j / kActGroup] = (uint8_t)e;
                            if (e == 255u)
                                set_status(c.status, TURNOPD_ERR_NONFINITE);
                        }
                    }
                }
            }
        }
}

// The value of a code, no further than the type reaches: a group next to its end may have codes that stand for more.
template <typename TX> __device__ __forceinline__ float worth(float code, float scale)
{
    constexpr float kMost = sizeof(TX) == 2 ? 0x1.fep+127f : 0x1.fffffep+127f;
    const float v = code * scale;
    return v > kMost ? kMost : v < -kMost ? -kMost : v;  // NaN stays
}

template <typename TX, bool VEC> __global__ void __launch_bounds__(32 * kWarps, 4) k_act8_load(Act8Call c)
{
    const int lane = threadIdx.x & 31;
    const int64_t d = c.d, groups = (d + kActGroup - 1) / kActGroup;
    const bool e4m3 = c.code_dtype == TURNOPD_E4M3;
    for (int64_t strip = (int64_t)blockIdx.y * kStrip; strip < d; strip += (int64_t)gridDim.y * kStrip)
        for (int64_t row = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5); row < c.T; row += (int64_t)gridDim.x * kWarps) {
            uint2 code[kUnits];
            uint32_t exp[kUnits];
            if constexpr (VEC) {
#pragma unroll
                for (int q = 0; q < kUnits; ++q) {
                    const int64_t j = (strip + q * kChunk) + lane * 8;
                    if (j + 8 <= d) {
                        code[q] = __ldcs(reinterpret_cast<const uint2 *>(static_cast<const uint8_t *>(c.codes) + row * c.ldc + j));
                        exp[q] = c.exps[row * groups + j / kActGroup];
                    }
                }
            }
#pragma unroll
            for (int q = 0; q < kUnits; ++q) {
                TX *x = static_cast<TX *>(c.out) + row * c.ldx;
                const uint8_t *codes = static_cast<const uint8_t *>(c.codes) + row * c.ldc, *exps = c.exps + row * groups;
                const auto one = [&](int64_t j) {
                    const float v = e4m3 ? decode_e4m3(codes[j]) : (float)(int8_t)codes[j];
                    x[j] = from_float<TX>(worth<TX>(v, act_scale(exps[j / kActGroup])));
                };
                if constexpr (VEC) {
                    const int64_t j = (strip + q * kChunk) + lane * 8;
                    if (j + 8 <= d) {
                        float v[8];
                        decode8(code[q], e4m3, v);
                        const float s = act_scale(exp[q]);
#pragma unroll
                        for (int k = 0; k < 8; ++k)
                            v[k] = worth<TX>(v[k], s);
                        store8(x + j, v);
                    } else {
                        for (int k = 0; k < 8; ++k)
                            if (j + k < d)
                                one(j + k);
                    }
                } else {
#pragma unroll
                    for (int g = 0; g < 8; ++g)
                        if ((strip + q * kChunk) + g * kActGroup + lane < d)
                            one((strip + q * kChunk) + g * kActGroup + lane);
                }
            }
        }
}

bool on_boundaries(const Act8Call &c)
{
    const int64_t esz = c.x_dtype == TURNOPD_BF16 ? 2 : 4;
    const void *x = c.x ? c.x : c.out;
    return reinterpret_cast<uintptr_t>(x) % 16 == 0 && c.ldx * esz % 16 == 0 && reinterpret_cast<uintptr_t>(c.codes) % 8 == 0 &&
           c.ldc % 8 == 0;
}

template <bool STORE> cudaError_t launch(const Act8Call &c, cudaStream_t stream)
{
    const int64_t strips = (c.d + kStrip - 1) / kStrip, blocks = (c.T + kWarps - 1) / kWarps;
    const dim3 grid((unsigned)std::min<int64_t>(blocks, std::max<int64_t>((int64_t)device_sm_count() * 8 / strips, 1)),
                    (unsigned)std::min<int64_t>(strips, 65535));
    const bool vec = on_boundaries(c);
    const auto go = [&](auto x) {
        using X = decltype(x);
        auto kernel = STORE ? (vec ? k_act8_store<X, true> : k_act8_store<X, false>)
                            : (vec ? k_act8_load<X, true> : k_act8_load<X, false>);
        kernel<<<grid, 32 * kWarps, 0, stream>>>(c);
    };
    if (c.x_dtype == TURNOPD_BF16)
        go(__nv_bfloat16());
    else
        go(float());
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_act8_store(const Act8Call &c, cudaStream_t stream) { return launch<true>(c, stream); }
cudaError_t launch_act8_load(const Act8Call &c, cudaStream_t stream) { return launch<false>(c, stream); }

}  // namespace turnopd
