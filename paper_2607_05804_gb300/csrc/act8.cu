// Activations kept in 8 bits between the forward and the backward pass.
//
// 32 columns of a row share the exponent k = the smallest integer, -126 at least, with amax <= M 2^k (M = 448 for e4m3, 127
// for int8); a code is x 2^-k, rounded to the nearest even one.  Scaling by a power of two is exact, so the code's is the
// only rounding: |x - x~| <= 2^-4 |x| from 2^(k-6) on and 2^(k-10) below (e4m3), 2^(k-1) (int8).  A scale that is no power
// of two would spare int8 up to one of its seven bits, but round twice and depend on how the quotient is formed.

#include <algorithm>
#include <type_traits>

#include "columns.cuh"
#include "common.cuh"
#include "kernels.h"
#include "packed.cuh"

namespace turnopd {
namespace {

constexpr int kWarps = 8;
constexpr int kChunk = 256;  // columns of a row, eight groups, that a warp takes together

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

// Eight columns as they are stored.
template <typename TX> struct Raw;
template <> struct Raw<__nv_bfloat16> {
    uint4 u;
    __device__ void load(const __nv_bfloat16 *p) { u = __ldcs(reinterpret_cast<const uint4 *>(p)); }
    __device__ void put(int k, __nv_bfloat16 x)
    {
        const uint32_t b = __bfloat16_as_ushort(x), w = k & 1 ? b << 16 : b;
        (k < 4 ? (k < 2 ? u.x : u.y) : (k < 6 ? u.z : u.w)) |= w;
    }
    // the largest magnitude as the bits of a float; of sixteen bits as whole numbers NaN is the largest
    __device__ uint32_t largest() const
    {
        const uint32_t m = 0x7fff7fffu;
        const uint32_t a = __vmaxu2(__vmaxu2(u.x & m, u.y & m), __vmaxu2(u.z & m, u.w & m));
        return max(a << 16, a & 0xffff0000u);
    }
    __device__ float2 pair(int k) const { return unpack2(word(u, k)); }
};
template <> struct Raw<float> {
    float4 a, b;
    __device__ void load(const float *p)
    {
        a = __ldcs(reinterpret_cast<const float4 *>(p));
        b = __ldcs(reinterpret_cast<const float4 *>(p) + 1);
    }
    __device__ void put(int k, float x)
    {
        float4 &v = k < 4 ? a : b;
        (k & 2 ? (k & 1 ? v.w : v.z) : (k & 1 ? v.y : v.x)) = x;
    }
    __device__ uint32_t largest() const
    {
        return max(max(max(magnitude(a.x), magnitude(a.y)), max(magnitude(a.z), magnitude(a.w))),
                   max(max(magnitude(b.x), magnitude(b.y)), max(magnitude(b.z), magnitude(b.w))));
    }
    __device__ float2 pair(int k) const
    {
        const float4 &v = k < 2 ? a : b;
        return k & 1 ? make_float2(v.z, v.w) : make_float2(v.x, v.y);
    }
};

// Rows of x on 16-byte boundaries, of codes on 8-byte ones: a warp takes strips of U chunks of a row, eight columns to a lane,
// four lanes to a group.  A block's strips begin at one column: no division tells a row from its columns (with one for each
// chunk 32,768 x 4,096 bf16 took 132 us).
//
// Bound: HBM, with instruction issue behind it (0.66 of the slots).  32,768 x 4,096 bf16: storing 64 us (407 MB, 6,350 GB/s),
// loading 63; fp32 236 for both (0.84 of the copy rate); rows of 1,001 columns, off boundaries, 87 for both (0.34).
template <typename TX, bool E4M3, int U> __global__ void __launch_bounds__(32 * kWarps) k_act8_store(Act8Call c)
{
    const int lane = threadIdx.x & 31;
    const int64_t d = c.d, groups = (d + kActGroup - 1) / kActGroup;
    for (int64_t strip = (int64_t)blockIdx.y * U * kChunk; strip < d; strip += (int64_t)gridDim.y * U * kChunk)
        for (int64_t row = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5); row < c.T; row += (int64_t)gridDim.x * kWarps) {
            const bool on = !c.mask || c.mask[row];
            const int64_t first = strip + lane * 8;
            const TX *x = static_cast<const TX *>(c.x) + row * c.ldx + first;
            uint8_t *codes = static_cast<uint8_t *>(c.codes) + row * c.ldc + first, *exps = c.exps + row * groups;
            Raw<TX> v[U];
#pragma unroll
            for (int q = 0; q < U; ++q) {
                const int64_t left = d - first - q * kChunk;
                if (on && left >= 8) {
                    v[q].load(x + q * kChunk);
                } else {
                    v[q] = Raw<TX>{};
#pragma unroll
                    for (int k = 0; k < 8; ++k)
                        if (on && k < left)
                            v[q].put(k, x[q * kChunk + k]);
                }
            }
            uint32_t e[U];
#pragma unroll
            for (int q = 0; q < U; ++q) {
                const int64_t left = d - first - q * kChunk;
                uint32_t amax = v[q].largest();
                amax = max(amax, __shfl_xor_sync(~0u, amax, 1));
                amax = max(amax, __shfl_xor_sync(~0u, amax, 2));
                e[q] = on ? exponent_byte(amax, E4M3) : 0u;
                const float s = inverse_scale(e[q]);
                uint2 w;
                const float2 p0 = v[q].pair(0), p1 = v[q].pair(1), p2 = v[q].pair(2), p3 = v[q].pair(3);
                w.x = encode2(p0.x * s, p0.y * s, E4M3) | encode2(p1.x * s, p1.y * s, E4M3) << 16;
                w.y = encode2(p2.x * s, p2.y * s, E4M3) | encode2(p3.x * s, p3.y * s, E4M3) << 16;
                if (e[q] == 255u) {
                    w = make_uint2(0u, 0u);
                    if (left > 0)
                        set_status(c.status, TURNOPD_ERR_NONFINITE);
                }
                if (left >= 8) {
                    __stcs(reinterpret_cast<uint2 *>(codes + q * kChunk), w);
                } else {
#pragma unroll
                    for (int k = 0; k < 8; ++k)
                        if (k < left)
                            codes[q * kChunk + k] = (uint8_t)((k < 4 ? w.x : w.y) >> (8 * (k & 3)));
                }
            }
            // the strip's 8 U exponents in one store: lane 4 g + q has that of group g of chunk q
            const int q = lane & 3;
            const int64_t at = (strip + q * kChunk) / kActGroup + (lane >> 2);
            if (q < U && at < groups)
                exps[at] = (uint8_t)(U == 1 || q == 0 ? e[0] : q == 1 ? e[U > 1 ? 1 : 0] : q == 2 ? e[U > 2 ? 2 : 0] : e[U > 3 ? 3 : 0]);
        }
}

// Any rows: a column to a lane, a group at a time, U chunks of a row at once.
template <typename TX, int U> __global__ void __launch_bounds__(32 * kWarps) k_act8_store_any(Act8Call c)
{
    const int lane = threadIdx.x & 31;
    const int64_t d = c.d, groups = (d + kActGroup - 1) / kActGroup;
    const bool e4m3 = c.code_dtype == TURNOPD_E4M3;
    for (int64_t strip = (int64_t)blockIdx.y * U * kChunk; strip < d; strip += (int64_t)gridDim.y * U * kChunk)
        for (int64_t row = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5); row < c.T; row += (int64_t)gridDim.x * kWarps) {
            const bool on = !c.mask || c.mask[row];
            const int left = (int)min(d - strip, (int64_t)U * kChunk);
            const TX *x = static_cast<const TX *>(c.x) + row * c.ldx + strip;
            uint8_t *codes = static_cast<uint8_t *>(c.codes) + row * c.ldc + strip, *exps = c.exps + row * groups + strip / kActGroup;
            // (a column past the end counts as the last one, whose group is the same or is not written)
            TX raw[U * 8];
            float v[U * 8];
#pragma unroll
            for (int g = 0; g < U * 8; ++g)
                if (on)
                    raw[g] = x[min(g * kActGroup + lane, left - 1)];
#pragma unroll
            for (int g = 0; g < U * 8; ++g)
                v[g] = on && g * kActGroup < left ? to_float(raw[g]) : 0.f;
            // lane g has group g's largest magnitude, makes its exponent and writes it
            uint32_t mine = 0;
#pragma unroll
            for (int g = 0; g < U * 8; ++g) {
                const uint32_t amax = __reduce_max_sync(~0u, magnitude(v[g]));
                mine = lane == g ? amax : mine;
            }
            const uint32_t e = on ? exponent_byte(mine, e4m3) : 0u;
            const float s = inverse_scale(e);
            if (lane < U * 8 && lane * kActGroup < left) {
                exps[lane] = (uint8_t)e;
                if (e == 255u)
                    set_status(c.status, TURNOPD_ERR_NONFINITE);
            }
#pragma unroll
            for (int g = 0; g < U * 8; ++g) {
                const float scale = __shfl_sync(~0u, s, g);
                if (g * kActGroup + lane < left)
                    codes[g * kActGroup + lane] = (uint8_t)encode2(scale == 0.f ? 0.f : v[g] * scale, 0.f, e4m3);
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

// The same two layouts as for storing.
template <typename TX, int U> __global__ void __launch_bounds__(32 * kWarps, 4) k_act8_load(Act8Call c)
{
    const int lane = threadIdx.x & 31;
    const int64_t d = c.d, groups = (d + kActGroup - 1) / kActGroup;
    const bool e4m3 = c.code_dtype == TURNOPD_E4M3;
    for (int64_t strip = (int64_t)blockIdx.y * U * kChunk; strip < d; strip += (int64_t)gridDim.y * U * kChunk)
        for (int64_t row = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5); row < c.T; row += (int64_t)gridDim.x * kWarps) {
            const int64_t first = strip + lane * 8;
            const uint8_t *codes = static_cast<const uint8_t *>(c.codes) + row * c.ldc + first, *exps = c.exps + row * groups;
            TX *x = static_cast<TX *>(c.out) + row * c.ldx + first;
            uint2 code[U];
            uint32_t exp[U];
#pragma unroll
            for (int q = 0; q < U; ++q) {
                const int64_t left = d - first - q * kChunk;
                code[q] = make_uint2(0u, 0u);
                exp[q] = left > 0 ? exps[(first + q * kChunk) / kActGroup] : 0u;
                if (left >= 8)
                    code[q] = __ldcs(reinterpret_cast<const uint2 *>(codes + q * kChunk));
                else
                    for (int k = 0; k < left; ++k)
                        (k < 4 ? code[q].x : code[q].y) |= (uint32_t)codes[q * kChunk + k] << (8 * (k & 3));
            }
#pragma unroll
            for (int q = 0; q < U; ++q) {
                const int64_t left = d - first - q * kChunk;
                float v[8];
                decode8(code[q], e4m3, v);
                const float s = act_scale(exp[q]);
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    v[k] = worth<TX>(v[k], s);
                if (left >= 8) {
                    store8(x + q * kChunk, v);
                } else {
#pragma unroll
                    for (int k = 0; k < 8; ++k)
                        if (k < left)
                            x[q * kChunk + k] = from_float<TX>(v[k]);
                }
            }
        }
}

template <typename TX, int U> __global__ void __launch_bounds__(32 * kWarps) k_act8_load_any(Act8Call c)
{
    const int lane = threadIdx.x & 31;
    const int64_t d = c.d, groups = (d + kActGroup - 1) / kActGroup;
    const bool e4m3 = c.code_dtype == TURNOPD_E4M3;
    for (int64_t strip = (int64_t)blockIdx.y * U * kChunk; strip < d; strip += (int64_t)gridDim.y * U * kChunk)
        for (int64_t row = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5); row < c.T; row += (int64_t)gridDim.x * kWarps) {
            const int left = (int)min(d - strip, (int64_t)U * kChunk);
            const uint8_t *codes = static_cast<const uint8_t *>(c.codes) + row * c.ldc + strip;
            TX *x = static_cast<TX *>(c.out) + row * c.ldx + strip;
            uint8_t code[U * 8];
#pragma unroll
            for (int g = 0; g < U * 8; ++g)
                code[g] = codes[min(g * kActGroup + lane, left - 1)];
            float s = 0.f;
            if (lane < U * 8 && lane * kActGroup < left)
                s = act_scale(c.exps[row * groups + strip / kActGroup + lane]);
#pragma unroll
            for (int g = 0; g < U * 8; ++g) {
                const float scale = __shfl_sync(~0u, s, g);
                if (g * kActGroup + lane < left)
                    x[g * kActGroup + lane] = from_float<TX>(worth<TX>(e4m3 ? decode_e4m3(code[g]) : (float)(int8_t)code[g], scale));
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

// Strips of four chunks where there are enough for every warp to have several, else of one.
template <typename F> void with_grid(const Act8Call &c, F &&go)
{
    const int64_t chunks = (c.d + kChunk - 1) / kChunk, blocks = (c.T + kWarps - 1) / kWarps, sms = device_sm_count();
    const bool four = chunks >= 3 && blocks * ((chunks + 3) / 4) >= 8 * sms;
    const int64_t strips = four ? (chunks + 3) / 4 : chunks;
    const dim3 grid((unsigned)std::min<int64_t>(blocks, std::max<int64_t>(sms * 16 / strips, 1)), (unsigned)std::min<int64_t>(strips, 65535));
    if (four)
        go(grid, std::integral_constant<int, 4>());
    else
        go(grid, std::integral_constant<int, 1>());
}

template <typename F> cudaError_t with_type(int32_t dtype, F &&go)
{
    if (dtype == TURNOPD_BF16)
        go(__nv_bfloat16());
    else
        go(float());
    return cudaGetLastError();
}

}  // namespace

cudaError_t launch_act8_store(const Act8Call &c, cudaStream_t stream)
{
    const bool vec = on_boundaries(c);
    return with_type(c.x_dtype, [&](auto x) {
        with_grid(c, [&](dim3 grid, auto units) {
            using X = decltype(x);
            constexpr int U = decltype(units)::value;
            auto kernel = !vec                             ? k_act8_store_any<X, U>
                          : c.code_dtype == TURNOPD_E4M3 ? k_act8_store<X, true, U>
                                                           : k_act8_store<X, false, U>;
            kernel<<<grid, 32 * kWarps, 0, stream>>>(c);
        });
    });
}

cudaError_t launch_act8_load(const Act8Call &c, cudaStream_t stream)
{
    const bool vec = on_boundaries(c);
    return with_type(c.x_dtype, [&](auto x) {
        with_grid(c, [&](dim3 grid, auto units) {
            using X = decltype(x);
            constexpr int U = decltype(units)::value;
            auto kernel = vec ? k_act8_load<X, U> : k_act8_load_any<X, U>;
            kernel<<<grid, 32 * kWarps, 0, stream>>>(c);
        });
    });
}

}  // namespace turnopd
