// Columns of rows of hidden states: eight at a time, of either element type, and from 8-bit codes.
#pragma once

#include <cuda_fp8.h>

#include "common.cuh"

namespace turnopd {

__device__ __forceinline__ float param(const void *p, int32_t dtype, int64_t j)
{
    return dtype == TURNOPD_BF16 ? __bfloat162float(static_cast<const __nv_bfloat16 *>(p)[j])
                                 : static_cast<const float *>(p)[j];
}

// Eight columns from or to 16-byte aligned memory.
__device__ __forceinline__ void load8(const __nv_bfloat16 *p, float *v)
{
    const uint4 u = *reinterpret_cast<const uint4 *>(p);
    v[0] = bf16lo(u.x), v[1] = bf16hi(u.x), v[2] = bf16lo(u.y), v[3] = bf16hi(u.y);
    v[4] = bf16lo(u.z), v[5] = bf16hi(u.z), v[6] = bf16lo(u.w), v[7] = bf16hi(u.w);
}
__device__ __forceinline__ void load8(const float *p, float *v)
{
    const float4 a = reinterpret_cast<const float4 *>(p)[0], b = reinterpret_cast<const float4 *>(p)[1];
    v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w;
    v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
}
__device__ __forceinline__ void store8(__nv_bfloat16 *p, const float *v)
{
    __stcs(reinterpret_cast<uint4 *>(p), make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]),
                                                    pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])));
}
__device__ __forceinline__ void store8(float *p, const float *v)
{
    __stcs(reinterpret_cast<float4 *>(p), make_float4(v[0], v[1], v[2], v[3]));
    __stcs(reinterpret_cast<float4 *>(p) + 1, make_float4(v[4], v[5], v[6], v[7]));
}
__device__ __forceinline__ void cp16(void *smem, const void *gmem)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(smem)), "l"(gmem)
                 : "memory");
}

// Barrier of the n threads of one group (barriers 1 .. 8; 0 is the block's).
__device__ __forceinline__ void group_barrier(int group, int n)
{
    asm volatile("bar.sync %0, %1;" ::"r"(group + 1), "r"(n) : "memory");
}

// ---------------------------------------------------------------- activations in 8 bits

constexpr int kActGroup = 32;  // columns of a row that share one exponent

// 2^(e - 127) of an exponent byte; 0 for a masked token's, NaN for a group that held no finite numbers.
__device__ __forceinline__ float act_scale(uint32_t e) { return __uint_as_float(e == 255u ? 0x7fc00000u : e << 23); }

__device__ __forceinline__ float decode_e4m3(uint8_t b)
{
    return __half2float(__half(__nv_cvt_fp8_to_halfraw(b, __NV_E4M3)));
}

// Two codes from the low half of a word.
__device__ __forceinline__ float2 decode2_e4m3(uint32_t u)
{
    return __half22float2(__half2(__nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)u, __NV_E4M3)));
}

// Eight codes (exact in fp32, unscaled).
__device__ __forceinline__ void decode8(uint2 u, bool e4m3, float *v)
{
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const uint32_t w = h ? u.y : u.x;
        if (e4m3) {
            const float2 a = decode2_e4m3(w & 0xffffu), b = decode2_e4m3(w >> 16);
            v[4 * h] = a.x, v[4 * h + 1] = a.y, v[4 * h + 2] = b.x, v[4 * h + 3] = b.y;
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k)
                // the byte plus 128 as the last bits of 2^23: no conversion, of which an SM does few at a time
                v[4 * h + k] = __uint_as_float(__byte_perm(w ^ 0x80808080u, 0x4b000000u, 0x7440 | k)) - 8388736.f;
        }
    }
}

// ---------------------------------------------------------------- launches

// f(x type, second type) with values of the element types that two dtype codes name
template <typename F> void with_types(int32_t a, int32_t b, F &&f)
{
    if (a == TURNOPD_BF16 && b == TURNOPD_BF16)
        f(__nv_bfloat16(), __nv_bfloat16());
    else if (a == TURNOPD_BF16)
        f(__nv_bfloat16(), float());
    else if (b == TURNOPD_BF16)
        f(float(), __nv_bfloat16());
    else
        f(float(), float());
}

// Dynamic shared memory of a kernel up to `most`, the largest amount that any call of this kernel asks for: every call sets
// the same limit, since another host thread's call may come between one that sets it and its launch.  (From 40 KB: with the
// kernel's static shared memory it may pass the default limit of 48 KB.)
template <typename K> cudaError_t allow_shared(K kernel, size_t most)
{
    return most > 40 * 1024 ? cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)most) : cudaSuccess;
}

}  // namespace turnopd
