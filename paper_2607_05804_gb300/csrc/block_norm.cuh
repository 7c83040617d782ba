// What the kernels of the norms around a block share.
#pragma once

#include <initializer_list>

#include "columns.cuh"
#include "common.cuh"
#include "kernels.h"
#include "packed.cuh"

namespace turnopd {

constexpr int kBlockMaxRow = 8192;   // longest rows that a block of threads holds
constexpr int kBlockMaxParts = 320;  // CTAs of the backward pass, at most

// N numbers that are added up together.
template <int N> struct Numbers {
    float v[N];
};
// Sums over the warp's lanes.  Of two numbers each half of the warp takes one on after the first exchange, and of four each
// quarter after the second: 5 + 2 shuffles for two numbers, not 10.
__device__ __forceinline__ float halve(float a, float b, int lane, int o)
{
    const bool upper = lane & o;
    return (upper ? b : a) + __shfl_xor_sync(~0u, upper ? a : b, o);
}
template <int N> __device__ __forceinline__ float spread_sum(const Numbers<N> &x)  // number N lane / 32 of this lane
{
    const int lane = threadIdx.x & 31;
    float v;
    if constexpr (N == 4)
        v = halve(halve(x.v[0], x.v[2], lane, 16), halve(x.v[1], x.v[3], lane, 16), lane, 8);
    else if constexpr (N == 2)
        v = halve(x.v[0], x.v[1], lane, 16);
    else
        v = x.v[0];
#pragma unroll
    for (int o = 16 / N; o > 0; o >>= 1)
        v += __shfl_xor_sync(~0u, v, o);
    return v;
}
template <int N> __device__ __forceinline__ Numbers<N> gather_sums(float v)
{
    Numbers<N> x;
#pragma unroll
    for (int k = 0; k < N; ++k)
        x.v[k] = N == 1 ? v : __shfl_sync(~0u, v, k * (32 / N));
    return x;
}

// Sums over the `warps` warps of a group, the same values in every thread; red: an entry per warp of the block, free again
// two sums later.  The warps' sums are added up like the lanes': a lane reads one of them each.
template <int N> __device__ __forceinline__ Numbers<N> group_sum(Numbers<N> x, Numbers<N> *red, int group, int warps)
{
    float v = spread_sum(x);
    if (warps > 1) {
        const int lane = threadIdx.x & 31;
        if (lane % (32 / N) == 0)
            red[threadIdx.x >> 5].v[lane / (32 / N)] = v;
        group_barrier(group, warps * 32);
        x = Numbers<N>{};
        if (lane < warps)
            x = red[group * warps + lane];
        v = spread_sum(x);
    }
    return gather_sums<N>(v);
}
__device__ __forceinline__ float group_sum(float x, float *red, int group, int warps)
{
    return group_sum(Numbers<1>{{x}}, reinterpret_cast<Numbers<1> *>(red), group, warps).v[0];
}

// Eight columns of a parameter from j on (those past the last one are some numbers), without conditions between the loads, or
// one would wait for another.
template <typename T> __device__ __forceinline__ void eight_of(const T *p, int j, int d, float *v)
{
    if (j + 8 <= d && (reinterpret_cast<uintptr_t>(p + j) & 15) == 0) {
        load8(p + j, v);
        return;
    }
    T raw[8];
#pragma unroll
    for (int e = 0; e < 8; ++e)
        raw[e] = p[min(j + e, d - 1)];
#pragma unroll
    for (int e = 0; e < 8; ++e)
        v[e] = to_float(raw[e]);
}
__device__ __forceinline__ void param8(const void *p, int32_t dtype, int j, int d, float *v)
{
    if (dtype == TURNOPD_BF16)
        eight_of(static_cast<const __nv_bfloat16 *>(p), j, d, v);
    else
        eight_of(static_cast<const float *>(p), j, d, v);
}

// Column j of row i of an array of any type; 8-bit codes with their exponents.
__device__ __forceinline__ float element(const void *p, int32_t dtype, int64_t ld, const uint8_t *exps, int64_t d, int64_t i, int64_t j)
{
    if (dtype == TURNOPD_BF16 || dtype == TURNOPD_F32)
        return param(p, dtype, i * ld + j);
    const uint8_t b = static_cast<const uint8_t *>(p)[i * ld + j];
    const float s = act_scale(exps[i * ((d + kActGroup - 1) / kActGroup) + j / kActGroup]);
    return (dtype == TURNOPD_E4M3 ? decode_e4m3(b) : (float)(int8_t)b) * s;
}

__device__ __forceinline__ void put(void *p, int32_t dtype, int64_t at, float v)
{
    if (dtype == TURNOPD_BF16)
        static_cast<__nv_bfloat16 *>(p)[at] = __float2bfloat16_rn(v);
    else
        static_cast<float *>(p)[at] = v;
}

// Whether row i takes part: supervised, and its statistics were finite.
__device__ __forceinline__ bool takes_part(const BlockGradCall &c, int64_t i, float4 &stats)
{
    if (c.mask && !c.mask[i])
        return false;
    stats = c.stats ? reinterpret_cast<const float4 *>(c.stats)[i] : make_float4(0.f, 0.f, 0.f, 0.f);
    return (!c.gamma_post || stats.y > 0.f) && (!c.gamma_pre || stats.w > 0.f);
}

inline int stored_bytes(int32_t dtype) { return dtype == TURNOPD_F32 ? 4 : dtype == TURNOPD_BF16 ? 2 : 1; }

// The element of a group of eight at which row 0 of an array begins, and by how many the next row begins later.  Where they
// are 0 each row begins at a boundary that eight columns can be copied from (16 bytes, 8 for codes).
struct Phase {
    bool given;
    int at, step;
    Phase(const void *p, int64_t ld, int32_t dtype)
        : given(p), at((int)(reinterpret_cast<uintptr_t>(p) / stored_bytes(dtype) & 7)), step((int)(ld & 7))
    {
    }
};

// The phase that all arrays of a call share, if they do.
struct Phases {
    bool alike = true;
    int at = 0, step = 0;
    Phases(std::initializer_list<Phase> all)
    {
        bool first = true;
        for (const Phase &p : all) {
            if (!p.given)
                continue;
            if (first)
                at = p.at, step = p.step;
            alike = alike && p.at == at && p.step == step;
            first = false;
        }
    }
};

// The row kernels of the forward pass, by the types of r and y.
template <typename TR, typename TY> cudaError_t launch_block_rows_fwd(const BlockCall &c, const Phases &phases, cudaStream_t stream);

// The row kernels of the backward pass, by the types of dr' and of dh; *parts: rows of partial sums that they leave in the
// workspace, 4 d floats each (dh xh_pre, dh, X xh_post, X; the second and fourth only where block_bwd_bias says).  *taken:
// whether they take such rows.
bool block_bwd_bias(const BlockGradCall &c);
// whether a row needs more than the sums of g xh: the means of layer norms, the sums for betas, or beta in the gate's own
// gradient for every element, whose kernels add it
bool block_bwd_general(const BlockGradCall &c);
bool block_bwd_needs_y(const BlockGradCall &c);
template <typename TR, typename TY>
cudaError_t launch_block_rows_bwd(const BlockGradCall &c, int *parts, bool *taken, cudaStream_t stream);

}  // namespace turnopd
