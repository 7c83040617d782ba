// Layer norm and root-mean-square norm of hidden states, and their backward pass.
//
// Row x[0..d): mu = mean x (0 in the root-mean-square form), r = (mean (x - mu)^2 + eps)^{-1/2},
// xh = (x - mu) r, y = xh gamma + beta.  With g = dy gamma:
//   dx = r (g - mean g - xh mean(g xh))   (root-mean-square form: without mean g),
//   dgamma = sum_i dy_i xh_i, dbeta = sum_i dy_i over the rows.
// The variance is a second pass over x - mu, so a mean much larger than the deviation costs no digits.

#include <algorithm>

#include "common.cuh"
#include "kernels.h"

namespace turnopd {
namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kMaxPartials = 608;  // rows of partial dgamma / dbeta sums in the workspace

__device__ __forceinline__ float param(const void *p, int32_t dtype, int64_t j)
{
    return dtype == TURNOPD_BF16 ? __bfloat162float(static_cast<const __nv_bfloat16 *>(p)[j])
                                 : static_cast<const float *>(p)[j];
}

// Sum over the block in a fixed order, the same value in every thread.
__device__ __forceinline__ float block_sum(float v, float *red)
{
    v = warp_sum_f(v);
    __syncthreads();
    if ((threadIdx.x & 31) == 0)
        red[threadIdx.x >> 5] = v;
    __syncthreads();
    float s = red[0];
#pragma unroll
    for (int w = 1; w < kWarps; ++w)
        s += red[w];
    return s;
}

template <typename TX, typename TY> __global__ void __launch_bounds__(kThreads) k_norm_fwd(NormCall c)
{
    __shared__ float red[kWarps];
    const bool layer = c.kind == TURNOPD_LAYER_NORM;
    for (int64_t i = blockIdx.x; i < c.T; i += gridDim.x) {
        const TX *x = static_cast<const TX *>(c.x) + i * c.ldx;
        TY *y = static_cast<TY *>(c.y) + i * c.ldy;
        float mu = 0.f, r = 0.f;
        bool fine = !c.mask || c.mask[i];
        if (fine) {
            if (layer) {
                float s = 0.f;
                for (int64_t j = threadIdx.x; j < c.d; j += kThreads)
                    s += to_float(x[j]);
                mu = block_sum(s, red) / (float)c.d;
            }
            float q = 0.f;
            for (int64_t j = threadIdx.x; j < c.d; j += kThreads) {
                const float t = to_float(x[j]) - mu;
                q = fmaf(t, t, q);
            }
            r = 1.f / sqrtf(block_sum(q, red) / (float)c.d + c.eps);
            if (!(isfinite(mu) && isfinite(r) && r > 0.f)) {
                fine = false;
                mu = r = 0.f;
                if (threadIdx.x == 0)
                    set_status(c.status, TURNOPD_ERR_NONFINITE);
            }
        }
        for (int64_t j = threadIdx.x; j < c.d; j += kThreads) {
            float o = 0.f;
            if (fine) {
                o = (to_float(x[j]) - mu) * r * param(c.gamma, c.param_dtype, j);
                if (c.beta)
                    o += param(c.beta, c.param_dtype, j);
            }
            y[j] = from_float<TY>(o);
        }
        if (threadIdx.x == 0) {
            if (c.mean)
                c.mean[i] = mu;
            if (c.rstd)
                c.rstd[i] = r;
        }
    }
}

// Whether token i takes part: supervised, and the forward pass found it finite.
__device__ __forceinline__ bool takes_part(const NormGradCall &c, int64_t i)
{
    return (!c.mask || c.mask[i]) && c.rstd[i] > 0.f;
}

template <typename TX, typename TDY, typename TDX>
__global__ void __launch_bounds__(kThreads) k_norm_dx(NormGradCall c)
{
    __shared__ float red[kWarps];
    const bool layer = c.kind == TURNOPD_LAYER_NORM;
    for (int64_t i = blockIdx.x; i < c.T; i += gridDim.x) {
        const TX *x = static_cast<const TX *>(c.x) + i * c.ldx;
        const TDY *dy = static_cast<const TDY *>(c.dy) + i * c.lddy;
        TDX *dx = static_cast<TDX *>(c.dx) + i * c.lddx;
        if (!takes_part(c, i)) {
            for (int64_t j = threadIdx.x; j < c.d; j += kThreads)
                dx[j] = from_float<TDX>(0.f);
            continue;
        }
        const float mu = layer ? c.mean[i] : 0.f, r = c.rstd[i];
        float sg = 0.f, sgx = 0.f;
        for (int64_t j = threadIdx.x; j < c.d; j += kThreads) {
            const float g = to_float(dy[j]) * param(c.gamma, c.param_dtype, j);
            sg += g;
            sgx = fmaf(g, (to_float(x[j]) - mu) * r, sgx);
        }
        sgx = block_sum(sgx, red) / (float)c.d;
        sg = layer ? block_sum(sg, red) / (float)c.d : 0.f;
        for (int64_t j = threadIdx.x; j < c.d; j += kThreads) {
            const float g = to_float(dy[j]) * param(c.gamma, c.param_dtype, j);
            const float xh = (to_float(x[j]) - mu) * r;
            dx[j] = from_float<TDX>(r * (g - sg - xh * sgx));
        }
    }
}

// Partial sums over the tokens blockIdx.y, blockIdx.y + gridDim.y, ... of 256 columns.
template <typename TX, typename TDY> __global__ void __launch_bounds__(kThreads) k_norm_params(NormGradCall c)
{
    const int64_t j = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    float sg = 0.f, sb = 0.f;
    for (int64_t i = blockIdx.y; i < c.T; i += gridDim.y) {
        if (j >= c.d || !takes_part(c, i))
            continue;
        const float dy = to_float(static_cast<const TDY *>(c.dy)[i * c.lddy + j]);
        const float t = to_float(static_cast<const TX *>(c.x)[i * c.ldx + j]) -
                        (c.kind == TURNOPD_LAYER_NORM ? c.mean[i] : 0.f);
        sg = fmaf(dy, t * c.rstd[i], sg);
        sb += dy;
    }
    float *part = static_cast<float *>(c.workspace) + (int64_t)blockIdx.y * 2 * c.d;
    if (j < c.d) {
        part[j] = sg;
        part[c.d + j] = sb;
    }
}

__global__ void __launch_bounds__(kThreads) k_norm_params_sum(NormGradCall c, int n)
{
    const int64_t j = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (j >= c.d)
        return;
    const float *part = static_cast<const float *>(c.workspace);
    float sg = 0.f, sb = 0.f;
    for (int k = 0; k < n; ++k) {
        sg += part[(int64_t)k * 2 * c.d + j];
        sb += part[(int64_t)k * 2 * c.d + c.d + j];
    }
    if (c.dgamma)
        c.dgamma[j] = sg;
    if (c.dbeta)
        c.dbeta[j] = sb;
}

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

}  // namespace

size_t norm_bwd_workspace_bytes(int64_t T, int64_t d)
{
    return align256(sizeof(float) * 2 * (size_t)d * (size_t)std::min<int64_t>(std::max<int64_t>(T, 1), kMaxPartials));
}

cudaError_t launch_norm_fwd(const NormCall &c, cudaStream_t stream)
{
    const int grid = (int)std::min<int64_t>(c.T, (int64_t)device_sm_count() * 8);
    with_types(c.x_dtype, c.y_dtype, [&](auto x, auto y) {
        k_norm_fwd<decltype(x), decltype(y)><<<grid, kThreads, 0, stream>>>(c);
    });
    return cudaGetLastError();
}

cudaError_t launch_norm_bwd(const NormGradCall &c, cudaStream_t stream)
{
    with_types(c.x_dtype, c.dy_dtype, [&](auto x, auto dy) {
        using X = decltype(x);
        using DY = decltype(dy);
        const int grid = (int)std::min<int64_t>(c.T, (int64_t)device_sm_count() * 8);
        if (c.dx && c.T > 0) {
            if (c.dx_dtype == TURNOPD_BF16)
                k_norm_dx<X, DY, __nv_bfloat16><<<grid, kThreads, 0, stream>>>(c);
            else
                k_norm_dx<X, DY, float><<<grid, kThreads, 0, stream>>>(c);
        }
        if (c.dgamma || c.dbeta) {
            const unsigned cols = (unsigned)((c.d + kThreads - 1) / kThreads);
            const int n = (int)std::min<int64_t>(std::max<int64_t>(c.T, 1), 64);
            k_norm_params<X, DY><<<dim3(cols, n), kThreads, 0, stream>>>(c);
            k_norm_params_sum<<<cols, kThreads, 0, stream>>>(c, n);
        }
    });
    return cudaGetLastError();
}

}  // namespace turnopd
