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
constexpr int kE = 16;  // columns of a row that one thread holds
constexpr int kMaxFwd = 1024 * kE;  // longest rows of the register kernels
constexpr int kMaxBwd = 512 * kE;

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
__device__ __forceinline__ void load_params8(const void *p, int32_t dtype, int64_t j, float *v)
{
    if (dtype == TURNOPD_BF16)
        load8(static_cast<const __nv_bfloat16 *>(p) + j, v);
    else
        load8(static_cast<const float *>(p) + j, v);
}

// The columns of thread t among n that share a row: in pieces of eight, a piece of each thread in turn (rows on
// 16-byte boundaries, d a multiple of 8), or one by one (any rows).  f(column, first of the thread's kE values).
template <bool VEC, typename F> __device__ __forceinline__ void each_piece(int t, int n, int64_t d, F &&f)
{
    constexpr int W = VEC ? 8 : 1;
#pragma unroll
    for (int k = 0; k < kE / W; ++k) {
        const int j = (k * n + t) * W;
        if (j < d)
            f(j, k * W);
    }
}

// Sum over the `warps` warps of a row's group, the same value in every thread; red: one entry per warp of the block.
// Every thread of the block calls it where a row has more than one warp.
__device__ __forceinline__ float group_sum(float v, float *red, int first, int warps)
{
    v = warp_sum_f(v);
    if (warps == 1)
        return v;
    if ((threadIdx.x & 31) == 0)
        red[threadIdx.x >> 5] = v;
    __syncthreads();
    float s = red[first];
    for (int w = 1; w < warps; ++w)
        s += red[first + w];
    return s;
}

// One row per group of n threads (a multiple of 32), kE columns to a thread, one read of x.
template <typename TX, typename TY, bool VEC>
__global__ void __launch_bounds__(1024) k_norm_fwd(NormCall c, int n)
{
    __shared__ float red[2][32];
    const int t = threadIdx.x % n, group = threadIdx.x / n, warps = n / 32;
    const int64_t i = (int64_t)blockIdx.x * (blockDim.x / n) + group;
    const bool layer = c.kind == TURNOPD_LAYER_NORM;
    const bool on = i < c.T && (!c.mask || c.mask[i]);
    const TX *x = static_cast<const TX *>(c.x) + i * c.ldx;
    const float inv_d = 1.f / (float)c.d;
    float v[kE], g[kE];
    if (on) {
        each_piece<VEC>(t, n, c.d, [&](int j, int k) {
            if constexpr (VEC)
                load8(x + j, v + k);
            else
                v[k] = to_float(x[j]);
        });
        each_piece<VEC>(t, n, c.d, [&](int j, int k) {
            if constexpr (VEC)
                load_params8(c.gamma, c.param_dtype, j, g + k);
            else
                g[k] = param(c.gamma, c.param_dtype, j);
        });
    }
    float mu = 0.f, q = 0.f;
    if (layer) {
        float s = 0.f;
        if (on)
            each_piece<VEC>(t, n, c.d, [&](int, int k) {
#pragma unroll
                for (int e = 0; e < (VEC ? 8 : 1); ++e)
                    s += v[k + e];
            });
        mu = group_sum(s, red[0], group * warps, warps) * inv_d;
    }
    if (on)
        each_piece<VEC>(t, n, c.d, [&](int, int k) {
#pragma unroll
            for (int e = 0; e < (VEC ? 8 : 1); ++e)
                q = fmaf(v[k + e] - mu, v[k + e] - mu, q);
        });
    q = group_sum(q, red[1], group * warps, warps);
    if (i >= c.T)
        return;
    float r = 0.f;
    if (on) {
        r = 1.f / sqrtf(q * inv_d + c.eps);
        if (!(isfinite(mu) && isfinite(r) && r > 0.f)) {
            r = 0.f;
            if (t == 0)
                set_status(c.status, TURNOPD_ERR_NONFINITE);
        }
    }
    if (r == 0.f)
        mu = 0.f;
    TY *y = static_cast<TY *>(c.y) + i * c.ldy;
    each_piece<VEC>(t, n, c.d, [&](int j, int k) {
        constexpr int W = VEC ? 8 : 1;
        float o[W], b[W];
#pragma unroll
        for (int e = 0; e < W; ++e)
            b[e] = 0.f;
        if (c.beta && r != 0.f) {
            if constexpr (VEC)
                load_params8(c.beta, c.param_dtype, j, b);
            else
                b[0] = param(c.beta, c.param_dtype, j);
        }
#pragma unroll
        for (int e = 0; e < W; ++e)
            o[e] = r != 0.f ? fmaf((v[k + e] - mu) * r, g[k + e], b[e]) : 0.f;
        if constexpr (VEC)
            store8(y + j, o);
        else
            y[j] = from_float<TY>(o[0]);
    });
    if (t == 0) {
        if (c.mean)
            c.mean[i] = mu;
        if (c.rstd)
            c.rstd[i] = r;
    }
}

// Rows longer than that: three reads, of which the second and third come from the caches.
template <typename TX, typename TY> __global__ void __launch_bounds__(kThreads) k_norm_fwd_long(NormCall c)
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

__device__ __forceinline__ void cp16(void *smem, const void *gmem)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(smem)), "l"(gmem)
                 : "memory");
}

constexpr int kStages = 3;  // rows in flight per group: the one at hand and two ahead

// One pass over x and dy: every thread keeps its columns of gamma, dgamma and dbeta in registers from row to row.
// Group b of all takes rows b, b + groups, ... of the list of supervised tokens (of all tokens, without a list), so that
// the sums are in a fixed order.  Aligned rows come through a ring in shared memory, in which each thread copies and
// reads its own columns only: no barrier but the one of the row's two sums.
template <typename TX, typename TDY, typename TDX, bool VEC, bool WIDE>
__global__ void __launch_bounds__(WIDE ? 512 : 320, WIDE ? 1 : 2) k_norm_bwd(NormGradCall c, const int4 *__restrict__ rows,
                                                  const int32_t *__restrict__ nvalid, int n)
{
    extern __shared__ __align__(16) char ring[];
    __shared__ float2 red[2][16];
    const int t = threadIdx.x % n, group = threadIdx.x / n, warps = n / 32, per = blockDim.x / n;
    const int64_t groups = (int64_t)gridDim.x * per, b = (int64_t)blockIdx.x * per + group;
    const int64_t count = rows ? *nvalid : c.T, steps = (count + groups - 1) / groups;
    const bool layer = c.kind == TURNOPD_LAYER_NORM;
    const float inv_d = 1.f / (float)c.d;
    const size_t xbytes = sizeof(TX) * n * kE, stage = (sizeof(TX) + sizeof(TDY)) * n * kE;
    char *own = ring + group * kStages * stage;

    float gamma[kE], dg[kE], db[kE];
#pragma unroll
    for (int k = 0; k < kE; ++k)
        gamma[k] = dg[k] = db[k] = 0.f;
    each_piece<VEC>(t, n, c.d, [&](int j, int k) {
        if constexpr (VEC)
            load_params8(c.gamma, c.param_dtype, j, gamma + k);
        else
            gamma[k] = param(c.gamma, c.param_dtype, j);
    });

    // the row of a step: -1 for none
    const auto row_of = [&](int64_t m) -> int64_t {
        const int64_t at = m * groups + b;
        if (at >= count)
            return -1;
        return rows ? rows[at].x : at;
    };
    const auto on = [&](int64_t i) { return i >= 0 && (rows || !c.mask || c.mask[i]); };
    const auto copy = [&](int64_t i, int s) {
        if (on(i)) {
            const TX *x = static_cast<const TX *>(c.x) + i * c.ldx;
            const TDY *dy = static_cast<const TDY *>(c.dy) + i * c.lddy;
            char *to = own + s * stage;
            each_piece<true>(t, n, c.d, [&](int j, int) {
#pragma unroll
                for (int h = 0; h < (int)sizeof(TX) / 2; ++h)
                    cp16(to + j * sizeof(TX) + 16 * h, reinterpret_cast<const char *>(x + j) + 16 * h);
#pragma unroll
                for (int h = 0; h < (int)sizeof(TDY) / 2; ++h)
                    cp16(to + xbytes + j * sizeof(TDY) + 16 * h, reinterpret_cast<const char *>(dy + j) + 16 * h);
            });
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    int64_t i = row_of(0), i1 = row_of(1), i2 = row_of(2);
    if constexpr (VEC) {
        copy(i, 0);
        copy(i1, 1);
    }
    float mu = 0.f, r = 0.f;
    if (on(i)) {
        mu = layer ? c.mean[i] : 0.f;
        r = c.rstd[i];
    }
    int s = 0;
    for (int64_t m = 0; m < steps; ++m) {
        const int64_t i3 = row_of(m + 3);
        if constexpr (VEC)
            copy(i2, s >= 1 ? s - 1 : s + 2);
        float mu1 = 0.f, r1 = 0.f;
        if (on(i1)) {
            mu1 = layer ? c.mean[i1] : 0.f;
            r1 = c.rstd[i1];
        }
        const bool part = r > 0.f;
        float x[kE], dy[kE];
        if constexpr (VEC) {
            asm volatile("cp.async.wait_group 2;" ::: "memory");
            if (part)
                each_piece<true>(t, n, c.d, [&](int j, int k) {
                    load8(reinterpret_cast<const TX *>(own + s * stage) + j, x + k);
                    load8(reinterpret_cast<const TDY *>(own + s * stage + xbytes) + j, dy + k);
                });
        } else if (part) {
            each_piece<false>(t, n, c.d, [&](int j, int k) {
                x[k] = to_float(static_cast<const TX *>(c.x)[i * c.ldx + j]);
                dy[k] = to_float(static_cast<const TDY *>(c.dy)[i * c.lddy + j]);
            });
        }
        float sg = 0.f, sx = 0.f;
        if (part)
            each_piece<VEC>(t, n, c.d, [&](int, int k0) {
#pragma unroll
                for (int e = 0; e < (VEC ? 8 : 1); ++e) {
                    const int k = k0 + e;
                    x[k] = (x[k] - mu) * r;
                    const float g = dy[k] * gamma[k];
                    sg += g;
                    sx = fmaf(g, x[k], sx);
                    dg[k] = fmaf(dy[k], x[k], dg[k]);
                    db[k] += dy[k];
                }
            });
        if (c.dx) {
            sg = warp_sum_f(sg);
            sx = warp_sum_f(sx);
            if (warps > 1) {
                float2 *to = red[m & 1];
                if ((threadIdx.x & 31) == 0)
                    to[threadIdx.x >> 5] = make_float2(sg, sx);
                __syncthreads();
                const int first = group * warps;
                sg = to[first].x;
                sx = to[first].y;
                for (int w = 1; w < warps; ++w) {
                    sg += to[first + w].x;
                    sx += to[first + w].y;
                }
            }
            sg = layer ? sg * inv_d : 0.f;
            sx *= inv_d;
            if (i >= 0) {
                TDX *dx = static_cast<TDX *>(c.dx) + i * c.lddx;
                each_piece<VEC>(t, n, c.d, [&](int j, int k) {
                    constexpr int W = VEC ? 8 : 1;
                    float o[W];
#pragma unroll
                    for (int e = 0; e < W; ++e)
                        o[e] = part ? r * (fmaf(dy[k + e], gamma[k + e], -sg) - x[k + e] * sx) : 0.f;
                    if constexpr (VEC)
                        store8(dx + j, o);
                    else
                        dx[j] = from_float<TDX>(o[0]);
                });
            }
        }
        i = i1;
        i1 = i2;
        i2 = i3;
        mu = mu1;
        r = r1;
        s = s == 2 ? 0 : s + 1;
    }
    if (c.dgamma || c.dbeta) {
        float *part = static_cast<float *>(c.workspace) + b * 2 * c.d;
        each_piece<VEC>(t, n, c.d, [&](int j, int k) {
#pragma unroll
            for (int e = 0; e < (VEC ? 8 : 1); ++e) {
                part[j + e] = dg[k + e];
                part[c.d + j + e] = db[k + e];
            }
        });
    }
    // rows of tokens that are not in the list
    if (rows && c.dx) {
        const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, nw = blockDim.x >> 5;
        const int64_t all = (int64_t)gridDim.x * nw, w0 = (int64_t)blockIdx.x * nw + warp;
        for (int64_t k = w0; k < c.T; k += 32 * all) {
            const int64_t mine = k + lane * all;
            unsigned off = __ballot_sync(~0u, mine < c.T && !c.mask[mine]);
            while (off) {
                const int64_t z = k + (__ffs(off) - 1) * all;
                off &= off - 1;
                TDX *dx = static_cast<TDX *>(c.dx) + z * c.lddx;
                if constexpr (VEC) {
                    const float zero[8] = {};
                    for (int64_t j = lane * 8; j < c.d; j += 256)
                        store8(dx + j, zero);
                } else {
                    for (int64_t j = lane; j < c.d; j += 32)
                        dx[j] = from_float<TDX>(0.f);
                }
            }
        }
    }
}

// dgamma and dbeta from n rows of partial sums: 32 columns to a block, the rows shared by its warps.
__global__ void __launch_bounds__(1024) k_norm_bwd_sum(NormGradCall c, int n)
{
    __shared__ float part[32][33];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t j = (int64_t)blockIdx.x * 32 + lane;
    const float *p = static_cast<const float *>(c.workspace) + j;
    float s = 0.f;
    if (j < 2 * c.d) {
#pragma unroll 4
        for (int k = warp; k < n; k += 32)
            s += p[(int64_t)k * 2 * c.d];
    }
    part[warp][lane] = s;
    __syncthreads();
    s = warp_sum_f(part[lane][warp]);  // column `warp` of the block
    const int64_t col = (int64_t)blockIdx.x * 32 + warp;
    if (lane == 0 && col < 2 * c.d) {
        if (col < c.d) {
            if (c.dgamma)
                c.dgamma[col] = s;
        } else if (c.dbeta) {
            c.dbeta[col - c.d] = s;
        }
    }
}

// Rows longer than kMaxBwd.
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

constexpr int kMaxGrid = 320;         // CTAs of the backward pass, at most
constexpr int kLongParts = 64;        // partial sums of the kernels for long rows
constexpr int64_t kListFrom = 4096;   // tokens from which a loss mask is turned into a list of rows

int row_threads(int64_t d) { return (int)((d + kE * 32 - 1) / (kE * 32)) * 32; }
int rows_per_cta(int64_t d) { return std::max(1, kThreads / row_threads(d)); }

int64_t partial_rows(int64_t T, int64_t d)
{
    if (d > kMaxBwd)
        return std::min<int64_t>(std::max<int64_t>(T, 1), kLongParts);
    const int64_t per = rows_per_cta(d);
    return std::min<int64_t>((T + per - 1) / per, kMaxGrid) * per;
}

bool on16(const void *p, int64_t ld, int32_t dtype)
{
    return (reinterpret_cast<uintptr_t>(p) & 15) == 0 && ld * (dtype == TURNOPD_BF16 ? 2 : 4) % 16 == 0;
}

template <typename X, typename DY, typename DX>
cudaError_t launch_bwd(const NormGradCall &c, bool vec, const int4 *rows, const int32_t *nvalid, int *parts,
                       cudaStream_t stream)
{
    const int n = row_threads(c.d), per = rows_per_cta(c.d);
    const int64_t most = std::min<int64_t>(2 * device_sm_count(), kMaxGrid);
    const int grid = (int)std::min<int64_t>((c.T + per - 1) / per, most);
    *parts = grid * per;
    const size_t smem = vec ? (sizeof(X) + sizeof(DY)) * n * per * kE * kStages : 0;
    const bool wide = n * per > 320;  // one CTA per SM then, else two
    auto kernel = wide ? (vec ? k_norm_bwd<X, DY, DX, true, true> : k_norm_bwd<X, DY, DX, false, true>)
                       : (vec ? k_norm_bwd<X, DY, DX, true, false> : k_norm_bwd<X, DY, DX, false, false>);
    if (smem > 48 * 1024) {
        const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (e != cudaSuccess)
            return e;
    }
    kernel<<<grid, n * per, smem, stream>>>(c, rows, nvalid, n);
    return cudaGetLastError();
}

}  // namespace

size_t norm_bwd_workspace_bytes(int64_t T, int64_t d)
{
    const int64_t nblk = (T + kCompactBlock - 1) / kCompactBlock;
    return align256(sizeof(float) * 2 * (size_t)d * (size_t)partial_rows(T, d)) +
           (T >= kListFrom ? align256(sizeof(int4) * (size_t)T) + align256(sizeof(int32_t) * (size_t)(nblk + 1)) + 256 : 0);
}

cudaError_t launch_norm_fwd(const NormCall &c, cudaStream_t stream)
{
    const bool vec = c.d % 8 == 0 && on16(c.x, c.ldx, c.x_dtype) && on16(c.y, c.ldy, c.y_dtype) &&
                     on16(c.gamma, 8, c.param_dtype) && on16(c.beta, 8, c.param_dtype);
    with_types(c.x_dtype, c.y_dtype, [&](auto x, auto y) {
        using X = decltype(x);
        using Y = decltype(y);
        if (c.d > kMaxFwd) {
            const int grid = (int)std::min<int64_t>(c.T, (int64_t)device_sm_count() * 8);
            k_norm_fwd_long<X, Y><<<grid, kThreads, 0, stream>>>(c);
            return;
        }
        const int n = row_threads(c.d), per = rows_per_cta(c.d);
        const unsigned grid = (unsigned)((c.T + per - 1) / per);
        if (vec)
            k_norm_fwd<X, Y, true><<<grid, n * per, 0, stream>>>(c, n);
        else
            k_norm_fwd<X, Y, false><<<grid, n * per, 0, stream>>>(c, n);
    });
    return cudaGetLastError();
}

cudaError_t launch_norm_bwd(const NormGradCall &c, cudaStream_t stream)
{
    cudaError_t e = cudaSuccess;
    int parts = 0;
    const bool sums = c.dgamma || c.dbeta;
    if (c.d > kMaxBwd) {
        with_types(c.x_dtype, c.dy_dtype, [&](auto x, auto dy) {
            using X = decltype(x);
            using DY = decltype(dy);
            const int grid = (int)std::min<int64_t>(c.T, (int64_t)device_sm_count() * 8);
            if (c.dx && c.dx_dtype == TURNOPD_BF16)
                k_norm_dx<X, DY, __nv_bfloat16><<<grid, kThreads, 0, stream>>>(c);
            else if (c.dx)
                k_norm_dx<X, DY, float><<<grid, kThreads, 0, stream>>>(c);
            parts = (int)partial_rows(c.T, c.d);
            if (sums)
                k_norm_params<X, DY><<<dim3((unsigned)((c.d + kThreads - 1) / kThreads), parts), kThreads, 0, stream>>>(c);
        });
        e = cudaGetLastError();
    } else {
        int4 *rows = nullptr;
        int32_t *nvalid = nullptr;
        // Many rows: the supervised ones are listed first, so that every CTA has as many of them.  (Without sums there
        // may be no workspace.)
        if (c.mask && c.T >= kListFrom && sums) {
            const int64_t nblk = (c.T + kCompactBlock - 1) / kCompactBlock;
            char *p = static_cast<char *>(c.workspace) + align256(sizeof(float) * 2 * (size_t)c.d * (size_t)partial_rows(c.T, c.d));
            rows = reinterpret_cast<int4 *>(p);
            p += align256(sizeof(int4) * (size_t)c.T);
            int32_t *blk_count = reinterpret_cast<int32_t *>(p);
            p += align256(sizeof(int32_t) * (size_t)(nblk + 1));
            nvalid = reinterpret_cast<int32_t *>(p);
            LossArgs a{};
            a.mask = c.mask;
            a.num_rows = a.T = c.T;
            a.vocab = 1;
            a.mode = TURNOPD_FULL_VOCAB;
            e = launch_compaction(a, rows, blk_count, nvalid, stream);
            if (e != cudaSuccess)
                return e;
        }
        const bool vec = c.d % 8 == 0 && on16(c.x, c.ldx, c.x_dtype) && on16(c.dy, c.lddy, c.dy_dtype) &&
                         (!c.dx || on16(c.dx, c.lddx, c.dx_dtype)) && on16(c.gamma, 8, c.param_dtype);
        with_types(c.x_dtype, c.dy_dtype, [&](auto x, auto dy) {
            using X = decltype(x);
            using DY = decltype(dy);
            e = c.dx_dtype == TURNOPD_BF16 ? launch_bwd<X, DY, __nv_bfloat16>(c, vec, rows, nvalid, &parts, stream)
                                           : launch_bwd<X, DY, float>(c, vec, rows, nvalid, &parts, stream);
        });
    }
    if (e == cudaSuccess && sums) {
        k_norm_bwd_sum<<<(unsigned)((2 * c.d + 31) / 32), 1024, 0, stream>>>(c, parts);
        e = cudaGetLastError();
    }
    return e;
}

}  // namespace turnopd
