// The norms around a block with its gate and residual connection, and their backward pass.
//
// Row of the residual stream r, of the block's output y:
//   b = N_post(y) (or y), r' = alpha r + s gate b, h = N_pre(r'),   N(x) = (x - mu) r gamma + beta.
// h is taken from r' in fp32, before r' is rounded to the stream's type: each output is rounded once.
// Back, with D = dr' + J_pre^T dh and E = s gate D:
//   dr = alpha D, dy = J_post^T E, dgamma_pre = sum dh xh_pre, dbeta_pre = sum dh, dgamma_post = sum E xh_post,
//   dbeta_post = sum E, dgate = s b D,   J^T g' = r (g - mean g - xh mean(g xh)) with g = g' gamma (no mean g in the
// root-mean-square form).  With a gate per channel the sums over rows are those of D xh_post and D alone:
//   dgamma_post = s gate S, dbeta_post = s gate Z, dgate = s (gamma_post S + beta_post Z).

#include <algorithm>

#include "block_norm.cuh"

namespace turnopd {
namespace {

constexpr int kThreads = 256;

// Sum of two numbers over the block in a fixed order, the same values in every thread.
__device__ __forceinline__ float2 block_sum2(float2 v, float2 *red)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
        v = fadd2(v, make_float2(__shfl_xor_sync(~0u, v.x, o), __shfl_xor_sync(~0u, v.y, o)));
    __syncthreads();
    if ((threadIdx.x & 31) == 0)
        red[threadIdx.x >> 5] = v;
    __syncthreads();
    v = red[0];
#pragma unroll
    for (int w = 1; w < kThreads / 32; ++w)
        v = fadd2(v, red[w]);
    return v;
}

// ---------------------------------------------------------------- rows of any length, column by column

// For rows of more than 8,192 columns, and arrays whose rows begin at different elements of a group of eight: a block to a row,
// whose columns are computed anew for each of its four passes; each thread comes back to its own columns, so r' may be
// written over r.  Bound: instruction issue (every element asks for its arrays' types); 4,096 x 12,288 bf16 540 us, the
// backward pass 1,815 (0.11 and 0.05 of the copy rate).
__global__ void __launch_bounds__(kThreads) k_block_fwd_long(BlockCall c)
{
    __shared__ float2 red[kThreads / 32];
    const int64_t d = c.d;
    const float inv_d = 1.f / (float)d;
    const bool layer = c.kind == TURNOPD_LAYER_NORM;
    for (int64_t i = blockIdx.x; i < c.T; i += gridDim.x) {
        // one thread looks, and all go by what it saw: the sums are the block's
        bool fine = __syncthreads_or(threadIdx.x == 0 && (!c.mask || c.mask[i]));
        float mu[2] = {0.f, 0.f}, r[2] = {0.f, 0.f};
        const auto output = [&](int64_t j) { return param(c.y, c.y_dtype, i * c.ldy + j); };
        const auto stream = [&](int64_t j) {
            float b = output(j);
            if (c.gamma_post)
                b = fmaf((b - mu[0]) * r[0], param(c.gamma_post, c.param_dtype, j),
                         c.beta_post ? param(c.beta_post, c.param_dtype, j) : 0.f);
            float g = c.branch_scale;
            if (c.gate)
                g *= c.ldg ? param(c.gate, c.y_dtype, i * c.ldg + j) : param(c.gate, c.param_dtype, j);
            return fmaf(g, b, c.resid_scale * param(c.resid, c.resid_dtype, i * c.ldr + j));
        };
        const auto statistics = [&](int k, const auto &x) {
            float s = 0.f;
            if (layer) {
                for (int64_t j = threadIdx.x; j < d; j += kThreads)
                    s += x(j);
                mu[k] = block_sum2(make_float2(s, 0.f), red).x / (float)d;
            }
            s = 0.f;
            for (int64_t j = threadIdx.x; j < d; j += kThreads) {
                const float v = x(j) - mu[k];
                s = fmaf(v, v, s);
            }
            r[k] = 1.f / sqrtf(block_sum2(make_float2(s, 0.f), red).x * inv_d + c.eps);
            return isfinite(mu[k]) && isfinite(r[k]) && r[k] > 0.f;
        };
        bool finite = true;
        if (fine && c.gamma_post)
            finite = statistics(0, output);
        if (fine && finite && c.gamma_pre)
            finite = statistics(1, stream);
        if (!finite) {
            fine = false;
            if (threadIdx.x == 0)
                set_status(c.status, TURNOPD_ERR_NONFINITE);
        }
        for (int64_t j = threadIdx.x; j < d; j += kThreads) {
            const float v = fine ? stream(j) : 0.f;
            put(c.resid_out, c.resid_dtype, i * c.ldro + j, v);
            if (c.gamma_pre)
                put(c.h, c.y_dtype, i * c.ldh + j,
                    fine ? fmaf((v - mu[1]) * r[1], param(c.gamma_pre, c.param_dtype, j),
                                c.beta_pre ? param(c.beta_pre, c.param_dtype, j) : 0.f)
                         : 0.f);
        }
        if (c.stats && threadIdx.x == 0)
            reinterpret_cast<float4 *>(c.stats)[i] = fine ? make_float4(mu[0], r[0], mu[1], r[1]) : make_float4(0.f, 0.f, 0.f, 0.f);
    }
}

// ---------------------------------------------------------------- backward, rows of any length

// What the backward pass needs of one column of a row.
struct GradColumn {
    const BlockGradCall &c;
    int64_t i;
    float4 stats;
    __device__ float xh_pre(int64_t j) const
    {
        return (element(c.resid, c.resid_dtype, c.ldr, c.resid_exps, c.d, i, j) - stats.z) * stats.w;
    }
    __device__ float dh(int64_t j) const { return param(c.dh, c.grad_y_dtype, i * c.lddh + j); }
    __device__ float y(int64_t j) const { return element(c.y, c.y_dtype, c.ldy, c.y_exps, c.d, i, j); }
    __device__ float xh_post(int64_t j) const { return c.gamma_post ? (y(j) - stats.x) * stats.y : y(j); }
    // D, given the means of g and of g xh
    __device__ float stream(int64_t j, float2 mean) const
    {
        float v = c.d_resid_out ? param(c.d_resid_out, c.grad_r_dtype, i * c.lddro + j) : 0.f;
        if (c.gamma_pre)
            v = fmaf(fmaf(-xh_pre(j), mean.y, dh(j) * param(c.gamma_pre, c.param_dtype, j) - mean.x), stats.w, v);
        return v;
    }
    __device__ float token_gate(int64_t j) const { return c.gate && c.ldg ? param(c.gate, c.grad_y_dtype, i * c.ldg + j) : 1.f; }
    __device__ float gate(int64_t j) const
    {
        return c.branch_scale * (c.gate && !c.ldg ? param(c.gate, c.param_dtype, j) : token_gate(j));
    }
};

// means of g and of g xh of the norm before the next block
__device__ float2 pre_means(const GradColumn &g, float2 *red, bool layer)
{
    float2 v = make_float2(0.f, 0.f);
    if (!g.c.gamma_pre)
        return v;
    for (int64_t j = threadIdx.x; j < g.c.d; j += kThreads) {
        const float a = g.dh(j) * param(g.c.gamma_pre, g.c.param_dtype, j);
        v.x += a;
        v.y = fmaf(a, g.xh_pre(j), v.y);
    }
    v = block_sum2(v, red);
    return make_float2(layer ? v.x / (float)g.c.d : 0.f, v.y / (float)g.c.d);
}

// A block to a row.  means (or null): where the rows' means of g and g xh go; without it the gradients are written.
__global__ void __launch_bounds__(kThreads) k_block_bwd_long(BlockGradCall c, float2 *means)
{
    __shared__ float2 red[kThreads / 32];
    const int64_t d = c.d;
    const bool layer = c.kind == TURNOPD_LAYER_NORM;
    for (int64_t i = blockIdx.x; i < c.T; i += gridDim.x) {
        GradColumn g{c, i, make_float4(0.f, 0.f, 0.f, 0.f)};
        const bool on = takes_part(c, i, g.stats);
        const bool fine = __syncthreads_or(threadIdx.x == 0 && on);
        const float2 mean = fine ? pre_means(g, red, layer) : make_float2(0.f, 0.f);
        if (means) {
            if (threadIdx.x == 0)
                means[i] = mean;
            continue;
        }
        float2 post = make_float2(0.f, 0.f);
        if (fine && c.gamma_post && c.dy) {
            for (int64_t j = threadIdx.x; j < d; j += kThreads) {
                const float a = g.stream(j, mean) * g.gate(j) * param(c.gamma_post, c.param_dtype, j);
                post.x += a;
                post.y = fmaf(a, g.xh_post(j), post.y);
            }
            post = block_sum2(post, red);
            post = make_float2(layer ? post.x / (float)d : 0.f, post.y / (float)d);
        }
        const bool token_gate = c.gate && c.ldg && c.dgate;
        for (int64_t j = threadIdx.x; j < d; j += kThreads) {
            const float D = fine ? g.stream(j, mean) : 0.f;
            if (c.dy) {
                float e = fine ? D * g.gate(j) : 0.f;
                if (fine && c.gamma_post)
                    e = g.stats.y * fmaf(-g.xh_post(j), post.y, e * param(c.gamma_post, c.param_dtype, j) - post.x);
                put(c.dy, c.grad_y_dtype, i * c.lddy + j, e);
            }
            if (token_gate) {
                float b = 0.f;
                if (fine) {
                    b = g.xh_post(j);
                    if (c.gamma_post)
                        b = fmaf(b, param(c.gamma_post, c.param_dtype, j), c.beta_post ? param(c.beta_post, c.param_dtype, j) : 0.f);
                }
                put(c.dgate, c.grad_y_dtype, i * c.lddg + j, c.branch_scale * D * b);
            }
            if (c.d_resid)
                put(c.d_resid, c.grad_r_dtype, i * c.lddr + j, c.resid_scale * D);
        }
    }
}

// Partial sums over the rows blockIdx.y, blockIdx.y + gridDim.y, ... of 256 columns: of dh xh_pre and dh, of X xh_post and X,
// where X is D (times the gate where it is each token's own).
__global__ void __launch_bounds__(kThreads) k_block_params(BlockGradCall c, const float2 *means)
{
    const int64_t j = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (j >= c.d)
        return;
    const bool pre = c.dgamma_pre || c.dbeta_pre;
    const bool post = c.dgamma_post || c.dbeta_post || (c.dgate && !c.ldg), xh_post = c.dgamma_post || (c.dgate && !c.ldg);
    float s[4] = {0.f, 0.f, 0.f, 0.f};
    for (int64_t i = blockIdx.y; i < c.T; i += gridDim.y) {
        GradColumn g{c, i, make_float4(0.f, 0.f, 0.f, 0.f)};
        if (!takes_part(c, i, g.stats))
            continue;
        if (pre) {
            const float dh = g.dh(j);
            s[0] = fmaf(dh, g.xh_pre(j), s[0]);
            s[1] += dh;
        }
        if (post) {
            const float x = g.stream(j, means[i]) * g.token_gate(j);
            if (xh_post)
                s[2] = fmaf(x, g.xh_post(j), s[2]);
            s[3] += x;
        }
    }
    float *part = static_cast<float *>(c.workspace) + (int64_t)blockIdx.y * 4 * c.d;
    for (int k = 0; k < 4; ++k)
        part[k * c.d + j] = s[k];
}

// The parameters' gradients from n rows of partial sums: 32 columns to a block, the rows shared by its 32 warps (152 rows of
// 4 x 5,120: 10 us with eight).
__global__ void __launch_bounds__(1024) k_block_bwd_sum(BlockGradCall c, int n, bool bias)
{
    __shared__ float part[4][32][33];
    pdl_begin();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t first = (int64_t)blockIdx.x * 32;
    {
        const float *p = static_cast<const float *>(c.workspace) + min(first + lane, c.d - 1);
        float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
        for (int k = warp; k < n; k += 32)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                if (bias || !(q & 1))
                    s[q] += p[((int64_t)k * 4 + q) * c.d];
#pragma unroll
        for (int q = 0; q < 4; ++q)
            part[q][warp][lane] = s[q];
    }
    __syncthreads();
    const int64_t j = first + warp;  // a column to each warp
    float s[4];
#pragma unroll
    for (int q = 0; q < 4; ++q)
        s[q] = warp_sum_f(part[q][lane][warp]);
    if (lane || j >= c.d)
        return;
    if (c.dgamma_pre)
        c.dgamma_pre[j] = s[0];
    if (c.dbeta_pre)
        c.dbeta_pre[j] = s[1];
    const bool channel = c.gate && !c.ldg;
    const float g = c.branch_scale * (channel ? param(c.gate, c.param_dtype, j) : 1.f);
    if (c.dgamma_post)
        c.dgamma_post[j] = g * s[2];
    if (c.dbeta_post)
        c.dbeta_post[j] = g * s[3];
    if (channel && c.dgate) {
        float b = s[2];
        if (c.gamma_post)
            b = fmaf(param(c.gamma_post, c.param_dtype, j), b, c.beta_post ? param(c.beta_post, c.param_dtype, j) * s[3] : 0.f);
        static_cast<float *>(c.dgate)[j] = c.branch_scale * b;
    }
}

constexpr int kLongParts = 64;

int64_t partial_rows(int64_t T, int64_t d)
{
    // (eight groups of rows at least where the rows begin anywhere)
    return d > kBlockMaxRow ? std::min<int64_t>(std::max<int64_t>(T, 1), kLongParts) : std::min<int64_t>(T + 8, kBlockMaxParts);
}

}  // namespace

bool block_bwd_bias(const BlockGradCall &c) { return c.dbeta_pre || c.dbeta_post || (c.dgate && !c.ldg && c.beta_post); }

bool block_bwd_general(const BlockGradCall &c)
{
    return c.kind == TURNOPD_LAYER_NORM || block_bwd_bias(c) || (c.dgate && c.ldg && c.beta_post);
}

bool block_bwd_needs_y(const BlockGradCall &c) { return c.gamma_post ? c.dy || c.dgamma_post || c.dgate : c.dgate != nullptr; }

size_t block_bwd_workspace_bytes(int64_t T, int64_t d)
{
    return align256(sizeof(float) * 4 * (size_t)d * (size_t)partial_rows(T, d)) + align256(sizeof(float2) * (size_t)T);
}

cudaError_t launch_block_fwd(const BlockCall &c, cudaStream_t stream)
{
    const Phases phases{Phase(c.resid, c.ldr, c.resid_dtype), Phase(c.y, c.ldy, c.y_dtype), Phase(c.resid_out, c.ldro, c.resid_dtype),
                        Phase(c.h, c.ldh, c.y_dtype), Phase(c.ldg ? c.gate : nullptr, c.ldg, c.y_dtype)};
    if (c.d > kBlockMaxRow || !phases.alike) {
        const unsigned grid = (unsigned)std::min<int64_t>(c.T, (int64_t)device_sm_count() * 8);
        k_block_fwd_long<<<grid, kThreads, 0, stream>>>(c);
        return cudaGetLastError();
    }
    cudaError_t e = cudaSuccess;
    with_types(c.resid_dtype, c.y_dtype, [&](auto r, auto y) { e = launch_block_rows_fwd<decltype(r), decltype(y)>(c, phases, stream); });
    return e;
}

cudaError_t launch_block_bwd(const BlockGradCall &c, cudaStream_t stream)
{
    const bool sums = c.dgamma_pre || c.dbeta_pre || c.dgamma_post || c.dbeta_post || (c.dgate && !c.ldg);
    int parts = 0;
    cudaError_t e = cudaSuccess;
    bool bias = block_bwd_bias(c), taken = false;
    if (c.d <= kBlockMaxRow)
        with_types(c.grad_r_dtype, c.grad_y_dtype,
                   [&](auto r, auto y) { e = launch_block_rows_bwd<decltype(r), decltype(y)>(c, &parts, &taken, stream); });
    if (!taken && e == cudaSuccess) {
        const unsigned grid = (unsigned)std::min<int64_t>(c.T, (int64_t)device_sm_count() * 8);
        parts = (int)std::min<int64_t>(c.T, kLongParts);
        bias = true;
        if (sums) {
            // before d_resid is written, which may be d_resid_out
            float2 *means = reinterpret_cast<float2 *>(static_cast<char *>(c.workspace) +
                                                       align256(sizeof(float) * 4 * (size_t)c.d * (size_t)partial_rows(c.T, c.d)));
            k_block_bwd_long<<<grid, kThreads, 0, stream>>>(c, means);
            k_block_params<<<dim3((unsigned)((c.d + kThreads - 1) / kThreads), parts), kThreads, 0, stream>>>(c, means);
        }
        if (c.d_resid || c.dy || (c.dgate && c.ldg))
            k_block_bwd_long<<<grid, kThreads, 0, stream>>>(c, nullptr);
        e = cudaGetLastError();
    }
    if (e == cudaSuccess && sums)
        e = launch_dependent(k_block_bwd_sum, dim3((unsigned)((c.d + 31) / 32)), dim3(1024), 0, stream, c, parts, bias);
    return e;
}

}  // namespace turnopd
