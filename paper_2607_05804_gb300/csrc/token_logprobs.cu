// Log probabilities of given tokens with the row's entropy and top alternatives, and their
// gradient with respect to the logits.
//
// Row z[0..V), m = max z, S = sum e^{z-m}:
//   log p_v = (z_v - m) - log S,   H = log S - A / S,   A = sum e^{z-m} (z - m),
//   dL/dz_v = dL/dlp (delta_vy - p_v) - dL/dH p_v (log p_v + H).
// The sums leave the given token y out and take its term at the end: where y is all but certain,
// log p_y = -log1p(S') with S' = sum_{v != y} e^{z-m} keeps its relative precision, and so does
// H = log1p(S') - A / S, whose two terms then have one sign.

#include <algorithm>

#include "common.cuh"
#include "kernels.h"

namespace turnopd {
namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;

// A row whose largest logit lies at or below this holds nothing but masked values.
constexpr float kMaskedBelow = -0x1.8p+126f;

struct Row {
    int32_t token, r, y;
    bool ok;
};

// Item k of the row list; without one (no loss mask) token k itself, its indexes checked here.
template <typename Call> __device__ __forceinline__ Row get_row(const Call &c, const int4 *rows, int64_t k)
{
    if (rows) {
        const int4 v = rows[k];
        return Row{v.x, v.y, v.z, true};
    }
    Row o{(int32_t)k, c.row_of_token ? c.row_of_token[k] : (int32_t)k, c.token_ids ? c.token_ids[k] : -1, true};
    o.ok = o.r >= 0 && o.r < c.num_rows && (!c.token_ids || (o.y >= 0 && o.y < c.vocab));
    if (!o.ok && threadIdx.x == 0)
        set_status(c.status, TURNOPD_ERR_TOKEN_RANGE);
    return o;
}

// Running maximum, S and A of part of a row.
struct Part {
    float m, s, a;
};

__device__ __forceinline__ Part part_merge(Part x, Part y)
{
    const float m = fmaxf(x.m, y.m);
    if (m == -INFINITY)
        return x;
    Part o{m, 0.f, 0.f};
    if (x.m != -INFINITY) {
        const float f = expf(x.m - m);
        o.s = x.s * f;
        o.a = f == 0.f ? 0.f : fmaf(x.s, x.m - m, x.a) * f;
    }
    if (y.m != -INFINITY) {
        const float f = expf(y.m - m);
        o.s += y.s * f;
        o.a += f == 0.f ? 0.f : fmaf(y.s, y.m - m, y.a) * f;
    }
    return o;
}

// Order of the alternatives: by logit, then the lower id first.
__device__ __forceinline__ uint64_t top_key(float z, int64_t v)
{
    const uint32_t u = __float_as_uint(z + 0.f);  // -0 becomes +0
    const uint32_t k = (u & 0x80000000u) ? ~u : (u | 0x80000000u);
    return ((uint64_t)k << 32) | (0xffffffffu - (uint32_t)v);
}
__device__ __forceinline__ uint32_t key_id(uint64_t k) { return 0xffffffffu - (uint32_t)k; }
__device__ __forceinline__ float key_logit(uint64_t k)
{
    const uint32_t u = (uint32_t)(k >> 32);
    return __uint_as_float((u & 0x80000000u) ? (u & 0x7fffffffu) : ~u);
}

// A token without a distribution: masked (m = 0), or out of range or of a row that is not finite (m = -inf, by
// which the backward pass knows it).
__device__ __forceinline__ void write_nothing(const LogprobCall &c, int64_t i, float m)
{
    if (c.logprob)
        c.logprob[i] = 0.f;
    if (c.entropy)
        c.entropy[i] = 0.f;
    if (c.stats) {
        c.stats[2 * i] = m;
        c.stats[2 * i + 1] = 0.f;
    }
    for (int k = 0; k < c.n_top; ++k) {
        c.top_ids[i * c.n_top + k] = -1;
        c.top_logprob[i * c.n_top + k] = 0.f;
    }
}

template <typename TIn>
__global__ void __launch_bounds__(kThreads) k_logprobs(LogprobCall c, const int4 *__restrict__ rows,
                                                       const int32_t *__restrict__ nvalid)
{
    __shared__ Part parts[kWarps];
    __shared__ uint64_t keys[kWarps];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t n = rows ? *nvalid : c.T;
    for (int64_t k = blockIdx.x; k < n; k += gridDim.x) {
        const Row row = get_row(c, rows, k);
        if (!row.ok) {
            if (threadIdx.x == 0)
                write_nothing(c, row.token, -INFINITY);
            continue;
        }
        const TIn *z = static_cast<const TIn *>(c.logits) + (int64_t)row.r * c.ld;
        Part p{-INFINITY, 0.f, 0.f};
        for (int64_t v = threadIdx.x; v < c.vocab; v += kThreads) {
            const float x = to_float(z[v]);
            if (v == row.y || x == -INFINITY)
                continue;
            if (!(x < INFINITY))
                p.m = INFINITY;  // NaN or +inf: the row is reported
            if (x > p.m)
                p = part_merge(p, Part{x, 0.f, 0.f});
            const float e = expf(x - p.m);
            p.s += e;
            p.a = e == 0.f ? p.a : fmaf(e, x - p.m, p.a);
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1)
            p = part_merge(p, Part{__shfl_xor_sync(~0u, p.m, o), __shfl_xor_sync(~0u, p.s, o),
                                   __shfl_xor_sync(~0u, p.a, o)});
        __syncthreads();
        if (lane == 0)
            parts[warp] = p;
        __syncthreads();
        p = parts[0];
        for (int w = 1; w < kWarps; ++w)
            p = part_merge(p, parts[w]);
        const float zy = row.y >= 0 ? to_float(z[row.y]) : -INFINITY;
        const Part all = part_merge(p, Part{zy, row.y >= 0 ? 1.f : 0.f, 0.f});
        const float logs = row.y >= 0 && zy == all.m ? log1pf(p.m == -INFINITY ? 0.f : p.s * expf(p.m - zy))
                                                     : logf(all.s);
        const bool fine = all.m > kMaskedBelow && all.m < INFINITY && isfinite(logs) && isfinite(all.a) && zy == zy;
        if (!fine) {
            if (threadIdx.x == 0) {
                set_status(c.status, TURNOPD_ERR_NONFINITE);
                write_nothing(c, row.token, -INFINITY);
            }
            continue;
        }
        const int64_t i = row.token;
        if (threadIdx.x == 0) {
            if (c.logprob)
                c.logprob[i] = (zy - all.m) - logs;
            if (c.entropy)
                c.entropy[i] = logs - all.a / all.s;
            if (c.stats) {
                c.stats[2 * i] = all.m;
                c.stats[2 * i + 1] = logs;
            }
        }
        uint64_t below = ~0ull;
        for (int t = 0; t < c.n_top; ++t) {
            uint64_t best = 0;
            for (int64_t v = threadIdx.x; v < c.vocab; v += kThreads) {
                const uint64_t key = top_key(to_float(z[v]), v);
                if (key < below && key > best)
                    best = key;
            }
#pragma unroll
            for (int o = 16; o > 0; o >>= 1)
                best = max(best, (uint64_t)__shfl_xor_sync(~0u, (unsigned long long)best, o));
            __syncthreads();
            if (lane == 0)
                keys[warp] = best;
            __syncthreads();
            for (int w = 0; w < kWarps; ++w)
                best = max(best, keys[w]);
            below = best;
            if (threadIdx.x == 0) {
                c.top_ids[i * c.n_top + t] = (int32_t)key_id(best);
                c.top_logprob[i * c.n_top + t] = (key_logit(best) - all.m) - logs;
            }
        }
    }
    // tokens that are not in the row list
    if (rows) {
        for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < c.T; i += (int64_t)gridDim.x * kThreads) {
            const bool on = c.mask[i] != 0;
            bool listed = on;
            if (listed && c.row_of_token)
                listed = c.row_of_token[i] >= 0 && c.row_of_token[i] < c.num_rows;
            if (listed && c.token_ids)
                listed = c.token_ids[i] >= 0 && c.token_ids[i] < c.vocab;
            if (!listed)
                write_nothing(c, i, on ? -INFINITY : 0.f);
        }
    }
}

template <typename TIn, typename TOut>
__global__ void __launch_bounds__(kThreads) k_logprobs_bwd(LogprobGradCall c, const int4 *__restrict__ rows,
                                                           const int32_t *__restrict__ nvalid)
{
    const int64_t n = rows ? *nvalid : c.T;
    for (int64_t k = blockIdx.x; k < n; k += gridDim.x) {
        const Row row = get_row(c, rows, k);
        if (!row.ok)
            continue;
        // no __restrict__: the gradient may be written over the logits
        const TIn *z = static_cast<const TIn *>(c.logits) + (int64_t)row.r * c.ld;
        TOut *g = static_cast<TOut *>(c.grad) + (int64_t)row.r * c.ld;
        const int64_t i = row.token;
        const float m = c.stats[2 * i], logs = c.stats[2 * i + 1];
        const bool fine = m > -INFINITY;
        const float gl = c.d_logprob ? c.d_logprob[i] : 0.f;
        const float gh = c.d_entropy ? c.d_entropy[i] : 0.f, H = c.d_entropy ? c.entropy[i] : 0.f;
        for (int64_t v = threadIdx.x; v < c.vocab; v += kThreads) {
            const float lp = fmaxf((to_float(z[v]) - m) - logs, -1e4f);
            const float p = expf(lp);
            float o = -p * fmaf(gh, lp + H, gl);
            if (v == row.y && c.d_logprob)
                o = fmaf(-gl, expm1f(c.logprob[i]), -p * (gh * (lp + H)));
            g[v] = from_float<TOut>(fine ? o : 0.f);
        }
    }
}

template <typename Call> struct Lists {
    int4 *rows = nullptr;
    int32_t *nvalid = nullptr;
    cudaError_t make(const Call &c, cudaStream_t stream)
    {
        if (!c.mask)
            return cudaSuccess;
        const int64_t nblk = (c.T + kCompactBlock - 1) / kCompactBlock;
        char *p = static_cast<char *>(c.workspace);
        rows = reinterpret_cast<int4 *>(p);
        p += align256(sizeof(int4) * (size_t)c.T);
        int32_t *blk_count = reinterpret_cast<int32_t *>(p);
        p += align256(sizeof(int32_t) * (size_t)(nblk + 1));
        nvalid = reinterpret_cast<int32_t *>(p);
        LossArgs a{};
        a.mask = c.mask;
        a.row_of_token = c.row_of_token;
        a.sampled_ids = c.token_ids;
        a.num_rows = c.num_rows;
        a.vocab = c.vocab;
        a.T = c.T;
        a.mode = c.token_ids ? TURNOPD_SAMPLED_TOKEN : TURNOPD_FULL_VOCAB;
        a.status = c.status;
        return launch_compaction(a, rows, blk_count, nvalid, stream);
    }
};

}  // namespace

size_t logprob_workspace_bytes(int64_t T)
{
    const int64_t nblk = (T + kCompactBlock - 1) / kCompactBlock;
    return align256(sizeof(int4) * (size_t)T) + align256(sizeof(int32_t) * (size_t)(nblk + 1)) + 256;
}

cudaError_t launch_token_logprobs(const LogprobCall &c, cudaStream_t stream)
{
    Lists<LogprobCall> l;
    const cudaError_t e = l.make(c, stream);
    if (e != cudaSuccess)
        return e;
    const int grid = (int)std::min<int64_t>(c.T, (int64_t)device_sm_count() * 8);
    if (c.in_dtype == TURNOPD_BF16)
        k_logprobs<__nv_bfloat16><<<grid, kThreads, 0, stream>>>(c, l.rows, l.nvalid);
    else
        k_logprobs<float><<<grid, kThreads, 0, stream>>>(c, l.rows, l.nvalid);
    return cudaGetLastError();
}

cudaError_t launch_token_logprobs_bwd(const LogprobGradCall &c, cudaStream_t stream)
{
    Lists<LogprobGradCall> l;
    const cudaError_t e = l.make(c, stream);
    if (e != cudaSuccess)
        return e;
    if (c.mask && (c.flags & TURNOPD_ZERO_MASKED_GRAD))
        launch_zero_masked_grad(c.mask, c.row_of_token, c.T, c.num_rows, c.ld, c.vocab, c.grad, c.grad_dtype, stream);
    const int grid = (int)std::min<int64_t>(c.T, (int64_t)device_sm_count() * 8);
    const bool in16 = c.in_dtype == TURNOPD_BF16, out16 = c.grad_dtype == TURNOPD_BF16;
    if (in16 && out16)
        k_logprobs_bwd<__nv_bfloat16, __nv_bfloat16><<<grid, kThreads, 0, stream>>>(c, l.rows, l.nvalid);
    else if (in16)
        k_logprobs_bwd<__nv_bfloat16, float><<<grid, kThreads, 0, stream>>>(c, l.rows, l.nvalid);
    else if (out16)
        k_logprobs_bwd<float, __nv_bfloat16><<<grid, kThreads, 0, stream>>>(c, l.rows, l.nvalid);
    else
        k_logprobs_bwd<float, float><<<grid, kThreads, 0, stream>>>(c, l.rows, l.nvalid);
    return cudaGetLastError();
}

}  // namespace turnopd
