// Rows of the forward pass of the norms around a block, which a block's threads hold in their registers.
#pragma once

#include <algorithm>
#include <type_traits>

#include "block_norm.cuh"

namespace turnopd {
namespace {

// Eight columns of a row as they are stored.
template <typename T> struct Raw8 {
    static constexpr int kWords = sizeof(T) / 2;  // of 16 bytes
    uint4 w[kWords];
    __device__ void load(const T *p)
    {
#pragma unroll
        for (int k = 0; k < kWords; ++k)
            w[k] = __ldcs(reinterpret_cast<const uint4 *>(p) + k);
    }
    __device__ void clear()
    {
#pragma unroll
        for (int k = 0; k < kWords; ++k)
            w[k] = make_uint4(0u, 0u, 0u, 0u);
    }
    __device__ float2 pair(int e) const
    {
        if constexpr (sizeof(T) == 2)
            return unpack2(word(w[0], e));
        else
            return make_float2(__uint_as_float(word(w[e / 2], 2 * (e & 1))), __uint_as_float(word(w[e / 2], 2 * (e & 1) + 1)));
    }
};

// The vectors of the call in fp32, with the gate per channel and the branch's scale multiplied into those of the first norm:
//   r' = alpha r + factor xh [gate] + shift [gate],  h = gamma xh' + beta.
enum Vector { kFactor, kGamma, kShift, kBeta };
__device__ __forceinline__ float vector_column(const BlockCall &c, int v, int j)
{
    if (v == kGamma)
        return c.gamma_pre ? param(c.gamma_pre, c.param_dtype, j) : 0.f;
    if (v == kBeta)
        return c.beta_pre ? param(c.beta_pre, c.param_dtype, j) : 0.f;
    const float s = c.gate && !c.ldg ? c.branch_scale * param(c.gate, c.param_dtype, j) : c.branch_scale;
    if (v == kFactor)
        return c.gamma_post ? s * param(c.gamma_post, c.param_dtype, j) : s;
    return c.beta_post ? s * param(c.beta_post, c.param_dtype, j) : 0.f;
}

// Eight columns of them from j on.
template <int N> __device__ __forceinline__ void vector_columns(const BlockCall &c, int j, int d, float2 (&o)[N][4])
{
    float g[8], gate[8], beta[8];
    float *f[4];
#pragma unroll
    for (int v = 0; v < N; ++v)
        f[v] = reinterpret_cast<float *>(o[v]);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        g[e] = gate[e] = 1.f;
        beta[e] = f[kGamma][e] = 0.f;
        if (N > 2)
            f[N > 2 ? kBeta : 0][e] = 0.f;
    }
    if (c.gamma_post)
        param8(c.gamma_post, c.param_dtype, j, d, g);
    if (c.gate && !c.ldg)
        param8(c.gate, c.param_dtype, j, d, gate);
    if (N > 2 && c.beta_post)
        param8(c.beta_post, c.param_dtype, j, d, beta);
    if (c.gamma_pre)
        param8(c.gamma_pre, c.param_dtype, j, d, f[kGamma]);
    if (N > 2 && c.beta_pre)
        param8(c.beta_pre, c.param_dtype, j, d, f[N > 2 ? kBeta : 0]);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float s = c.branch_scale * gate[e];
        f[kFactor][e] = s * g[e];
        if (N > 2)
            f[N > 2 ? kShift : 0][e] = s * beta[e];
    }
}

// n threads take a row, P pieces of eight columns to a thread, kept as they were read until r' is there; then the loads of
// the group's next row go out, and that row's bytes arrive while this one's second norm is taken and its results are written.
// With several pieces the vectors lie in shared memory: the halves of the pieces in a plane each, so that neighbouring
// threads' lie next to each other.  With one piece, for few rows, a thread keeps its columns of them in registers.
//
// Bound: HBM.  32,768 x 4,096 bf16 with both norms and a gate per channel 171 us (6,270 GB/s, 0.92 of the copy rate), with an
// fp32 stream 269 (0.88), layer norms 205 (0.77: two more sums and two more vectors to a row), a gate for every element 221
// (0.90); 16,384 x 8,192 167 (0.95); 32,768 x 1,001 60 (0.65); one row of 4,096 3.0 on the device.
//
// ENDS: the rows begin anywhere, but in all arrays at the same element of a group of eight: pieces from the row's first
// boundary on, and the first threads one of the elements before and after them each.  The groups' number is a multiple of
// eight, so that all rows of one group begin at the same element.  The vectors lie in eight planes of every eighth column then.
// GENERAL: layer norms, or betas.
template <typename TR, typename TY, int P, bool GATE, bool ENDS, bool GENERAL, int MOST, int PER_SM>
__global__ void __launch_bounds__(MOST, PER_SM) k_block_fwd(BlockCall c, int n, int phase, int phase_step)
{
    constexpr int kVectors = GENERAL ? 4 : 2;
    constexpr bool kHeld = P == 1;
    extern __shared__ __align__(16) float vectors[];
    __shared__ float red[4][32];
    const int t = threadIdx.x % n, group = threadIdx.x / n, warps = n / 32, per = blockDim.x / n, d = (int)c.d;
    const int64_t groups = (int64_t)gridDim.x * per, b = (int64_t)blockIdx.x * per + group;
    const bool layer = GENERAL && c.kind == TURNOPD_LAYER_NORM, pre = c.gamma_pre, post = c.gamma_post;
    const float inv_d = 1.f / (float)d;
    int sums = 0;  // taken so far: the next one's place in `red`, which is free again two sums later

    const int head = ENDS ? min((8 - (int)((phase + b * phase_step) & 7)) & 7, d) : 0;
    const int whole = (d - head) / 8, ends = ENDS ? d - whole * 8 : 0;
    const int end = t < head ? t : whole * 8 + t;  // the single column of this thread, where t < ends
    const bool at_end = ENDS && t < ends;
    const int piece0 = (t >> 5) * 32 * P + (t & 31);
    const auto column = [&](int k) { return head + (piece0 + 32 * k) * 8; };  // the first of piece k
    const auto there = [&](int k) { return piece0 + 32 * k < whole; };

    Raw8<TR> r[P];
    Raw8<TY> y[P], g[GATE ? P : 1];
    float re = 0.f, ye = 0.f, ge = 0.f;
    bool on = false;
    const auto load = [&](int64_t i) {
        on = i < c.T && (!c.mask || c.mask[i]);
        const TR *rr = static_cast<const TR *>(c.resid) + i * c.ldr;
        const TY *yy = static_cast<const TY *>(c.y) + i * c.ldy, *gg = static_cast<const TY *>(c.gate) + i * c.ldg;
#pragma unroll
        for (int k = 0; k < P; ++k)
            if (on && there(k)) {
                y[k].load(yy + column(0) + k * 256);
                r[k].load(rr + column(0) + k * 256);
                if (GATE)
                    g[GATE ? k : 0].load(gg + column(0) + k * 256);
            } else {
                r[k].clear();
                y[k].clear();
                if (GATE)
                    g[GATE ? k : 0].clear();
            }
        if (ENDS) {
            re = on && at_end ? to_float(rr[end]) : 0.f;
            ye = on && at_end ? to_float(yy[end]) : 0.f;
            ge = GATE && on && at_end ? to_float(gg[end]) : 0.f;
        }
    };
    load(b);

    const int plane = ENDS ? d / 8 + 2 : (d + 7) / 8;  // floats, or groups of four
    float2 held[kHeld ? kVectors : 1][4];
    if constexpr (kHeld) {
        vector_columns<kVectors>(c, whole > 0 ? min(column(0), d - 8) : 0, d, held);
    } else {
        for (int piece = threadIdx.x; piece < (d + 7) / 8; piece += blockDim.x) {
            float2 o[kVectors][4];
            vector_columns<kVectors>(c, piece * 8, d, o);
#pragma unroll
            for (int v = 0; v < kVectors; ++v) {
                const float *f = reinterpret_cast<const float *>(o[v]);
                if constexpr (ENDS) {
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        vectors[(v * 8 + e) * plane + piece] = f[e];
                } else {
                    float4 *to = reinterpret_cast<float4 *>(vectors) + v * 2 * plane + piece;
                    to[0] = make_float4(f[0], f[1], f[2], f[3]);
                    to[plane] = make_float4(f[4], f[5], f[6], f[7]);
                }
            }
        }
        __syncthreads();
    }
    float end_of[kVectors];
#pragma unroll
    for (int v = 0; v < kVectors; ++v)
        end_of[v] = at_end ? vector_column(c, v, end) : 0.f;
    const auto vector = [&](int v, int k, float2 *o) {  // (of a missing piece: the first one's)
        const int at = there(k) ? piece0 + 32 * k : 0;
        if constexpr (kHeld) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                o[e] = held[v][e];
        } else if constexpr (ENDS) {
            const float *p = vectors + v * 8 * plane;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int j = head + e;
                reinterpret_cast<float *>(o)[e] = p[(j & 7) * plane + (j >> 3) + at];
            }
        } else {
            const float4 *p = reinterpret_cast<const float4 *>(vectors) + v * 2 * plane + at;
            const float4 x = p[0], z = p[plane];
            o[0] = make_float2(x.x, x.y), o[1] = make_float2(x.z, x.w);
            o[2] = make_float2(z.x, z.y), o[3] = make_float2(z.z, z.w);
        }
    };

    // mu and rho of the columns that x(k, e) gives in pairs, and of a single one; missing columns are zeros.  The sums are
    // taken for rows that do not take part too: no barrier stands under a condition that every thread reads from the
    // caller's memory for itself.
    const auto statistics = [&](const auto &x, float xe, float &mu, float &rho) {
        mu = 0.f;
        if (layer) {
            float2 s = make_float2(xe, 0.f);
#pragma unroll
            for (int k = 0; k < P; ++k)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    s = fadd2(s, x(k, e));
            // divided, not times 1/d: a sum that is exact (a row of equal numbers) has its exact mean
            mu = group_sum(s.x + s.y, red[sums++ & 3], group, warps) / (float)d;
        }
        float2 q = make_float2(at_end ? (xe - mu) * (xe - mu) : 0.f, 0.f);
#pragma unroll
        for (int k = 0; k < P; ++k)
            if (!GENERAL || there(k))
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float2 v = GENERAL ? fadd2(x(k, e), splat(-mu)) : x(k, e);
                    q = ffma2(v, v, q);
                }
        rho = rsqrtf(group_sum(q.x + q.y, red[sums++ & 3], group, warps) * inv_d + c.eps);  // within two units of the last place
        return isfinite(mu) && isfinite(rho) && rho > 0.f;
    };
    for (int64_t i = b; i < c.T; i += groups) {
        bool fine = on;
        float mu0 = 0.f, rho0 = 0.f, mu1 = 0.f, rho1 = 0.f;
        if (post)
            fine = statistics([&](int k, int e) { return y[k].pair(e); }, ye, mu0, rho0) && fine;
        const float scale = post ? rho0 : 1.f;
        float2 v[P][4];
#pragma unroll
        for (int k = 0; k < P; ++k) {
            float2 a[4];
            vector(kFactor, k, a);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                v[k][e] = y[k].pair(e);
                if (GENERAL)
                    v[k][e] = fadd2(v[k][e], splat(-mu0));
                v[k][e] = fmul2(v[k][e], splat(scale));
            }
            if (GENERAL) {
                float2 z[4];
                vector(kShift, k, z);
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    v[k][e] = ffma2(v[k][e], a[e], z[e]);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    v[k][e] = fmul2(v[k][e], a[e]);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e)
                v[k][e] = ffma2(r[k].pair(e), splat(c.resid_scale), GATE ? fmul2(v[k][e], g[GATE ? k : 0].pair(e)) : v[k][e]);
        }
        float ve = 0.f;
        if (ENDS) {
            ve = fmaf((ye - mu0) * scale, end_of[kFactor], GENERAL ? end_of[GENERAL ? kShift : 0] : 0.f);
            ve = at_end ? fmaf(re, c.resid_scale, GATE ? ve * ge : ve) : 0.f;
        }
        const bool took_part = on;
        load(i + groups);
        if (pre) {
            const bool finite = statistics([&](int k, int e) { return GENERAL && !there(k) ? make_float2(0.f, 0.f) : v[k][e]; }, ve, mu1, rho1);
            fine = finite && fine;
        }
        if (took_part && !fine && t == 0)
            set_status(c.status, TURNOPD_ERR_NONFINITE);
        TR *out = static_cast<TR *>(c.resid_out) + i * c.ldro;
        TY *h = static_cast<TY *>(c.h) + i * c.ldh;
        if (!fine) {
#pragma unroll
            for (int k = 0; k < P; ++k)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    v[k][e] = make_float2(0.f, 0.f);
            ve = mu0 = rho0 = mu1 = rho1 = 0.f;
        }
#pragma unroll
        for (int k = 0; k < P; ++k)
            if (there(k))
                store8(out + column(0) + k * 256, reinterpret_cast<const float *>(v[k]));
        if (at_end)
            out[end] = from_float<TR>(ve);
        if (pre) {
            if (fine) {
#pragma unroll
                for (int k = 0; k < P; ++k) {
                    float2 a[4];
                    vector(kGamma, k, a);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        if (GENERAL)
                            v[k][e] = fadd2(v[k][e], splat(-mu1));
                        v[k][e] = fmul2(v[k][e], splat(rho1));
                    }
                    if (GENERAL) {
                        float2 z[4];
                        vector(kBeta, k, z);
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            v[k][e] = ffma2(v[k][e], a[e], z[e]);
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            v[k][e] = fmul2(v[k][e], a[e]);
                    }
                }
                ve = fmaf((ve - mu1) * rho1, end_of[kGamma], GENERAL ? end_of[GENERAL ? kBeta : 0] : 0.f);
            }
#pragma unroll
            for (int k = 0; k < P; ++k)
                if (there(k))
                    store8(h + column(0) + k * 256, reinterpret_cast<const float *>(v[k]));
            if (at_end)
                h[end] = from_float<TY>(ve);
        }
        if (c.stats && t == 0)
            reinterpret_cast<float4 *>(c.stats)[i] = make_float4(mu0, rho0, mu1, rho1);
    }
}

template <typename TR, typename TY, bool GATE, int P, int MOST, int PER_SM>
cudaError_t launch_rows(const BlockCall &c, const Phases &phases, cudaStream_t stream)
{
    const int n = (int)((c.d + P * 256 - 1) / (P * 256)) * 32, per = std::max(1, 256 / n);
    const int64_t blocks = (c.T + per - 1) / per;
    const bool ends = phases.at || phases.step || c.d % 8;
    const bool general = c.kind == TURNOPD_LAYER_NORM || c.beta_post || c.beta_pre;
    const auto go = [&](auto kernel, auto has_ends, auto is_general) {
        constexpr bool E = decltype(has_ends)::value;
        constexpr size_t kVectorBytes = sizeof(float) * (decltype(is_general)::value ? 4 : 2) * 8;
        const auto bytes = [&](int64_t d) { return P == 1 ? (size_t)0 : kVectorBytes * (size_t)(E ? d / 8 + 2 : (d + 7) / 8); };
        // as many CTAs as are resident at once, of which each SM's shared memory limits some
        const size_t smem = bytes(c.d);
        const int resident = std::min<int>(std::max((P == 1 && n == 32 ? 1024 : PER_SM * MOST) / (n * per), 1), (int)(220 * 1024 / (smem + 1024)));
        int64_t grid = std::min<int64_t>(blocks, (int64_t)device_sm_count() * resident);
        if (E)
            grid = (grid * per + 7) / 8 * 8 / per;  // a multiple of eight groups
        const cudaError_t e = allow_shared(kernel, bytes(kBlockMaxRow));
        if (e != cudaSuccess)
            return e;
        kernel<<<(unsigned)grid, n * per, smem, stream>>>(c, n, phases.at, phases.step);
        return cudaGetLastError();
    };
    const auto with_general = [&](auto has_ends) {
        constexpr bool E = decltype(has_ends)::value;
        if (general)
            return go(k_block_fwd<TR, TY, P, GATE, E, true, MOST, PER_SM>, has_ends, std::true_type());
        return go(k_block_fwd<TR, TY, P, GATE, E, false, MOST, PER_SM>, has_ends, std::false_type());
    };
    return ends ? with_general(std::true_type()) : with_general(std::false_type());
}

// Many rows: as many pieces to a thread as its registers hold (and the row has), so that many rows are in flight; few rows:
// one, so that each answers sooner.
template <typename TR, typename TY, bool GATE> cudaError_t launch_gated(const BlockCall &c, const Phases &phases, cudaStream_t stream)
{
    const bool few = c.T * ((c.d + 1023) / 1024) < 4 * device_sm_count();
    if (c.d <= 256 || (few && c.d <= 4096))
        return launch_rows<TR, TY, GATE, 1, 512, 1>(c, phases, stream);
    if (few)
        return launch_rows<TR, TY, GATE, 1, 1024, 1>(c, phases, stream);
    // bf16 layer norms with a gate per channel, rows on boundaries, 32,768 x 512: 40 us with four pieces, 29 with two; x 1,024:
    // 50, 63; x 4,096: 204, 251; 16,384 x 5,120: 185, 220; x 8,192: 317, 268 (two copies of their four vectors do not fit beside
    // each other)
    const bool general = c.kind == TURNOPD_LAYER_NORM || c.beta_post || c.beta_pre;
    if constexpr (sizeof(TR) + sizeof(TY) * (GATE ? 2 : 1) <= 6)
        if (c.d > 512 && (!general || c.d <= 5120))
            return launch_rows<TR, TY, GATE, 4, 256, 2>(c, phases, stream);
    return launch_rows<TR, TY, GATE, 2, 512, 1>(c, phases, stream);
}

}  // namespace

template <typename TR, typename TY> cudaError_t launch_block_rows_fwd(const BlockCall &c, const Phases &phases, cudaStream_t stream)
{
    return c.gate && c.ldg ? launch_gated<TR, TY, true>(c, phases, stream) : launch_gated<TR, TY, false>(c, phases, stream);
}

}  // namespace turnopd
