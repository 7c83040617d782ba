// Rows of the backward pass of the norms around a block: everything of a row in one pass over its arrays.
#pragma once

#include <algorithm>

#include "block_norm.cuh"

namespace turnopd {
namespace {

constexpr int kE = 16;       // columns of a row that one thread holds, in two pieces of eight
constexpr int kPieces = kE / 8;

__device__ __forceinline__ void cp8(void *smem, const void *gmem)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"((uint32_t)__cvta_generic_to_shared(smem)), "l"(gmem) : "memory");
}

// One array of a row in the ring.
struct RingPart {
    const char *p;   // row 0, null: not read
    int64_t pitch;   // bytes from row to row
    int at;          // bytes into a stage
    int bytes;       // of one column
};

struct Ring {
    RingPart resid, y, dh, dro, gate;
    int stage;  // bytes of a stage of one group
    int depth;  // rows in flight ahead of the one at hand
};

// Eight columns from the ring; codes without their scale.
__device__ __forceinline__ void from_ring(const char *stage, const RingPart &p, int dtype, int piece, float2 *v)
{
    float *f = reinterpret_cast<float *>(v);
    const char *at = stage + p.at + piece * 8 * p.bytes;
    if (dtype == TURNOPD_BF16)
        load8(reinterpret_cast<const __nv_bfloat16 *>(at), f);
    else if (dtype == TURNOPD_F32)
        load8(reinterpret_cast<const float *>(at), f);
    else
        decode8(*reinterpret_cast<const uint2 *>(at), dtype == TURNOPD_E4M3, f);
}

// One column of a row of any array, by its type; codes without their scale.
__device__ __forceinline__ float one_column(const RingPart &p, int dtype, int64_t i, int j)
{
    const char *at = p.p + i * p.pitch + (int64_t)j * p.bytes;
    if (dtype == TURNOPD_BF16)
        return __bfloat162float(*reinterpret_cast<const __nv_bfloat16 *>(at));
    if (dtype == TURNOPD_F32)
        return *reinterpret_cast<const float *>(at);
    const uint8_t b = *reinterpret_cast<const uint8_t *>(at);
    return dtype == TURNOPD_E4M3 ? decode_e4m3(b) : (float)(int8_t)b;
}

// A thread keeps its columns of gamma and of the sums over rows in registers from row to row.  Group b of all takes rows b,
// b + groups, ..., so that every sum has a fixed order.  A row's arrays come through a ring in shared memory, in which each
// thread copies and reads its own pieces only: no barrier but those of the row's two sums.
//
// ENDS: the rows begin anywhere, but in all arrays at the same element of a group of eight.  The groups' number is a multiple
// of eight then, so all rows of one group begin at the same element, and a thread keeps the same columns from row to row:
// pieces of eight from the first boundary on, and the first threads one of the elements before and after them each.
template <typename TR, typename TY, bool ENDS, bool BIAS, int MOST, int PER_SM>
__global__ void __launch_bounds__(MOST, PER_SM) k_block_bwd(BlockGradCall c, Ring ring, int n, int phase, int phase_step)
{
    extern __shared__ __align__(128) char shared[];
    __shared__ float2 red[2][16];
    const int t = threadIdx.x % n, group = threadIdx.x / n, warps = n / 32, per = blockDim.x / n, d = (int)c.d;
    const int64_t groups = (int64_t)gridDim.x * per, b = (int64_t)blockIdx.x * per + group;
    const bool layer = c.kind == TURNOPD_LAYER_NORM, pre = c.gamma_pre, post = c.gamma_post;
    const bool token_gate = c.gate && c.ldg, dgate = token_gate && c.dgate;
    const bool post_sums = c.dgamma_post || c.dbeta_post || (c.dgate && !c.ldg);
    const bool needs_y = ring.y.p, needs_stream = c.d_resid || c.dy || c.dgate || post_sums;
    const float inv_d = 1.f / (float)d, s = c.branch_scale;
    const int64_t exps_per_row = (c.d + kActGroup - 1) / kActGroup;
    char *own = shared + group * (ring.depth + 1) * ring.stage;
    const int head = ENDS ? min((8 - (int)((phase + b * phase_step) & 7)) & 7, d) : 0;
    const int whole = (d - head) / 8, ends = ENDS ? d - whole * 8 : 0;
    const int end = t < head ? t : whole * 8 + t;  // the single column of this thread, where t < ends
    const auto column = [&](int k) { return head + (k * n + t) * 8; };  // the first of piece k
    const auto there = [&](int k) { return k * n + t < whole; };

    constexpr int kSums = BIAS ? 4 : 2, kPostSum = BIAS ? 2 : 1;  // dh xh_pre, (dh,) X xh_post (, X)
    float2 gamma[kE / 2], cpost[kE / 2], sums[kSums][kE / 2];
    float sums_end[kSums] = {};
#pragma unroll
    for (int k = 0; k < kE / 2; ++k)
#pragma unroll
        for (int q = 0; q < kSums; ++q)
            sums[q][k] = make_float2(0.f, 0.f);
    // s gamma_post gate of a column (without those that there are not)
    const auto post_factor = [&](int j) {
        float p = s * (post ? param(c.gamma_post, c.param_dtype, j) : 1.f);
        return c.gate && !c.ldg ? p * param(c.gate, c.param_dtype, j) : p;
    };
#pragma unroll
    for (int k = 0; k < kPieces; ++k)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int j = column(k) + e;
            reinterpret_cast<float *>(gamma)[k * 8 + e] = there(k) && pre ? param(c.gamma_pre, c.param_dtype, j) : 0.f;
            reinterpret_cast<float *>(cpost)[k * 8 + e] = there(k) ? post_factor(j) : 0.f;
        }
    const bool at_end = ENDS && t < ends;
    const float gamma_end = at_end && pre ? param(c.gamma_pre, c.param_dtype, end) : 0.f, cpost_end = at_end ? post_factor(end) : 0.f;

    const auto copy = [&](int64_t i, int stage) {
        if (i < c.T && (!c.mask || c.mask[i])) {
            char *to = own + stage * ring.stage;
            const auto part = [&](const RingPart &p) {
                if (!p.p)
                    return;
                const char *row = p.p + i * p.pitch + head * p.bytes;
#pragma unroll
                for (int k = 0; k < kPieces; ++k) {
                    if (!there(k))
                        continue;
                    const int at = (k * n + t) * 8 * p.bytes;
                    if (p.bytes == 1) {
                        cp8(to + p.at + at, row + at);
                    } else {
                        cp16(to + p.at + at, row + at);
                        if (p.bytes == 4)
                            cp16(to + p.at + at + 16, row + at + 16);
                    }
                }
            };
            part(ring.resid);
            part(ring.dh);
            part(ring.dro);
            part(ring.y);
            part(ring.gate);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    // a row's statistics, its exponents (a byte to each piece, whose columns may lie in two groups of them: the first's in the
    // low half) and this thread's single column are read a row ahead
    struct Numbers {
        float4 stats;
        uint32_t er, ey;
        float resid, y, dh, dro, gate;
        bool fine;
    };
    const bool code_r = pre && c.resid_dtype >= TURNOPD_E4M3, code_y = needs_y && c.y_dtype >= TURNOPD_E4M3;
    const auto numbers = [&](int64_t i) {
        Numbers m{};
        if (i < c.T) {
            m.fine = takes_part(c, i, m.stats);
            if (m.fine) {
#pragma unroll
                for (int k = 0; k < kPieces; ++k)
                    if (there(k)) {
                        const int64_t at = i * exps_per_row;
                        const int g = column(k) / kActGroup, h = ENDS ? (column(k) + 7) / kActGroup : g;
                        if (code_r)
                            m.er |= (uint32_t)c.resid_exps[at + g] << (8 * k) | (ENDS ? (uint32_t)c.resid_exps[at + h] << (8 * k + 16) : 0u);
                        if (code_y)
                            m.ey |= (uint32_t)c.y_exps[at + g] << (8 * k) | (ENDS ? (uint32_t)c.y_exps[at + h] << (8 * k + 16) : 0u);
                    }
                if (at_end) {
                    const int64_t at = i * exps_per_row + end / kActGroup;
                    if (pre) {
                        m.resid = one_column(ring.resid, c.resid_dtype, i, end) * (code_r ? act_scale(c.resid_exps[at]) : 1.f);
                        m.dh = one_column(ring.dh, c.grad_y_dtype, i, end);
                    }
                    if (ring.dro.p)
                        m.dro = one_column(ring.dro, c.grad_r_dtype, i, end);
                    if (needs_y)
                        m.y = one_column(ring.y, c.y_dtype, i, end) * (code_y ? act_scale(c.y_exps[at]) : 1.f);
                    if (token_gate)
                        m.gate = one_column(ring.gate, c.grad_y_dtype, i, end);
                }
            }
        }
        return m;
    };
    for (int k = 0; k < ring.depth; ++k)
        copy(b + k * groups, k);
    Numbers m = numbers(b);
    int stage = 0, odd = 0;
    for (int64_t i = b; i < c.T; i += groups) {
        copy(i + ring.depth * groups, stage ? stage - 1 : ring.depth);
        const Numbers next = numbers(i + groups);
        if (ring.depth == 3)
            asm volatile("cp.async.wait_group 3;" ::: "memory");
        else if (ring.depth == 2)
            asm volatile("cp.async.wait_group 2;" ::: "memory");
        else if (ring.depth == 1)
            asm volatile("cp.async.wait_group 1;" ::: "memory");
        else
            asm volatile("cp.async.wait_group 0;" ::: "memory");
        const char *at = own + stage * ring.stage;
        const float mu0 = m.stats.x, r0 = m.stats.y, mu1 = m.stats.z, r1 = m.stats.w;
        // eight columns of an array; missing ones are zeros
        const auto activation = [&](const RingPart &part, int dtype, uint32_t exps, int k, float2 *v) {
            if (!there(k)) {
                v[0] = v[1] = v[2] = v[3] = make_float2(0.f, 0.f);
                return;
            }
            from_ring(at, part, dtype, k * n + t, v);
            if (dtype >= TURNOPD_E4M3) {
                const float lo = act_scale(exps >> (8 * k) & 255u), hi = ENDS ? act_scale(exps >> (8 * k + 16) & 255u) : lo;
                const int first = ENDS ? kActGroup - (column(k) & (kActGroup - 1)) : 8;  // columns of the first group
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    v[e] = fmul2(v[e], make_float2(2 * e < first ? lo : hi, 2 * e + 1 < first ? lo : hi));
            }
        };
        const auto gradient = [&](auto type, const RingPart &part, int k, float2 *v) {
            if (there(k))
                load8(reinterpret_cast<const decltype(type) *>(at + part.at) + (k * n + t) * 8, reinterpret_cast<float *>(v));
            else
                v[0] = v[1] = v[2] = v[3] = make_float2(0.f, 0.f);
        };
        const auto put8 = [&](auto *p, int64_t ld, int k, const float2 *v) {
            if (there(k))
                store8(p + i * ld + column(k), reinterpret_cast<const float *>(v));
        };
        const auto put1 = [&](auto *p, int64_t ld, float v) {
            using T = std::remove_reference_t<decltype(*p)>;
            if (at_end)
                p[i * ld + end] = from_float<T>(v);
        };
        const auto xh_pre = [&](int k, float2 *v) {
            activation(ring.resid, c.resid_dtype, m.er, k, v);
#pragma unroll
            for (int e = 0; e < 4; ++e)
                v[e] = fmul2(fadd2(v[e], splat(-mu1)), splat(r1));
        };
        const auto xh_post = [&](int k, float2 *v) {
            activation(ring.y, c.y_dtype, m.ey, k, v);
            if (post)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    v[e] = fmul2(fadd2(v[e], splat(-mu0)), splat(r0));
        };

        // (the sums over the row are taken whatever the mask and the statistics say: no barrier stands under a condition
        // that every thread reads from the caller's memory for itself)
        float2 mean = make_float2(0.f, 0.f);
        const float xe_pre = ENDS && m.fine && at_end ? (m.resid - mu1) * r1 : 0.f;
        const float xe_post = ENDS && m.fine && at_end ? (post ? (m.y - mu0) * r0 : m.y) : 0.f;
        if (pre) {
            float2 sg = make_float2(0.f, 0.f), sx = sg;
            if (m.fine) {
#pragma unroll
                for (int k = 0; k < kPieces; ++k) {
                    float2 x[4], g[4];
                    xh_pre(k, x);
                    gradient(TY(), ring.dh, k, g);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        sums[0][4 * k + e] = ffma2(g[e], x[e], sums[0][4 * k + e]);
                        if (BIAS)
                            sums[1][4 * k + e] = fadd2(g[e], sums[1][4 * k + e]);
                        g[e] = fmul2(g[e], gamma[4 * k + e]);
                        sg = fadd2(sg, g[e]);
                        sx = ffma2(g[e], x[e], sx);
                    }
                }
                if (ENDS) {
                    sums_end[0] = fmaf(m.dh, xe_pre, sums_end[0]);
                    if (BIAS)
                        sums_end[1] += m.dh;
                    sg.x += m.dh * gamma_end;
                    sx.x = fmaf(m.dh * gamma_end, xe_pre, sx.x);
                }
            }
            if (needs_stream) {
                mean = group_sum2(make_float2(sg.x + sg.y, sx.x + sx.y), red[odd], group, warps);
                odd ^= 1;
            }
        }
        if (needs_stream) {
            // D = dr' + r (g - mean g - xh mean(g xh)), then X = D times the gate that each token has of its own, and E
            const float2 c0 = splat(layer ? -r1 * (mean.x * inv_d) : 0.f), c1 = splat(-r1 * (mean.y * inv_d));
            float2 E[kE / 2];
            float E_end = 0.f;
            float2 sg = make_float2(0.f, 0.f), sx = sg;
#pragma unroll
            for (int k = 0; k < kPieces; ++k) {
                float2 D[4], x[4];
                D[0] = D[1] = D[2] = D[3] = make_float2(0.f, 0.f);
                if (m.fine) {
                    if (ring.dro.p)
                        gradient(TR(), ring.dro, k, D);
                    if (pre) {
                        float2 g[4];
                        xh_pre(k, x);
                        gradient(TY(), ring.dh, k, g);
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            D[e] = fadd2(D[e], ffma2(fmul2(g[e], gamma[4 * k + e]), splat(r1), ffma2(x[e], c1, c0)));
                    }
                }
                if (c.d_resid) {
                    float2 o[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        o[e] = fmul2(D[e], splat(c.resid_scale));
                    put8(static_cast<TR *>(c.d_resid), c.lddr, k, o);
                }
                if (needs_y) {
                    if (m.fine)
                        xh_post(k, x);
                    else
                        x[0] = x[1] = x[2] = x[3] = make_float2(0.f, 0.f);
                }
                if (token_gate) {
                    if (dgate) {
                        float2 o[4];
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            float w = reinterpret_cast<const float *>(x)[e];
                            if (post && there(k))
                                w = fmaf(w, param(c.gamma_post, c.param_dtype, column(k) + e),
                                         c.beta_post ? param(c.beta_post, c.param_dtype, column(k) + e) : 0.f);
                            reinterpret_cast<float *>(o)[e] = s * reinterpret_cast<const float *>(D)[e] * w;
                        }
                        put8(static_cast<TY *>(c.dgate), c.lddg, k, o);
                    }
                    if (m.fine) {
                        float2 g[4];
                        gradient(TY(), ring.gate, k, g);
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            D[e] = fmul2(D[e], g[e]);
                    }
                }
                if (post_sums) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        if (needs_y)
                            sums[kPostSum][4 * k + e] = ffma2(D[e], x[e], sums[kPostSum][4 * k + e]);
                        if (BIAS)
                            sums[kSums - 1][4 * k + e] = fadd2(D[e], sums[kSums - 1][4 * k + e]);
                    }
                }
                if (c.dy) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float2 g = fmul2(D[e], cpost[4 * k + e]);
                        E[4 * k + e] = g;
                        sg = fadd2(sg, g);
                        if (post)
                            sx = ffma2(g, x[e], sx);
                    }
                    if (!post)
                        put8(static_cast<TY *>(c.dy), c.lddy, k, E + 4 * k);
                }
            }
            if (ENDS) {
                float D = 0.f;
                if (m.fine)
                    D = m.dro + (pre ? fmaf(m.dh * gamma_end, r1, fmaf(xe_pre, c1.x, c0.x)) : 0.f);
                if (c.d_resid)
                    put1(static_cast<TR *>(c.d_resid), c.lddr, D * c.resid_scale);
                if (dgate) {
                    float w = xe_post;
                    if (post && at_end)
                        w = fmaf(w, param(c.gamma_post, c.param_dtype, end), c.beta_post ? param(c.beta_post, c.param_dtype, end) : 0.f);
                    put1(static_cast<TY *>(c.dgate), c.lddg, s * D * w);
                }
                if (token_gate)
                    D *= m.gate;
                if (!at_end)
                    D = 0.f;
                sums_end[kPostSum] = fmaf(D, xe_post, sums_end[kPostSum]);
                if (BIAS)
                    sums_end[kSums - 1] += D;
                E_end = D * cpost_end;
                sg.x += E_end;
                sx.x = fmaf(E_end, xe_post, sx.x);
                if (c.dy && !post)
                    put1(static_cast<TY *>(c.dy), c.lddy, E_end);
            }
            if (c.dy && post) {
                const float2 v = group_sum2(make_float2(sg.x + sg.y, sx.x + sx.y), red[odd], group, warps);
                odd ^= 1;
                const float2 a0 = splat(layer ? -r0 * (v.x * inv_d) : 0.f), a1 = splat(-r0 * (v.y * inv_d));
#pragma unroll
                for (int k = 0; k < kPieces; ++k) {
                    float2 x[4], o[4];
                    if (m.fine)
                        xh_post(k, x);
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        o[e] = m.fine ? ffma2(E[4 * k + e], splat(r0), ffma2(x[e], a1, a0)) : make_float2(0.f, 0.f);
                    put8(static_cast<TY *>(c.dy), c.lddy, k, o);
                }
                if (ENDS)
                    put1(static_cast<TY *>(c.dy), c.lddy, m.fine ? fmaf(E_end, r0, fmaf(xe_post, a1.x, a0.x)) : 0.f);
            }
        }
        m = next;
        stage = stage == ring.depth ? 0 : stage + 1;
    }
    if (!c.workspace)
        return;
    // the block's groups are added up in their order, in shared memory: one row of partial sums per block
    asm volatile("cp.async.wait_all;" ::: "memory");
    __syncthreads();
    float *out = static_cast<float *>(c.workspace) + (int64_t)blockIdx.x * 4 * d;
#pragma unroll
    for (int q = 0; q < kSums; ++q) {
        const int row = BIAS ? q : 2 * q;
        float *part = per == 1 ? out + (int64_t)row * d : reinterpret_cast<float *>(shared) + group * d;
#pragma unroll
        for (int k = 0; k < kPieces; ++k)
            if (there(k))
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    part[column(k) + e] = reinterpret_cast<const float *>(sums[q])[k * 8 + e];
        if (at_end)
            part[end] = sums_end[q];
        if (per > 1) {
            __syncthreads();
            for (int j = threadIdx.x; j < d; j += blockDim.x) {
                float sum = reinterpret_cast<const float *>(shared)[j];
                for (int g = 1; g < per; ++g)
                    sum += reinterpret_cast<const float *>(shared)[g * d + j];
                out[(int64_t)row * d + j] = sum;
            }
            __syncthreads();
        }
    }
}

}  // namespace

template <typename TR, typename TY> cudaError_t launch_block_rows_bwd(const BlockGradCall &given, int *parts, bool *taken, cudaStream_t stream)
{
    BlockGradCall c = given;
    const bool sums = c.dgamma_pre || c.dbeta_pre || c.dgamma_post || c.dbeta_post || (c.dgate && !c.ldg);
    const bool needs_y = c.gamma_post ? c.dy || c.dgamma_post || c.dgate : c.dgate != nullptr;
    const bool token_gate = c.gate && c.ldg;
    if (!sums)
        c.workspace = nullptr;
    Ring ring{};
    const int n = (int)((c.d + kE * 32 - 1) / (kE * 32)) * 32, per = std::max(1, 256 / n);
    const auto add = [&](RingPart &part, const void *p, int64_t ld, int32_t dtype) {
        if (!p)
            return;
        part.p = static_cast<const char *>(p);
        part.bytes = stored_bytes(dtype);
        part.pitch = ld * part.bytes;
        part.at = ring.stage;
        ring.stage += n * kE * part.bytes;
    };
    const void *resid = c.gamma_pre ? c.resid : nullptr, *y = needs_y ? c.y : nullptr, *gate = token_gate ? c.gate : nullptr;
    add(ring.resid, resid, c.ldr, c.resid_dtype);
    add(ring.dh, c.dh, c.lddh, c.grad_y_dtype);
    add(ring.dro, c.d_resid_out, c.lddro, c.grad_r_dtype);
    add(ring.y, y, c.ldy, c.y_dtype);
    add(ring.gate, gate, c.ldg, c.grad_y_dtype);
    const Phases phases{Phase(resid, c.ldr, c.resid_dtype),
                        Phase(c.dh, c.lddh, c.grad_y_dtype),
                        Phase(c.d_resid_out, c.lddro, c.grad_r_dtype),
                        Phase(y, c.ldy, c.y_dtype),
                        Phase(gate, c.ldg, c.grad_y_dtype),
                        Phase(c.d_resid, c.lddr, c.grad_r_dtype),
                        Phase(c.dy, c.lddy, c.grad_y_dtype),
                        Phase(token_gate ? c.dgate : nullptr, c.lddg, c.grad_y_dtype)};
    *taken = phases.alike;
    if (!*taken)
        return cudaSuccess;
    const bool ends = phases.at || phases.step || c.d % 8;
    // two CTAs per SM up to 256 threads, if each then has room for a row in flight ahead of the one at hand
    constexpr size_t kRoom = 220 * 1024;
    const int threads = n * per;
    const size_t stage = (size_t)per * std::max(ring.stage, 1);
    const int per_sm = threads <= 256 && 2 * 2 * stage <= kRoom ? 2 : 1;
    ring.depth = (int)std::min<size_t>(3, kRoom / per_sm / stage - 1);
    const size_t smem = std::max<size_t>(stage * (ring.depth + 1),
                                         sums && per > 1 ? sizeof(float) * per * (size_t)c.d : 0);
    const int64_t blocks = (c.T + per - 1) / per;
    const int64_t most = std::min<int64_t>((int64_t)per_sm * device_sm_count(), kBlockMaxParts);
    int grid = (int)std::min<int64_t>(blocks > device_sm_count() ? (blocks + 1) / 2 : blocks, most);
    if (ends)
        grid = std::min((grid * per + 7) / 8 * 8 / per, kBlockMaxParts);  // a multiple of eight groups
    *parts = grid;
    const bool bias = block_bwd_bias(c);
    const auto go = [&](auto kernel) {
        const cudaError_t e = allow_shared(kernel, kRoom);
        if (e != cudaSuccess)
            return e;
        kernel<<<grid, threads, smem, stream>>>(c, ring, n, phases.at, phases.step);
        return cudaGetLastError();
    };
    if (threads <= 256)
        return ends ? (bias ? go(k_block_bwd<TR, TY, true, true, 256, 2>) : go(k_block_bwd<TR, TY, true, false, 256, 2>))
                    : (bias ? go(k_block_bwd<TR, TY, false, true, 256, 2>) : go(k_block_bwd<TR, TY, false, false, 256, 2>));
    if (threads <= 384)
        return ends ? (bias ? go(k_block_bwd<TR, TY, true, true, 384, 1>) : go(k_block_bwd<TR, TY, true, false, 384, 1>))
                    : (bias ? go(k_block_bwd<TR, TY, false, true, 384, 1>) : go(k_block_bwd<TR, TY, false, false, 384, 1>));
    return ends ? (bias ? go(k_block_bwd<TR, TY, true, true, 512, 1>) : go(k_block_bwd<TR, TY, true, false, 512, 1>))
                : (bias ? go(k_block_bwd<TR, TY, false, true, 512, 1>) : go(k_block_bwd<TR, TY, false, false, 512, 1>));
}

}  // namespace turnopd
