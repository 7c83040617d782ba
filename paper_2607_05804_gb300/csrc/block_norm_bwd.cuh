// Rows of the backward pass of the norms around a block: everything of a row in one pass over its arrays.
#pragma once

#include <algorithm>
#include <type_traits>

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
    int dtype;
    int bytes;       // of one column
};

struct Ring {
    RingPart resid, y, dh, dro, gate;
    int stage;  // bytes of a stage of one group
    int depth;  // rows in flight ahead of the one at hand
};

// Eight columns from the ring; codes without their scale.
__device__ __forceinline__ void from_ring(const char *at, int dtype, float2 *v)
{
    float *f = reinterpret_cast<float *>(v);
    if (dtype == TURNOPD_BF16)
        load8(reinterpret_cast<const __nv_bfloat16 *>(at), f);
    else if (dtype == TURNOPD_F32)
        load8(reinterpret_cast<const float *>(at), f);
    else
        decode8(*reinterpret_cast<const uint2 *>(at), dtype == TURNOPD_E4M3, f);
}

template <typename T> constexpr int type_code() { return sizeof(T) == 2 ? TURNOPD_BF16 : TURNOPD_F32; }

// One column of a row of any array, by its type; codes without their scale.
__device__ __forceinline__ float one_column(const RingPart &p, int64_t i, int j)
{
    const char *at = p.p + i * p.pitch + (int64_t)j * p.bytes;
    const int dtype = p.dtype;
    if (dtype == TURNOPD_BF16)
        return __bfloat162float(*reinterpret_cast<const __nv_bfloat16 *>(at));
    if (dtype == TURNOPD_F32)
        return *reinterpret_cast<const float *>(at);
    const uint8_t b = *reinterpret_cast<const uint8_t *>(at);
    return dtype == TURNOPD_E4M3 ? decode_e4m3(b) : (float)(int8_t)b;
}

// A thread keeps its columns of the sums over rows and of the factor after the first norm in registers from row to row, and
// of gamma_pre in shared memory, in pieces of four (its registers would not hold both).  Group b of all takes rows b,
// b + groups, ..., so that every sum has a fixed order.  A row's arrays come through a ring in shared memory, in which each
// thread copies and reads its own pieces only: no barrier but those of the row's two sums.  A warp's pieces lie 256 columns
// apart, so that they are found at constant offsets.
//
// ENDS: the rows begin anywhere, but in all arrays at the same element of a group of eight.  The groups' number is a multiple
// of eight then, so all rows of one group begin at the same element, and a thread keeps the same columns from row to row:
// pieces of eight from the first boundary on, and the first threads one of the elements before and after them each.
// GENERAL: layer norms, or sums for betas; without it the mean of g and those sums are left out.
// STORED: r' and y are of the gradients' types; else of any, codes among them.
template <typename TR, typename TY, bool STORED, bool ENDS, bool GENERAL, int MOST, int PER_SM>
__global__ void __launch_bounds__(MOST, PER_SM) k_block_bwd(BlockGradCall c, Ring ring, int n, int phase, int phase_step)
{
    using V = std::conditional_t<GENERAL, float2, float>;  // sums over a row: (of g, of g xh) or the second alone
    extern __shared__ __align__(128) char shared[];
    __shared__ V red[2][16];
    const int t = threadIdx.x % n, group = threadIdx.x / n, warps = n / 32, per = blockDim.x / n, d = (int)c.d;
    const int64_t groups = (int64_t)gridDim.x * per, b = (int64_t)blockIdx.x * per + group;
    const bool layer = GENERAL && c.kind == TURNOPD_LAYER_NORM, pre = c.gamma_pre, post = c.gamma_post;
    const bool token_gate = ring.gate.p, dgate = token_gate && c.dgate;
    const bool post_sums = c.dgamma_post || c.dbeta_post || (c.dgate && !c.ldg);
    const bool needs_y = ring.y.p, needs_stream = c.d_resid || c.dy || c.dgate || post_sums;
    const float inv_d = 1.f / (float)d, s = c.branch_scale;
    const int64_t exps_per_row = (c.d + kActGroup - 1) / kActGroup;
    const int head = ENDS ? min((8 - (int)((phase + b * phase_step) & 7)) & 7, d) : 0;
    const int whole = (d - head) / 8, ends = ENDS ? d - whole * 8 : 0;
    const int end = t < head ? t : whole * 8 + t;  // the single column of this thread, where t < ends
    const int piece0 = (t >> 5) * 32 * kPieces + (t & 31);
    const auto column = [&](int k) { return head + (piece0 + 32 * k) * 8; };  // the first of piece k
    const auto there = [&](int k) { return piece0 + 32 * k < whole; };
    const bool at_end = ENDS && t < ends;

    char *own = shared + (size_t)group * ((ring.depth + 1) * ring.stage + n * kE * (int)sizeof(float));
    float4 *gamma = reinterpret_cast<float4 *>(own + (ring.depth + 1) * ring.stage) + t;  // n apart
    constexpr int kSums = GENERAL ? 4 : 2, kPostSum = GENERAL ? 2 : 1;  // dh xh_pre, (dh,) X xh_post (, X)
    float2 cpost[kE / 2], sums[kSums][kE / 2];
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
    for (int k = 0; k < kPieces; ++k) {
        float g[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int j = column(k) + e;
            g[e] = there(k) && pre ? param(c.gamma_pre, c.param_dtype, j) : 0.f;
            reinterpret_cast<float *>(cpost)[k * 8 + e] = there(k) ? post_factor(j) : 0.f;
        }
        gamma[2 * k * n] = make_float4(g[0], g[1], g[2], g[3]);
        gamma[(2 * k + 1) * n] = make_float4(g[4], g[5], g[6], g[7]);
    }
    const float gamma_end = at_end && pre ? param(c.gamma_pre, c.param_dtype, end) : 0.f, cpost_end = at_end ? post_factor(end) : 0.f;
    // missing pieces are zeros in every stage
#pragma unroll
    for (int k = 0; k < kPieces; ++k)
        if (!there(k))
            for (int q = 0; q <= ring.depth; ++q)
                for (const RingPart *p : {&ring.resid, &ring.y, &ring.dh, &ring.dro, &ring.gate})
                    if (p->p)
                        for (int h = 0; h < p->bytes; ++h)
                            *reinterpret_cast<uint2 *>(own + q * ring.stage + p->at + (piece0 + 32 * k) * 8 * p->bytes + 8 * h) =
                                make_uint2(0u, 0u);

    // One array's pieces of a row: `from` is this thread's first one there, which goes on by a step of the groups.
    struct Source {
        const char *from;
        int64_t step;
    };
    const auto source = [&](const RingPart &p) { return Source{p.p + b * p.pitch + column(0) * p.bytes, groups * p.pitch}; };
    Source resid = source(ring.resid), y = source(ring.y), dh = source(ring.dh), dro = source(ring.dro), gate = source(ring.gate);
    int64_t ahead = b;  // the next row to copy
    const auto copy = [&](int stage) {
        const bool on = ahead < c.T && (!c.mask || c.mask[ahead]);
        char *to = own + stage * ring.stage;
        const auto part = [&](Source &src, const RingPart &p, int bytes) {
            if (!p.p)
                return;
#pragma unroll
            for (int k = 0; k < kPieces; ++k) {
                if (!on || !there(k))
                    continue;
                char *dst = to + p.at + piece0 * 8 * bytes + k * 256 * bytes;
                const char *at = src.from + k * 256 * bytes;
                if (bytes == 1) {
                    cp8(dst, at);
                } else {
                    cp16(dst, at);
                    if (bytes == 4)
                        cp16(dst + 16, at + 16);
                }
            }
            src.from += src.step;
        };
        part(resid, ring.resid, STORED ? (int)sizeof(TR) : ring.resid.bytes);
        part(dh, ring.dh, sizeof(TY));
        part(dro, ring.dro, sizeof(TR));
        part(y, ring.y, STORED ? (int)sizeof(TY) : ring.y.bytes);
        part(gate, ring.gate, sizeof(TY));
        ahead += groups;
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
    const bool code_r = !STORED && pre && ring.resid.dtype >= TURNOPD_E4M3, code_y = !STORED && needs_y && ring.y.dtype >= TURNOPD_E4M3;
    const auto numbers = [&](int64_t i) {
        Numbers m{};
        if (i < c.T) {
            m.fine = takes_part(c, i, m.stats);
            if (m.fine) {
                if (!STORED) {
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
                }
                if (at_end) {
                    const int64_t at = i * exps_per_row + end / kActGroup;
                    if (pre) {
                        m.resid = one_column(ring.resid, i, end) * (code_r ? act_scale(c.resid_exps[at]) : 1.f);
                        m.dh = one_column(ring.dh, i, end);
                    }
                    if (ring.dro.p)
                        m.dro = one_column(ring.dro, i, end);
                    if (needs_y)
                        m.y = one_column(ring.y, i, end) * (code_y ? act_scale(c.y_exps[at]) : 1.f);
                    if (token_gate)
                        m.gate = one_column(ring.gate, i, end);
                }
            }
        }
        return m;
    };
    for (int k = 0; k < ring.depth; ++k)
        copy(k);
    Numbers m = numbers(b);
    int stage = 0, odd = 0;
    for (int64_t i = b; i < c.T; i += groups) {
        copy(stage ? stage - 1 : ring.depth);
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
        // eight columns of an array
        const auto activation = [&](const RingPart &part, int stored, uint32_t exps, int k, float2 *v) {
            const int dtype = STORED ? stored : part.dtype, bytes = STORED ? (stored == TURNOPD_BF16 ? 2 : 4) : part.bytes;
            from_ring(at + part.at + piece0 * 8 * bytes + k * 256 * bytes, dtype, v);
            if (!STORED && dtype >= TURNOPD_E4M3) {
                const float lo = act_scale(exps >> (8 * k) & 255u), hi = ENDS ? act_scale(exps >> (8 * k + 16) & 255u) : lo;
                const int first = ENDS ? kActGroup - (column(k) & (kActGroup - 1)) : 8;  // columns of the first group
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    v[e] = fmul2(v[e], make_float2(2 * e < first ? lo : hi, 2 * e + 1 < first ? lo : hi));
            }
        };
        const auto gradient = [&](auto type, const RingPart &part, int k, float2 *v) {
            using T = decltype(type);
            load8(reinterpret_cast<const T *>(at + part.at) + piece0 * 8 + k * 256, reinterpret_cast<float *>(v));
        };
        const auto put8 = [&](auto *p, int64_t ld, int k, const float2 *v) {
            if (there(k))
                store8(p + i * ld + column(0) + k * 256, reinterpret_cast<const float *>(v));
        };
        const auto put1 = [&](auto *p, int64_t ld, float v) {
            using T = std::remove_reference_t<decltype(*p)>;
            if (at_end)
                p[i * ld + end] = from_float<T>(v);
        };
        const auto normed = [&](float2 *v, float mu, float r) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (GENERAL)
                    v[e] = fadd2(v[e], splat(-mu));
                v[e] = fmul2(v[e], splat(r));
            }
        };
        const auto xh_pre = [&](int k, float2 *v) {
            activation(ring.resid, type_code<TR>(), m.er, k, v);
            normed(v, mu1, r1);
        };
        const auto xh_post = [&](int k, float2 *v) {
            activation(ring.y, type_code<TY>(), m.ey, k, v);
            if (post)
                normed(v, mu0, r0);
        };
        const auto times_gamma = [&](int k, float2 *g) {
            const float4 a = gamma[2 * k * n], z = gamma[(2 * k + 1) * n];
            g[0] = fmul2(g[0], make_float2(a.x, a.y));
            g[1] = fmul2(g[1], make_float2(a.z, a.w));
            g[2] = fmul2(g[2], make_float2(z.x, z.y));
            g[3] = fmul2(g[3], make_float2(z.z, z.w));
        };
        const auto row_sum = [&](float2 sg, float2 sx) -> float2 {
            float2 v;
            if constexpr (GENERAL) {
                v = group_sum(make_float2(sg.x + sg.y, sx.x + sx.y), red[odd], group, warps);
            } else {
                v = make_float2(0.f, group_sum(sx.x + sx.y, red[odd], group, warps));
            }
            odd ^= 1;
            return v;
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
                        if (GENERAL)
                            sums[1][4 * k + e] = fadd2(g[e], sums[1][4 * k + e]);
                    }
                    times_gamma(k, g);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        if (GENERAL)
                            sg = fadd2(sg, g[e]);
                        sx = ffma2(g[e], x[e], sx);
                    }
                }
                if (ENDS) {
                    sums_end[0] = fmaf(m.dh, xe_pre, sums_end[0]);
                    if (GENERAL)
                        sums_end[1] += m.dh;
                    sg.x += m.dh * gamma_end;
                    sx.x = fmaf(m.dh * gamma_end, xe_pre, sx.x);
                }
            }
            if (needs_stream)
                mean = row_sum(sg, sx);
        }
        if (needs_stream) {
            // D = dr' + r (g - mean g - xh mean(g xh)), then X = D times the gate that each token has of its own, and E
            const float2 c0 = splat(layer ? -r1 * (mean.x * inv_d) : 0.f), c1 = splat(-r1 * (mean.y * inv_d));
            float2 E[kE / 2];
            float E_end = 0.f;
            float2 sg = make_float2(0.f, 0.f), sx = sg;
            if (m.fine) {
#pragma unroll
                for (int k = 0; k < kPieces; ++k) {
                    float2 D[4], x[4];
                    if (ring.dro.p)
                        gradient(TR(), ring.dro, k, D);
                    else
                        D[0] = D[1] = D[2] = D[3] = make_float2(0.f, 0.f);
                    if (pre) {
                        float2 g[4];
                        xh_pre(k, x);
                        gradient(TY(), ring.dh, k, g);
                        times_gamma(k, g);
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            D[e] = fadd2(D[e], ffma2(g[e], splat(r1), GENERAL ? ffma2(x[e], c1, c0) : fmul2(x[e], c1)));
                    }
                    if (c.d_resid) {
                        float2 o[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            o[e] = fmul2(D[e], splat(c.resid_scale));
                        put8(static_cast<TR *>(c.d_resid), c.lddr, k, o);
                    }
                    if (needs_y)
                        xh_post(k, x);
                    if (token_gate) {
                        float2 g[4];
                        if (dgate) {
#pragma unroll
                            for (int e = 0; e < 8; ++e) {
                                float w = reinterpret_cast<const float *>(x)[e];
                                if (post && there(k))
                                    w = fmaf(w, param(c.gamma_post, c.param_dtype, column(k) + e),
                                             c.beta_post ? param(c.beta_post, c.param_dtype, column(k) + e) : 0.f);
                                reinterpret_cast<float *>(g)[e] = s * reinterpret_cast<const float *>(D)[e] * w;
                            }
                            put8(static_cast<TY *>(c.dgate), c.lddg, k, g);
                        }
                        gradient(TY(), ring.gate, k, g);
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            D[e] = fmul2(D[e], g[e]);
                    }
                    if (post_sums) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            if (needs_y)
                                sums[kPostSum][4 * k + e] = ffma2(D[e], x[e], sums[kPostSum][4 * k + e]);
                            if (GENERAL)
                                sums[kSums - 1][4 * k + e] = fadd2(D[e], sums[kSums - 1][4 * k + e]);
                        }
                    }
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float2 g = fmul2(D[e], cpost[4 * k + e]);
                        E[4 * k + e] = g;
                        if (GENERAL)
                            sg = fadd2(sg, g);
                        if (post)
                            sx = ffma2(g, x[e], sx);
                    }
                    if (c.dy && !post)
                        put8(static_cast<TY *>(c.dy), c.lddy, k, E + 4 * k);
                }
                if (ENDS) {
                    float D = m.dro + (pre ? fmaf(m.dh * gamma_end, r1, fmaf(xe_pre, c1.x, c0.x)) : 0.f);
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
                    if (GENERAL)
                        sums_end[kSums - 1] += D;
                    E_end = D * cpost_end;
                    sg.x += E_end;
                    sx.x = fmaf(E_end, xe_post, sx.x);
                    if (c.dy && !post)
                        put1(static_cast<TY *>(c.dy), c.lddy, E_end);
                }
            } else {
                const float2 zero[4] = {};
#pragma unroll
                for (int k = 0; k < kPieces; ++k) {
                    if (c.d_resid)
                        put8(static_cast<TR *>(c.d_resid), c.lddr, k, zero);
                    if (c.dy)
                        put8(static_cast<TY *>(c.dy), c.lddy, k, zero);
                    if (dgate)
                        put8(static_cast<TY *>(c.dgate), c.lddg, k, zero);
                }
                if (ENDS) {
                    if (c.d_resid)
                        put1(static_cast<TR *>(c.d_resid), c.lddr, 0.f);
                    if (c.dy)
                        put1(static_cast<TY *>(c.dy), c.lddy, 0.f);
                    if (dgate)
                        put1(static_cast<TY *>(c.dgate), c.lddg, 0.f);
                }
            }
            if (c.dy && post) {
                const float2 v = row_sum(sg, sx);
                if (m.fine) {
                    const float2 a0 = splat(layer ? -r0 * (v.x * inv_d) : 0.f), a1 = splat(-r0 * (v.y * inv_d));
#pragma unroll
                    for (int k = 0; k < kPieces; ++k) {
                        float2 x[4];
                        xh_post(k, x);
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            x[e] = ffma2(E[4 * k + e], splat(r0), GENERAL ? ffma2(x[e], a1, a0) : fmul2(x[e], a1));
                        put8(static_cast<TY *>(c.dy), c.lddy, k, x);
                    }
                    if (ENDS)
                        put1(static_cast<TY *>(c.dy), c.lddy, fmaf(E_end, r0, fmaf(xe_post, a1.x, a0.x)));
                }
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
        const int row = GENERAL ? q : 2 * q;
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
        part.dtype = dtype;
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
    const size_t stage = (size_t)per * std::max(ring.stage, 1), gamma = sizeof(float) * kE * threads;
    const int per_sm = threads <= 256 && 2 * (2 * stage + gamma) <= kRoom ? 2 : 1;
    ring.depth = (int)std::min<size_t>(3, (kRoom / per_sm - gamma) / stage - 1);
    const size_t smem = std::max<size_t>(stage * (ring.depth + 1) + gamma, sums && per > 1 ? sizeof(float) * per * (size_t)c.d : 0);
    const int64_t blocks = (c.T + per - 1) / per;
    const int64_t most = std::min<int64_t>((int64_t)per_sm * device_sm_count(), kBlockMaxParts);
    int grid = (int)std::min<int64_t>(blocks > device_sm_count() ? (blocks + 1) / 2 : blocks, most);
    if (ends)
        grid = std::min((grid * per + 7) / 8 * 8 / per, kBlockMaxParts);  // a multiple of eight groups
    *parts = grid;
    const bool general = c.kind == TURNOPD_LAYER_NORM || block_bwd_bias(c);
    const bool stored = (!resid || c.resid_dtype == c.grad_r_dtype) && (!y || c.y_dtype == c.grad_y_dtype);
    const auto go = [&](auto kernel) {
        const cudaError_t e = allow_shared(kernel, kRoom);
        if (e != cudaSuccess)
            return e;
        kernel<<<grid, threads, smem, stream>>>(c, ring, n, phases.at, phases.step);
        return cudaGetLastError();
    };
    const auto wide = [&](auto is_stored, auto has_ends, auto is_general) {
        constexpr bool S = decltype(is_stored)::value, E = decltype(has_ends)::value, G = decltype(is_general)::value;
        return threads <= 256 ? go(k_block_bwd<TR, TY, S, E, G, 256, 2>) : go(k_block_bwd<TR, TY, S, E, G, 512, 1>);
    };
    const auto with_general = [&](auto is_stored, auto has_ends) {
        return general ? wide(is_stored, has_ends, std::true_type()) : wide(is_stored, has_ends, std::false_type());
    };
    const auto with_ends = [&](auto is_stored) {
        return ends ? with_general(is_stored, std::true_type()) : with_general(is_stored, std::false_type());
    };
    return stored ? with_ends(std::true_type()) : with_ends(std::false_type());
}

}  // namespace turnopd
