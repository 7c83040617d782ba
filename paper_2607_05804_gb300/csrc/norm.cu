// Layer norm and root-mean-square norm of hidden states, and their backward pass.
//
// Row x[0..d): mu = mean x (0 in the root-mean-square form), r = (mean (x - mu)^2 + eps)^{-1/2},
// xh = (x - mu) r, y = xh gamma + beta.  With g = dy gamma:
//   dx = r (g - mean g - xh mean(g xh))   (root-mean-square form: without mean g),
//   dgamma = sum_i dy_i xh_i, dbeta = sum_i dy_i over the rows.
// The variance and xh are taken from x - mu in a second pass, so a mean much larger than the deviation costs no digits but
// those of mu's own rounding.

#include <algorithm>

#include "columns.cuh"
#include "common.cuh"
#include "kernels.h"
#include "packed.cuh"

namespace turnopd {
namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kE = 16;  // columns of a row that one thread holds
constexpr int kMaxRow = 512 * kE;  // longest rows that a block holds

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

// ---------------------------------------------------------------- forward

// 16 bytes of a row: W elements as pairs of floats.
template <typename T> struct Piece {
    static constexpr int W = 16 / (int)sizeof(T);
    static __device__ float2 pair(const uint4 &u, int j)
    {
        if constexpr (sizeof(T) == 2)
            return unpack2(word(u, j));
        else
            return make_float2(__uint_as_float(word(u, 2 * j)), __uint_as_float(word(u, 2 * j + 1)));
    }
};

template <int W, typename TY> __device__ __forceinline__ void store_piece(TY *p, const float2 (&o)[W / 2])
{
    if constexpr (W == 8) {
        store8(p, reinterpret_cast<const float *>(o));
    } else if constexpr (sizeof(TY) == 4) {
        __stcs(reinterpret_cast<float4 *>(p), make_float4(o[0].x, o[0].y, o[1].x, o[1].y));
    } else {
        __stcs(reinterpret_cast<uint2 *>(p), make_uint2(pack_bf16x2(o[0].x, o[0].y), pack_bf16x2(o[1].x, o[1].y)));
    }
}

// gamma and beta are kept in shared memory as fp32 pairs, in W planes of every W-th column: the pieces of a row that
// starts off a 16-byte boundary begin at any column, and in this layout neighbouring threads' columns lie next to each
// other wherever they begin.
template <int W> __host__ __device__ constexpr int plane_size(int d) { return d / W + 2; }

// Sum over a row, the same value in every one of its N threads; red: an entry per warp of the block.
template <int N> __device__ __forceinline__ float group_sum(float v, float *red, int group)
{
    constexpr int kLanes = N < 32 ? N : 32;
    const unsigned lanes = N < 32 ? ((1u << (N & 31)) - 1u) << (threadIdx.x & 31 & ~(N - 1)) : ~0u;
#pragma unroll
    for (int o = kLanes / 2; o > 0; o >>= 1)
        v += __shfl_xor_sync(lanes, v, o);
    if (N <= 32)
        return v;
    if ((threadIdx.x & 31) == 0)
        red[threadIdx.x >> 5] = v;
    group_barrier(group, N);
    float s = red[group * (N / 32)];
#pragma unroll
    for (int w = 1; w < N / 32; ++w)
        s += red[group * (N / 32) + w];
    return s;
}

// CTAs of 256 threads per SM: what the registers allow, but for up to 56 bytes of spills with twelve pieces (32,768 x
// 5,120 bf16 layer norm: 124 us with three CTAs and twelve pieces, 130 with two and sixteen).
constexpr int fwd_per_sm(int pieces) { return pieces > 12 ? 2 : pieces > 4 ? 3 : 4; }

// N threads take a row, P of its whole 16-byte pieces to a thread, kept as they were read: one read of x, all of it
// asked for at once, and with N <= 32 no barrier.  The elements before and after the whole pieces go to the row's first
// threads, one to each.  A group takes `reps` rows in turn.
//
// Bound: HBM.  32,768 x 4,096 bf16 take 92 us (5,850 GB/s) as layer norm, 76 (5,670) as root-mean-square norm with 0.6 of
// the rows supervised; 32,768 x 8,192 184 (5,830); with rows off 16-byte boundaries the 4,096 columns take 96.  Fewer
// warps (14 per SM) with all of a row's loads out beat many: the pieces stay packed, and converting them twice is cheaper
// than the registers of their values (137 us at 4,096 with spills).
template <typename TX, typename TY, int N, int P>
__global__ void __launch_bounds__(256, fwd_per_sm(P)) k_norm_fwd(NormCall c, int reps)
{
    using X = Piece<TX>;
    constexpr int W = X::W, kPer = 256 / N;
    static_assert(N >= 2 * (W - 1), "a thread to each end");
    extern __shared__ __align__(16) float2 planes[];
    __shared__ float red[4][8];
    const int t = threadIdx.x % N, group = threadIdx.x / N, d = (int)c.d, S = plane_size<W>(d);
    const bool layer = c.kind == TURNOPD_LAYER_NORM;
    const float inv_d = 1.f / (float)d;
    for (int j = threadIdx.x; j < d; j += 256)
        planes[(j & (W - 1)) * S + j / W] =
            make_float2(param(c.gamma, c.param_dtype, j), c.beta ? param(c.beta, c.param_dtype, j) : 0.f);
    __syncthreads();
    int sums = 0;  // taken so far: the next one's place in `red`, which is free again two sums later
    for (int rep = 0; rep < reps; ++rep) {
        const int64_t i = ((int64_t)blockIdx.x * reps + rep) * kPer + group;
        if (i >= c.T)
            break;
        const TX *x = static_cast<const TX *>(c.x) + i * c.ldx;
        TY *y = static_cast<TY *>(c.y) + i * c.ldy;
        const int head = min((int)((16 - (reinterpret_cast<uintptr_t>(x) & 15)) & 15) / (int)sizeof(TX), d);
        const int whole = (d - head) / W, ends = d - whole * W;
        const int end = t < head ? t : whole * W + t;  // the column of this thread's single element
        constexpr int kOut = (int)sizeof(TY) * W < 16 ? (int)sizeof(TY) * W : 16;  // a piece's store is aligned to this
        const bool vector_out = (reinterpret_cast<uintptr_t>(y + head) & (kOut - 1)) == 0;
        const auto put = [&](int k, const float2(&o)[W / 2]) {
            TY *to = y + head + (k * N + t) * W;
            if (vector_out) {
                store_piece<W>(to, o);
            } else {
#pragma unroll
                for (int h = 0; h < W; ++h)
                    to[h] = from_float<TY>(h & 1 ? o[h / 2].y : o[h / 2].x);
            }
        };
        // The sums are taken for masked rows too (of nothing): no barrier stands under a condition that every thread
        // reads from the caller's memory for itself.
        const bool on = !c.mask || c.mask[i];
        float mu = 0.f, r = 0.f, z = 0.f;
        uint4 v[P];
        if (on) {
            const uint4 *p = reinterpret_cast<const uint4 *>(x + head) + t;
#pragma unroll
            for (int k = 0; k < P; ++k)
                v[k] = k * N + t < whole ? __ldcs(p + k * N) : make_uint4(0u, 0u, 0u, 0u);
            if (t < ends)
                z = to_float(x[end]);
        }
        if (layer) {
            float2 s = make_float2(z, 0.f);
            if (on) {
#pragma unroll
                for (int k = 0; k < P; ++k)
#pragma unroll
                    for (int j = 0; j < W / 2; ++j)
                        s = fadd2(s, X::pair(v[k], j));
            }
            // divided, not times 1/d: a sum that is exact (a row of equal numbers) has its exact mean
            mu = group_sum<N>(s.x + s.y, red[sums++ & 3], group) / (float)d;
        }
        // in a block of its own: in one with the loop above the compiler keeps the unpacked pieces, and spills
        float2 q = make_float2(t < ends ? (z - mu) * (z - mu) : 0.f, 0.f);
        if (on) {
#pragma unroll
            for (int k = 0; k < P; ++k)
                if (k * N + t < whole)
#pragma unroll
                    for (int j = 0; j < W / 2; ++j) {
                        const float2 u = fadd2(X::pair(v[k], j), splat(-mu));
                        q = ffma2(u, u, q);
                    }
        }
        const float squares = group_sum<N>(q.x + q.y, red[sums++ & 3], group) * inv_d;
        if (on) {
            r = 1.f / sqrtf(squares + c.eps);
            if (!(isfinite(mu) && isfinite(r) && r > 0.f)) {
                r = 0.f;
                if (t == 0)
                    set_status(c.status, TURNOPD_ERR_NONFINITE);
            }
        }
        if (r == 0.f)
            mu = 0.f;
        if (r != 0.f) {
            // xh = (x - mu) r, as the backward pass takes it: x r - mu r would be off by half a unit of mu r
            int at[W];  // gamma and beta of the h-th columns of this thread's pieces
#pragma unroll
            for (int h = 0; h < W; ++h)
                at[h] = ((head + h) & (W - 1)) * S + (head + h) / W + t;
#pragma unroll
            for (int k = 0; k < P; ++k) {
                if (k * N + t >= whole)
                    break;
                float2 o[W / 2];
#pragma unroll
                for (int j = 0; j < W / 2; ++j) {
                    const float2 a = planes[at[2 * j] + k * N], b = planes[at[2 * j + 1] + k * N];
                    const float2 xh = fmul2(fadd2(X::pair(v[k], j), splat(-mu)), splat(r));
                    o[j].x = fmaf(xh.x, a.x, a.y);
                    o[j].y = fmaf(xh.y, b.x, b.y);
                }
                put(k, o);
            }
            if (t < ends) {
                const float2 a = planes[(end & (W - 1)) * S + end / W];
                y[end] = from_float<TY>(fmaf((z - mu) * r, a.x, a.y));
            }
        } else {
            const float2 zero[W / 2] = {};
            for (int k = 0; k * N + t < whole; ++k)
                put(k, zero);
            if (t < ends)
                y[end] = from_float<TY>(0.f);
        }
        if (t == 0) {
            if (c.mean)
                c.mean[i] = mu;
            if (c.rstd)
                c.rstd[i] = r;
        }
    }
}

// Rows longer than kMaxRow: three reads, of which the second and third come from the caches.
template <typename TX, typename TY> __global__ void __launch_bounds__(kThreads) k_norm_fwd_long(NormCall c)
{
    __shared__ float red[kWarps];
    const bool layer = c.kind == TURNOPD_LAYER_NORM;
    for (int64_t i = blockIdx.x; i < c.T; i += gridDim.x) {
        const TX *x = static_cast<const TX *>(c.x) + i * c.ldx;
        TY *y = static_cast<TY *>(c.y) + i * c.ldy;
        float mu = 0.f, r = 0.f;
        // one thread looks, and all go by what it saw: the sums below are the block's
        bool fine = __syncthreads_or(threadIdx.x == 0 && (!c.mask || c.mask[i]));
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

constexpr int kBwdSingles = 8;  // columns of a thread where they are read one by one
constexpr int kStages = 3;  // rows in flight per group: the one at hand and two ahead

__device__ __forceinline__ float2 sum2(float2 v)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
        v = fadd2(v, make_float2(__shfl_xor_sync(~0u, v.x, o), __shfl_xor_sync(~0u, v.y, o)));
    return v;
}

// One pass over x and dy: every thread keeps its columns of gamma, dgamma and dbeta in registers from row to row.
// Group b of all takes rows b, b + groups, ... of the list of supervised tokens (of all tokens, without a list), so that
// the sums are in a fixed order.
//
// kPieces: the three arrays' rows begin at the same element of a group of eight.  The groups' number is a multiple of eight,
// so all rows of one group begin there too, and a thread keeps the same columns from row to row wherever the rows begin:
// pieces of eight from the row's first boundary on, and the first threads one of the elements before and after the whole
// pieces each.  (With a list of rows, only where every row begins at a boundary.)  The pieces come through a ring in
// shared memory, in which each thread copies and reads its own only: no barrier but the one of the row's two sums.
// kWhole is the same without ends, and kSingles reads column by column.  Missing columns are zeros throughout.
//
// Bound: HBM, with the arithmetic of both dx and dgamma close behind (0.57 of the issue slots).  32,768 x 5,120, bf16 x and
// dx, fp32 dy, 0.6 of the rows supervised: 159 us with the sum over blocks, 5,930 GB/s.  16,384 x 4,096 with rows off
// boundaries: kPieces 140 us, kSingles 268.
enum BwdForm {
    kSingles,  // any rows, column by column
    kPieces,   // rows that begin anywhere, but in all three arrays alike
    kWhole,    // rows that begin at boundaries, d a multiple of eight: no ends
};

template <typename TX, typename TDY, typename TDX, BwdForm FORM, bool WIDE>
__global__ void __launch_bounds__(FORM ? (WIDE ? 512 : 320) : (WIDE ? 1024 : 512), FORM && !WIDE ? 2 : 1)
k_norm_bwd(NormGradCall c, const int4 *__restrict__ rows, const int32_t *__restrict__ nvalid, int n)
{
    constexpr bool VEC = FORM != kSingles, ENDS = FORM == kPieces;
    constexpr int kE = VEC ? turnopd::kE : kBwdSingles;
    // 128 bytes: 32,768 x 5,120 take 159 us, and 170 with a ring that begins 16 bytes off
    extern __shared__ __align__(128) char ring[];
    __shared__ __align__(16) float2 red[2][32];
    __shared__ int list_length;
    constexpr int W = VEC ? 8 : 1, P = kE / W;  // columns to a piece, pieces to a thread
    const int t = threadIdx.x % n, group = threadIdx.x / n, warps = n / 32, per = blockDim.x / n;
    const int groups = gridDim.x * per, b = blockIdx.x * per + group, d = (int)c.d;
    // one thread reads the list's length and all go by what it read: it says how often the groups meet at their barriers
    if (rows) {
        if (threadIdx.x == 0)
            list_length = *nvalid;
        __syncthreads();
    }
    const int count = rows ? list_length : (int)c.T;
    const bool layer = c.kind == TURNOPD_LAYER_NORM;
    const float inv_d = 1.f / (float)d;
    const int xbytes = (int)sizeof(TX) * n * kE, stage = (int)(sizeof(TX) + sizeof(TDY)) * n * kE;
    char *own = ring + group * kStages * stage;
    const int head = ENDS ? min((int)(-(reinterpret_cast<intptr_t>(static_cast<const TX *>(c.x) + b * c.ldx) / (int)sizeof(TX)) & 7), d) : 0;
    const int whole = VEC ? (d - head) / 8 : d, ends = ENDS ? d - whole * 8 : 0;
    const int end = t < head ? t : whole * 8 + t;  // the single column of this thread, where t < ends
    const auto column = [&](int k) { return head + (k * n + t) * W; };  // of piece k
    const auto there = [&](int k) { return k * n + t < whole; };

    float2 gamma[kE / 2], dg[kE / 2], db[kE / 2];
#pragma unroll
    for (int k = 0; k < kE / 2; ++k)
        gamma[k] = dg[k] = db[k] = make_float2(0.f, 0.f);
    float *gam = reinterpret_cast<float *>(gamma);
    const auto load_gamma = [&](const auto *g) {
#pragma unroll
        for (int k = 0; k < P; ++k)
            if (there(k)) {
                if (FORM == kWhole && (reinterpret_cast<uintptr_t>(g) & 15) == 0) {
                    if constexpr (FORM == kWhole)
                        load8(g + column(k), gam + k * W);
                } else {
#pragma unroll
                    for (int e = 0; e < W; ++e)
                        gam[k * W + e] = to_float(__ldg(g + column(k) + e));
                }
            }
    };
    if (c.param_dtype == TURNOPD_BF16)
        load_gamma(static_cast<const __nv_bfloat16 *>(c.gamma));
    else
        load_gamma(static_cast<const float *>(c.gamma));
    const float gamma_end = ENDS && t < ends ? param(c.gamma, c.param_dtype, end) : 0.f;
    float dg_end = 0.f, db_end = 0.f;
    if constexpr (VEC) {
#pragma unroll
        for (int k = 0; k < P; ++k)
            if (!there(k))
                for (int s = 0; s < kStages; ++s) {
                    const int at = (k * n + t) * 8;
                    for (int h = 0; h < (int)sizeof(TX) / 2; ++h)
                        reinterpret_cast<uint4 *>(own + s * stage + at * sizeof(TX))[h] = make_uint4(0, 0, 0, 0);
                    for (int h = 0; h < (int)sizeof(TDY) / 2; ++h)
                        reinterpret_cast<uint4 *>(own + s * stage + xbytes + at * sizeof(TDY))[h] = make_uint4(0, 0, 0, 0);
                }
    }

    // the row at a place of the list, -1 past its end (32 bits hold three groups' steps beyond 2^31 - 1)
    const auto row_of = [&](uint32_t at) -> int {
        if (at >= (uint32_t)count)
            return -1;
        return rows ? rows[at].x : (int)at;
    };
    const auto on = [&](int i) { return i >= 0 && (rows || !c.mask || c.mask[i]); };
    const auto copy = [&](int i, int s) {
        if (on(i)) {
            const TX *x = static_cast<const TX *>(c.x) + i * c.ldx;
            const TDY *dy = static_cast<const TDY *>(c.dy) + i * c.lddy;
            char *to = own + s * stage;
#pragma unroll
            for (int k = 0; k < P; ++k) {
                if (!there(k))
                    continue;
                const int j = column(k), at = (k * n + t) * 8;
#pragma unroll
                for (int h = 0; h < 8; h += 16 / (int)sizeof(TX))
                    cp16(to + (at + h) * (int)sizeof(TX), x + j + h);
#pragma unroll
                for (int h = 0; h < 8; h += 16 / (int)sizeof(TDY))
                    cp16(to + xbytes + (at + h) * (int)sizeof(TDY), dy + j + h);
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    int i = row_of(b), i1 = row_of(b + groups), i2 = row_of(b + 2 * groups);
    if constexpr (VEC) {
        copy(i, 0);
        copy(i1, 1);
    }
    // a row's numbers and this thread's single column are read a row ahead
    float mu = 0.f, r = 0.f, xe = 0.f, dye = 0.f;
    const auto numbers = [&](int i, float &mu, float &r, float &xe, float &dye) {
        mu = r = xe = dye = 0.f;
        if (on(i)) {
            mu = layer ? c.mean[i] : 0.f;
            r = c.rstd[i];
            if (ENDS && t < ends) {
                xe = to_float(static_cast<const TX *>(c.x)[i * c.ldx + end]);
                dye = to_float(static_cast<const TDY *>(c.dy)[i * c.lddy + end]);
            }
        }
    };
    numbers(i, mu, r, xe, dye);
    int s = 0;
    for (uint32_t at = b, odd = 0; at < (uint32_t)count; at += groups, odd ^= 1) {
        const int i3 = row_of(at + 3 * groups);
        if constexpr (VEC)
            copy(i2, s >= 1 ? s - 1 : s + 2);
        float mu1, r1, xe1, dye1;
        numbers(i1, mu1, r1, xe1, dye1);
        if constexpr (VEC)
            asm volatile("cp.async.wait_group 2;" ::: "memory");
        TDX *dx = static_cast<TDX *>(c.dx) + i * c.lddx;
        // (as in the forward pass, the sums are taken whatever rstd says)
        float2 sg = make_float2(0.f, 0.f), sx = sg;
        float2 x[kE / 2], dy[kE / 2];  // xh and dy; pieces are read from the ring once more for dx instead
        if (r > 0.f) {
#pragma unroll
            for (int k = 0; k < P; ++k) {
                if constexpr (VEC) {
                    float2 *xk = x + k * W / 2, *dyk = dy + k * W / 2;
                    load8(reinterpret_cast<const TX *>(own + s * stage) + (k * n + t) * 8, reinterpret_cast<float *>(xk));
                    load8(reinterpret_cast<const TDY *>(own + s * stage + xbytes) + (k * n + t) * 8, reinterpret_cast<float *>(dyk));
                } else {
                    const int j = column(k);
                    reinterpret_cast<float *>(x)[k] = j < d ? to_float(static_cast<const TX *>(c.x)[i * c.ldx + j]) : 0.f;
                    reinterpret_cast<float *>(dy)[k] = j < d ? to_float(static_cast<const TDY *>(c.dy)[i * c.lddy + j]) : 0.f;
                }
            }
#pragma unroll
            for (int k = 0; k < kE / 2; ++k) {
                x[k] = fmul2(fadd2(x[k], splat(-mu)), splat(r));
                const float2 g = fmul2(dy[k], gamma[k]);
                sg = fadd2(sg, g);
                sx = ffma2(g, x[k], sx);
                dg[k] = ffma2(dy[k], x[k], dg[k]);
                db[k] = fadd2(db[k], dy[k]);
            }
            if (ENDS) {
                xe = t < ends ? (xe - mu) * r : 0.f;
                const float g = dye * gamma_end;
                sg.x += g;
                sx.x = fmaf(g, xe, sx.x);
                dg_end = fmaf(dye, xe, dg_end);
                db_end += dye;
            }
        }
        if (c.dx) {
            float2 v = sum2(make_float2(sg.x + sg.y, sx.x + sx.y));
            if (warps > 1) {
                float2 *to = red[odd];
                const int first = group * warps;
                if ((threadIdx.x & 31) == 0)
                    to[threadIdx.x >> 5] = v;
                group_barrier(group, n);
                v = to[first];
#pragma unroll 2
                for (int w = 1; w < warps; ++w)
                    v = fadd2(v, to[first + w]);
            }
            if (r > 0.f) {
                // dx = r g + xh (-r mean(g xh)) - r mean g
                const float2 c0 = splat(layer ? -r * (v.x * inv_d) : 0.f), c1 = splat(-r * (v.y * inv_d));
#pragma unroll
                for (int k = 0; k < P; ++k) {
                    const int j = column(k);
                    if constexpr (VEC) {
                        float2 xk[4], dyk[4];
                        load8(reinterpret_cast<const TX *>(own + s * stage) + (k * n + t) * 8, reinterpret_cast<float *>(xk));
                        load8(reinterpret_cast<const TDY *>(own + s * stage + xbytes) + (k * n + t) * 8, reinterpret_cast<float *>(dyk));
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const float2 xh = fmul2(fadd2(xk[e], splat(-mu)), splat(r));
                            xk[e] = ffma2(fmul2(dyk[e], gamma[4 * k + e]), splat(r), ffma2(xh, c1, c0));
                        }
                        if (there(k))
                            store8(dx + j, reinterpret_cast<const float *>(xk));
                    } else if (j < d) {
                        const float g = reinterpret_cast<const float *>(dy)[k] * gam[k];
                        dx[j] = from_float<TDX>(fmaf(g, r, fmaf(reinterpret_cast<const float *>(x)[k], c1.x, c0.x)));
                    }
                }
                if (ENDS && t < ends)
                    dx[end] = from_float<TDX>(fmaf(dye * gamma_end, r, fmaf(xe, c1.x, c0.x)));
            } else {
                const float zero[8] = {};
#pragma unroll
                for (int k = 0; k < P; ++k) {
                    if (there(k)) {
                        if constexpr (VEC)
                            store8(dx + column(k), zero);
                        else
                            dx[column(k)] = from_float<TDX>(0.f);
                    }
                }
                if (ENDS && t < ends)
                    dx[end] = from_float<TDX>(0.f);
            }
        }
        i = i1;
        i1 = i2;
        i2 = i3;
        mu = mu1;
        r = r1;
        xe = xe1;
        dye = dye1;
        s = s == 2 ? 0 : s + 1;
    }
    if (c.dgamma || c.dbeta) {
        // the block's groups are added up first, in shared memory, in their order: one row of partial sums per block
        // (rows that begin anywhere go there too, to be written out in order)
        const bool one = per == 1 && FORM != kPieces;
        float *part = one ? static_cast<float *>(c.workspace) + (int64_t)blockIdx.x * 2 * d
                          : reinterpret_cast<float *>(ring) + group * 2 * d;
        if (!one) {
            if constexpr (VEC)
                asm volatile("cp.async.wait_all;" ::: "memory");
            __syncthreads();
        }
        const float *dgs = reinterpret_cast<const float *>(dg), *dbs = reinterpret_cast<const float *>(db);
#pragma unroll
        for (int k = 0; k < P; ++k)
            if (there(k)) {
                float *g = part + column(k), *e = g + d;
                if constexpr (FORM == kWhole) {
#pragma unroll
                    for (int h = 0; h < 8; h += 4) {
                        const float *a = dgs + k * W + h, *z = dbs + k * W + h;
                        *reinterpret_cast<float4 *>(g + h) = make_float4(a[0], a[1], a[2], a[3]);
                        *reinterpret_cast<float4 *>(e + h) = make_float4(z[0], z[1], z[2], z[3]);
                    }
                } else {
#pragma unroll
                    for (int h = 0; h < W; ++h) {
                        g[h] = dgs[k * W + h];
                        e[h] = dbs[k * W + h];
                    }
                }
            }
        if (ENDS && t < ends) {
            part[end] = dg_end;
            part[d + end] = db_end;
        }
        if (!one) {
            __syncthreads();
            const float *all = reinterpret_cast<const float *>(ring);
            for (int j = threadIdx.x; j < 2 * d; j += blockDim.x) {
                float sum = all[j];
                for (int g = 1; g < per; ++g)
                    sum += all[g * 2 * d + j];
                static_cast<float *>(c.workspace)[(int64_t)blockIdx.x * 2 * d + j] = sum;
            }
        }
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
                    for (int j = lane * 8; j + 8 <= d; j += 256)
                        store8(dx + j, zero);
                    if (lane < (d & 7))
                        dx[(d & ~7) + lane] = from_float<TDX>(0.f);
                } else {
                    for (int j = lane; j < d; j += 32)
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
    pdl_begin();
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

// Rows longer than kMaxRow.
template <typename TX, typename TDY, typename TDX>
__global__ void __launch_bounds__(kThreads) k_norm_dx(NormGradCall c)
{
    __shared__ float red[kWarps];
    const bool layer = c.kind == TURNOPD_LAYER_NORM;
    for (int64_t i = blockIdx.x; i < c.T; i += gridDim.x) {
        const TX *x = static_cast<const TX *>(c.x) + i * c.ldx;
        const TDY *dy = static_cast<const TDY *>(c.dy) + i * c.lddy;
        TDX *dx = static_cast<TDX *>(c.dx) + i * c.lddx;
        if (!__syncthreads_or(threadIdx.x == 0 && takes_part(c, i))) {
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

constexpr int kMaxGrid = 320;         // CTAs of the backward pass, at most
constexpr int kLongParts = 64;        // partial sums of the kernels for long rows
// Elements from which a loss mask is turned into a list of rows, two launches that take 5 us.  bf16 x, fp32 dy, 0.6 of the
// rows supervised, us without a list and with one.  Below the limit: 8,192 x 1,024 16.0 and 20.5, 1,024 x 8,192 21.3 and
// 24.2, 2,048 x 5,120 23.2 and 25.1, but 2,048 x 6,000 30.2 and 27.1.  From it on: 32,768 x 640 37.5 and 35.2, 2,048 x 8,192
// 33.2 and 31.4, 4,096 x 5,120 37.1 and 36.9, 8,192 x 2,560 41.4 and 36.5, 16,384 x 5,120 109 and 89, but 16,384 x 1,024 23.7
// and 26.7, 4,096 x 4,096 29.1 and 29.5, 65,536 x 256 30.4 and 30.8.  These four exceptions cost 13 % at most.
constexpr int64_t kListFrom = 1 << 24;

int row_threads(int64_t d, int columns = kE) { return (int)((d + columns * 32 - 1) / (columns * 32)) * 32; }
int rows_per_cta(int64_t d, int columns = kE) { return std::max(1, kThreads / row_threads(d, columns)); }

int64_t partial_rows(int64_t T, int64_t d)
{
    return d > kMaxRow ? std::min<int64_t>(std::max<int64_t>(T, 1), kLongParts) : std::min<int64_t>(T + 8, kMaxGrid);
}

// The element of a group of eight at which row 0 of an array begins, and by how many the next row begins later.
struct Start {
    int at, step;
    Start(const void *p, int64_t ld, int32_t dtype)
        : at((int)(reinterpret_cast<uintptr_t>(p) / (dtype == TURNOPD_BF16 ? 2 : 4) & 7)), step((int)(ld & 7))
    {
    }
    bool operator==(const Start &o) const { return at == o.at && step == o.step; }
    bool boundary() const { return at == 0 && step == 0; }
};

template <typename X, typename Y, int N, int P> cudaError_t launch_fwd_rows(const NormCall &c, cudaStream_t stream)
{
    constexpr int W = Piece<X>::W, kPer = 256 / N;
    const int64_t ctas = (c.T + kPer - 1) / kPer;
    // every CTA lays gamma and beta out first: for several rows where there are many, but in several rounds of CTAs, so
    // that those with more masked rows do not leave the device idle at the end
    const int64_t round = device_sm_count() * fwd_per_sm(P);
    const int reps = (int)std::min<int64_t>(16, std::max<int64_t>(1, ctas / (4 * round)));
    const size_t smem = sizeof(float2) * W * plane_size<W>((int)c.d);
    auto kernel = k_norm_fwd<X, Y, N, P>;
    const cudaError_t e = allow_shared(kernel, sizeof(float2) * W * plane_size<W>(N * P * W));  // d / W <= N P pieces
    if (e != cudaSuccess)
        return e;
    kernel<<<(unsigned)((ctas + reps - 1) / reps), 256, smem, stream>>>(c, reps);
    return cudaGetLastError();
}

// Many rows: as few threads to a row as hold it, so that many rows are in flight and most need no barrier.  Few rows:
// many threads to each, which answer sooner (300 rows x 4,096 bf16: 4.2 us with 128 threads, 5.4 with 32; 2,000 rows: 9.3
// and 7.7).
template <typename X, typename Y> cudaError_t launch_fwd(const NormCall &c, cudaStream_t stream)
{
    const int64_t pieces = c.d / Piece<X>::W;
    const bool few = c.T * ((pieces + 511) / 512) < 8 * device_sm_count();
    if (c.d > kMaxRow) {
        const int grid = (int)std::min<int64_t>(c.T, (int64_t)device_sm_count() * 8);
        k_norm_fwd_long<X, Y><<<grid, kThreads, 0, stream>>>(c);
        return cudaGetLastError();
    }
    if (pieces <= 16 * 4)
        return launch_fwd_rows<X, Y, 16, 4>(c, stream);
    if (pieces <= 32 * 4)
        return launch_fwd_rows<X, Y, 32, 4>(c, stream);
    if (few && pieces <= 128 * 4)
        return launch_fwd_rows<X, Y, 128, 4>(c, stream);
    if (few && pieces <= 256 * 4)
        return launch_fwd_rows<X, Y, 256, 4>(c, stream);
    if (pieces <= 32 * 8)
        return launch_fwd_rows<X, Y, 32, 8>(c, stream);
    if (pieces <= 32 * 12)
        return launch_fwd_rows<X, Y, 32, 12>(c, stream);
    if (pieces <= 32 * 16)
        return launch_fwd_rows<X, Y, 32, 16>(c, stream);
    if (pieces <= 64 * 12)
        return launch_fwd_rows<X, Y, 64, 12>(c, stream);
    if (pieces <= 64 * 16)
        return launch_fwd_rows<X, Y, 64, 16>(c, stream);
    return launch_fwd_rows<X, Y, 128, 16>(c, stream);
}

template <typename X, typename DY, typename DX>
cudaError_t launch_bwd(const NormGradCall &c, BwdForm form, const int4 *rows, const int32_t *nvalid, int *parts,
                       cudaStream_t stream)
{
    const bool vec = form != kSingles;
    const int columns = vec ? kE : kBwdSingles, n = row_threads(c.d, columns), per = rows_per_cta(c.d, columns);
    const bool wide = vec ? n * per > 320 : n * per > 512;  // one CTA per SM then, else two
    const int64_t most = std::min<int64_t>((wide ? 1 : 2) * device_sm_count(), kMaxGrid);
    // two rows to a group at least, once there is one for every SM: each block's partial sums are written and read again
    // (512 rows x 4,096: one row 10.8 us, two 9.9, eight 13.6)
    const int64_t blocks = (c.T + per - 1) / per;
    int grid = (int)std::min<int64_t>(blocks > device_sm_count() ? (blocks + 1) / 2 : blocks, most);
    if (form == kPieces)
        grid = std::min((grid * per + 7) / 8 * 8 / per, kMaxGrid);  // a multiple of eight groups
    *parts = grid;
    const size_t row = (sizeof(X) + sizeof(DY)) * n * columns;
    const size_t smem = per * std::max<size_t>(vec ? kStages * row : 0, per > 1 ? sizeof(float) * 2 * (size_t)c.d : 0);
    auto kernel = form == kWhole    ? (wide ? k_norm_bwd<X, DY, DX, kWhole, true> : k_norm_bwd<X, DY, DX, kWhole, false>)
                  : form == kPieces ? (wide ? k_norm_bwd<X, DY, DX, kPieces, true> : k_norm_bwd<X, DY, DX, kPieces, false>)
                                    : (wide ? k_norm_bwd<X, DY, DX, kSingles, true> : k_norm_bwd<X, DY, DX, kSingles, false>);
    // pieces: the ring of a whole block, and no less than a group's 8 d bytes of sums with n * 16 >= d; single columns: the
    // sums of the groups of 256 threads
    const cudaError_t e = allow_shared(kernel, vec ? kStages * (sizeof(X) + sizeof(DY)) * (wide ? 512 : 320) * kE
                                                   : sizeof(float) * 2 * kThreads * kBwdSingles);
    if (e != cudaSuccess)
        return e;
    kernel<<<grid, n * per, smem, stream>>>(c, rows, nvalid, n);
    return cudaGetLastError();
}

}  // namespace

size_t norm_bwd_workspace_bytes(int64_t T, int64_t d)
{
    const int64_t nblk = (T + kCompactBlock - 1) / kCompactBlock;
    return align256(sizeof(float) * 2 * (size_t)d * (size_t)partial_rows(T, d)) +
           (T * d >= kListFrom ? align256(sizeof(int4) * (size_t)T) + align256(sizeof(int32_t) * (size_t)(nblk + 1)) + 256 : 0);
}

cudaError_t launch_norm_fwd(const NormCall &c, cudaStream_t stream)
{
    cudaError_t e = cudaSuccess;
    with_types(c.x_dtype, c.y_dtype, [&](auto x, auto y) { e = launch_fwd<decltype(x), decltype(y)>(c, stream); });
    return e;
}

cudaError_t launch_norm_bwd(const NormGradCall &c, cudaStream_t stream)
{
    cudaError_t e = cudaSuccess;
    int parts = 0;
    const bool sums = c.dgamma || c.dbeta;
    if (c.d > kMaxRow) {
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
        const Start x0(c.x, c.ldx, c.x_dtype);
        const bool vec = x0 == Start(c.dy, c.lddy, c.dy_dtype) && (!c.dx || x0 == Start(c.dx, c.lddx, c.dx_dtype));
        const BwdForm form = !vec ? kSingles : x0.boundary() && c.d % 8 == 0 ? kWhole : kPieces;
        if (c.mask && c.T * c.d >= kListFrom && sums && (!vec || x0.boundary())) {
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
        with_types(c.x_dtype, c.dy_dtype, [&](auto x, auto dy) {
            using X = decltype(x);
            using DY = decltype(dy);
            e = c.dx_dtype == TURNOPD_BF16 ? launch_bwd<X, DY, __nv_bfloat16>(c, form, rows, nvalid, &parts, stream)
                                           : launch_bwd<X, DY, float>(c, form, rows, nvalid, &parts, stream);
        });
    }
    if (e == cudaSuccess && sums) {
        e = launch_dependent(k_norm_bwd_sum, dim3((unsigned)((2 * c.d + 31) / 32)), dim3(1024), 0, stream, c, parts);
    }
    return e;
}

}  // namespace turnopd
