// Log probabilities of given tokens with the row's entropy and top alternatives, and their
// gradient with respect to the logits.
//
// Row z[0..V), m = max z, S = sum e^{z-m}:
//   log p_v = (z_v - m) - log S,   H = log S - A / S,   A = sum e^{z-m} (z - m),
//   dL/dz_v = dL/dlp (delta_vy - p_v) - dL/dH p_v (log p_v + H).
// The sums leave the given token y out and take its term at the end: where y is all but certain,
// log p_y = -log1p(S') with S' = sum_{v != y} e^{z-m} keeps its relative precision, and so does
// H = log1p(S') - A / S, whose two terms then have one sign.

#include <cooperative_groups.h>

#include <algorithm>

#include "common.cuh"
#include "kernels.h"
#include "packed.cuh"

namespace turnopd {
namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;

// Logits at or below this are masked values: they have probability 0, and a row with nothing else has no distribution.
// It is where the running maximum starts.  Lower logits (-inf, the type's lowest value) are raised to kClamp for the
// sums, so that z - m and e^{z-m} (z - m) stay finite, for maxima up to -kMaskedBelow.
constexpr float kMaskedBelow = -0x1p+126f;
constexpr float kClamp = -0x1.8p+126f;
constexpr uint32_t kClampBf16x2 = 0xfec0fec0u;

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

// Part of a row: its largest logit m, S = sum e^{z-m} and A = sum e^{z-m} (z - m) log2 e.
struct Part {
    float m, s, a;
};

__device__ __forceinline__ Part part_empty() { return Part{kMaskedBelow, 0.f, 0.f}; }

// The part's sums about another reference m.
__device__ __forceinline__ Part part_about(Part p, float m)
{
    const float d = (p.m - m) * kLog2e, f = ex2(d);
    return Part{m, p.s * f, fmaf(d, p.s, p.a) * f};
}

// Merges across the warp: the exact maximum, one change of reference, then sums (a fixed tree).
__device__ __forceinline__ Part part_warp(Part p)
{
    p = part_about(p, warp_max_f(p.m));
    return Part{p.m, warp_sum_f(p.s), warp_sum_f(p.a)};
}

__device__ __forceinline__ uint4 ldg_stream(const uint4 *p)
{
    uint4 v;
    asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
                 : "l"(p));
    return v;
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

// ---------------------------------------------------------------- 16-byte vectors of logits

__device__ __forceinline__ uint32_t max_nan_bf16x2(uint32_t a, uint32_t b)
{
    uint32_t d;
    asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
__device__ __forceinline__ float max_nan(float a, float b)
{
    float d;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
    return d;
}

// Two logits into the sums about m (NaN stays NaN).
__device__ __forceinline__ void fold2(float2 z, float2 minus_m, float2 &S, float2 &A)
{
    const float2 x = fmul2(fadd2(z, minus_m), splat(kLog2e));
    const float2 e = ex2x2(x);
    S = fadd2(S, e);
    A = ffma2(e, x, A);
}

template <typename TIn> struct Logits;
template <> struct Logits<__nv_bfloat16> {
    static constexpr int N = 8;
    static constexpr uint32_t kHole = 0xff80ff80u;  // -inf
    template <int U> __device__ static float max_of(const uint4 (&v)[U])
    {
        uint32_t m = hmax4(v[0]);
#pragma unroll
        for (int u = 1; u < U; ++u)
            m = hmax2u(m, hmax4(v[u]));
        return fmaxf(bf16lo(m), bf16hi(m));
    }
    __device__ static void fold(const uint4 &v, float2 minus_m, float2 &S, float2 &A)
    {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            fold2(unpack2(max_nan_bf16x2(word(v, j), kClampBf16x2)), minus_m, S, A);
    }
    __device__ static float at(const uint4 &v, int j)
    {
        const uint32_t w = word(v, j >> 1);
        return j & 1 ? bf16hi(w) : bf16lo(w);
    }
    __device__ static uint32_t without(uint32_t w, int j) { return j & 1 ? (w & 0xffffu) | 0xff800000u : (w & 0xffff0000u) | 0xff80u; }
    __device__ static int word_of(int j) { return j >> 1; }
};
template <> struct Logits<float> {
    static constexpr int N = 4;
    static constexpr uint32_t kHole = 0xff800000u;
    template <int U> __device__ static float max_of(const uint4 (&v)[U])
    {
        float m = -INFINITY;
#pragma unroll
        for (int u = 0; u < U; ++u)
            m = fmaxf(m, fmaxf(fmaxf(at(v[u], 0), at(v[u], 1)), fmaxf(at(v[u], 2), at(v[u], 3))));
        return m;
    }
    __device__ static void fold(const uint4 &v, float2 minus_m, float2 &S, float2 &A)
    {
#pragma unroll
        for (int j = 0; j < 4; j += 2)
            fold2(make_float2(max_nan(at(v, j), kClamp), max_nan(at(v, j + 1), kClamp)), minus_m, S, A);
    }
    __device__ static float at(const uint4 &v, int j) { return __uint_as_float(word(v, j)); }
    __device__ static uint32_t without(uint32_t, int) { return kHole; }
    __device__ static int word_of(int j) { return j; }
};

// ---------------------------------------------------------------- alternatives
//
// The n best of a row in one pass.  Each chunk of the row is in the threads' registers.  On the first chunk the n-th
// best of the threads' own best logits is a bound that n logits reach, and since fewer than n threads have a better
// one, at most 31 threads' logits (32 each) lie above it: those go to a list in shared memory, and its n-th best is the
// bound from then on.  Later logits have higher ids, so only those strictly above the bound can matter.  The list
// is cut back to n, and the bound raised, when it has grown; a chunk with more logits above the bound than the list
// holds is taken like a first chunk.  Keys are unique, so the outcome does not depend on the order of the list.

constexpr int kU = 4;                             // vectors per thread and chunk
constexpr int kChunk = kU * kThreads;
#ifndef LP_PERSM
#define LP_PERSM 3
#endif
constexpr int kPerSm = LP_PERSM;
constexpr int kListCap = 1088;                    // 32 kept + 31 threads' 32 logits + 1, and the row's ends
constexpr int kListCut = 160;                     // cut the list back from here
constexpr int kTopMax = TURNOPD_TOP_ALTERNATIVES_MAX;

struct TopShared {
    uint64_t list[kListCap];
    uint64_t runs[kThreads];      // kWarps runs of 32 keys in descending order
    uint64_t sorted[kTopMax];
    uint64_t bound;
    int count;
};

// Place of a key, entry `at` of run `own`, among all of kWarps runs of 32 keys in descending order.  Keys differ, but
// for empty entries (0), which have no place.
__device__ __forceinline__ int place_among(uint64_t key, int own, int at, const uint64_t *runs)
{
    int place = at;
#pragma unroll
    for (int w = 1; w < kWarps; ++w) {
        const int o = (own + w) & (kWarps - 1);
        const uint64_t *run = runs + 32 * o;
        int lo = 0;
#pragma unroll
        for (int h = 16; h > 0; h >>= 1)
            lo += run[lo + h - 1] > key ? h : 0;
        place += lo + (lo == 31 && run[31] > key);
    }
    return place;
}

// n-th largest of kThreads keys, one per thread (0: none), in every thread; 0 if there are fewer.
__device__ __forceinline__ uint64_t block_nth(uint64_t key, int n, TopShared &t)
{
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int k = 2; k <= 32; k <<= 1) {
#pragma unroll
        for (int j = k >> 1; j > 0; j >>= 1) {
            const uint64_t o = __shfl_xor_sync(~0u, (unsigned long long)key, j);
            const bool up = (lane & k) != 0 && k < 32;  // this run ascends
            const bool low = (lane & j) == 0;
            key = (low != up) == (key > o) ? key : o;
        }
    }
    if (threadIdx.x == 0)
        t.bound = 0;
    t.runs[threadIdx.x] = key;
    __syncthreads();
    if (key && place_among(key, threadIdx.x >> 5, lane, t.runs) == n - 1)
        t.bound = key;
    __syncthreads();
    return t.bound;
}

// Cuts the list to its n best, in order; the n-th best is the bound.  Entries of ids from `from` on are dropped.
__device__ __forceinline__ void cut_list(int n, TopShared &t, int64_t from = INT64_MAX)
{
    __syncthreads();
    const int m = min(t.count, kListCap);
    if (threadIdx.x < kTopMax)
        t.sorted[threadIdx.x] = 0;
    if (from != INT64_MAX)
        for (int i = threadIdx.x; i < m; i += kThreads)
            if (key_id(t.list[i]) >= from)
                t.list[i] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < m; i += kThreads) {
        const uint64_t key = t.list[i];
        int place = 0;
        for (int j = 0; j < m; ++j)
            place += t.list[j] > key;
        if (place < n)
            t.sorted[place] = key;
    }
    __syncthreads();
    if (threadIdx.x < n)
        t.list[threadIdx.x] = t.sorted[threadIdx.x];
    if (threadIdx.x == 0) {
        t.count = n;
        t.bound = t.sorted[n - 1];
    }
    __syncthreads();
}

__device__ __forceinline__ int list_add(uint64_t key, TopShared &t)
{
    const int at = atomicAdd(&t.count, 1);
    if (at < kListCap)
        t.list[at] = key;
    return at;
}

// A first chunk: vector u of the thread holds ids id0 + u stride + 0..N-1 (none where u >= held).
template <typename TIn>
__device__ __noinline__ void top_chunk(const uint4 (&v)[kU], int held, int64_t id0, int64_t stride, int n, TopShared &t)
{
    using X = Logits<TIn>;
    uint64_t best = 0;
#pragma unroll
    for (int u = 0; u < kU; ++u)
#pragma unroll
        for (int j = 0; j < X::N; ++j)
            if (u < held)
                best = max(best, top_key(X::at(v[u], j), id0 + u * stride + j));
    const uint64_t kept = t.bound;  // of the chunks before, 0 at the row's start
    __syncthreads();
    const uint64_t bound = max(block_nth(best, n, t), kept);
    if (best >= bound && best != 0) {
#pragma unroll
        for (int u = 0; u < kU; ++u)
#pragma unroll
            for (int j = 0; j < X::N; ++j)
                if (u < held) {
                    const uint64_t key = top_key(X::at(v[u], j), id0 + u * stride + j);
                    if (key >= bound)
                        list_add(key, t);
                }
    }
    cut_list(n, t);
}

// ---------------------------------------------------------------- forward kernel

// A row's share of one CTA: `len` of the row's whole 16-byte vectors, from the row's q0-th on; the first starts after
// `head` logits.  CTA 0 of the cluster also takes the logits before and after the row's `nvec` vectors one by one.
struct Share {
    const char *row;
    int32_t head, nvec, q0, len, chunks, token, y;
    float zy;
    bool ok;
};

template <typename TIn>
__device__ __forceinline__ Share get_share(const LogprobCall &c, const int4 *rows, int64_t k, int rank, int ctas)
{
    constexpr int N = Logits<TIn>::N;
    const Row r = get_row(c, rows, k);
    Share s;
    s.token = r.token;
    s.y = r.y;
    s.ok = r.ok;
    const TIn *z = static_cast<const TIn *>(c.logits) + (r.ok ? (int64_t)r.r * c.ld : 0);
    s.row = reinterpret_cast<const char *>(z);
    const int V = r.ok ? (int)c.vocab : 0;
    s.head = min((int)((16 - (reinterpret_cast<uintptr_t>(z) & 15)) & 15) / (int)sizeof(TIn), V);
    s.nvec = (V - s.head) / N;
    const int per = (s.nvec + ctas - 1) / ctas;
    s.q0 = min(s.nvec, rank * per);
    s.len = min(s.nvec, s.q0 + per) - s.q0;
    s.chunks = (s.len + kChunk - 1) / kChunk;
    s.zy = r.ok && r.y >= 0 ? to_float(z[r.y]) : -INFINITY;
    return s;
}

template <typename TIn>
__device__ __forceinline__ void load_chunk(const Share &s, int chunk, uint4 (&v)[kU])
{
    const int q = chunk * kChunk + threadIdx.x;
    const uint4 *p = reinterpret_cast<const uint4 *>(s.row + s.head * sizeof(TIn)) + s.q0 + q;
    const int left = s.len - q;
#pragma unroll
    for (int u = 0; u < kU; ++u) {
        constexpr uint32_t h = Logits<TIn>::kHole;
        v[u] = u * kThreads < left ? ldg_stream(p + u * kThreads) : make_uint4(h, h, h, h);
    }
}

template <typename TIn, bool TOP>
__global__ void __launch_bounds__(kThreads, kPerSm) k_logprobs(LogprobCall c, const int4 *__restrict__ rows,
                                                          const int32_t *__restrict__ nvalid)
{
    using X = Logits<TIn>;
    __shared__ Part parts[kWarps];
    __shared__ Part whole;      // this CTA's part of the row
    __shared__ float norm[3];   // m, log S of the row, 1 if it is fine
    __shared__ TopShared top;
    __shared__ Share shares[2][kWarps];  // each warp its own: no barrier between a row's share and the next one's
    namespace cg = cooperative_groups;
    cg::cluster_group cluster = cg::this_cluster();
    const int rank = (int)cluster.block_rank(), ctas = (int)cluster.num_blocks();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int64_t n = rows ? *nvalid : c.T;
    const int64_t first = blockIdx.x / ctas, step = gridDim.x / ctas;
    uint4 ahead[kU];
    int slot = 0;
    if (first < n) {
        if (lane == 0)
            shares[0][warp] = get_share<TIn>(c, rows, first, rank, ctas);
        __syncwarp();
        load_chunk<TIn>(shares[0][warp], 0, ahead);
    }
    for (int64_t k = first; k < n; k += step, slot ^= 1) {
        const bool more = k + step < n;
        const Share &s = shares[slot][warp], &next = shares[slot ^ 1][warp];
        if (more && lane == 0)
            shares[slot ^ 1][warp] = get_share<TIn>(c, rows, k + step, rank, ctas);
        __syncwarp();
        // where y lies: in this thread's vector uy of chunk cy, or nowhere
        int cy = -1, uy = 0;
        if (s.y >= s.head) {
            const int f = (s.y - s.head) / X::N - s.q0;
            if (f >= 0 && f < s.len && (f & (kThreads - 1)) == (int)threadIdx.x) {
                cy = f / kChunk;
                uy = f / kThreads & (kU - 1);
            }
        }
        const int chunks = s.chunks;
        if (TOP && threadIdx.x == 0) {
            top.count = 0;
            top.bound = 0;
        }
        float m = kMaskedBelow;
        float2 S = splat(0.f), A = splat(0.f);
        float bound = -INFINITY;
        for (int chunk = 0; chunk < chunks; ++chunk) {
            uint4 v[kU];
#pragma unroll
            for (int u = 0; u < kU; ++u)
                v[u] = ahead[u];
            const bool last = chunk + 1 == chunks;
            if (!last || more)
                load_chunk<TIn>(last ? next : s, last ? 0 : chunk + 1, ahead);
            const float vm = X::max_of(v);
            if (TOP) {
                const int q = chunk * kChunk + threadIdx.x;
                const int64_t id0 = s.head + (int64_t)(s.q0 + q) * X::N;
                constexpr int stride = kThreads * X::N;
                const int held = q >= s.len ? 0 : min(kU, (s.len - q + kThreads - 1) / kThreads);
                bool grown = chunk == 0;
                if (vm > bound && chunk > 0) {
#pragma unroll
                    for (int u = 0; u < kU; ++u)
#pragma unroll
                        for (int j = 0; j < X::N; ++j) {
                            const float x = X::at(v[u], j);
                            if (x > bound)
                                grown |= list_add(top_key(x, id0 + u * stride + j), top) >= kListCut;
                        }
                }
                if (__syncthreads_or(grown)) {
                    if (chunk == 0) {
                        top_chunk<TIn>(v, held, id0, stride, c.n_top, top);
                    } else if (top.count <= kListCap) {
                        cut_list(c.n_top, top);
                    } else {
                        // more than the list holds: without this chunk's, then the chunk as a first one
                        cut_list(c.n_top, top, s.head + (int64_t)(s.q0 + chunk * kChunk) * X::N);
                        top_chunk<TIn>(v, held, id0, stride, c.n_top, top);
                    }
                    bound = top.bound ? key_logit(top.bound) : -INFINITY;
                }
            }
            if (chunk == cy) {
                const int j = (s.y - s.head) & (X::N - 1);
#pragma unroll
                for (int u = 0; u < kU; ++u) {
                    if (u != uy)
                        continue;
                    uint32_t w[4] = {v[u].x, v[u].y, v[u].z, v[u].w};
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        w[i] = i == X::word_of(j) ? X::without(w[i], j) : w[i];
                    v[u] = make_uint4(w[0], w[1], w[2], w[3]);
                }
            }
            const float tm = chunk == cy ? X::max_of(v) : vm;
            if (tm > m) {
                const float d = (m - tm) * kLog2e;
                const float2 f = splat(ex2(d));
                A = fmul2(ffma2(splat(d), S, A), f);
                S = fmul2(S, f);
                m = tm;
            }
#pragma unroll
            for (int u = 0; u < kU; ++u)
                X::fold(v[u], splat(-m), S, A);
        }
        if (chunks == 0 && more)
            load_chunk<TIn>(next, 0, ahead);
        Part p{m, S.x + S.y, A.x + A.y};
        // the row's ends, before its first and after its last whole vector
        const int tail = s.ok ? (int)c.vocab - s.head - s.nvec * X::N : 0;
        if (TOP)
            __syncthreads();
        if (rank == 0 && (int)threadIdx.x < s.head + tail) {
            const int v = (int)threadIdx.x < s.head ? threadIdx.x : s.nvec * X::N + threadIdx.x;
            const float x = to_float(reinterpret_cast<const TIn *>(s.row)[v]);
            if (TOP) {
                const uint64_t key = top_key(x, v);
                if (key > top.bound)
                    list_add(key, top);
            }
            if (v != s.y) {
                const float zc = max_nan(x, kClamp);
                if (zc > p.m)
                    p = part_about(p, zc);
                const float t = (zc - p.m) * kLog2e, e = ex2(t);
                p.s += e;
                p.a = fmaf(e, t, p.a);
            }
        }
        p = part_warp(p);
        if (lane == 0)
            parts[warp] = p;
        __syncthreads();
        if (warp == 0) {
            p = part_warp(lane < kWarps ? parts[lane] : part_empty());
            if (lane == 0)
                whole = p;
        }
        if (TOP && (top.count > c.n_top || chunks == 0))
            cut_list(c.n_top, top);
        if (ctas > 1)
            cluster.sync();
        else
            __syncthreads();
        if (rank == 0) {
            if (warp == 0) {
                p = whole;
                if (ctas > 1)
                    p = part_warp(lane < ctas ? *cluster.map_shared_rank(&whole, lane) : part_empty());
                // y's own term at the end
                const float M = fmaxf(p.m, s.zy), zc = fmaxf(s.zy, kClamp);
                p = part_about(p, M);
                const float ty = (zc - M) * kLog2e, ey = s.y >= 0 ? ex2(ty) : 0.f;
                const float total = p.s + ey;
                const float logs = ey == 1.f ? log1pf(p.s) : logf(total);
                const float H = logs - kLn2 * (fmaf(ey, ty, p.a) / total);
                const bool fine = s.ok && M > kMaskedBelow && M < -kMaskedBelow && isfinite(logs) && isfinite(H) &&
                                  s.zy == s.zy;
                if (lane == 0) {
                    norm[0] = M;
                    norm[1] = logs;
                    norm[2] = fine ? 1.f : 0.f;
                    const int64_t i = s.token;
                    if (fine) {
                        if (c.logprob)
                            c.logprob[i] = (s.zy - M) - logs;
                        if (c.entropy)
                            c.entropy[i] = H;
                        if (c.stats) {
                            c.stats[2 * i] = M;
                            c.stats[2 * i + 1] = logs;
                        }
                    } else {
                        if (s.ok)
                            set_status(c.status, TURNOPD_ERR_NONFINITE);
                        write_nothing(c, i, -INFINITY);
                    }
                }
            }
            if (TOP) {
                __syncthreads();
                // the CTAs' n best, each list in order: merged by the places of their keys
                static_assert(kWarps * 32 == kThreads && kTopMax == 32, "one list to a run");
                top.runs[threadIdx.x] = warp < ctas ? cluster.map_shared_rank(top.sorted, warp)[lane] : 0;
                __syncthreads();
                const uint64_t key = top.runs[threadIdx.x];
                if (key != 0 && norm[2] != 0.f) {
                    const int place = ctas > 1 ? place_among(key, warp, lane, top.runs) : lane;
                    if (place < c.n_top) {
                        c.top_ids[(int64_t)s.token * c.n_top + place] = (int32_t)key_id(key);
                        c.top_logprob[(int64_t)s.token * c.n_top + place] = (key_logit(key) - norm[0]) - norm[1];
                    }
                }
            }
        }
        if (ctas > 1)
            cluster.sync();
        else
            __syncthreads();
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

// Few rows: each is shared by a cluster of CTAs, so that the device's SMs all have some of it.
template <typename TIn>
cudaError_t launch_fwd(const LogprobCall &c, const int4 *rows, const int32_t *nvalid, cudaStream_t stream)
{
    const int sms = device_sm_count();
    const int64_t vecs = c.vocab / Logits<TIn>::N;
    int ctas = 1;
    while (ctas < 8 && c.T * ctas * 2 <= 2 * sms && vecs >= ctas * 2 * kThreads)
        ctas *= 2;
    const int64_t want = c.T * ctas, most = (int64_t)sms * kPerSm / ctas * ctas;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = ctas;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = ctas > 1 ? 1 : 0;
    cfg.gridDim = dim3((unsigned)std::min(want, most));
    cfg.blockDim = dim3(kThreads);
    cfg.stream = stream;
    return c.n_top > 0 ? cudaLaunchKernelEx(&cfg, k_logprobs<TIn, true>, c, rows, nvalid)
                       : cudaLaunchKernelEx(&cfg, k_logprobs<TIn, false>, c, rows, nvalid);
}

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
    return c.in_dtype == TURNOPD_BF16 ? launch_fwd<__nv_bfloat16>(c, l.rows, l.nvalid, stream)
                                      : launch_fwd<float>(c, l.rows, l.nvalid, stream);
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
