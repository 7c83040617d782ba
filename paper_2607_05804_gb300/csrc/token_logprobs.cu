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

// Logits at or below this are masked values: they have probability 0, and a row with nothing else has no distribution.
// It is where the running maximum starts.  Lower logits (-inf, the type's lowest value) are raised to kClamp for the
// sums, so that z - m and e^{z-m} (z - m) stay finite, for maxima up to -kMaskedBelow.
constexpr float kMaskedBelow = -0x1p+126f;
constexpr float kClamp = -0x1.8p+126f;
constexpr uint32_t kClampBf16x2 = 0xfec0fec0u;

enum RowState : int32_t { kRowBad = 0, kRowFine = 1, kRowMasked = 2 };

struct Row {
    int32_t token, r, y, state;
};

// Item k of the row list; without one token k itself, its mask and indexes checked here.
template <typename Call> __device__ __forceinline__ Row get_row(const Call &c, const int4 *rows, int64_t k)
{
    if (rows) {
        const int4 v = rows[k];
        return Row{v.x, v.y, v.z, kRowFine};
    }
    if (c.mask && !c.mask[k])
        return Row{(int32_t)k, (int32_t)k, -1, kRowMasked};
    Row o{(int32_t)k, c.row_of_token ? c.row_of_token[k] : (int32_t)k, c.token_ids ? c.token_ids[k] : -1, kRowFine};
    if (!(o.r >= 0 && o.r < c.num_rows && (!c.token_ids || (o.y >= 0 && o.y < c.vocab)))) {
        o.state = kRowBad;
        if (threadIdx.x == 0)
            set_status(c.status, TURNOPD_ERR_TOKEN_RANGE);
    }
    return o;
}

// Part of a row: its largest logit m, S = sum e^{z-m} and A = sum e^{z-m} (z - m) log2 e.
struct Part {
    float m, s, a;
};

__device__ __forceinline__ Part part_empty() { return Part{kMaskedBelow, 0.f, 0.f}; }

// A change of reference by d (in powers of two).  2^-1000 is 0: bounded there, d times a sum stays finite, and a sum about a
// reference far below the new one (-1e37, as forbidden tokens are filled with) becomes 0 and not -inf times 0.
__device__ __forceinline__ float shift(float from, float to) { return fmaxf((from - to) * kLog2e, -1000.f); }

// The part's sums about another reference m.
__device__ __forceinline__ Part part_about(Part p, float m)
{
    const float d = shift(p.m, m), f = ex2(d);
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
    __device__ static float max_of_one(const uint4 &v)
    {
        const uint32_t m = hmax4(v);
        return fmaxf(bf16lo(m), bf16hi(m));
    }
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
    // Which of vector u's logits reach `low` (bf16, or NaN: none): bit 4 u + word, upper halves 16 bits up.
    __device__ static uint32_t reach(const uint4 &v, float low, int u)
    {
        const __nv_bfloat162 l = __float2bfloat162_rn(low);
        uint32_t hits = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t w = word(v, j);
            hits |= __hge2_mask(*reinterpret_cast<const __nv_bfloat162 *>(&w), l) & (0x00010001u << (4 * u + j));
        }
        return hits;
    }
    __device__ static int vector_of(int p) { return (p & 15) >> 2; }
    __device__ static int place_of(int p) { return (p & 3) * 2 + (p >> 4); }
    __device__ static float at_run_time(const uint4 &v, int j)
    {
        const uint32_t w = j < 4 ? (j < 2 ? v.x : v.y) : (j < 6 ? v.z : v.w);
        return j & 1 ? bf16hi(w) : bf16lo(w);
    }
    __device__ static uint32_t without(uint32_t w, int j) { return j & 1 ? (w & 0xffffu) | 0xff800000u : (w & 0xffff0000u) | 0xff80u; }
    __device__ static int word_of(int j) { return j >> 1; }
};
template <> struct Logits<float> {
    static constexpr int N = 4;
    static constexpr uint32_t kHole = 0xff800000u;
    __device__ static float max_of_one(const uint4 &v)
    {
        return fmaxf(fmaxf(at(v, 0), at(v, 1)), fmaxf(at(v, 2), at(v, 3)));
    }
    template <int U> __device__ static float max_of(const uint4 (&v)[U])
    {
        float m = max_of_one(v[0]);
#pragma unroll
        for (int u = 1; u < U; ++u)
            m = fmaxf(m, max_of_one(v[u]));
        return m;
    }
    __device__ static void fold(const uint4 &v, float2 minus_m, float2 &S, float2 &A)
    {
#pragma unroll
        for (int j = 0; j < 4; j += 2)
            fold2(make_float2(max_nan(at(v, j), kClamp), max_nan(at(v, j + 1), kClamp)), minus_m, S, A);
    }
    __device__ static float at(const uint4 &v, int j) { return __uint_as_float(word(v, j)); }
    __device__ static uint32_t reach(const uint4 &v, float low, int u)
    {
        uint32_t hits = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            hits |= at(v, j) >= low ? 1u << (4 * u + j) : 0u;
        return hits;
    }
    __device__ static int vector_of(int p) { return p >> 2; }
    __device__ static int place_of(int p) { return p & 3; }
    __device__ static float at_run_time(const uint4 &v, int j)
    {
        return __uint_as_float(j < 2 ? (j < 1 ? v.x : v.y) : (j < 3 ? v.z : v.w));
    }
    __device__ static uint32_t without(uint32_t, int) { return kHole; }
    __device__ static int word_of(int j) { return j; }
};

// ---------------------------------------------------------------- alternatives
//
// The n best of a row in one pass.  Each chunk of the row is in the threads' registers.  The first chunk sets a bound:
// the threads of one lane index are a group, and the n-th best of the 32 groups' best logits is reached by n logits at
// least and, in a row in no particular order, by few more.  Those are added to a list in shared memory.  Later logits have
// higher ids, so only those strictly above the bound can matter; they are added without a barrier, and after 2, 4, 8, ...
// chunks or 4, 16, ... the list is cut back to its n best and the bound raised to the n-th: n or 3 n logits, about, are
// added from one cut to the next.  A row that adds more than the list holds
// (one that ascends, or whose first chunk is forbidden) is read again with each chunk taken like a first one, and if
// even that adds too many, n times.  Keys are unique, so the outcome does not depend on the order of the list.

constexpr int kU = 4;                             // vectors per thread and chunk
constexpr int kListCap = 1024;
constexpr int kTopMax = TURNOPD_TOP_ALTERNATIVES_MAX;
constexpr int kMaxCtas = 8;                       // of a cluster

template <int NT> struct alignas(16) TopShared {
    uint64_t list[kListCap + 2];
    uint64_t lanes[NT];                     // the threads' best keys
    uint64_t groups[(NT / 32)][32];                  // each warp's copy of the groups' best
    uint64_t merge[kMaxCtas * kTopMax];           // CTA 0: every CTA's n best
    int count;
    bool lost;                                    // the list was full
};

// The lowest value above b.
__device__ __forceinline__ float next_above(float b, __nv_bfloat16)
{
    const uint32_t u = __float_as_uint(b) & 0xffff0000u;
    return __uint_as_float((u << 1) == 0 ? 0x00010000u : (u & 0x80000000u) ? u - 0x10000u : u + 0x10000u);
}
__device__ __forceinline__ float next_above(float b, float)
{
    const uint32_t u = __float_as_uint(b);
    return __uint_as_float((u << 1) == 0 ? 1u : (u & 0x80000000u) ? u - 1u : u + 1u);
}

// Cuts the list to its n best, in order (the 32 best, rather, with zeros after the last; the list's count is n).
template <int NT> __device__ __forceinline__ void cut_list(int n, TopShared<NT> &t)
{
    __syncthreads();
    const int m = min(t.count, kListCap), tid = threadIdx.x;
    // blocks of NT entries, each but the first beginning with the 32 best of those before
    for (int start = 0;; start += NT - kTopMax) {
        uint64_t *block = t.list + start;
        const int len = min(m - start, NT);
        // a key's place is the number of keys above it, counted by `lanes` neighbouring threads
        const int bits = len > 1 ? 32 - __clz(len - 1) : 0, lanes = min(NT >> bits, 32);
        const int at = tid / lanes, lane = tid & (lanes - 1);
        const uint64_t key = at < len ? block[at] : 0;
        int place = 0;
#pragma unroll 4
        for (int j = 2 * lane; j < len; j += 2 * lanes) {
            const ulonglong2 o = *reinterpret_cast<const ulonglong2 *>(block + j);
            place += (o.x > key) + (o.y > key && j + 1 < len);
        }
        for (int o = lanes >> 1; o > 0; o >>= 1)
            place += __shfl_xor_sync(~0u, place, o);
        __syncthreads();
        const bool done = start + NT >= m;
        uint64_t *to = done ? t.list : block + NT - kTopMax;
        if (lane == 0 && key != 0 && place < kTopMax)
            to[place] = key;
        if (done && tid >= len && tid < kTopMax)
            to[tid] = 0;
        if (done)
            break;
        __syncthreads();
    }
    if (tid == 0) {
        if (t.count > kListCap)
            t.lost = true;
        t.count = n;
    }
    __syncthreads();
}

template <int NT> __device__ __forceinline__ void list_add(uint64_t key, TopShared<NT> &t)
{
    const int at = atomicAdd(&t.count, 1);
    if (at < kListCap)
        t.list[at] = key;
}

__device__ __forceinline__ uint4 pick(const uint4 (&v)[kU], int u)
{
    uint4 w = v[0];
#pragma unroll
    for (int k = 1; k < kU; ++k)
        if (u == k)
            w = v[k];
    return w;
}

// Adds the logits of a chunk that reach `above` and, where equal to it, have ids up to tie_id, and whose keys reach
// `least`.  Vector u of the thread holds ids id0 + u stride + 0..N-1 (none where u >= held).
template <typename TIn, int NT>
__device__ __forceinline__ void list_add_chunk(const uint4 (&v)[kU], int held, uint32_t id0, float above, uint32_t tie_id,
                                               uint64_t least, TopShared<NT> &t)
{
    using X = Logits<TIn>;
    constexpr uint32_t stride = NT * X::N;
    // bit p: element of word p % 16, upper half from bit 16 on (bf16); element p (fp32)
    uint32_t hits = 0;
#pragma unroll
    for (int u = 0; u < kU; ++u) {
        const float low = u >= held ? NAN : id0 + u * stride <= tie_id ? above : next_above(above, TIn());
        hits |= X::reach(v[u], low, u);
    }
    while (hits) {
        const int p = __ffs(hits) - 1;
        hits &= hits - 1;
        const int u = X::vector_of(p), j = X::place_of(p);
        const uint64_t key = top_key(X::at_run_time(pick(v, u), j), id0 + u * stride + j);
        if (key >= least)
            list_add(key, t);
    }
}

// A chunk that sets its own bound; vm is the largest of the thread's logits, `bound` the n-th best so far.
template <typename TIn, int NT>
__device__ __forceinline__ void top_first_chunk(const uint4 (&v)[kU], float vm, int held, uint32_t id0, int n, TopShared<NT> &t,
                                                float &bound)
{
    using X = Logits<TIn>;
    constexpr uint32_t stride = NT * X::N;
    // the thread's best: its logit, and an id not below its own (the last of its vector)
    int u0 = kU - 1;
#pragma unroll
    for (int u = kU - 2; u >= 0; --u)
        u0 = X::max_of_one(v[u]) == vm ? u : u0;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    t.lanes[threadIdx.x] = held > 0 && vm == vm ? top_key(vm, id0 + u0 * stride + X::N - 1) : 0;
    __syncthreads();
    uint64_t best = 0;
#pragma unroll
    for (int w = 0; w < (NT / 32); ++w)
        best = max(best, t.lanes[32 * w + lane]);
    t.groups[warp][lane] = best;
    __syncwarp();
    int place = 0;
#pragma unroll
    for (int j = 0; j < 32; j += 2) {
        const ulonglong2 o = *reinterpret_cast<const ulonglong2 *>(&t.groups[warp][j]);
        place += (o.x > best) + (o.y > best);
    }
    const unsigned who = __ballot_sync(~0u, best != 0 && place == n - 1);
    uint64_t least = 0;  // 0: fewer than n groups, all of them are added
    if (who)
        least = __shfl_sync(~0u, (unsigned long long)best, __ffs(who) - 1);
    const float own = least ? key_logit(least) : -INFINITY;
    float above = next_above(bound, TIn());
    uint32_t tie_id = ~0u;
    if (bound == -INFINITY || own >= above) {
        above = own;
        tie_id = least ? key_id(least) : ~0u;
    } else {
        least = 0;
    }
    if (vm >= above)
        list_add_chunk<TIn>(v, held, id0, above, tie_id, least, t);
    if (least != 0)
        bound = own;  // n logits of this chunk reach it, with lower ids than any later one
}

// ---------------------------------------------------------------- forward kernel

// CTAs of NT threads per SM: what the registers allow without spills.
constexpr int per_sm(bool top, int nt) { return nt == 128 ? 7 : top ? 3 : 4; }

// A row's share of one CTA: `len` of the row's whole 16-byte vectors, from the row's q0-th on; the first starts after
// `head` logits.  CTA 0 of the cluster also takes the logits before and after the row's `nvec` vectors one by one.
struct Share {
    const char *row;
    int32_t head, nvec, q0, len, chunks, token, y, state;
};

template <typename TIn, int NT> __device__ __forceinline__ Share get_share(const LogprobCall &c, Row r, int rank, int ctas)
{
    constexpr int N = Logits<TIn>::N;
    Share s;
    s.token = r.token;
    s.y = r.y;
    s.state = r.state;
    const TIn *z = static_cast<const TIn *>(c.logits) + (r.state == kRowFine ? (int64_t)r.r * c.ld : 0);
    s.row = reinterpret_cast<const char *>(z);
    const int V = r.state == kRowFine ? (int)c.vocab : 0;
    s.head = min((int)((16 - (reinterpret_cast<uintptr_t>(z) & 15)) & 15) / (int)sizeof(TIn), V);
    s.nvec = (V - s.head) / N;
    const int per = (s.nvec + ctas - 1) / ctas;
    s.q0 = min(s.nvec, rank * per);
    s.len = min(s.nvec, s.q0 + per) - s.q0;
    s.chunks = (s.len + (kU * NT) - 1) / (kU * NT);
    return s;
}

template <typename TIn, int NT>
__device__ __forceinline__ void load_chunk(const Share &s, int chunk, uint4 (&v)[kU])
{
    const int q = chunk * (kU * NT) + threadIdx.x;
    const uint4 *p = reinterpret_cast<const uint4 *>(s.row + s.head * sizeof(TIn)) + s.q0 + q;
    const int left = s.len - q;
#pragma unroll
    for (int u = 0; u < kU; ++u) {
        constexpr uint32_t h = Logits<TIn>::kHole;
        v[u] = u * NT < left ? ldg_stream(p + u * NT) : make_uint4(h, h, h, h);
    }
}

// The alternatives of a row whose list was full: every chunk like a first one, and if that fails too, the best logit
// below the last one, n times.
template <typename TIn, int NT>
__device__ __noinline__ void top_again(const Share &s, bool has_end, float end_z, int end_id, int n, TopShared<NT> &t)
{
    constexpr int N = Logits<TIn>::N;
    const uint64_t end_key = has_end ? top_key(end_z, end_id) : 0;
    __syncthreads();
    if (threadIdx.x == 0) {
        t.count = 0;
        t.lost = false;
    }
    __syncthreads();
    float bound = -INFINITY;
    for (int chunk = 0; chunk < s.chunks; ++chunk) {
        uint4 v[kU];
        load_chunk<TIn, NT>(s, chunk, v);
        const int q = chunk * (kU * NT) + threadIdx.x;
        const int held = q >= s.len ? 0 : min(kU, (s.len - q + NT - 1) / NT);
        top_first_chunk<TIn>(v, Logits<TIn>::max_of(v), held, s.head + (uint32_t)(s.q0 + q) * N, n, t, bound);
        cut_list(n, t);
        bound = t.list[n - 1] ? key_logit(t.list[n - 1]) : -INFINITY;
    }
    if (end_key != 0)
        list_add(end_key, t);
    cut_list(n, t);
    if (!t.lost)
        return;
    const TIn *z = reinterpret_cast<const TIn *>(s.row) + s.head + (int64_t)s.q0 * N;
    uint64_t below = ~0ull;
    for (int k = 0; k < n; ++k) {
        uint64_t best = end_key < below ? end_key : 0;
        // (unsigned: the step after the last may pass 2^31 - 1)
        for (uint32_t i = threadIdx.x; i < (uint32_t)s.len * N; i += NT) {
            const uint64_t key = top_key(to_float(z[i]), (uint32_t)(s.head + s.q0 * N) + i);
            best = key < below ? max(best, key) : best;
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1)
            best = max(best, (uint64_t)__shfl_xor_sync(~0u, (unsigned long long)best, o));
        if ((threadIdx.x & 31) == 0)
            t.lanes[threadIdx.x >> 5] = best;
        __syncthreads();
        for (int w = 0; w < (NT / 32); ++w)
            best = max(best, t.lanes[w]);
        below = best;
        if (threadIdx.x == 0)
            t.list[k] = best;
        __syncthreads();
    }
    if ((int)threadIdx.x >= n && threadIdx.x < kTopMax)
        t.list[threadIdx.x] = 0;
    __syncthreads();
}

// One pass over each row: chunks of kU 16-byte vectors to a thread, the next one's loads out while one is summed.  A CTA or
// a cluster takes rows in turn; a cluster's CTAs push their parts to CTA 0, which writes the row's outputs.
//
// Bound: HBM with many rows, 9,830 x 151,936 bf16 in 455 us (6,570 GB/s, 0.97 of a copy).  With alternatives the issue
// rate: 2,458 x 50,304 bf16 take 46 us without, 67 with 10, 100 with 32 (14 instructions to a logit, not 8).  With few rows
// latency: one row of 151,936 takes 4.3 us, 7.9 with five alternatives, of which the exchange and cold code are most.
template <typename TIn, bool TOP, int NT, bool CLUSTER>
__global__ void __launch_bounds__(NT, per_sm(TOP, NT)) k_logprobs(LogprobCall c, const int4 *__restrict__ rows,
                                                          const int32_t *__restrict__ nvalid)
{
    using X = Logits<TIn>;
    __shared__ Part parts[(NT / 32)];
    __shared__ Part whole[kMaxCtas];  // CTA 0: the parts of the row
    __shared__ float norm[3];   // m, log S of the row, 1 if it is fine
    __shared__ TopShared<NT> top;
    // Thread 0 reads a row's indexes and all go by what it read.  The share of the row after next is laid out while a row
    // is worked on; the barrier at the row's end publishes it.
    __shared__ Share shares[3];
    namespace cg = cooperative_groups;
    cg::cluster_group cluster = cg::this_cluster();
    const int rank = CLUSTER ? (int)cluster.block_rank() : 0, ctas = CLUSTER ? (int)cluster.num_blocks() : 1;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    // One thread reads the list's length too: it says how many barriers there are.  (A cluster has no list.)
    __shared__ int list_length;
    if (!CLUSTER && rows) {
        if (threadIdx.x == 0)
            list_length = *nvalid;
        __syncthreads();
    }
    // (32 bits hold three steps beyond 2^31 - 1; 64 cost registers: 2,458 x 50,304 with 10 alternatives 67.6 us and 68.4)
    const uint32_t n = !CLUSTER && rows ? list_length : (int)c.T;
    const uint32_t first = blockIdx.x / ctas, step = gridDim.x / ctas;
    uint4 ahead[kU];
    int slot = 0;
    // Chunks before which the list is cut: powers of four where few rows are shared out and a cut's barriers count (64 fp32
    // rows with 20 alternatives: 18.1 us, with powers of two 18.3), of two where many rows keep the SMs busy (2,458 rows x
    // 50,304 with 32: 100 us and 107).  With many alternatives after the first too: its bound is a loose one.
    constexpr int kCuts = NT == 256 ? 0x55555555 : -1;
    const int first_cut = c.n_top > 16 ? 1 : NT == 256 ? 4 : 2;
    if (CLUSTER)
        asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
    Row coming{};  // thread 0: the row whose share is laid out next
    if (first < n) {
        if (threadIdx.x == 0) {
            shares[0] = get_share<TIn, NT>(c, get_row(c, rows, first), rank, ctas);
            if (first + step < n)
                shares[1] = get_share<TIn, NT>(c, get_row(c, rows, first + step), rank, ctas);
            if (first + 2 * step < n)
                coming = get_row(c, rows, first + 2 * step);
        }
        __syncthreads();
        load_chunk<TIn, NT>(shares[0], 0, ahead);
    }
    for (uint32_t k = first; k < n; k += step, slot = slot == 2 ? 0 : slot + 1) {
        const bool more = k + step < n;
        const Share &s = shares[slot], &next = shares[slot == 2 ? 0 : slot + 1];
        if (threadIdx.x == 0 && k + 2 * step < n) {
            shares[slot == 0 ? 2 : slot - 1] = get_share<TIn, NT>(c, coming, rank, ctas);
            if (k + 3 * step < n)
                coming = get_row(c, rows, k + 3 * step);
        }
        // the row's ends, before its first and after its last whole vector, and y's logit: needed last, asked for first
        const TIn *z = reinterpret_cast<const TIn *>(s.row);
        const int ends = rank == 0 && s.state == kRowFine ? (int)c.vocab - s.nvec * X::N : 0;
        const int end_id = (int)threadIdx.x < s.head ? threadIdx.x : s.nvec * X::N + threadIdx.x;
        const float end_z = (int)threadIdx.x < ends ? to_float(z[end_id]) : 0.f;
        const float zy = warp == 0 && s.state == kRowFine && s.y >= 0 ? to_float(z[s.y]) : -INFINITY;
        // where y lies: in this thread's vector uy of chunk cy, or nowhere
        int cy = -1, uy = 0;
        if (s.y >= s.head) {
            const int f = (s.y - s.head) / X::N - s.q0;
            if (f >= 0 && f < s.len && (f & (NT - 1)) == (int)threadIdx.x) {
                cy = f / (kU * NT);
                uy = f / NT & (kU - 1);
            }
        }
        const int chunks = s.chunks;
        if (TOP && threadIdx.x == 0) {
            top.count = 0;
            top.lost = false;
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
                load_chunk<TIn, NT>(last ? next : s, last ? 0 : chunk + 1, ahead);
            const float vm = X::max_of(v);
            if (TOP) {
                if (chunk >= first_cut && (chunk & (chunk - 1)) == 0 && (chunk & kCuts)) {
                    cut_list(c.n_top, top);
                    bound = key_logit(top.list[c.n_top - 1]);
                }
                if (chunk == 0 || vm > bound) {
                    const int q = chunk * (kU * NT) + threadIdx.x;
                    const int held = q >= s.len ? 0 : min(kU, (s.len - q + NT - 1) / NT);
                    const uint32_t id0 = s.head + (uint32_t)(s.q0 + q) * X::N;
                    if (chunk == 0)
                        top_first_chunk<TIn>(v, vm, held, id0, c.n_top, top, bound);
                    else
                        list_add_chunk<TIn>(v, held, id0, next_above(bound, TIn()), ~0u, 0, top);
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
                const float d = shift(m, tm);
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
            load_chunk<TIn, NT>(next, 0, ahead);
        Part p{m, S.x + S.y, A.x + A.y};
        if (TOP)
            __syncthreads();
        if ((int)threadIdx.x < ends) {
            if (TOP && end_z >= bound)
                list_add(top_key(end_z, end_id), top);
            if (end_id != s.y) {
                const float zc = max_nan(end_z, kClamp);
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
        if (TOP && (top.count > c.n_top || chunks <= first_cut))  // else it is as the last cut left it
            cut_list(c.n_top, top);
        if (TOP && top.lost)
            top_again<TIn>(s, (int)threadIdx.x < ends, end_z, end_id, c.n_top, top);
        // what CTA 0 needs of this one goes into its shared memory, once it runs
        if (CLUSTER && k == first)
            asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
        if (warp == 0) {
            p = part_warp(lane < (NT / 32) ? parts[lane] : part_empty());
            if (lane == 0)
                *(CLUSTER ? cluster.map_shared_rank(&whole[rank], 0) : &whole[0]) = p;
        }
        if (TOP && CLUSTER && (int)threadIdx.x < kTopMax)
            cluster.map_shared_rank(top.merge, 0)[kTopMax * rank + threadIdx.x] = top.list[threadIdx.x];
        if (CLUSTER)
            cluster.sync();
        else
            __syncthreads();
        if (rank == 0) {
            if (warp == 0) {
                p = part_warp(lane < ctas ? whole[lane] : part_empty());
                // y's own term at the end
                const float M = fmaxf(p.m, zy), zc = fmaxf(zy, kClamp);
                p = part_about(p, M);
                const float ty = (zc - M) * kLog2e, ey = s.y >= 0 ? ex2(ty) : 0.f;
                const float total = p.s + ey;
                const float logs = ey == 1.f ? log1pf(p.s) : logf(total);
                const float H = logs - kLn2 * (fmaf(ey, ty, p.a) / total);
                const bool fine = s.state == kRowFine && M > kMaskedBelow && M < -kMaskedBelow && isfinite(logs) && isfinite(H) &&
                                  zy == zy;
                if (lane == 0) {
                    norm[0] = M;
                    norm[1] = logs;
                    norm[2] = fine ? 1.f : 0.f;
                    const int64_t i = s.token;
                    if (fine) {
                        if (c.logprob)
                            c.logprob[i] = (zy - M) - logs;
                        if (c.entropy)
                            c.entropy[i] = H;
                        if (c.stats) {
                            c.stats[2 * i] = M;
                            c.stats[2 * i + 1] = logs;
                        }
                    } else {
                        if (s.state == kRowFine)
                            set_status(c.status, TURNOPD_ERR_NONFINITE);
                        write_nothing(c, i, s.state == kRowMasked ? 0.f : -INFINITY);
                    }
                }
            }
            if (TOP) {
                // the CTAs' lists, each in order: a key's place among all is the number of keys above it, which every
                // other list is searched for (side by side: one search alone waits for shared memory at each step)
                int place = threadIdx.x % kTopMax;
                uint64_t key = 0;
                if constexpr (CLUSTER) {
                    static_assert(!CLUSTER || kMaxCtas * kTopMax == NT, "a thread to every key");
                    const int own = threadIdx.x / kTopMax;
                    key = own < ctas ? top.merge[threadIdx.x] : 0;
                    if (key != 0) {
                        int lo[kMaxCtas] = {};
#pragma unroll
                        for (int h = 16; h > 0; h >>= 1)
#pragma unroll
                            for (int w = 0; w < kMaxCtas; ++w)
                                if (w < ctas)
                                    lo[w] += top.merge[kTopMax * w + lo[w] + h - 1] > key ? h : 0;
#pragma unroll
                        for (int w = 0; w < kMaxCtas; ++w)
                            if (w < ctas && w != own)
                                place += lo[w] + (lo[w] == 31 && top.merge[kTopMax * w + 31] > key);
                    }
                } else if (threadIdx.x < kTopMax) {
                    key = top.list[threadIdx.x];
                }
                __syncthreads();
                if (key != 0 && place < c.n_top && norm[2] != 0.f) {
                    c.top_ids[(int64_t)s.token * c.n_top + place] = (int32_t)key_id(key);
                    c.top_logprob[(int64_t)s.token * c.n_top + place] = (key_logit(key) - norm[0]) - norm[1];
                }
            }
        }
        // CTA 0's memory is written again for the next row
        if (more) {
            if (CLUSTER)
                cluster.sync();
            else
                __syncthreads();
        }
    }
    // tokens that are not in the row list
    if (rows) {
        for (int64_t i = (int64_t)blockIdx.x * NT + threadIdx.x; i < c.T; i += (int64_t)gridDim.x * NT) {
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

// ---------------------------------------------------------------- gradient kernel
//
// One read and one write per logit: the row's statistics are given.  CTAs take chunks of rows in turn, so few long rows
// and many short ones fill the device alike; the row's numbers are read one chunk ahead.  No __restrict__ and no
// read-only loads: the gradient may be written over the logits, each vector by the thread that read it.

struct GradRow {
    Row row;
    float m, logs, gl, gh, H, lp;
};

__device__ __forceinline__ GradRow get_grad_row(const LogprobGradCall &c, const int4 *rows, int64_t k)
{
    GradRow g{};
    g.row = get_row(c, rows, k);
    const int64_t i = g.row.token;
    g.m = c.stats[2 * i];
    g.logs = c.stats[2 * i + 1];
    if (c.d_logprob) {
        g.gl = c.d_logprob[i];
        g.lp = c.logprob[i];
    }
    if (c.d_entropy) {
        g.gh = c.d_entropy[i];
        g.H = c.entropy[i];
    }
    return g;
}

// -p (gl + gh (log p + H)) of two logits.
template <bool ENT> __device__ __forceinline__ float2 grad2(float2 z, const GradRow &g)
{
    float2 lp = fadd2(fadd2(z, splat(-g.m)), splat(-g.logs));
    if (ENT) {  // p = 0: keeps 0 times log p finite
        lp.x = max_nan(lp.x, -1e4f);
        lp.y = max_nan(lp.y, -1e4f);
    }
    const float2 p = ex2x2(fmul2(lp, splat(kLog2e)));
    const float2 f = ENT ? ffma2(splat(-g.gh), fadd2(lp, splat(g.H)), splat(-g.gl)) : splat(-g.gl);
    return fmul2(p, f);
}
// y's own: gl (1 - p) - gh p (log p + H), with 1 - p = -expm1(log p)
__device__ __forceinline__ float grad_y(float z, const GradRow &g)
{
    const float lp = fmaxf((z - g.m) - g.logs, -1e4f), p = expf(lp);
    return fmaf(-g.gl, expm1f(g.lp), -p * (g.gh * (lp + g.H)));
}

constexpr int kGradU = 4;
constexpr int kGradChunk = kGradU * kThreads;  // vectors

__device__ __forceinline__ uint4 ld_once(const uint4 *p)
{
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
                 : "l"(p)
                 : "memory");
    return v;
}

template <int N> __device__ __forceinline__ void st_once(float *p, const float (&g)[N])
{
#pragma unroll
    for (int j = 0; j < N; j += 4)
        __stcs(reinterpret_cast<float4 *>(p + j), make_float4(g[j], g[j + 1], g[j + 2], g[j + 3]));
}
template <int N> __device__ __forceinline__ void st_once(__nv_bfloat16 *p, const float (&g)[N])
{
    if constexpr (N == 8)
        __stcs(reinterpret_cast<uint4 *>(p), make_uint4(pack_bf16x2(g[0], g[1]), pack_bf16x2(g[2], g[3]),
                                                        pack_bf16x2(g[4], g[5]), pack_bf16x2(g[6], g[7])));
    else
        __stcs(reinterpret_cast<uint2 *>(p), make_uint2(pack_bf16x2(g[0], g[1]), pack_bf16x2(g[2], g[3])));
}

// Items of one chunk of one row, taken in turn, so that long and short rows load every SM alike; an item's statistics come
// with its first loads, one item ahead.  Each logit is read before its place is written: grad may be the logits.
// DIRECT: a loss mask without a list, looked at here.
//
// Bound: HBM.  4,915 x 151,936 bf16 with the entropy's term: 445 us (6,710 GB/s, 0.99 of a copy), in place 450.
template <typename TIn, typename TOut, bool ENT, bool DIRECT>
__global__ void __launch_bounds__(kThreads, 4) k_logprobs_bwd(LogprobGradCall c, const int4 *__restrict__ rows,
                                                              const int32_t *__restrict__ nvalid)
{
    using X = Logits<TIn>;
    constexpr int N = X::N;
    constexpr int kOutAlign = sizeof(TOut) * N < 16 ? sizeof(TOut) * N : 16;
    const int64_t n = rows ? *nvalid : c.T;
    const int V = (int)c.vocab;
    const int chunks = (V / N + kGradChunk - 1) / kGradChunk + (V < N);  // of the longest row
    int64_t k = blockIdx.x / chunks;
    int chunk = blockIdx.x % chunks;
    const int64_t dk = gridDim.x / chunks;
    const int dc = gridDim.x % chunks;
    GradRow next{};
    if (k < n)
        next = get_grad_row(c, rows, k);
    while (k < n) {
        const GradRow g = next;
        const int here = chunk;
        k += dk;
        chunk += dc;
        if (chunk >= chunks) {
            chunk -= chunks;
            ++k;
        }
        // without a list a masked token's row may be zeroed here (one that a token -> row map names is zeroed before,
        // since the map may send a masked token to a supervised one's row)
        const bool zeros = DIRECT && g.row.state == kRowMasked && !c.row_of_token && (c.flags & TURNOPD_ZERO_MASKED_GRAD);
        const bool listed = g.row.state == kRowFine || zeros;
        const TIn *z = static_cast<const TIn *>(c.logits) + (listed ? (int64_t)g.row.r * c.ld : 0);
        TOut *out = static_cast<TOut *>(c.grad) + (listed ? (int64_t)g.row.r * c.ld : 0);
        const int len = listed ? V : 0;
        const int head = min((int)((16 - (reinterpret_cast<uintptr_t>(z) & 15)) & 15) / (int)sizeof(TIn), len);
        const int nvec = (len - head) / N;
        const bool aligned = ((reinterpret_cast<uintptr_t>(out + head)) & (kOutAlign - 1)) == 0;
        const int q = here * kGradChunk + threadIdx.x;
        const uint4 *p = reinterpret_cast<const uint4 *>(z + head) + q;
        uint4 v[kGradU];
#pragma unroll
        for (int u = 0; u < kGradU; ++u)
            if (q + u * kThreads < nvec)
                v[u] = ld_once(p + u * kThreads);
        if (k < n)
            next = get_grad_row(c, rows, k);
        const bool fine = !zeros && g.m > -INFINITY;
        const int y = c.d_logprob ? g.row.y : -1;
        // the row's ends
        const int ends = here == 0 ? len - nvec * N : 0;
        if ((int)threadIdx.x < ends) {
            const int e = (int)threadIdx.x < head ? threadIdx.x : nvec * N + threadIdx.x;
            const float x = to_float(z[e]);
            const float o = e == y ? grad_y(x, g) : grad2<ENT>(splat(x), g).x;
            out[e] = from_float<TOut>(fine ? o : 0.f);
        }
#pragma unroll
        for (int u = 0; u < kGradU; ++u) {
            if (q + u * kThreads >= nvec)
                break;
            const int id0 = head + (q + u * kThreads) * N;
            float o[N];
#pragma unroll
            for (int j = 0; j < N; j += 2) {
                const float2 w = grad2<ENT>(make_float2(X::at(v[u], j), X::at(v[u], j + 1)), g);
                o[j] = w.x;
                o[j + 1] = w.y;
            }
            if ((unsigned)(y - id0) < (unsigned)N) {
#pragma unroll
                for (int j = 0; j < N; ++j)
                    if (id0 + j == y)
                        o[j] = grad_y(X::at(v[u], j), g);
            }
            if (!fine) {
#pragma unroll
                for (int j = 0; j < N; ++j)
                    o[j] = 0.f;
            }
            if (aligned) {
                st_once(out + id0, o);
            } else {
#pragma unroll
                for (int j = 0; j < N; ++j)
                    out[id0 + j] = from_float<TOut>(o[j]);
            }
        }
    }
}

template <typename Call> struct Lists {
    int4 *rows = nullptr;
    int32_t *nvalid = nullptr;
    // `direct`: a CTA to every token, which looks at the mask itself (300 bf16 rows x 8,192, 0.6 of them supervised: 3.8 us,
    // with a list 8.5; the gradient of 64 x 1,024 fp32 2.3 and 6.7)
    cudaError_t make(const Call &c, bool direct, cudaStream_t stream)
    {
        if (!c.mask || direct)
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

// Few rows: each is shared by a cluster of CTAs, so that the device's SMs all have some of it, up to 8 CTAs for 3 SMs.
// Powers of two: 64 fp32 rows x 151,936 with 20 alternatives take 18.1 us with 4 CTAs to a row, 19.8 with 2, 24.9 with 8;
// 200 bf16 rows with ten 22.3 with 2, 23.6 with one.  The slices are a chunk long at least: below that the exchange costs
// more than it saves (152 rows x 8,192: one CTA 3.4 us, two 4.2).
int cluster_ctas(const LogprobCall &c)
{
    const int64_t vecs = c.vocab / (c.in_dtype == TURNOPD_BF16 ? 8 : 4);
    int ctas = 1;
    while (ctas < kMaxCtas && 3 * c.T * ctas * 2 <= 8 * device_sm_count() && vecs >= ctas * 2 * kU * 256)
        ctas *= 2;
    return ctas;
}

template <typename TIn, int NT, bool CLUSTER>
cudaError_t launch_fwd(const LogprobCall &c, int ctas, const int4 *rows, const int32_t *nvalid, cudaStream_t stream)
{
    const int64_t want = c.T * ctas;
    const int64_t most = (int64_t)device_sm_count() * per_sm(c.n_top > 0, NT) / ctas * ctas;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = ctas;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = CLUSTER ? 1 : 0;
    cfg.gridDim = dim3((unsigned)std::min(want, most));
    cfg.blockDim = dim3(NT);
    cfg.stream = stream;
    return c.n_top > 0 ? cudaLaunchKernelEx(&cfg, k_logprobs<TIn, true, NT, CLUSTER>, c, rows, nvalid)
                       : cudaLaunchKernelEx(&cfg, k_logprobs<TIn, false, NT, CLUSTER>, c, rows, nvalid);
}

// Rows enough for four CTAs on every SM: CTAs of 128 threads, of which one row's merge hides behind more of the others'
// reads (5,000 rows x 8,192 bf16 with ten alternatives 38 us, with 256 threads 59; 2,458 x 50,304 67 and 81).
template <typename TIn>
cudaError_t launch_fwd(const LogprobCall &c, int ctas, const int4 *rows, const int32_t *nvalid, cudaStream_t stream)
{
    if (ctas > 1)
        return launch_fwd<TIn, 256, true>(c, ctas, rows, nvalid, stream);
    return c.T >= 4 * device_sm_count() ? launch_fwd<TIn, 128, false>(c, ctas, rows, nvalid, stream)
                                        : launch_fwd<TIn, 256, false>(c, ctas, rows, nvalid, stream);
}

constexpr int kGradPerSm = 4;

template <typename TIn, typename TOut>
void launch_grad(const LogprobGradCall &c, const int4 *rows, const int32_t *nvalid, int64_t items, cudaStream_t stream)
{
    const int grid = (int)std::min<int64_t>(items, (int64_t)device_sm_count() * kGradPerSm);
    const bool direct = c.mask && !rows;
    auto kernel = c.d_entropy ? (direct ? k_logprobs_bwd<TIn, TOut, true, true> : k_logprobs_bwd<TIn, TOut, true, false>)
                              : (direct ? k_logprobs_bwd<TIn, TOut, false, true> : k_logprobs_bwd<TIn, TOut, false, false>);
    kernel<<<grid, kThreads, 0, stream>>>(c, rows, nvalid);
}

}  // namespace

size_t logprob_workspace_bytes(int64_t T)
{
    const int64_t nblk = (T + kCompactBlock - 1) / kCompactBlock;
    return align256(sizeof(int4) * (size_t)T) + align256(sizeof(int32_t) * (size_t)(nblk + 1)) + 256;
}

cudaError_t launch_token_logprobs(const LogprobCall &c, cudaStream_t stream)
{
    const int ctas = cluster_ctas(c);
    Lists<LogprobCall> l;
    // (clusters are for fewer tokens than that)
    const bool direct = ctas > 1 || c.T <= (int64_t)device_sm_count() * per_sm(c.n_top > 0, 256);
    const cudaError_t e = l.make(c, direct, stream);
    if (e != cudaSuccess)
        return e;
    return c.in_dtype == TURNOPD_BF16 ? launch_fwd<__nv_bfloat16>(c, ctas, l.rows, l.nvalid, stream)
                                      : launch_fwd<float>(c, ctas, l.rows, l.nvalid, stream);
}

cudaError_t launch_token_logprobs_bwd(const LogprobGradCall &c, cudaStream_t stream)
{
    const bool in16 = c.in_dtype == TURNOPD_BF16, out16 = c.grad_dtype == TURNOPD_BF16;
    const int64_t items = c.T * (c.vocab / (in16 ? 8 : 4) / kGradChunk + 1);
    Lists<LogprobGradCall> l;
    const bool direct = items <= (int64_t)device_sm_count() * kGradPerSm;
    const cudaError_t e = l.make(c, direct, stream);
    if (e != cudaSuccess)
        return e;
    if (c.mask && (c.row_of_token || !direct) && (c.flags & TURNOPD_ZERO_MASKED_GRAD))
        launch_zero_masked_grad(c.mask, c.row_of_token, c.T, c.num_rows, c.ld, c.vocab, c.grad, c.grad_dtype, stream);
    if (in16 && out16)
        launch_grad<__nv_bfloat16, __nv_bfloat16>(c, l.rows, l.nvalid, items, stream);
    else if (in16)
        launch_grad<__nv_bfloat16, float>(c, l.rows, l.nvalid, items, stream);
    else if (out16)
        launch_grad<float, __nv_bfloat16>(c, l.rows, l.nvalid, items, stream);
    else
        launch_grad<float, float>(c, l.rows, l.nvalid, items, stream);
    return cudaGetLastError();
}

}  // namespace turnopd
