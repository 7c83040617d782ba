// Embedding lookup with scaling, and its gradient by sorted tokens.
//
// out[i] = s W[id_i].  dW[v] = s sum_{i: id_i = v} dout[i]: the tokens are sorted by id (stable, so a row's terms come in
// token order), tiles of the sorted list are added up each by itself, runs of one id that pass a tile's end leave partial
// sums, and those are added up in the tiles' order.  No sum's order depends on which thread comes first, and a token that
// the batch repeats thousands of times (a chat template's) is shared by as many tiles.

#include <algorithm>
#include <atomic>

#include "columns.cuh"
#include "common.cuh"
#include "kernels.h"
#include "ptx.cuh"

namespace turnopd {
namespace {

// ---------------------------------------------------------------- lookup

constexpr int kFwdWarps = 4;
constexpr int kPieces = 4;                  // pieces of eight columns that a lane has in flight
constexpr int kFwdChunk = 256 * kPieces;    // columns that a warp copies at once

// A warp copies a row, or 1,024 columns of it, four pieces of a lane in flight.  VEC: rows of both arrays begin on 16-byte
// boundaries.  Bound: HBM.  32,768 x 5,120 bf16 of 14,100 distinct rows 77 us on the device (480 MB, 6,200 GB/s); 64 rows of
// 4,096 2.0; 32,768 x 1,001, off boundaries, 30 (0.44 of the copy rate).
template <typename TW, typename TO, bool VEC> __global__ void __launch_bounds__(32 * kFwdWarps) k_embed(EmbedCall c)
{
    const int lane = threadIdx.x & 31;
    const int64_t d = c.d;
    for (int64_t first = (int64_t)blockIdx.y * kFwdChunk; first < d; first += (int64_t)gridDim.y * kFwdChunk)
        for (int64_t i = (int64_t)blockIdx.x * kFwdWarps + (threadIdx.x >> 5); i < c.T; i += (int64_t)gridDim.x * kFwdWarps) {
            int id = -1;
            if (!c.mask || c.mask[i]) {
                id = c.ids[i];
                if (id < 0 || id >= c.vocab) {
                    if (lane == 0)
                        set_status(c.status, TURNOPD_ERR_TOKEN_RANGE);
                    id = -1;
                }
            }
            const TW *w = static_cast<const TW *>(c.w) + (int64_t)max(id, 0) * c.ldw;
            TO *out = static_cast<TO *>(c.out) + i * c.ldo;
            const auto one = [&](int64_t j) { out[j] = from_float<TO>(id < 0 ? 0.f : to_float(w[j]) * c.scale); };
            if constexpr (VEC) {
                float v[kPieces][8] = {};
#pragma unroll
                for (int k = 0; k < kPieces; ++k) {
                    const int64_t j = first + k * 256 + lane * 8;
                    if (id >= 0 && j + 8 <= d)
                        load8(w + j, v[k]);
                }
#pragma unroll
                for (int k = 0; k < kPieces; ++k) {
                    const int64_t j = first + k * 256 + lane * 8;
                    if (j + 8 <= d) {
#pragma unroll
                        for (int h = 0; h < 8; ++h)
                            v[k][h] *= c.scale;
                        if (id < 0)
                            for (int h = 0; h < 8; ++h)
                                v[k][h] = 0.f;
                        store8(out + j, v[k]);
                    } else {
                        for (int64_t h = j; h < d; ++h)
                            one(h);
                    }
                }
            } else {
                // sixteen loads before the first store: the compiler cannot know that the arrays do not overlap
                const int n = (int)min((int64_t)kFwdChunk, d - first);
                const TW *from = w + first;
                TO *to = out + first;
                for (int j = lane; j < n; j += 16 * 32) {
                    TW v[16];
#pragma unroll
                    for (int k = 0; k < 16; ++k)
                        v[k] = from[min(j + 32 * k, n - 1)];
#pragma unroll
                    for (int k = 0; k < 16; ++k)
                        if (j + 32 * k < n)
                            to[j + 32 * k] = from_float<TO>(id < 0 ? 0.f : to_float(v[k]) * c.scale);
                }
            }
        }
}

// ---------------------------------------------------------------- tokens sorted by id

constexpr int kSortThreads = 1024, kSortWarps = 32;
constexpr int kMaxCtas = 16, kPortableCtas = 8;  // of the sort's cluster, and where one of 16 cannot be placed
constexpr int64_t kZeroBytes = 128 << 20;  // written beside the sort at most
constexpr int kRadixBits = 9;     // at most, of one pass
constexpr int kSortBatch = 8;     // keys of a lane in flight

struct SortBuffers {
    uint2 *list[2];  // (key, token)
};

// Zeros from CTA `cta` of `ctas` into the first `rows` rows of dw.
template <typename TW> __device__ __forceinline__ void zero_rows(const EmbedGradCall &c, int64_t rows, int64_t cta, int64_t ctas)
{
    TW *w = static_cast<TW *>(c.dw);
    constexpr int W = 16 / (int)sizeof(TW);
    const int64_t thread = cta * blockDim.x + threadIdx.x, threads = ctas * blockDim.x;
    if (c.ldw == c.d && reinterpret_cast<uintptr_t>(w) % 16 == 0) {
        const int64_t n = rows * c.d;
        for (int64_t j = thread; j < n / W; j += threads)
            __stcs(reinterpret_cast<uint4 *>(w) + j, make_uint4(0u, 0u, 0u, 0u));
        if (thread < n % W)
            w[n / W * W + thread] = from_float<TW>(0.f);
        return;
    }
    const int lane = threadIdx.x & 31;
    const bool vec = reinterpret_cast<uintptr_t>(w) % 16 == 0 && c.ldw % W == 0;
    for (int64_t v = thread / 32; v < rows; v += threads / 32) {
        TW *row = w + v * c.ldw;
        const int64_t whole = vec ? c.d / W : 0;
        for (int64_t j = lane; j < whole; j += 32)
            __stcs(reinterpret_cast<uint4 *>(row) + j, make_uint4(0u, 0u, 0u, 0u));
        for (int64_t j = whole * W + lane; j < c.d; j += 32)
            row[j] = from_float<TW>(0.f);
    }
}

// The first cluster sorts all tokens, least significant digits first: each CTA takes a part of the list and each of its warps a
// part of that, in order.  A warp counts its digits, the counts are summed up over the warps, the CTAs and the digits, and the
// warp puts its keys where they belong.  Tokens that are masked or whose id is out of range get the key `vocab` and come last.
// The last pass leaves the list in buffer (passes & 1).  Meanwhile the other clusters write zeros into the first rows_zeroed
// rows of the table; those of them that occur are written over by the sums, which costs less than to wait for the list.
// present: a bit for each id that occurs from row rows_zeroed on.
//
// Bound: latency, a chain of some six round trips to the L2 cache or to the cluster's shared memory for each of two digits.
// 256 tokens 10 us under ncu, 8,192 15, 32,768 22 (eight CTAs 29), 131,072 43.
__global__ void __launch_bounds__(kSortThreads) k_sort_tokens(EmbedGradCall c, SortBuffers b, int passes, int bits, uint32_t ctas,
                                                              int64_t rows_zeroed, uint32_t *present)
{
    extern __shared__ uint32_t counts[];  // [kSortWarps][bins]
    __shared__ uint32_t total[1 << kRadixBits], base[1 << kRadixBits], warp_total[kSortWarps];
    pdl_begin();
    if (blockIdx.x >= ctas) {
        if (c.dw_dtype == TURNOPD_BF16)
            zero_rows<__nv_bfloat16>(c, rows_zeroed, blockIdx.x - ctas, gridDim.x - ctas);
        else
            zero_rows<float>(c, rows_zeroed, blockIdx.x - ctas, gridDim.x - ctas);
        return;
    }
    if (rows_zeroed < c.vocab)
        for (int64_t w = (int64_t)cluster_ctarank() * kSortThreads + threadIdx.x; w < (c.vocab + 31) / 32; w += (int64_t)ctas * kSortThreads)
            present[w] = 0;
    const int64_t T = c.T, vocab = c.vocab;
    const int bins = 1 << bits, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t rank = cluster_ctarank();
    const int64_t seg = ((T + (int64_t)ctas * kSortWarps - 1) / ((int64_t)ctas * kSortWarps) + 31) / 32 * 32;
    const int64_t lo = min(T, ((int64_t)rank * kSortWarps + warp) * seg), hi = min(T, lo + seg);
    uint32_t *mine = counts + warp * bins;
    for (int p = 0; p < passes; ++p) {
        const uint2 *from = b.list[p & 1];
        const auto entry = [&](int64_t i) -> uint2 {
            if (i >= hi)
                return make_uint2(0u, 0u);
            if (p)
                return __ldcg(from + i);
            uint32_t key = (uint32_t)vocab;
            if (!c.mask || c.mask[i]) {
                const int id = c.ids[i];
                if (id >= 0 && id < vocab)
                    key = (uint32_t)id;
                else
                    set_status(c.status, TURNOPD_ERR_TOKEN_RANGE);
            }
            return make_uint2(key, (uint32_t)i);
        };
        uint2 list[kSortBatch];  // the last batch read, which is the only one up to 256 keys to a warp
        const bool once = seg <= 32 * kSortBatch;
        const int shift = p * bits;
        for (int k = lane; k < bins; k += 32)
            mine[k] = 0;
        __syncwarp();
        for (int64_t first = lo; first < hi; first += 32 * kSortBatch) {
#pragma unroll
            for (int k = 0; k < kSortBatch; ++k)
                list[k] = entry(first + 32 * k + lane);
#pragma unroll
            for (int k = 0; k < kSortBatch; ++k) {
                const bool there = first + 32 * k + lane < hi;
                if (first + 32 * k >= hi)
                    break;
                const uint32_t digit = there ? (list[k].x >> shift) & (bins - 1) : ~0u;
                const uint32_t peers = __match_any_sync(~0u, digit);
                if (there && lane == __ffs(peers) - 1)
                    mine[digit] += __popc(peers);
                __syncwarp();
            }
        }
        __syncthreads();
        // per digit: the sum over the warps, and each warp's place in it
        const int bin = threadIdx.x;
        if (bin < bins) {
            uint32_t n[kSortWarps], sum = 0;
#pragma unroll
            for (int w = 0; w < kSortWarps; ++w)
                n[w] = counts[w * bins + bin];
#pragma unroll
            for (int w = 0; w < kSortWarps; ++w) {
                counts[w * bins + bin] = sum;
                sum += n[w];
            }
            total[bin] = sum;
        }
        cluster_sync();
        uint32_t before = 0, all = 0;
        if (bin < bins) {
            uint32_t n[kMaxCtas];
#pragma unroll
            for (uint32_t r = 0; r < kMaxCtas; ++r) {
                n[r] = 0;
                if (r < ctas)
                    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(n[r]) : "r"(mapa(smem_u32(total + bin), r)));
            }
#pragma unroll
            for (uint32_t r = 0; r < kMaxCtas; ++r) {
                before += r < rank ? n[r] : 0u;
                all += n[r];
            }
        }
        uint32_t scan = all;
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t n = __shfl_up_sync(~0u, scan, o);
            scan += lane >= o ? n : 0u;
        }
        if (lane == 31)
            warp_total[warp] = scan;
        __syncthreads();
        if (bin < bins) {
            for (int w = 0; w < warp; ++w)
                before += warp_total[w];
            base[bin] = before + scan - all;
        }
        __syncthreads();
        for (int64_t first = lo; first < hi; first += 32 * kSortBatch) {
            if (!once)
#pragma unroll
                for (int k = 0; k < kSortBatch; ++k)
                    list[k] = entry(first + 32 * k + lane);
#pragma unroll
            for (int k = 0; k < kSortBatch; ++k) {
                const bool there = first + 32 * k + lane < hi;
                if (first + 32 * k >= hi)
                    break;
                const uint32_t digit = there ? (list[k].x >> shift) & (bins - 1) : ~0u;
                const uint32_t peers = __match_any_sync(~0u, digit);
                uint32_t to = 0;
                if (there)
                    to = base[digit] + mine[digit] + __popc(peers & ((1u << lane) - 1u));
                __syncwarp();
                if (there) {
                    if (lane == __ffs(peers) - 1)
                        mine[digit] += __popc(peers);
                    __stcg(b.list[~p & 1] + to, list[k]);
                }
                __syncwarp();
            }
        }
        cluster_sync();
    }
    if (rows_zeroed < vocab)
        for (int64_t i = (int64_t)rank * kSortThreads + threadIdx.x; i < T; i += (int64_t)ctas * kSortThreads) {
            const uint32_t key = __ldcg(&b.list[passes & 1][i].x);
            if (key < vocab && (i == 0 || __ldcg(&b.list[passes & 1][i - 1].x) != key))
                atomicOr(present + key / 32, 1u << (key & 31));
        }
}

// ---------------------------------------------------------------- sums

constexpr int kSumThreads = 256;
constexpr int kMinTile = 8, kMaxTile = 512;  // positions
constexpr int kBusyWarps = 8192;             // that keep the device's memory busy
constexpr int kListed = 1024;  // tiles that a block of the last kernel looks at together

// Eight columns of a thread: consecutive ones (VEC), or `step` apart.
template <bool VEC> struct Columns {
    int64_t first, d;
    int step;
    __device__ int64_t at(int k) const { return VEC ? first + k : first + (int64_t)k * step; }
    template <typename T> __device__ void load(const T *p, float *v) const
    {
        if (VEC && first + 8 <= d) {
            load8(p + first, v);
            return;
        }
#pragma unroll
        for (int k = 0; k < 8; ++k)
            v[k] = at(k) < d ? to_float(p[at(k)]) : 0.f;
    }
    template <typename T> __device__ void store(T *p, const float *v) const
    {
        if (VEC && first + 8 <= d) {
            store8(p + first, v);
            return;
        }
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (at(k) < d)
                p[at(k)] = from_float<T>(v[k]);
    }
};

template <typename TW, bool VEC>
__device__ __forceinline__ void put_row(const EmbedGradCall &c, const Columns<VEC> &cols, uint32_t id, float *sum)
{
    TW *w = static_cast<TW *>(c.dw) + (int64_t)id * c.ldw;
#pragma unroll
    for (int k = 0; k < 8; ++k)
        sum[k] *= c.scale;
    if (c.accumulate) {
        float old[8];
        cols.load(w, old);
#pragma unroll
        for (int k = 0; k < 8; ++k)
            sum[k] += old[k];
    }
    cols.store(w, sum);
}

constexpr int kRows = 8;       // in flight
constexpr int kZeroRows = 64;  // of a CTA that writes zeros

// A tile of the sorted list and a slice of the columns.  A tile owns the runs that begin in it, and goes on with its last run
// through the next tile.  A run that ends by then goes to dW; a longer one leaves the sum of its owner's two tiles in partial
// row 2 t + 1, and of each later tile that it reaches in that tile's row 2 t.  The rows come through a ring in shared memory,
// in which each thread copies and reads its own columns (bf16 rows that begin at odd elements: a row ahead, in registers).
// Every so many CTAs one writes zeros instead, into the rows from rows_zeroed on that do not occur, 64 of them: the sums wait
// for their rows while the zeros go out.
//
// Bound: HBM.  151,936 x 4,096 bf16 from 32,768 tokens, the rest of the zeros among them, 228 us (1.33 GB, 5,850 GB/s).
template <typename TG, typename TW, bool VEC>
__global__ void __launch_bounds__(kSumThreads) k_embed_sums(EmbedGradCall c, const uint2 *__restrict__ list, int tile, int slices, float *partial,
                                                            int64_t ldp, int64_t rows_zeroed, const uint32_t *__restrict__ present,
                                                            int zero_ctas)
{
    constexpr bool kRing = VEC || sizeof(TG) == 4;
    extern __shared__ __align__(16) char ring[];
    __shared__ uint32_t key[2 * kMaxTile + 2];  // from the position before the tile to the one after the next tile
    __shared__ int32_t at[2 * kMaxTile];
    pdl_begin();
    const int64_t T = c.T, d = c.d;
    const uint32_t none = (uint32_t)c.vocab;
    const int zeros = (int)((int64_t)blockIdx.x * zero_ctas / gridDim.x);  // CTAs before this one that write them
    if ((int64_t)(blockIdx.x + 1) * zero_ctas / gridDim.x > zeros) {
        const int lane = threadIdx.x & 31;
        const int64_t v0 = rows_zeroed + (int64_t)zeros * kZeroRows;
        for (int64_t v = v0 + (threadIdx.x >> 5); v < min(v0 + kZeroRows, c.vocab); v += blockDim.x >> 5) {
            if (present[v / 32] >> (v & 31) & 1)
                continue;
            TW *row = static_cast<TW *>(c.dw) + v * c.ldw;
            constexpr int W = 16 / (int)sizeof(TW);
            const int64_t pieces = VEC ? d / W : 0;
            for (int64_t j = lane; j < pieces; j += 32)
                __stcs(reinterpret_cast<uint4 *>(row) + j, make_uint4(0u, 0u, 0u, 0u));
            for (int64_t j = pieces * W + lane; j < d; j += 32)
                row[j] = from_float<TW>(0.f);
        }
        return;
    }
    const int t = (blockIdx.x - zeros) / slices, slice = (blockIdx.x - zeros) % slices;
    const int64_t base = (int64_t)slice * 8 * blockDim.x, lo = (int64_t)t * tile;
    const Columns<VEC> cols{base + (VEC ? threadIdx.x * 8 : threadIdx.x), d, (int)blockDim.x};
    const int size = (int)min(T - lo, (int64_t)tile), most = (int)min(T - lo, (int64_t)2 * tile);  // positions of the tile, and of both
    for (int q = threadIdx.x; q < most + 2; q += blockDim.x) {
        const int64_t p = lo - 1 + q;
        const uint2 entry = p >= 0 && p < T ? list[p] : make_uint2(none, 0u);
        key[q] = entry.x;
        if (q > 0 && q <= most)
            at[q - 1] = (int)entry.y;
    }
    const bool long_ago = t > 1 && list[lo - tile - 1].x == list[lo].x;
    __syncthreads();
    uint32_t run = key[1];
    if (run == none)
        return;
    const uint32_t last = key[size];
    bool leading = lo > 0 && key[0] == run;        // begun before this tile:
    bool skip = leading && !long_ago;              // in the last one, whose it is then
    const bool all_leading = leading && last == run;
    const bool skip_first = skip;
    const uint32_t first = run;
    const auto wanted = [&](int q) {
        const uint32_t k = key[q + 1];
        return q < most && k != none && (q < size || (k == last && !all_leading)) && !(skip_first && k == first);
    };
    float sum[8] = {};
    TG ahead[kRing ? 1 : 8];  // as it is stored: converting it would wait for it
    int32_t places[kRing ? 1 : 8];
    if (!kRing)
#pragma unroll
        for (int h = 0; h < (kRing ? 1 : 8); ++h)
            places[h] = (int32_t)(min(cols.at(h), d - 1));
    const auto issue = [&](int q) {
        const TG *row = static_cast<const TG *>(c.dout) + (wanted(q) ? (int64_t)at[q] * c.ldg : 0);
        if constexpr (kRing) {
            if (wanted(q)) {
                if (VEC && cols.first + 8 <= d) {
                    char *to = ring + ((q % kRows) * blockDim.x + threadIdx.x) * 8 * sizeof(TG);
#pragma unroll
                    for (int h = 0; h < (int)sizeof(TG) / 2; ++h)
                        cp16(to + 16 * h, reinterpret_cast<const char *>(row + cols.first) + 16 * h);
                } else if (!VEC) {
#pragma unroll
                    for (int h = 0; h < 8; ++h)
                        if (cols.at(h) < d)
                            asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(
                                             (uint32_t)__cvta_generic_to_shared(ring + (((q % kRows) * 8 + h) * blockDim.x + threadIdx.x) * 4)),
                                         "l"(row + cols.at(h))
                                         : "memory");
                }
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
        } else if (wanted(q)) {
#pragma unroll
            for (int h = 0; h < (kRing ? 1 : 8); ++h)
                ahead[h] = row[places[h]];
        }
    };
    const auto add = [&](int q) {
        float v[8];
        if constexpr (kRing) {
            asm volatile("cp.async.wait_group %0;" ::"n"(kRows - 1) : "memory");
            if (VEC && cols.first + 8 <= d) {
                load8(reinterpret_cast<const TG *>(ring) + ((q % kRows) * blockDim.x + threadIdx.x) * 8, v);
            } else if (VEC) {
                cols.load(static_cast<const TG *>(c.dout) + (int64_t)at[q] * c.ldg, v);  // the last columns of a row
            } else {
#pragma unroll
                for (int h = 0; h < 8; ++h)
                    v[h] = cols.at(h) < d ? reinterpret_cast<const float *>(ring)[((q % kRows) * 8 + h) * blockDim.x + threadIdx.x] : 0.f;
            }
        } else {
#pragma unroll
            for (int h = 0; h < 8; ++h)
                v[h] = cols.at(h) < d ? to_float(ahead[kRing ? 0 : h]) : 0.f;
        }
        if (kRing || q + 1 < most)
            issue(kRing ? q + kRows : q + 1);
        if (!skip)
#pragma unroll
            for (int h = 0; h < 8; ++h)
                sum[h] += v[h];
    };
    const auto flush = [&](bool goes_on) {
        if (!skip) {
            if (leading || goes_on)
                cols.store(partial + (2 * (int64_t)t + (leading ? 0 : 1)) * ldp, sum);
            else
                put_row<TW, VEC>(c, cols, run, sum);
        }
#pragma unroll
        for (int h = 0; h < 8; ++h)
            sum[h] = 0.f;
        leading = skip = false;
    };
    for (int q = 0; q < (kRing ? kRows : 1); ++q)
        issue(q);
#pragma unroll 1
    for (int q = 0;; ++q) {
        const uint32_t k = key[q + 1];  // past both tiles: the position after them
        const bool over = q >= most || k == none || (q >= size && (k != run || leading || skip));
        if (k != run || over) {
            flush(over && k == run);
            if (over)
                break;
            run = k;
        }
        add(q);
    }
    if (kRing)
        asm volatile("cp.async.wait_all;" ::: "memory");
}

// Runs over more than two tiles: the partial sums of the tile they began in and of those they go on in.  32 threads take 256
// columns, the block's eight warps share the tiles of a run, and their sums are added up in order.  A row of blocks looks at
// 1,024 tiles.  Bound: latency (10 us for 512 tiles of 4,096 columns: the list of runs, then few rows each).
template <typename TW>
__global__ void __launch_bounds__(256) k_embed_join(EmbedGradCall c, const uint2 *__restrict__ list, int tile, int tiles,
                                                    int slices, const float *__restrict__ partial, int64_t ldp)
{
    __shared__ int owner[kListed], first_of[kListed / 32 + 1];
    __shared__ float part[8][256];
    pdl_begin();
    const int64_t d = c.d;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    static_assert(kListed == 32 * 32, "one warp adds up the counts");
    for (int64_t t0 = (int64_t)blockIdx.y * kListed; t0 + 2 < tiles; t0 += (int64_t)gridDim.y * kListed) {
        // tile t owns a run that begins in it and goes on in tile t + 2; every block lists the owners in the same order
        __syncthreads();
#pragma unroll
        for (int w = warp; w < kListed / 32; w += 8) {
            const int t = (int)t0 + w * 32 + lane;
            bool owns = false;
            if (t + 2 < tiles) {
                const uint32_t k = list[(int64_t)(t + 1) * tile - 1].x, later = list[(int64_t)(t + 2) * tile].x;
                const uint32_t earlier = t ? list[(int64_t)t * tile - 1].x : ~0u;
                owns = k < (uint32_t)c.vocab && later == k && earlier != k;
            }
            const uint32_t owners = __ballot_sync(~0u, owns);
            if (lane == 0)
                first_of[w + 1] = (int)owners;
        }
        __syncthreads();
        if (warp == 0) {
            const uint32_t owners = (uint32_t)first_of[lane + 1];
            int scan = __popc(owners);
            for (int o = 1; o < 32; o <<= 1) {
                const int n = __shfl_up_sync(~0u, scan, o);
                scan += lane >= o ? n : 0;
            }
            int place = scan - __popc(owners);
            for (uint32_t left = owners; left; left &= left - 1)
                owner[place++] = (int)t0 + lane * 32 + __ffs(left) - 1;
            __syncwarp();
            first_of[lane + 1] = scan;
        }
        __syncthreads();
        const int n = first_of[kListed / 32] * slices;
        for (int item = blockIdx.x; item < n; item += gridDim.x) {
            const int t = owner[item / slices], slice = item % slices;
            const uint32_t k = list[(int64_t)(t + 1) * tile - 1].x;
            const Columns<true> cols{(int64_t)slice * 256 + lane * 8, ldp, 1};  // of the partial sums, whose rows are padded
            float sum[8] = {};
            for (int s0 = t + 2 + warp; s0 < tiles; s0 += 32) {
                bool in[4];
                float v[4][8];
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    in[q] = s0 + 8 * q < tiles && list[(int64_t)(s0 + 8 * q) * tile].x == k;
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    if (in[q] && cols.first < ldp)
                        cols.load(partial + 2 * (int64_t)(s0 + 8 * q) * ldp, v[q]);
#pragma unroll
                for (int q = 0; q < 4; ++q)
                    if (in[q] && cols.first < ldp)
#pragma unroll
                        for (int h = 0; h < 8; ++h)
                            sum[h] += v[q][h];
                if (!in[3])
                    break;
            }
#pragma unroll
            for (int h = 0; h < 8; ++h)
                part[warp][h * 32 + lane] = sum[h];
            __syncthreads();
            const int64_t j = (int64_t)slice * 256 + threadIdx.x;
            if (j < d) {
                float s = partial[(2 * (int64_t)t + 1) * ldp + j];
#pragma unroll
                for (int w = 0; w < 8; ++w)
                    s += part[w][(threadIdx.x & 7) * 32 + (threadIdx.x >> 3)];
                TW *w = static_cast<TW *>(c.dw) + (int64_t)k * c.ldw + j;
                s *= c.scale;
                *w = from_float<TW>(c.accumulate ? to_float(*w) + s : s);
            }
            __syncthreads();
        }
    }
}

int sum_threads(int64_t d) { return (int)std::min<int64_t>(kSumThreads, (d + 255) / 256 * 32); }
int sum_slices(int64_t d) { return (int)((d + 8 * sum_threads(d) - 1) / (8 * sum_threads(d))); }

int64_t tile_warps(int64_t d) { return (int64_t)sum_slices(d) * (sum_threads(d) / 32); }

// Positions of a tile: as many as leave 8,192 warps; each run that passes two tiles' ends costs partial sums
// (32,768 x 4,096: 64 positions).
int tile_size(int64_t T, int64_t d)
{
    int n = kMinTile;
    while (n < kMaxTile && (T + 2 * n - 1) / (2 * n) * tile_warps(d) >= kBusyWarps)
        n *= 2;
    return n;
}

// Tiles of T tokens, or of any fewer, at most: tiles stay shorter than kMaxTile only while `doubled` tiles of twice their
// length hold all tokens.  (Fewer tokens can be more tiles: of 4,096 columns 8,176 tokens are 1,022, 8,192 are 512.)
int64_t most_tiles(int64_t T, int64_t d)
{
    const int64_t doubled = (kBusyWarps - 1) / tile_warps(d);
    return std::min((T + kMinTile - 1) / kMinTile, std::max(2 * doubled, (T + kMaxTile - 1) / kMaxTile));
}

// Whether the sort's largest cluster, of a size that is not portable, can be placed: a part of a device may have too few SMs.
cudaError_t largest_cluster_fits(bool *fits)
{
    static std::atomic<int> known[64];  // by device: 1 no, 2 yes
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess)
        return e;
    if (dev >= 64)
        return cudaErrorInvalidDevice;
    if (!known[dev]) {
        cudaLaunchConfig_t cfg = {};
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = kMaxCtas;
        attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
        cfg.gridDim = dim3(kMaxCtas);
        cfg.blockDim = dim3(kSortThreads);
        cfg.dynamicSmemBytes = sizeof(uint32_t) * kSortWarps << kRadixBits;
        int clusters = 0;
        e = cudaOccupancyMaxActiveClusters(&clusters, k_sort_tokens, &cfg);
        if (e != cudaSuccess && e != cudaErrorInvalidClusterSize)
            return e;
        if (e != cudaSuccess)
            cudaGetLastError();  // that is the answer
        known[dev] = e == cudaSuccess && clusters > 0 ? 2 : 1;
    }
    *fits = known[dev] == 2;
    return cudaSuccess;
}

bool boundary(const void *p, int64_t ld, int32_t dtype)
{
    return reinterpret_cast<uintptr_t>(p) % 16 == 0 && ld * (dtype == TURNOPD_BF16 ? 2 : 4) % 16 == 0;
}

struct Workspace {
    SortBuffers sort;
    uint32_t *present;
    float *partial;
    int64_t ldp;
    size_t bytes;
    Workspace(void *ws, int64_t T, int64_t d, int64_t vocab) : ldp((d + 7) / 8 * 8)
    {
        char *p = static_cast<char *>(ws);
        const auto take = [&](size_t n) {
            char *at = p + bytes;
            bytes += align256(n);
            return at;
        };
        bytes = 0;
        for (uint2 *&list : sort.list)
            list = reinterpret_cast<uint2 *>(take(sizeof(uint2) * (size_t)T));
        present = reinterpret_cast<uint32_t *>(take(sizeof(uint32_t) * (size_t)((vocab + 31) / 32)));
        partial = reinterpret_cast<float *>(take(sizeof(float) * 2 * (size_t)ldp * (size_t)most_tiles(T, d)));
    }
};

}  // namespace

size_t embed_bwd_workspace_bytes(int64_t T, int64_t d, int64_t vocab) { return Workspace(nullptr, T, d, vocab).bytes; }

cudaError_t launch_embed(const EmbedCall &c, cudaStream_t stream)
{
    const int64_t chunks = (c.d + kFwdChunk - 1) / kFwdChunk, blocks = (c.T + kFwdWarps - 1) / kFwdWarps;
    const dim3 grid((unsigned)std::min<int64_t>(blocks, std::max<int64_t>((int64_t)device_sm_count() * 16 / chunks, 1)),
                    (unsigned)std::min<int64_t>(chunks, 65535));
    const bool vec = boundary(c.w, c.ldw, c.w_dtype) && boundary(c.out, c.ldo, c.out_dtype);
    with_types(c.w_dtype, c.out_dtype, [&](auto w, auto o) {
        using W = decltype(w);
        using O = decltype(o);
        auto kernel = vec ? k_embed<W, O, true> : k_embed<W, O, false>;
        kernel<<<grid, 32 * kFwdWarps, 0, stream>>>(c);
    });
    return cudaGetLastError();
}

cudaError_t launch_embed_bwd(const EmbedGradCall &c, cudaStream_t stream)
{
    const Workspace ws(c.workspace, c.T, c.d, c.vocab);
    int key_bits = 1;
    while ((int64_t)1 << key_bits <= c.vocab)
        ++key_bits;
    const int passes = (key_bits + kRadixBits - 1) / kRadixBits, bits = (key_bits + passes - 1) / passes;
    cudaError_t e = allow_shared(k_sort_tokens, sizeof(uint32_t) * kSortWarps << kRadixBits);
    if (e == cudaSuccess)
        e = cudaFuncSetAttribute(k_sort_tokens, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e != cudaSuccess)
        return e;
    // As many zeros beside the sort as go out in its time (a small table whole), 32 KB to a CTA at least.
    const int64_t row_bytes = c.d * (c.dw_dtype == TURNOPD_BF16 ? 2 : 4);
    unsigned ctas = c.T > 8 * kSortThreads ? kMaxCtas : c.T > kSortThreads ? kPortableCtas : 1;
    if (ctas > kPortableCtas) {
        bool fits = false;
        e = largest_cluster_fits(&fits);
        if (e != cudaSuccess)
            return e;
        if (!fits || c.portable)
            ctas = kPortableCtas;
    }
    int64_t rows_zeroed = c.accumulate ? 0 : c.vocab;
    if (c.T > 0 && rows_zeroed * row_bytes > kZeroBytes)
        rows_zeroed = kZeroBytes / row_bytes / kZeroRows * kZeroRows;
    const int zero_ctas = c.accumulate ? 0 : (int)((c.vocab - rows_zeroed + kZeroRows - 1) / kZeroRows);
    const unsigned fill = (unsigned)std::min<int64_t>((rows_zeroed * row_bytes + 32767) / 32768, (int64_t)device_sm_count() * 2 - kMaxCtas);
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[2];
    cfg.gridDim = (ctas + fill + ctas - 1) / ctas * ctas;
    cfg.blockDim = kSortThreads;
    cfg.dynamicSmemBytes = sizeof(uint32_t) * kSortWarps << bits;
    cfg.stream = stream;
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = ctas;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    e = cudaLaunchKernelEx(&cfg, k_sort_tokens, c, ws.sort, passes, bits, (uint32_t)ctas, c.accumulate ? c.vocab : rows_zeroed, ws.present);
    if (e != cudaSuccess || c.T == 0)
        return e;
    const uint2 *list = ws.sort.list[passes & 1];
    const int tile = tile_size(c.T, c.d), tiles = (int)((c.T + tile - 1) / tile);
    const int threads = sum_threads(c.d), slices = sum_slices(c.d);
    const bool vec = boundary(c.dout, c.ldg, c.dout_dtype) && boundary(c.dw, c.ldw, c.dw_dtype);
    with_types(c.dout_dtype, c.dw_dtype, [&](auto g, auto w) {
        using G = decltype(g);
        using W = decltype(w);
        const size_t smem = vec || sizeof(G) == 4 ? sizeof(G) * 8 * kRows * (size_t)threads : 0;
        auto sums = vec ? k_embed_sums<G, W, true> : k_embed_sums<G, W, false>;
        e = allow_shared(sums, sizeof(G) * 8 * kRows * kSumThreads);
        if (e != cudaSuccess)
            return;
        e = launch_dependent(sums, dim3((unsigned)((int64_t)tiles * slices + zero_ctas)), dim3(threads), smem, stream, c,
                             list, tile, slices, ws.partial, ws.ldp, rows_zeroed, (const uint32_t *)ws.present, zero_ctas);
        if (e == cudaSuccess && tiles > 2) {
            const int n = (int)((c.d + 255) / 256);
            const int64_t lists = std::min<int64_t>((tiles - 2 + kListed - 1) / kListed, 65535);
            const int64_t items = (int64_t)std::min(tiles - 2, kListed) * n, most = std::max<int64_t>(device_sm_count() * 4 / lists, 1);
            const dim3 grid((unsigned)std::min(items, most), (unsigned)lists);
            e = launch_dependent(k_embed_join<W>, grid, dim3(256), 0, stream, c, list, tile, tiles, n, (const float *)ws.partial, ws.ldp);
        }
    });
    return e;
}

}  // namespace turnopd
