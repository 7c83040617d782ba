// Embedding lookup with scaling, and its gradient by sorted tokens.
//
// out[i] = s W[id_i].  dW[v] = s sum_{i: id_i = v} dout[i]: the tokens are sorted by id (stable, so a row's terms come in
// token order), tiles of the sorted list are added up each by itself, runs of one id that pass a tile's end leave partial
// sums, and those are added up in the tiles' order.  No sum's order depends on which thread comes first, and a token that
// the batch repeats thousands of times (a chat template's) is shared by as many tiles.

#include <algorithm>

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

// VEC: rows of both arrays begin on 16-byte boundaries.
template <typename TW, typename TO, bool VEC> __global__ void __launch_bounds__(32 * kFwdWarps) k_embed(EmbedCall c, int64_t chunks)
{
    const int lane = threadIdx.x & 31;
    const int64_t d = c.d, units = c.T * chunks;
    for (int64_t u = (int64_t)blockIdx.x * kFwdWarps + (threadIdx.x >> 5); u < units; u += (int64_t)gridDim.x * kFwdWarps) {
        const int64_t i = u / chunks, first = (u - i * chunks) * kFwdChunk;
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
#pragma unroll 8
            for (int64_t j = first + lane; j < min(first + kFwdChunk, d); j += 32)
                one(j);
        }
    }
}

// ---------------------------------------------------------------- tokens sorted by id

constexpr int kSortThreads = 1024, kSortWarps = 32;
constexpr int kMaxCtas = 8;       // of the sort's cluster
constexpr int kRadixBits = 9;     // at most, of one pass

struct SortBuffers {
    uint32_t *key[2];
    int32_t *at[2];
};

// One cluster sorts all tokens, least significant digits first: each CTA takes a part of the list and each of its warps a part
// of that, in order.  A warp counts its digits, the counts are summed up over the warps, the CTAs and the digits, and the warp
// puts its keys where they belong.  Tokens that are masked or whose id is out of range get the key `vocab` and come last.
// The last pass leaves the list in buffer (passes & 1).  present (or null): a bit for each id that occurs.
__global__ void __launch_bounds__(kSortThreads) k_sort_tokens(const int32_t *__restrict__ ids, const uint8_t *__restrict__ mask,
                                                              int64_t T, int64_t vocab, SortBuffers b, int passes, int bits,
                                                              uint32_t *present, int32_t *status)
{
    extern __shared__ uint32_t counts[];  // [kSortWarps][bins]
    __shared__ uint32_t total[1 << kRadixBits], warp_total[kSortWarps];
    const int bins = 1 << bits, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t rank = cluster_ctarank(), ctas = gridDim.x;
    const int64_t seg = ((T + (int64_t)ctas * kSortWarps - 1) / ((int64_t)ctas * kSortWarps) + 31) / 32 * 32;
    const int64_t lo = min(T, ((int64_t)rank * kSortWarps + warp) * seg), hi = min(T, lo + seg);
    uint32_t *mine = counts + warp * bins;
    if (present)
        for (int64_t w = (int64_t)rank * kSortThreads + threadIdx.x; w < (vocab + 31) / 32; w += (int64_t)ctas * kSortThreads)
            present[w] = 0;
    for (int p = 0; p < passes; ++p) {
        const uint32_t *from = b.key[p & 1];
        const auto key_of = [&](int64_t i) -> uint32_t {
            if (p)
                return __ldcg(from + i);
            if (mask && !mask[i])
                return (uint32_t)vocab;
            const int id = ids[i];
            if (id >= 0 && id < vocab)
                return (uint32_t)id;
            set_status(status, TURNOPD_ERR_TOKEN_RANGE);
            return (uint32_t)vocab;
        };
        const int shift = p * bits;
        for (int k = lane; k < bins; k += 32)
            mine[k] = 0;
        __syncwarp();
        for (int64_t i = lo + lane; i - lane < hi; i += 32) {
            const uint32_t digit = i < hi ? (key_of(i) >> shift) & (bins - 1) : ~0u;
            const uint32_t peers = __match_any_sync(~0u, digit);
            if (i < hi && lane == __ffs(peers) - 1)
                mine[digit] += __popc(peers);
            __syncwarp();
        }
        __syncthreads();
        // per digit: the sum over the warps, and each warp's place in it
        const int bin = threadIdx.x;
        if (bin < bins) {
            uint32_t sum = 0;
            for (int w = 0; w < kSortWarps; ++w) {
                const uint32_t n = counts[w * bins + bin];
                counts[w * bins + bin] = sum;
                sum += n;
            }
            total[bin] = sum;
        }
        cluster_sync();
        uint32_t before = 0, all = 0;
        if (bin < bins)
            for (uint32_t r = 0; r < ctas; ++r) {
                uint32_t n;
                asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(n) : "r"(mapa(smem_u32(total + bin), r)) : "memory");
                before += r < rank ? n : 0u;
                all += n;
            }
        uint32_t scan = all;
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t n = __shfl_up_sync(~0u, scan, o);
            scan += lane >= o ? n : 0u;
        }
        if (lane == 31)
            warp_total[warp] = scan;
        __syncthreads();
        for (int w = 0; w < warp; ++w)
            before += warp_total[w];
        if (bin < bins)
            for (int w = 0; w < kSortWarps; ++w)
                counts[w * bins + bin] += before + scan - all;
        __syncthreads();
        for (int64_t i = lo + lane; i - lane < hi; i += 32) {
            const uint32_t key = i < hi ? key_of(i) : 0u, digit = i < hi ? (key >> shift) & (bins - 1) : ~0u;
            const uint32_t peers = __match_any_sync(~0u, digit);
            uint32_t to = 0;
            if (i < hi)
                to = mine[digit] + __popc(peers & ((1u << lane) - 1u));
            __syncwarp();
            if (i < hi) {
                if (lane == __ffs(peers) - 1)
                    mine[digit] += __popc(peers);
                __stcg(b.key[~p & 1] + to, key);
                __stcg(b.at[~p & 1] + to, p ? __ldcg(b.at[p & 1] + i) : (int32_t)i);
            }
            __syncwarp();
        }
        cluster_sync();
    }
    if (present)
        for (int64_t i = (int64_t)rank * kSortThreads + threadIdx.x; i < T; i += (int64_t)ctas * kSortThreads) {
            const uint32_t key = __ldcg(b.key[passes & 1] + i);
            if (key < vocab && (i == 0 || __ldcg(b.key[passes & 1] + i - 1) != key))
                atomicOr(present + key / 32, 1u << (key & 31));
        }
}

// ---------------------------------------------------------------- sums

constexpr int kSumThreads = 256;
constexpr int kMaxTiles = 1024;

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

// CTAs [0, tiles slices): a tile of the sorted list and a slice of the columns each.  A run that lies in the tile goes to dW;
// one that began before it leaves its sum in partial row 2 t, one that began in it and goes on in 2 t + 1.  The CTAs
// after them write the zeros of the ids that do not occur.
template <typename TG, typename TW, bool VEC>
__global__ void __launch_bounds__(kSumThreads) k_embed_sums(EmbedGradCall c, const uint32_t *__restrict__ key,
                                                            const int32_t *__restrict__ at, int tile, int tiles, int slices,
                                                            float *partial, int64_t ldp, const uint32_t *__restrict__ present)
{
    const int64_t T = c.T, d = c.d;
    if (blockIdx.x >= (unsigned)(tiles * slices)) {
        const int lane = threadIdx.x & 31, nw = blockDim.x >> 5;
        const int64_t warps = (int64_t)(gridDim.x - tiles * slices) * nw;
        for (int64_t w = (int64_t)(blockIdx.x - tiles * slices) * nw + (threadIdx.x >> 5); w < (c.vocab + 31) / 32; w += warps) {
            const int64_t left = c.vocab - w * 32;
            uint32_t off = ~present[w] & (left < 32 ? (1u << left) - 1u : ~0u);
            while (off) {
                const int k = __ffs(off) - 1;
                off &= off - 1;
                TW *row = static_cast<TW *>(c.dw) + (w * 32 + k) * c.ldw;
                const float zero[8] = {};
                for (int64_t j = VEC ? lane * 8 : lane; j < d; j += 256) {
                    const Columns<VEC> cols{j, d, 32};
                    cols.store(row, zero);
                }
            }
        }
        return;
    }
    const int t = blockIdx.x / slices, slice = blockIdx.x % slices;
    const int64_t base = (int64_t)slice * 8 * blockDim.x;
    const Columns<VEC> cols{base + (VEC ? threadIdx.x * 8 : threadIdx.x), d, (int)blockDim.x};
    const int64_t lo = (int64_t)t * tile, hi = min(T, lo + tile);
    float sum[8] = {};
    uint32_t run = key[lo];
    bool begun = lo > 0 && key[lo - 1] == run;  // before this tile
    const auto flush = [&](bool goes_on) {
        if (begun || goes_on) {
            float *p = partial + (2 * (int64_t)t + (begun ? 0 : 1)) * ldp;
            cols.store(p, sum);
        } else {
            put_row<TW, VEC>(c, cols, run, sum);
        }
#pragma unroll
        for (int k = 0; k < 8; ++k)
            sum[k] = 0.f;
        begun = false;
    };
    for (int64_t p = lo; p < hi; ++p) {
        const uint32_t k = key[p];
        if (k != run) {
            flush(false);
            run = k;
        }
        if (k >= (uint32_t)c.vocab)
            return;
        float v[8];
        cols.load(static_cast<const TG *>(c.dout) + (int64_t)at[p] * c.ldg, v);
#pragma unroll
        for (int h = 0; h < 8; ++h)
            sum[h] += v[h];
    }
    flush(hi < T && key[hi] == run);
}

// Runs over several tiles: the partial sums of the tile they began in and of those they go on in.  32 threads take 256
// columns, the block's eight warps share the tiles of a run, and their sums are added up in order.
template <typename TW>
__global__ void __launch_bounds__(256) k_embed_join(EmbedGradCall c, const uint32_t *__restrict__ key, int tile, int tiles,
                                                    int slices, const float *__restrict__ partial, int64_t ldp)
{
    __shared__ int owner[kMaxTiles], first_of[kMaxTiles / 32 + 1];
    __shared__ float part[8][256];
    const int64_t d = c.d;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    static_assert(kMaxTiles == 32 * 32, "one warp adds up the counts");
    // tile t owns a run that begins in it and goes on in tile t + 1; every block lists the owners in the same order
    for (int w = warp; w < kMaxTiles / 32; w += 8) {
        const int t = w * 32 + lane;
        bool owns = false;
        if (t + 1 < tiles) {
            const uint32_t k = key[(int64_t)(t + 1) * tile - 1];
            owns = k < (uint32_t)c.vocab && key[(int64_t)(t + 1) * tile] == k && (t == 0 || key[(int64_t)t * tile - 1] != k);
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
            owner[place++] = lane * 32 + __ffs(left) - 1;
        __syncwarp();
        first_of[lane + 1] = scan;
    }
    __syncthreads();
    const int n = first_of[kMaxTiles / 32] * slices;
    for (int item = blockIdx.x; item < n; item += gridDim.x) {
        const int t = owner[item / slices], slice = item % slices;
        const uint32_t k = key[(int64_t)(t + 1) * tile - 1];
        const Columns<true> cols{(int64_t)slice * 256 + lane * 8, ldp, 1};  // of the partial sums, whose rows are padded
        float sum[8] = {};
        for (int s = t + 1 + warp; s < tiles && key[(int64_t)s * tile] == k; s += 8) {
            float v[8];
            if (cols.first < ldp) {
                cols.load(partial + 2 * (int64_t)s * ldp, v);
#pragma unroll
                for (int h = 0; h < 8; ++h)
                    sum[h] += v[h];
            }
        }
#pragma unroll
        for (int h = 0; h < 8; ++h)
            part[warp][lane * 8 + h] = sum[h];
        __syncthreads();
        const int64_t j = (int64_t)slice * 256 + threadIdx.x;
        if (j < d) {
            float s = partial[(2 * (int64_t)t + 1) * ldp + j];
#pragma unroll
            for (int w = 0; w < 8; ++w)
                s += part[w][threadIdx.x];
            TW *w = static_cast<TW *>(c.dw) + (int64_t)k * c.ldw + j;
            s *= c.scale;
            *w = from_float<TW>(c.accumulate ? to_float(*w) + s : s);
        }
        __syncthreads();
    }
}

int tile_size(int64_t T)
{
    int n = 8;
    while ((T + n - 1) / n > kMaxTiles)
        n *= 2;
    return n;
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
        for (int k = 0; k < 2; ++k) {
            sort.key[k] = reinterpret_cast<uint32_t *>(take(sizeof(uint32_t) * (size_t)T));
            sort.at[k] = reinterpret_cast<int32_t *>(take(sizeof(int32_t) * (size_t)T));
        }
        present = reinterpret_cast<uint32_t *>(take(sizeof(uint32_t) * (size_t)((vocab + 31) / 32)));
        const int tile = tile_size(T);
        partial = reinterpret_cast<float *>(take(sizeof(float) * 2 * (size_t)ldp * (size_t)((T + tile - 1) / tile)));
    }
};

}  // namespace

size_t embed_bwd_workspace_bytes(int64_t T, int64_t d, int64_t vocab) { return Workspace(nullptr, T, d, vocab).bytes; }

cudaError_t launch_embed(const EmbedCall &c, cudaStream_t stream)
{
    const int64_t chunks = (c.d + kFwdChunk - 1) / kFwdChunk;
    const unsigned grid = (unsigned)std::min<int64_t>((c.T * chunks + kFwdWarps - 1) / kFwdWarps, (int64_t)device_sm_count() * 16);
    const bool vec = boundary(c.w, c.ldw, c.w_dtype) && boundary(c.out, c.ldo, c.out_dtype);
    with_types(c.w_dtype, c.out_dtype, [&](auto w, auto o) {
        using W = decltype(w);
        using O = decltype(o);
        auto kernel = vec ? k_embed<W, O, true> : k_embed<W, O, false>;
        kernel<<<grid, 32 * kFwdWarps, 0, stream>>>(c, chunks);
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
    if (e != cudaSuccess)
        return e;
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[1];
    cfg.gridDim = c.T > kSortThreads ? kMaxCtas : 1;
    cfg.blockDim = kSortThreads;
    cfg.dynamicSmemBytes = sizeof(uint32_t) * kSortWarps << bits;
    cfg.stream = stream;
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = cfg.gridDim.x;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    e = cudaLaunchKernelEx(&cfg, k_sort_tokens, c.ids, c.mask, c.T, c.vocab, ws.sort, passes, bits,
                           c.accumulate ? (uint32_t *)nullptr : ws.present, c.status);
    if (e != cudaSuccess)
        return e;
    const uint32_t *key = ws.sort.key[passes & 1];
    const int32_t *at = ws.sort.at[passes & 1];
    const int tile = tile_size(c.T), tiles = (int)((c.T + tile - 1) / tile);
    const int threads = (int)std::min<int64_t>(kSumThreads, (c.d + 255) / 256 * 32), slices = (int)((c.d + 8 * threads - 1) / (8 * threads));
    const int zero = c.accumulate ? 0 : (int)std::min<int64_t>((c.vocab + 255) / 256, (int64_t)device_sm_count() * 4);
    const bool vec = boundary(c.dout, c.ldg, c.dout_dtype) && boundary(c.dw, c.ldw, c.dw_dtype);
    with_types(c.dout_dtype, c.dw_dtype, [&](auto g, auto w) {
        using G = decltype(g);
        using W = decltype(w);
        auto sums = vec ? k_embed_sums<G, W, true> : k_embed_sums<G, W, false>;
        if (tiles * slices + zero > 0)
            sums<<<tiles * slices + zero, threads, 0, stream>>>(c, key, at, tile, tiles, slices, ws.partial, ws.ldp, ws.present);
        if (tiles > 1) {
            const int n = (int)((c.d + 255) / 256);
            const unsigned grid = (unsigned)std::min<int64_t>((int64_t)(tiles - 1) * n, (int64_t)device_sm_count() * 4);
            k_embed_join<W><<<grid, 256, 0, stream>>>(c, key, tile, tiles, n, ws.partial, ws.ldp);
        }
    });
    return cudaGetLastError();
}

}  // namespace turnopd
