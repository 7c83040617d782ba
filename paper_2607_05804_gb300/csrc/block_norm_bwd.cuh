// Rows of the backward pass of the norms around a block: everything of a row in one pass over its arrays.
#pragma once

#include <algorithm>
#include <type_traits>

#include "block_norm.cuh"

namespace turnopd {
namespace {

__device__ __forceinline__ void cp8(void *smem, const void *gmem)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"((uint32_t)__cvta_generic_to_shared(smem)), "l"(gmem) : "memory");
}
// Waits for all but the newest `pending` groups of copies.
__device__ __forceinline__ void wait_copies(int pending)
{
    if (pending == 0)
        asm volatile("cp.async.wait_group 0;" ::: "memory");
    else if (pending == 1)
        asm volatile("cp.async.wait_group 1;" ::: "memory");
    else
        asm volatile("cp.async.wait_group 2;" ::: "memory");
}

// One array of a row in the ring.
struct RingPart {
    const char *p;   // row 0, null: not read
    uint32_t pitch;  // bytes from row to row
    int at;          // bytes into a stage
    int dtype;
    int bytes;       // of one column
    bool direct;     // does not come through the ring: read from global memory when it is needed
};

struct Ring {
    RingPart resid, y, dh, dro, gate;
    uint32_t dr, dy, dgate;  // pitches of the results' rows
    int extra;   // bytes into a stage: for each warp its copy of the row's statistics and of its columns' exponents
    bool blocks; // rows are whole blocks of 256 columns, whose codes and exponents are copied by the warp
    int stage;   // bytes of a stage of one group
    int stages;  // 2 to 4: the row at hand, the next one, and those in flight
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

constexpr int extra_bytes(int pieces, bool codes) { return 16 + (codes ? 2 * 8 * pieces : 0); }  // of a warp: statistics, exponents

// Most threads of a block: 512 with 128 registers each, or 640 with 96, which one piece of eight columns to a thread will do with.
constexpr int kFew = 512, kMany = 640;

// What r' and y are stored in: the gradients' types, codes of one kind, or any.
enum Stored { kGradientTypes, kE4m3, kInt8, kAny };
template <Stored S, typename T> constexpr int type_code()
{
    return S == kGradientTypes ? (int)(sizeof(T) == 2 ? TURNOPD_BF16 : TURNOPD_F32) : (int)(S == kE4m3 ? TURNOPD_E4M3 : TURNOPD_INT8);
}
constexpr int type_bytes(int dtype) { return dtype == TURNOPD_F32 ? 4 : dtype == TURNOPD_BF16 ? 2 : 1; }

template <typename T> constexpr int gradient_type() { return sizeof(T) == 2 ? TURNOPD_BF16 : TURNOPD_F32; }

// One column of a row of any array as it is stored, and its value later, so that no instruction waits for the load
// before the value is needed.
__device__ __forceinline__ uint32_t raw_column(const RingPart &p, uint32_t i, int j)
{
    const char *at = p.p + (uint64_t)i * p.pitch + j * p.bytes;
    if (p.bytes == 2)
        return *reinterpret_cast<const unsigned short *>(at);
    if (p.bytes == 4)
        return *reinterpret_cast<const uint32_t *>(at);
    return *reinterpret_cast<const uint8_t *>(at);
}
__device__ __forceinline__ float column_value(uint32_t raw, int dtype, uint32_t exponent)
{
    if (dtype == TURNOPD_BF16)
        return __uint_as_float(raw << 16);
    if (dtype == TURNOPD_F32)
        return __uint_as_float(raw);
    return (dtype == TURNOPD_E4M3 ? decode_e4m3((uint8_t)raw) : (float)(int8_t)raw) * act_scale(exponent);
}

// One or two pieces of eight columns to a thread, which keeps their sums over rows in registers from row to row.  Group b of all
// takes rows b, b + groups, ..., so that every sum has a fixed order.  A row's arrays come through a ring in shared memory, in
// which each thread copies and reads its own pieces only (codes of r', and of y where it keeps them, in whole blocks each warp).
// The sums over the next row that D needs are taken together with those over the row at hand that dy needs: one barrier to a
// row.  gamma lies in shared memory, and values are read from the ring once more where they are needed again: a thread's
// registers would not hold them.  A warp's pieces lie 256 columns apart, so that they are found at constant offsets.
//
// Bound: instruction issue and its latencies beside HBM (ncu, 8,192 rows: 0.58 of the issue slots with 15 to 20 warps per SM).
// An element takes four arrays' unpacking, partly twice, 14 multiply-adds and a share of the row's sums, 40 to 52 instructions.
// 32,768 x 4,096 bf16 284 us with both norms (0.84 of the copy rate), 16,384 x 5,120 190 with a gate per channel (0.78), fp32
// stream 389 and 265 (0.91, 0.84), layer norms 345 and 271 (0.69, 0.55), from 8-bit codes 275 (0.72).  Rows that begin
// anywhere, 16,384 x 3,001: 177, where 3,000 columns take 133.
//
// ENDS: the rows begin anywhere, but in all arrays at the same element of a group of eight.  The groups' number is a multiple
// of eight then, so all rows of one group begin at the same element, and a thread keeps the same columns from row to row:
// pieces of eight from the first boundary on, and the first threads one of the elements before and after them each.
// GENERAL: layer norms, sums for betas, or beta in the gradient of a gate for every element; without it the means of g, those
// sums and that beta are left out.
// COMMON: dh and dr' come in, dr and dy go out, no gate for every element, so that nothing asks which there are.
template <typename TR, typename TY, int kPieces, int MOST, Stored STORED, bool ENDS, bool GENERAL, bool COMMON>
__global__ void __launch_bounds__(MOST, 1) k_block_bwd(BlockGradCall c, Ring ring, int n, int phase, int phase_step)
{
    // sums over a row: of g xh (and of g) of the norm after the block, and of the norm before the next one
    constexpr int kRowSums = GENERAL ? 4 : 2, kE = 8 * kPieces, kExtra = extra_bytes(kPieces, STORED != kGradientTypes);
    constexpr bool kMixed = STORED == kAny, kCodes = STORED == kE4m3 || STORED == kInt8;
    // Codes that a warp copied together are read before the warp meets in the middle of a row, since the next row's copies come
    // into their place from the row's end on.  y's are needed once more behind that, for dy: two pieces' are kept in registers
    // (32,768 x 4,096 from e4m3 275 us; copied by each thread for itself 296; with the warp meeting once more 282, and 526 with
    // an fp32 stream, which takes 410); one piece's, for which the registers are too few, and those of arrays of any type are
    // copied by each thread for itself (16,384 x 5,120 layer norms from int8 380 us; in registers 440; meeting once more 442).
    constexpr bool kKeepY = kCodes && !ENDS && kPieces == 2;
    constexpr int kTypeR = type_code<STORED, TR>(), kTypeY = type_code<STORED, TY>();
    extern __shared__ __align__(128) char shared[];
    __shared__ Numbers<kRowSums> red[2][MOST / 32];
    const int t = threadIdx.x % n, group = threadIdx.x / n, warps = n / 32, per = blockDim.x / n, d = (int)c.d;
    const uint32_t T = (uint32_t)c.T, groups = gridDim.x * per, b = blockIdx.x * per + group;  // rows: 2^31 at most, and a few steps more
    const bool layer = GENERAL && c.kind == TURNOPD_LAYER_NORM, pre = COMMON || c.gamma_pre, post = c.gamma_post;
    const bool token_gate = !COMMON && ring.gate.p, dgate = token_gate && c.dgate, has_dro = COMMON || ring.dro.p;
    const bool put_dr = COMMON || c.d_resid, put_dy = COMMON || c.dy, needs_y = ring.y.p;
    const bool post_sums = COMMON || c.dgamma_post || c.dbeta_post || (c.dgate && !c.ldg);
    const bool needs_stream = COMMON || put_dr || put_dy || c.dgate || post_sums;
    const float inv_d = 1.f / (float)d, s = c.branch_scale;
    const uint32_t exps_per_row = (d + kActGroup - 1) / kActGroup;
    const int head = ENDS ? min((8 - (int)((phase + b * phase_step) & 7)) & 7, d) : 0;
    const int whole = (d - head) / 8, ends = ENDS ? d - whole * 8 : 0;
    const int end = t < head ? t : whole * 8 + t;  // the single column of this thread, where t < ends
    const int piece0 = (t >> 5) * 32 * kPieces + (t & 31);
    // the first column of piece k; of a missing one that of the last piece, which is computed once more, with factors of 0,
    // and not stored
    int columns[kPieces];
#pragma unroll
    for (int k = 0; k < kPieces; ++k)
        columns[k] = head + min(piece0 + 32 * k, whole - 1) * 8;
    const auto column = [&](int k) { return columns[k]; };
    const auto there = [&](int k) { return piece0 + 32 * k < whole; };
    const bool at_end = ENDS && t < ends;

    char *own = shared + (size_t)group * (ring.stages * ring.stage + n * kE * (int)sizeof(float));
    float4 *gamma = reinterpret_cast<float4 *>(own + ring.stages * ring.stage) + t;  // n apart
    constexpr int kSums = GENERAL ? 4 : 2, kPostSum = GENERAL ? 2 : 1;  // dh xh_pre, (dh,) X xh_post (, X)
    float2 cpost[kE / 2], sums[kSums][kE / 2];
    float sums_end[kSums] = {};
#pragma unroll
    for (int k = 0; k < kE / 2; ++k)
#pragma unroll
        for (int q = 0; q < kSums; ++q)
            sums[q][k] = make_float2(0.f, 0.f);
    uint32_t ahead = b;  // the next row to copy, whose mask has been read before
    uint32_t ahead_on = ahead < T && c.mask ? c.mask[ahead] : 1u;
    int ahead_stage = 0;
    uint32_t ons = 0;  // whether the rows copied last are not masked, the newest in bit 0
    const bool code_r = kCodes ? pre : kMixed && pre && ring.resid.dtype >= TURNOPD_E4M3;
    const bool code_y = kCodes ? needs_y : kMixed && needs_y && ring.y.dtype >= TURNOPD_E4M3;
    const bool held_y = kKeepY && code_y && put_dy && post;  // wherever y is read for dy
    const auto copy = [&]() {
        if (ahead < T && ahead_on) {
            char *to = own + ahead_stage * ring.stage;
            const auto part = [&](const RingPart &p, int bytes, bool by_warp) {
                if (!p.p || (!COMMON && p.direct))
                    return;
                const char *from = p.p + (uint64_t)ahead * p.pitch;
                if (bytes == 1 && by_warp) {
                    // a warp's codes together, sixteen at a time: half as many copies
                    const int lane = t & 31;
                    if (lane < 16 * kPieces)
                        cp16(to + p.at + (t >> 5) * kPieces * 256 + lane * 16,
                             from + min(((t >> 5) * kPieces + (lane >> 4)) * 256, d - 256) + (lane & 15) * 16);
                    return;
                }
#pragma unroll
                for (int k = 0; k < kPieces; ++k) {
                    char *dst = to + p.at + piece0 * 8 * bytes + k * 256 * bytes;
                    const char *at = from + column(k) * bytes;
                    if (bytes == 1) {
                        cp8(dst, at);
                    } else {
                        cp16(dst, at);
                        if (bytes == 4)
                            cp16(dst + 16, at + 16);
                    }
                }
            };
            part(ring.resid, kMixed ? ring.resid.bytes : type_bytes(kTypeR), ring.blocks);
            part(ring.dh, sizeof(TY), false);
            part(ring.dro, sizeof(TR), false);
            part(ring.y, kMixed ? ring.y.bytes : type_bytes(kTypeY), kKeepY && ring.blocks);
            part(ring.gate, sizeof(TY), false);
            char *extra = to + ring.extra + (t >> 5) * kExtra;
            const int lane = t & 31, block = min((t >> 5) * kPieces + lane, d / 256 - 1);  // of 256 columns
            if (lane == 0 && (COMMON || c.stats))
                cp16(extra, c.stats + (uint64_t)ahead * 4);
            if ((kMixed || kCodes) && ring.blocks && lane < kPieces) {
                if (code_r)
                    cp8(extra + 16 + 8 * lane, c.resid_exps + (uint64_t)ahead * exps_per_row + block * 8);
                if (code_y)
                    cp8(extra + 16 + 8 * (kPieces + lane), c.y_exps + (uint64_t)ahead * exps_per_row + block * 8);
            }
        }
        ons = ons << 1 | (ahead < T && ahead_on);
        ahead += groups;
        ahead_stage = ahead_stage + 1 == ring.stages ? 0 : ahead_stage + 1;
        if (c.mask && ahead < T)
            ahead_on = c.mask[ahead];
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    for (int k = 0; k + 1 < ring.stages; ++k)
        copy();

    // gamma_pre, and s gamma_post gate (without those that there are not): 0 for missing pieces
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

    // What a thread needs of a row beside its pieces.  Exponents that do not come through the ring (of each piece, whose columns
    // may lie in two groups of them) and the thread's single column are read two rows ahead, of masked rows too, and looked at
    // when their turn comes.  (With the mask asked for first 32,768 x 4,096 from e4m3 took 1 % longer, 16,384 x 1,000 4 %.)
    struct Row {
        float4 stats;
        uint32_t er[kPieces], er2[ENDS ? kPieces : 1], ey[kPieces], ey2[ENDS ? kPieces : 1];
        uint32_t resid, y, dh, dro, gate, e_resid, e_y;
        bool fine;
    };
    const auto read_row = [&](uint32_t i) {
        Row m{};
        if (i >= T)
            return m;
        if ((kMixed || kCodes) && !ring.blocks) {
            const uint64_t at = (uint64_t)i * exps_per_row;
#pragma unroll
            for (int k = 0; k < kPieces; ++k) {
                const int g = column(k) / kActGroup, h = (column(k) + 7) / kActGroup;
                if (code_r) {
                    m.er[k] = c.resid_exps[at + g];
                    if (ENDS)
                        m.er2[ENDS ? k : 0] = c.resid_exps[at + h];
                }
                if (code_y) {
                    m.ey[k] = c.y_exps[at + g];
                    if (ENDS)
                        m.ey2[ENDS ? k : 0] = c.y_exps[at + h];
                }
            }
            if (at_end && code_r)
                m.e_resid = c.resid_exps[at + end / kActGroup];
            if (at_end && code_y)
                m.e_y = c.y_exps[at + end / kActGroup];
        }
        if (at_end) {
            if (pre) {
                m.resid = raw_column(ring.resid, i, end);
                m.dh = raw_column(ring.dh, i, end);
            }
            if (has_dro)
                m.dro = raw_column(ring.dro, i, end);
            if (needs_y)
                m.y = raw_column(ring.y, i, end);
            if (token_gate)
                m.gate = raw_column(ring.gate, i, end);
        }
        return m;
    };
    // the rest, from the ring (of a masked row that is of no use); on: the row is there and not masked
    const auto complete = [&](Row &m, const char *at, bool on) {
        const char *extra = at + ring.extra + (t >> 5) * kExtra;
        m.stats = COMMON || c.stats ? *reinterpret_cast<const float4 *>(extra) : make_float4(0.f, 0.f, 0.f, 0.f);
        m.fine = on && (!post || m.stats.y > 0.f) && (!pre || m.stats.w > 0.f);
        if ((kMixed || kCodes) && ring.blocks) {
            const int lane = t & 31;
#pragma unroll
            for (int k = 0; k < kPieces; ++k) {
                m.er[k] = static_cast<uint8_t>(extra[16 + 8 * k + (lane >> 2)]);
                m.ey[k] = static_cast<uint8_t>(extra[16 + 8 * (kPieces + k) + (lane >> 2)]);
            }
        }
    };

    // Eight columns of an activation of the row in a stage, less mu, but for a factor that is returned: the codes' scale, where
    // it is the same for all eight and nothing is taken off.
    const auto activation = [&](const char *at, uint32_t i, const RingPart &part, int stored, uint32_t exp, uint32_t exp2, float mu, int k,
                                float2 *v) {
        const int dtype = kMixed ? part.dtype : stored, bytes = kMixed ? part.bytes : type_bytes(stored);
        if (!COMMON && part.direct)
            from_ring(part.p + (uint64_t)i * part.pitch + column(k) * bytes, dtype, v);
        else
            from_ring(at + part.at + piece0 * 8 * bytes + k * 256 * bytes, dtype, v);
        if ((kMixed || kCodes) && dtype >= TURNOPD_E4M3) {
            const float lo = act_scale(exp);
            if (!ENDS && !GENERAL)
                return lo;
            const float hi = ENDS ? act_scale(exp2) : lo;
            const int first = ENDS ? kActGroup - (column(k) & (kActGroup - 1)) : 8;  // columns of the first group
#pragma unroll
            for (int e = 0; e < 4; ++e)
                v[e] = ffma2(v[e], make_float2(2 * e < first ? lo : hi, 2 * e + 1 < first ? lo : hi), splat(-mu));
        } else if (GENERAL) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                v[e] = fadd2(v[e], splat(-mu));
        }
        return 1.f;
    };
    const auto gradient = [&](auto type, const char *at, uint32_t i, const RingPart &part, int k, float2 *v) {
        if (!COMMON && part.direct) {
            load8(reinterpret_cast<const decltype(type) *>(part.p + (uint64_t)i * part.pitch) + column(k), reinterpret_cast<float *>(v));
            return;
        }
        load8(reinterpret_cast<const decltype(type) *>(at + part.at) + piece0 * 8 + k * 256, reinterpret_cast<float *>(v));
    };
    const auto centred_r = [&](const char *at, const Row &m, int k, float2 *v) {
        return activation(at, 0u, ring.resid, kTypeR, m.er[k], m.er2[ENDS ? k : 0], m.stats.z, k, v);
    };
    const auto centred_y = [&](const char *at, uint32_t i, const Row &m, int k, float2 *v) {  // mu is 0 without that norm
        return activation(at, i, ring.y, kTypeY, m.ey[k], m.ey2[ENDS ? k : 0], m.stats.x, k, v);
    };
    // the same from y's codes in registers
    const auto centred_codes = [&](uint2 codes, const Row &m, int k, float2 *v) {
        decode8(codes, kTypeY == TURNOPD_E4M3, reinterpret_cast<float *>(v));
        const float scale = act_scale(m.ey[k]);
        if (!GENERAL)
            return scale;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            v[e] = ffma2(v[e], splat(scale), splat(-m.stats.x));
        return 1.f;
    };
    const auto times_gamma = [&](int k, float2 *g) {
        const float4 a = gamma[2 * k * n], z = gamma[(2 * k + 1) * n];
        g[0] = fmul2(g[0], make_float2(a.x, a.y));
        g[1] = fmul2(g[1], make_float2(a.z, a.w));
        g[2] = fmul2(g[2], make_float2(z.x, z.y));
        g[3] = fmul2(g[3], make_float2(z.z, z.w));
    };
    // sums of g (r' - mu) and of g over a row of the norm before the next block, and the sums over rows
    const auto first_sums = [&](const char *at, const Row &m, float &sx, float &sg) {
        const float r1 = m.stats.w;
        sx = sg = 0.f;
#pragma unroll
        for (int k = 0; k < kPieces; ++k) {
            float2 x[4], g[4], x2 = make_float2(0.f, 0.f), g2 = x2;
            const float f = centred_r(at, m, k, x);
            gradient(TY(), at, 0u, ring.dh, k, g);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                sums[0][4 * k + e] = ffma2(fmul2(g[e], splat(r1 * f)), x[e], sums[0][4 * k + e]);
                if (GENERAL)
                    sums[1][4 * k + e] = fadd2(g[e], sums[1][4 * k + e]);
            }
            times_gamma(k, g);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (GENERAL)
                    g2 = fadd2(g2, g[e]);
                x2 = ffma2(g[e], x[e], x2);
            }
            sx = fmaf(x2.x + x2.y, f, sx);
            sg += g2.x + g2.y;
        }
        if (at_end) {
            const float x = column_value(m.resid, kMixed ? ring.resid.dtype : kTypeR, m.e_resid) - m.stats.z;
            const float g = column_value(m.dh, gradient_type<TY>(), 0u);
            sums_end[0] = fmaf(g * r1, x, sums_end[0]);
            if (GENERAL)
                sums_end[1] += g;
            sg += g * gamma_end;
            sx = fmaf(g * gamma_end, x, sx);
        }
    };

    Row m = read_row(b), next = read_row(b + groups);
    int stage = 0, odd = 0;
    // the sums of the first row are taken by themselves (those of rows that do not take part, of nothing: no barrier stands
    // under a condition that every thread reads from the caller's memory for itself)
    Numbers<kRowSums> row_sums{};
    wait_copies(ring.stages - 2);
    __syncwarp();  // the warp's copies of the statistics
    complete(m, own, ons >> (ring.stages - 2) & 1);
    if (pre && m.fine) {
        float sx, sg;
        first_sums(own, m, sx, sg);
        row_sums.v[1] = sx;
        if (GENERAL)
            row_sums.v[kRowSums - 1] = sg;
    }
    if (pre && needs_stream) {
        row_sums = group_sum(row_sums, red[odd], group, warps);
        odd ^= 1;
    }
    for (uint32_t i = b; i < T; i += groups) {
        copy();
        Row after = read_row(i + 2 * groups);
        const char *at = own + stage * ring.stage;
        const int next_stage = stage + 1 == ring.stages ? 0 : stage + 1;
        const bool fine = m.fine;
        const float r0 = m.stats.y, r1 = m.stats.w, scale = post ? r0 : 1.f;
        const auto put8 = [&](auto type, void *p, uint32_t pitch, int k, const float2 *v) {
            using R = decltype(type);
            if (there(k))
                store8(reinterpret_cast<R *>(static_cast<char *>(p) + (uint64_t)i * pitch) + column(k), reinterpret_cast<const float *>(v));
        };
        const auto put1 = [&](auto type, void *p, uint32_t pitch, float v) {
            using R = decltype(type);
            if (at_end)
                reinterpret_cast<R *>(static_cast<char *>(p) + (uint64_t)i * pitch)[end] = from_float<R>(v);
        };
        // D = dr' + r (g - mean g - xh mean(g xh)), then X = D times the gate that each token has of its own, and E
        const float c1 = -(row_sums.v[1] * inv_d * r1) * r1 * r1;  // of r' - mu
        const float c0 = layer ? -r1 * (row_sums.v[kRowSums - 1] * inv_d) : 0.f;
        float2 E[kE / 2];
        float E_end = 0.f, ye = 0.f;
        row_sums = Numbers<kRowSums>{};
        if (needs_stream && fine) {
            float2 sg = make_float2(0.f, 0.f), sx = sg;
#pragma unroll
            for (int k = 0; k < kPieces; ++k) {
                float2 D[4], x[4];
                if (has_dro)
                    gradient(TR(), at, 0u, ring.dro, k, D);
                else
                    D[0] = D[1] = D[2] = D[3] = make_float2(0.f, 0.f);
                if (pre) {
                    float2 g[4];
                    const float f = c1 * centred_r(at, m, k, x);
                    gradient(TY(), at, 0u, ring.dh, k, g);
                    times_gamma(k, g);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        D[e] = ffma2(x[e], splat(f), ffma2(g[e], splat(r1), D[e]));
                        if (GENERAL)
                            D[e] = fadd2(D[e], splat(c0));
                    }
                }
                if (put_dr) {
                    float2 o[4];
                    if (c.resid_scale == 1.f) {
                        put8(TR(), c.d_resid, ring.dr, k, D);
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            o[e] = fmul2(D[e], splat(c.resid_scale));
                        put8(TR(), c.d_resid, ring.dr, k, o);
                    }
                }
                if (needs_y) {
                    const float f = scale * centred_y(at, i, m, k, x);
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        x[e] = fmul2(x[e], splat(f));
                }
                if (token_gate) {
                    float2 g[4];
                    if (dgate) {
                        // s D (gamma xh + beta): the factor after that norm is s gamma here
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            g[e] = fmul2(x[e], cpost[4 * k + e]);
                        if (GENERAL && c.beta_post)
#pragma unroll
                            for (int e = 0; e < 8; ++e)
                                reinterpret_cast<float *>(g)[e] += s * param(c.beta_post, c.param_dtype, column(k) + e);
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            g[e] = fmul2(g[e], D[e]);
                        put8(TY(), c.dgate, ring.dgate, k, g);
                    }
                    gradient(TY(), at, i, ring.gate, k, g);
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
                if (put_dy && !post)
                    put8(TY(), c.dy, ring.dy, k, E + 4 * k);
            }
            if (at_end) {
                float D = has_dro ? column_value(m.dro, gradient_type<TR>(), 0u) : 0.f;
                if (pre) {
                    const float x = column_value(m.resid, kMixed ? ring.resid.dtype : kTypeR, m.e_resid) - m.stats.z;
                    D = fmaf(x, c1, fmaf(column_value(m.dh, gradient_type<TY>(), 0u) * gamma_end, r1, D)) + c0;
                }
                if (put_dr)
                    put1(TR(), c.d_resid, ring.dr, D * c.resid_scale);
                ye = needs_y ? (column_value(m.y, kMixed ? ring.y.dtype : kTypeY, m.e_y) - m.stats.x) * scale : 0.f;
                if (dgate) {
                    float w = ye * cpost_end;
                    if (GENERAL && c.beta_post)
                        w += s * param(c.beta_post, c.param_dtype, end);
                    put1(TY(), c.dgate, ring.dgate, D * w);
                }
                if (token_gate)
                    D *= column_value(m.gate, gradient_type<TY>(), 0u);
                sums_end[kPostSum] = fmaf(D, ye, sums_end[kPostSum]);
                if (GENERAL)
                    sums_end[kSums - 1] += D;
                E_end = D * cpost_end;
                sg.x += E_end;
                sx.x = fmaf(E_end, ye, sx.x);
                if (put_dy && !post)
                    put1(TY(), c.dy, ring.dy, E_end);
            }
            row_sums.v[0] = sx.x + sx.y;
            if (GENERAL)
                row_sums.v[kRowSums - 2] = sg.x + sg.y;
        } else if (needs_stream) {
            const float2 zero[4] = {};
#pragma unroll
            for (int k = 0; k < kPieces; ++k) {
                if (put_dr)
                    put8(TR(), c.d_resid, ring.dr, k, zero);
                if (put_dy)
                    put8(TY(), c.dy, ring.dy, k, zero);
                if (dgate)
                    put8(TY(), c.dgate, ring.dgate, k, zero);
            }
            if (put_dr)
                put1(TR(), c.d_resid, ring.dr, 0.f);
            if (put_dy)
                put1(TY(), c.dy, ring.dy, 0.f);
            if (dgate)
                put1(TY(), c.dgate, ring.dgate, 0.f);
        }
        uint2 y_codes[kKeepY ? kPieces : 1];
        if (held_y)
#pragma unroll
            for (int k = 0; k < kPieces; ++k)
                y_codes[kKeepY ? k : 0] = *reinterpret_cast<const uint2 *>(at + ring.y.at + piece0 * 8 + k * 256);
        wait_copies(ring.stages - 2);
        __syncwarp();
        complete(next, own + next_stage * ring.stage, ons >> (ring.stages - 2) & 1);
        if (pre && next.fine) {
            float sx, sg;
            first_sums(own + next_stage * ring.stage, next, sx, sg);
            row_sums.v[1] = sx;
            if (GENERAL)
                row_sums.v[kRowSums - 1] = sg;
        }
        if (needs_stream) {
            row_sums = group_sum(row_sums, red[odd], group, warps);
            odd ^= 1;
        }
        if (put_dy && post && fine) {
            const float a1 = -r0 * r0 * (row_sums.v[0] * inv_d), a0 = layer ? -r0 * (row_sums.v[kRowSums - 2] * inv_d) : 0.f;
#pragma unroll
            for (int k = 0; k < kPieces; ++k) {
                float2 x[4];
                const float f = a1 * (held_y ? centred_codes(y_codes[kKeepY ? k : 0], m, k, x) : centred_y(at, i, m, k, x));
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    x[e] = ffma2(x[e], splat(f), fmul2(E[4 * k + e], splat(r0)));
                    if (GENERAL)
                        x[e] = fadd2(x[e], splat(a0));
                }
                put8(TY(), c.dy, ring.dy, k, x);
            }
            if (ENDS)
                put1(TY(), c.dy, ring.dy, fmaf(E_end, r0, -r0 * (row_sums.v[0] * inv_d) * ye) + a0);
        }
        m = next;
        next = after;
        stage = next_stage;
    }
    if (!c.workspace)
        return;
    // the block's groups are added up in their order, in shared memory: one row of partial sums per block
    wait_copies(0);
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

template <typename TR, typename TY, int kPieces, int MOST> cudaError_t launch_rows(BlockGradCall c, const Phases &phases, int *parts, bool *taken, cudaStream_t stream)
{
    const bool sums = c.dgamma_pre || c.dbeta_pre || c.dgamma_post || c.dbeta_post || (c.dgate && !c.ldg);
    const bool needs_y = block_bwd_needs_y(c), token_gate = c.gate && c.ldg, ends = phases.at || phases.step || c.d % 8;
    if (!sums)
        c.workspace = nullptr;
    constexpr int kE = 8 * kPieces;
    Ring ring{};
    ring.dr = (uint32_t)(c.lddr * sizeof(TR));
    ring.dy = (uint32_t)(c.lddy * sizeof(TY));
    ring.dgate = (uint32_t)(c.lddg * sizeof(TY));
    const int n = (int)((c.d + kE * 32 - 1) / (kE * 32)) * 32, per = std::max(1, 256 / n), threads = n * per;
    const auto add = [&](RingPart &part, const void *p, int64_t ld, int32_t dtype, bool direct) {
        if (!p)
            return;
        part.p = static_cast<const char *>(p);
        part.dtype = dtype;
        part.bytes = stored_bytes(dtype);
        part.pitch = (uint32_t)(ld * part.bytes);
        part.at = ring.stage;
        part.direct = direct;
        ring.stage += direct ? 0 : n * kE * part.bytes;
    };
    const bool stored = (!c.gamma_pre || c.resid_dtype == c.grad_r_dtype) && (!needs_y || c.y_dtype == c.grad_y_dtype);
    // of a block that has an SM's shared memory to itself, or half of it beside a block's own kilobyte and its static arrays
    constexpr size_t kRoom = 226 * 1024, kHalf = 114 * 1024 - 1024 - 512;
    const size_t gamma = sizeof(float) * kE * threads;
    // y and a gate of its own for every element are read from global memory where two rows do not fit otherwise
    for (const bool direct : {false, true}) {
        ring.stage = 0;
        add(ring.resid, c.gamma_pre ? c.resid : nullptr, c.ldr, c.resid_dtype, false);
        add(ring.dh, c.dh, c.lddh, c.grad_y_dtype, false);
        add(ring.dro, c.d_resid_out, c.lddro, c.grad_r_dtype, false);
        add(ring.y, needs_y ? c.y : nullptr, c.ldy, c.y_dtype, direct);
        add(ring.gate, token_gate ? c.gate : nullptr, c.ldg, c.grad_y_dtype, direct);
        ring.extra = ring.stage;
        ring.stage += n / 32 * extra_bytes(kPieces, !stored);
        if (2 * (size_t)per * ring.stage + gamma <= kRoom)
            break;
    }
    const auto in_blocks = [](const RingPart &p, const uint8_t *exps) {
        return !p.p || p.bytes != 1 ||
               (reinterpret_cast<uintptr_t>(p.p) % 16 == 0 && p.pitch % 16 == 0 && reinterpret_cast<uintptr_t>(exps) % 8 == 0);
    };
    ring.blocks = c.d % 256 == 0 && !ends && in_blocks(ring.resid, c.resid_exps) && in_blocks(ring.y, c.y_exps);
    // two CTAs per SM up to 256 threads, if each then has room for a row in flight beside the two at hand
    const size_t stage = (size_t)per * ring.stage;
    const int per_sm = threads <= 256 && 3 * stage + gamma <= kHalf ? 2 : 1;
    ring.stages = (int)std::min<size_t>(4, ((per_sm == 2 ? kHalf : kRoom) - gamma) / stage);
    *taken = ring.stages >= 2;
    if (!*taken)
        return cudaSuccess;
    const size_t smem = std::max<size_t>(stage * ring.stages + gamma, sums && per > 1 ? sizeof(float) * per * (size_t)c.d : 0);
    const int64_t blocks = (c.T + per - 1) / per;
    const int64_t most = std::min<int64_t>((int64_t)per_sm * device_sm_count(), kBlockMaxParts);
    // six rows to a group at least, once there is one for every SM: each block's partial sums are written and read again
    // (512 rows x 4,096: 152 blocks 18 us, 256 blocks 22)
    const int64_t sms = device_sm_count();
    int grid = (int)std::min<int64_t>(blocks > sms ? std::max(sms, (blocks + 5) / 6) : blocks, most);
    if (ends)
        grid = std::min((grid * per + 7) / 8 * 8 / per, kBlockMaxParts);  // a multiple of eight groups
    *parts = grid;
    const bool general = block_bwd_general(c);
    const bool common = c.gamma_pre && c.d_resid_out && c.d_resid && c.dy && sums && !token_gate && !ring.y.direct;
    const auto go = [&](auto kernel) {
        const cudaError_t e = allow_shared(kernel, kRoom);
        if (e != cudaSuccess)
            return e;
        kernel<<<grid, threads, smem, stream>>>(c, ring, n, phases.at, phases.step);
        return cudaGetLastError();
    };
    const auto with_general = [&](auto stored, auto has_ends, auto is_common) {
        constexpr Stored S = decltype(stored)::value;
        constexpr bool E = decltype(has_ends)::value, C = decltype(is_common)::value;
        return general ? go(k_block_bwd<TR, TY, kPieces, MOST, S, E, true, C>) : go(k_block_bwd<TR, TY, kPieces, MOST, S, E, false, C>);
    };
    const std::integral_constant<Stored, kGradientTypes> gradient_types;
    const std::integral_constant<Stored, kAny> any;
    const auto with_ends = [&](auto stored_as, auto is_common) {
        return ends ? with_general(stored_as, std::true_type(), is_common) : with_general(stored_as, std::false_type(), is_common);
    };
    if (common && stored)
        return with_ends(gradient_types, std::true_type());
    if (common && c.resid_dtype == c.y_dtype && c.y_dtype == TURNOPD_E4M3)
        return with_ends(std::integral_constant<Stored, kE4m3>(), std::true_type());
    if (common && c.resid_dtype == c.y_dtype && c.y_dtype == TURNOPD_INT8)
        return with_ends(std::integral_constant<Stored, kInt8>(), std::true_type());
    return stored ? with_ends(gradient_types, std::false_type()) : with_ends(any, std::false_type());
}

}  // namespace

template <typename TR, typename TY> cudaError_t launch_block_rows_bwd(const BlockGradCall &c, int *parts, bool *taken, cudaStream_t stream)
{
    const bool token_gate = c.gate && c.ldg;
    const Phases phases{Phase(c.gamma_pre ? c.resid : nullptr, c.ldr, c.resid_dtype),
                        Phase(c.dh, c.lddh, c.grad_y_dtype),
                        Phase(c.d_resid_out, c.lddro, c.grad_r_dtype),
                        Phase(block_bwd_needs_y(c) ? c.y : nullptr, c.ldy, c.y_dtype),
                        Phase(token_gate ? c.gate : nullptr, c.ldg, c.grad_y_dtype),
                        Phase(c.d_resid, c.lddr, c.grad_r_dtype),
                        Phase(c.dy, c.lddy, c.grad_y_dtype),
                        Phase(token_gate ? c.dgate : nullptr, c.lddg, c.grad_y_dtype)};
    // rows less than 4 GB apart, so that a row's place is one product of 32 bits by 32, with a piece of eight columns at least
    const int64_t most = std::max({c.ldr, c.lddh, c.lddro, c.ldy, c.ldg, c.lddr, c.lddy, c.lddg});
    *taken = phases.alike && most < (int64_t)1 << 30 && c.d >= 16;
    if (!*taken)
        return cudaSuccess;
    // Two pieces to a thread up to 4,096 columns, with two blocks per SM where both have room, as beside four bf16 arrays (from
    // 8-bit activations, 32,768 x 4,096: 275 us, one piece and one block 352).  With a gate for every element mostly one block
    // of 256 threads has: 32,768 x 4,096 481 us, 0.66 of the copy rate, where two have 0.84 without such a gate.  Then one piece,
    // whose blocks have twice the warps (16,384 x 5,120 bf16: 192 us, two pieces 203), as long as a block's threads hold the row.
    // With the sums of layer norms or betas (32,768 x 4,096: two pieces 742 us, one 345), or in rows that begin anywhere
    // (16,384 x 3,001: 452 and 226), two pieces are more than the registers hold.  For few rows one piece answers sooner
    // (512 x 4,096: 18 us with two, 16.6 with one).
    const bool two = !block_bwd_general(c) && !phases.at && !phases.step && c.d % 8 == 0 && c.d > 256 &&
                     c.d <= 4096 && c.T >= 8 * device_sm_count();
    if (c.d > 8 * kMany || two)
        return launch_rows<TR, TY, 2, kFew>(c, phases, parts, taken, stream);
    return c.d <= 8 * kFew ? launch_rows<TR, TY, 1, kFew>(c, phases, parts, taken, stream)
                           : launch_rows<TR, TY, 1, kMany>(c, phases, parts, taken, stream);
}

}  // namespace turnopd
