// Attention of one new token per sequence over a paged 16-bit cache:  o = sum_t w_t v_t / sum_t w_t,  w_t = 2^(c q.k_t - m),
// c the softmax scale in log2 units, m a running reference of the row.  One pass; m moves only when a logit passes it by
// kRescaleSlack, so that the sums are rescaled a few times per unit instead of at every tile.
//
// A UNIT is a (sequence, KV head, block of 8 NT query heads).  The tiles of 16 tokens of all units lie end to end on an axis that
// is cut into stretches for the launch's CTAs, and those into equal parts for their warps, whatever the lengths: a warp streams the
// rows of its part through a ring of shared-memory stages of its own (16-byte asynchronous copies; page numbers are looked up one
// tile ahead) and never waits for another warp before its last tile.  The lengths are on the device, so every CTA adds them up for itself.
//
// Heads are the columns of the matrix instructions (m16n8k16): logits = K q^T with the 16 tokens of a tile as rows, and
// o^T = V^T w^T with the channels as rows, so that up to 8 query heads cost the same as one, K and V fragments are read with one
// ldmatrix per 16 x 16 block, and the weights of a tile become the second product's operand with one 8 x 8 transposition per
// eight tokens.  A weight enters as the sum of two 16-bit numbers (what the first loses the second holds): next to the rows'
// bytes the second product costs little (16 x 8192 fp16 tokens 2.4 of 174 us, 8 x 4001 bf16 ones 0.4 of 11.5), and with 8-bit mantissas (bf16) one rounding of the weights would be as large as the
// output's own.  Sums are fp32.
//
// A unit that begins and ends with one warp is written by that warp.  Pieces of a unit meet in their CTA.  Where there are few
// units a cluster of up to 16 CTAs takes one; its CTAs send one another their sums, and each adds up an equal share of the channels (1 x 32768
// tokens of 5 KV heads: 13.7 us; with one CTA that fetches and adds up all of it 16.5, through global records 27).  Where there are
// more units than that, CTAs take equal shares of the axis, a share's border moves to a unit's if that is near, and what is left over
// meets in records of the workspace: the CTA that delivers a unit's last record joins them, in the order of the axis whoever comes last.
//
// Bound: the rows' bytes, 4 D per token and KV head.  1.07 GB of 32 heads of 64 channels (16 x 8192 tokens, fp16, slot by slot) take 171 to 177 us,
// 6.1 to 6.3 TB/s or 0.92 to 0.96 of the copy rate; 0.79 GB of 8 heads of 128 (64 x 4096 at most, bf16) 133 us, 0.90.  Small calls are a chain of memory
// round trips (lengths, tables, rows), a tile's dependent instructions and the joins: 1 x 512 tokens 6.4 us.
#pragma once
#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include "kvq_common.cuh"
#include "kvq_pages.h"
#include "kvq_ptx.cuh"

namespace kvq {

constexpr int kAttnTile = 16;                          // tokens
constexpr int kAttnMaxCtas = 512;                      // of a launch
constexpr int kAttnAbreastLog2 = 1, kAttnAbreast = 1 << kAttnAbreastLog2;      // units that a CTA's warps take side by side at most
constexpr int kAttnCounters = kAttnMaxCtas * kAttnAbreast;     // arrival counters of a workspace
constexpr int kAttnJoinTiles = 10;                     // what a unit that goes on in another stretch costs, in tiles of a warp
constexpr int kAttnMaxCluster = 16;
constexpr int kAttnMinTilesLog2 = 1, kAttnMinTiles = 1 << kAttnMinTilesLog2;   // of a warp, where the work does not fill the
                                                       // launch (200 rows of 200 tokens: 11.0 us, with four 13.2, with one 11.0)
// How far a border may be from a unit's to move there: what a CTA streams in about the time that a join takes, 3 us (4096 rows of 122 tokens 182 us,
// 128 of up to 100 11.7; without it 186 and 15.1; with four times as much 182 and 11.7, but 16 x 8192 175 us instead of 174).
constexpr int kAttnSnapBytes = 131072;
constexpr float kLowest = -3.402823466e38f;
constexpr float kLn2 = 0.69314718055994531f;

// CTAs of 8 or 16 warps; 16 warps of 64 channels, or 8 of 128, fill an SM's shared memory.
template <int D, int W>
struct AttnGeom {
    static constexpr int kWarps = W, kThreads = 32 * W, kCtas = 1024 / (D * W);
    static constexpr int kStages = 3;
    static constexpr int kRowBytes = 2 * D, kTensorBytes = kAttnTile * kRowBytes, kStageBytes = 2 * kTensorBytes;
    static constexpr int kRingBytes = kStages * kStageBytes;               // of a warp
};
template <int D, int NT>
__host__ __device__ constexpr int attn_record_floats() { return 8 * NT * (D + 2); }            // o [D][8 NT], m [8 NT], l [8 NT]

// Shared memory: the rings, the rows' place on the axis and, where there are clusters, what CTAs send one another.
template <int D, int NT>
struct AttnSent {
    float o[D * 8 * NT];                               // [CTA][channels of this CTA][head]
    float m[kAttnMaxCluster][8 * NT], l[kAttnMaxCluster][8 * NT];
};
__host__ __device__ inline size_t attn_place_bytes(int batch) { return (sizeof(int64_t) * ((size_t)batch + 1) + 15) / 16 * 16; }
template <int D, int NT, int W>
inline size_t attn_smem(int batch, bool clusters) {
    return (size_t)W * AttnGeom<D, W>::kRingBytes + attn_place_bytes(batch) + (clusters ? sizeof(AttnSent<D, NT>) : 0);
}

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, bool there) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ void ldmatrix4(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldmatrix4_trans(uint32_t (&r)[4], uint32_t addr) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t v) {
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}
template <bool BF>
__device__ __forceinline__ void mma16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    if constexpr (BF)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// Two fp32 numbers as 16-bit ones (a in the low half), and back.
template <bool BF>
__device__ __forceinline__ uint32_t pack16(float a, float b) {
    uint32_t r;
    if constexpr (BF) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
    else asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
    return r;
}
template <bool BF>
__device__ __forceinline__ float2 unpack16(uint32_t v) {
    if constexpr (BF) return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u));
    else return __half22float2(*reinterpret_cast<const __half2*>(&v));
}
// Two fp16 numbers times a power of two.
__device__ __forceinline__ uint32_t scaled_half2(uint32_t v, float f) {
    const __half2 r = __hmul2(*reinterpret_cast<const __half2*>(&v), __float2half2_rn(f));
    return *reinterpret_cast<const uint32_t*>(&r);
}
template <bool BF>
__device__ __forceinline__ uint16_t round16(float v) {
    return (uint16_t)(pack16<BF>(v, 0.f) & 0xffffu);
}

// A place on the axis: tile t of unit (or bundle of units) u of row b.
struct AttnCursor {
    int b, u, t, tiles, len;
};

// A unit that a warp has part of: its number (-1: none) and its stretch of the axis.
struct AttnPiece {
    int unit;
    int64_t begin, end;
};

// grid: at most kAttnMaxCtas resident CTAs; those that the lengths leave without work return.
template <bool BF, int D, int NT, int W>
__global__ void __launch_bounds__(AttnGeom<D, W>::kThreads, AttnGeom<D, W>::kCtas) k_page_attn(const PageAttnParams P) {
    using G = AttnGeom<D, W>;
    // A weight of fp16 must not end where fp16 does, at 2^-24: where one token has nearly all of the weight, and values near zero, the many others
    // decide the output while the sum of weights counts them.  So the reference lies 2^7 below the largest weight (with the slack 2^15 at most),
    // and the second number of a weight is kept 2^11 times as large, which the values that it is multiplied with make up for: a weight is cut at
    // 2^-43 of the largest.  (Four multiplications for every 16 x 16 values: 16 x 8192 tokens 174.4 us, without 173.3, 32 of up to 8192 with 16 heads
    // per KV head 51.8 and 51.7; a sum of its own for the second product 65.3 there.)  bf16 weights
    // reach as far down as fp32, but so do the values upwards: the reference lies 2^8 above the largest weight, so that with the slack none passes one
    // and what is summed is no larger than n values.
    constexpr float kHead = BF ? -kRescaleSlack : 7.f, kMost = kRescaleSlack + kHead, kSecond = BF ? 1.f : 2048.f;
    constexpr int kMt = D / 16, kR = 8 * NT, kStages = G::kStages, kAttnWarps = G::kWarps, kAttnThreads = G::kThreads, kWarpsLog2 = W == 8 ? 3 : 4;
    namespace cg = cooperative_groups;
    // (powers of two throughout: a division of integers takes longer than all else between two round trips to memory)
    const int C = 1 << P.cluster_log2, group = (int)blockIdx.x >> P.cluster_log2, groups = (int)gridDim.x >> P.cluster_log2, rank = (int)blockIdx.x & (C - 1);
    constexpr int kVecs = D / 8, kRowsAtOnce = 32 / kVecs, kCopies = kAttnTile / kRowsAtOnce;     // 16-byte vectors of a row
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, q = lane & 3;
    extern __shared__ __align__(128) uint8_t s_ring_all[];
    // [batch + 1]: 16 times the tiles before a row, plus the tokens that its last tile lacks
    int64_t* s_place = reinterpret_cast<int64_t*>(s_ring_all + (size_t)kAttnWarps * G::kRingBytes);
    auto tiles_before = [&](int b) -> int64_t { return s_place[b] >> 4; };
    auto tiles_of = [&](int b) -> int { return (int)(tiles_before(b + 1) - tiles_before(b)); };
    auto len_of = [&](int b) -> int { return (tiles_of(b) - 1) * kAttnTile + (kAttnTile - (int)(s_place[b] & 15)); };
    __shared__ int64_t s_scan[kAttnWarps];
    __shared__ int s_longest[kAttnWarps];
    __shared__ uint32_t s_there[kAttnWarps][kStages];  // tokens of a stage that exist
    __shared__ AttnPiece s_piece[2 * kAttnWarps];      // a warp's first and last piece
    // Of every unit abreast, two may go on in other CTAs, one from before and one beyond: their first pieces, or -1
    __shared__ int s_open[2 * kAttnAbreast];
    __shared__ int s_first[2 * kAttnAbreast], s_last[2 * kAttnAbreast];    // stretches of such a unit that this CTA joins (last: -1, another does)

    pdl_launch_dependents();
    pdl_wait();

    // ---- lengths, and tiles before every row
    const int units_per_row = P.kv_heads * P.head_blocks;
    {
        const int per = (P.batch + kAttnThreads - 1) / kAttnThreads;       // neighbouring rows of a thread
        const long long room = (long long)P.width * P.page_size;
        auto tiles = [&](int n) { return (n + (long long)kAttnTile - 1) / kAttnTile; };
#pragma unroll 4
        for (int b = tid; b < P.batch; b += kAttnThreads) s_place[b] = min((long long)max(P.lens[b], 0), room);        // for now
        if (per > 1) __syncthreads();
        int64_t sum = 0;
        int most = 0;
        for (int k = 0; k < per; ++k) {
            const int b = tid * per + k;
            if (b >= P.batch) break;
            const int n = (int)s_place[b];
            sum += tiles(n);
            most = max(most, (int)tiles(n));
        }
        most = __reduce_max_sync(0xffffffffu, most);
        if (lane == 0) s_longest[warp] = most;
        int64_t upto = sum;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int64_t o = __shfl_up_sync(0xffffffffu, upto, d);
            if (lane >= d) upto += o;
        }
        if (lane == 31) s_scan[warp] = upto;
        if (tid < 2 * kAttnWarps) s_piece[tid].unit = -1;
        if (tid < 2 * kAttnAbreast) s_open[tid] = -1;
        __syncthreads();
        int64_t at = upto - sum;
        for (int w = 0; w < warp; ++w) at += s_scan[w];
        for (int k = 0; k < per; ++k) {
            const int b = tid * per + k;
            if (b >= P.batch) break;
            const int n = (int)s_place[b];
            s_place[b] = at * 16 + (tiles(n) * kAttnTile - n);
            at += tiles(n);
        }
        if (tid == kAttnThreads - 1) s_place[P.batch] = at * 16;
        __syncthreads();
    }
    uint16_t* const O = static_cast<uint16_t*>(P.O);
    auto inverse = [](float l) { return l > 0.f || l != l ? 1.f / l : 0.f; };      // (a row that sees nothing gives zeros, a NaN stays one)
    // rows without a token
    for (int b = blockIdx.x; b < P.batch; b += gridDim.x) {
        if (tiles_of(b) != 0) continue;
        for (int e = tid; e < P.q_heads * D; e += kAttnThreads) O[(size_t)b * P.q_heads * D + e] = 0;
        if (P.lse)
            for (int h = tid; h < P.q_heads; h += kAttnThreads) P.lse[(size_t)b * P.q_heads + h] = -INFINITY;
    }
    if (s_place[P.batch] == 0) return;
    // A cluster of CTAs (or one CTA) works on a stretch of the axis: a unit each, where there are no more units than clusters and
    // equal shares would not be shorter than the longest by more than joining them costs (2 units of 65536 tokens: 16.8 us in equal shares,
    // 19.0 one each; 48 of up to 6000: 25.1 and 16.9).
    int longest = 0;
#pragma unroll
    for (int w = 0; w < kAttnWarps; ++w) longest = max(longest, s_longest[w]);
    const int units = P.batch * units_per_row;
    const bool unit_each = units <= groups &&
                           (int64_t)longest * groups <= tiles_before(P.batch) * units_per_row + (int64_t)kAttnJoinTiles * C * kAttnWarps * groups;
    // With equal shares `abreast` units of a row that lie side by side in memory go abreast, each with its share of the CTA's warps
    // (member: which of them this warp works on); the axis then consists of such bundles of units.
    const int abreast_log2 = unit_each ? 0 : P.abreast_log2, abreast = 1 << abreast_log2, team = kAttnWarps >> abreast_log2;
    const int team_log2 = kWarpsLog2 - abreast_log2, member = warp >> team_log2;
    const int bundles_per_row = units_per_row >> abreast_log2, snap = (kAttnSnapBytes / G::kStageBytes) >> abreast_log2;
    const int warps_log2 = P.cluster_log2 + team_log2, warps = 1 << warps_log2;            // that share a stretch
    const int64_t total = tiles_before(P.batch) * bundles_per_row;
    const int stretches = unit_each ? units : (int)min((int64_t)groups, ((total + warps * kAttnMinTiles - 1) >> (warps_log2 + kAttnMinTilesLog2)));
    if (group >= stretches) return;
    auto locate = [&](int64_t at) -> AttnCursor {
        int b0 = 0, b1 = P.batch;
        while (b1 - b0 > 1) {
            const int mid = (b0 + b1) >> 1;
            if (tiles_before(mid) * bundles_per_row <= at) b0 = mid;
            else b1 = mid;
        }
        AttnCursor c;
        c.b = b0;
        c.tiles = tiles_of(b0);
        c.len = len_of(b0);
        const int64_t rest = at - tiles_before(b0) * bundles_per_row;
        c.u = (rest >> 32) == 0 ? (int)((uint32_t)rest / (uint32_t)c.tiles) : (int)(rest / c.tiles);
        c.t = (int)(rest - (int64_t)c.u * c.tiles);
        return c;
    };
    // The borders between equal shares move to the border of a unit that is no more than snap tiles away.
    const int64_t share_size = unit_each ? 0 : (total >> 32) == 0 ? (int64_t)((uint32_t)total / (uint32_t)stretches) : total / stretches;
    const int64_t share_more = total - share_size * stretches;             // (the first share_more have one tile more)
    auto share = [&](int c) -> int64_t { return share_size * c + min((int64_t)c, share_more); };
    auto border = [&](int c) -> int64_t {
        if (c == stretches) return total;
        const int64_t at = share(c);
        const AttnCursor x = locate(at);
        const int back = x.t, ahead = x.tiles - x.t;
        return min(back, ahead) > snap ? at : back <= ahead ? at - back : at + ahead;
    };
    int64_t lo, hi;
    AttnCursor first = {};                             // the unit, where there is one
    if (unit_each) {
        first.b = (int)P.by_units.div((uint32_t)group);
        first.u = group - first.b * units_per_row;
        first.tiles = tiles_of(first.b);
        first.len = len_of(first.b);
        lo = tiles_before(first.b) * units_per_row + (int64_t)first.u * first.tiles;
        hi = lo + first.tiles;
    } else {
        lo = border(group);
        hi = border(group + 1);
    }
    if (lo == hi) return;                              // (the same for the whole cluster)
    if (unit_each && C > 1 && hi - lo > 1) cg::this_cluster().barrier_arrive();            // (before they write one another's memory, all have to be there)
    auto warp_border = [&](int w) -> int64_t { return lo + (((hi - lo) * w) >> warps_log2); };     // of the cluster's warps
    auto cta_border = [&](int r) { return warp_border(r * team); };
    const int64_t wlo = warp_border(rank * team + (warp & (team - 1))), whi = warp_border(rank * team + (warp & (team - 1)) + 1);
    const int64_t cta_lo = cta_border(rank), cta_hi = cta_border(rank + 1);

    auto unit_of = [&](const AttnCursor& c) { return c.u * abreast + member; };        // this warp's, of the row
    auto next_unit = [&](AttnCursor& c) {
        c.t = 0;
        if (++c.u < bundles_per_row) return;
        c.u = 0;
        do ++c.b; while (c.b < P.batch && tiles_of(c.b) == 0);
        if (c.b >= P.batch) return;                    // (behind the last tile)
        c.tiles = tiles_of(c.b);
        c.len = len_of(c.b);
    };
    auto piece_at = [&](const AttnCursor& c, int64_t last) {       // behind its tile `last` of the axis
        AttnPiece p;
        p.unit = c.b * units_per_row + unit_of(c);
        p.begin = last + 1 - c.t;
        p.end = p.begin + c.tiles;
        return p;
    };
    uint8_t* const ring = s_ring_all + (size_t)warp * G::kRingBytes;
    const uint32_t ring_addr = smem_addr(ring);
    const int count = (int)(whi - wlo);
    if (count > 0) {
        // ---- copies: `ahead` is the tile whose page numbers are being looked up
        AttnCursor ahead = first;
        if (unit_each) ahead.t = (int)(wlo - lo);
        else ahead = locate(wlo);
        int looked = 0;                                // tiles looked up so far
        int page = -1, slot = 0, head = 0;
        auto look_up = [&]() {
            page = -1;
            if (looked >= count) return;
            const int pos = ahead.t * kAttnTile + (lane & 15);
            head = (int)P.by_blocks.div((uint32_t)unit_of(ahead));
            if (pos < ahead.len) {
                const int entry = (int)P.by_page.div((uint32_t)pos);
                slot = pos - entry * P.page_size;
                page = P.tables[(size_t)ahead.b * P.width + entry];
            }
            ++looked;
            if (++ahead.t == ahead.tiles) next_unit(ahead);
        };
        int issued = 0;
        auto issue = [&]() {
            if (issued < count) {
                const int stage = issued % kStages;
                const bool there = (uint32_t)page < (uint32_t)P.n_pages;
                const uint32_t mask = __ballot_sync(0xffffffffu, there);
                if (lane == 0) s_there[warp][stage] = mask;
                const int64_t at = there ? page * P.page_stride + slot * P.slot_stride + head * P.head_stride : 0;
                const uint32_t dst = ring_addr + stage * G::kStageBytes;
#pragma unroll
                for (int j = 0; j < kCopies; ++j) {
                    const int r = lane / kVecs + j * kRowsAtOnce, vec = lane % kVecs;
                    const int64_t from = __shfl_sync(0xffffffffu, at, r) + vec * 16;
                    const uint32_t to = dst + r * G::kRowBytes + ((vec ^ (r & 7)) << 4);
                    cp_async16(to, P.Kc + from, (mask >> r) & 1u);
                    cp_async16(to + G::kTensorBytes, P.Vc + from, (mask >> r) & 1u);
                }
            }
            cp_async_commit();
            ++issued;
            look_up();
        };
        AttnCursor at = ahead;
        look_up();
#pragma unroll
        for (int k = 0; k < kStages - 1; ++k) issue();

        uint32_t qf[kMt][NT][2];
        float o[kMt][NT][4], m[NT][2], l[NT][2];
        auto start_unit = [&]() {
            const int h0 = (int)P.by_blocks.div((uint32_t)unit_of(at)), hb = unit_of(at) - h0 * P.head_blocks;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const int r = hb * kR + nt * 8 + g;    // head within the group
                const uint32_t* src = reinterpret_cast<const uint32_t*>(
                    static_cast<const uint16_t*>(P.Q) + ((size_t)at.b * P.q_heads + h0 * P.group + min(r, P.group - 1)) * D) + q;
#pragma unroll
                for (int k = 0; k < kMt; ++k) {
                    qf[k][nt][0] = r < P.group ? __ldg(src + 8 * k) : 0u;
                    qf[k][nt][1] = r < P.group ? __ldg(src + 8 * k + 4) : 0u;
                }
                m[nt][0] = m[nt][1] = kLowest;
                l[nt][0] = l[nt][1] = 0.f;
#pragma unroll
                for (int k = 0; k < kMt; ++k) o[k][nt][0] = o[k][nt][1] = o[k][nt][2] = o[k][nt][3] = 0.f;
            }
        };
        auto sum_lanes = [&]() {                       // the lanes of a column each hold the weights of two tokens of a tile
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int c = 0; c < 2; ++c)
#pragma unroll
                    for (int d = 4; d < 32; d <<= 1) l[nt][c] += __shfl_xor_sync(0xffffffffu, l[nt][c], d);
        };
        auto deliver_piece = [&](float* rec) {         // o [D][kR], m [kR], l [kR]
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const int col = nt * 8 + 2 * q;
#pragma unroll
                for (int k = 0; k < kMt; ++k) {
                    *reinterpret_cast<float2*>(rec + (16 * k + g) * kR + col) = make_float2(o[k][nt][0], o[k][nt][1]);
                    *reinterpret_cast<float2*>(rec + (16 * k + g + 8) * kR + col) = make_float2(o[k][nt][2], o[k][nt][3]);
                }
                if (g == 0) {
                    *reinterpret_cast<float2*>(rec + D * kR + col) = make_float2(m[nt][0], m[nt][1]);
                    *reinterpret_cast<float2*>(rec + (D + 1) * kR + col) = make_float2(l[nt][0], l[nt][1]);
                }
            }
        };
        auto write_unit = [&]() {
            const int h0 = (int)P.by_blocks.div((uint32_t)unit_of(at)), hb = unit_of(at) - h0 * P.head_blocks;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const float i0 = inverse(l[nt][0]), i1 = inverse(l[nt][1]);
                const int r = hb * kR + nt * 8 + g;
                const size_t row = (size_t)at.b * P.q_heads + h0 * P.group + r;
#pragma unroll
                for (int k = 0; k < kMt; ++k) {        // after the transposition a lane holds two channels of head g
                    const uint32_t a = transpose8x8(pack16<BF>(o[k][nt][0] * i0, o[k][nt][1] * i1));
                    const uint32_t b = transpose8x8(pack16<BF>(o[k][nt][2] * i0, o[k][nt][3] * i1));
                    if (r < P.group) {
                        *reinterpret_cast<uint32_t*>(O + row * D + 16 * k + 2 * q) = a;
                        *reinterpret_cast<uint32_t*>(O + row * D + 16 * k + 8 + 2 * q) = b;
                    }
                }
                if (P.lse && g == 0)
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        const int rc = hb * kR + nt * 8 + 2 * q + c;
                        if (rc < P.group) P.lse[(size_t)at.b * P.q_heads + h0 * P.group + rc] = l[nt][c] == 0.f ? -INFINITY : m[nt][c] * kLn2 + logf(l[nt][c]);
                    }
            }
        };
        bool whole = at.t == 0;                        // the piece began with its unit
        start_unit();
#pragma unroll 1
        for (int i = 0; i < count; ++i) {
            cp_async_wait<kStages - 2>();
            __syncwarp();                              // (every lane's copies have arrived, and nobody reads the stage that is filled next)
            const int stage = i % kStages;
            const uint32_t there = s_there[warp][stage] & 0xffffu;
            issue();
            const uint32_t base = ring_addr + stage * G::kStageBytes;
            float s[NT][4];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) s[nt][0] = s[nt][1] = s[nt][2] = s[nt][3] = 0.f;
            {
                const int r = lane & 15;
#pragma unroll
                for (int k = 0; k < kMt; ++k) {
                    uint32_t a[4];
                    ldmatrix4(a, base + r * G::kRowBytes + (((2 * k + (lane >> 4)) ^ (r & 7)) << 4));
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) mma16<BF>(s[nt], a, qf[k][nt][0], qf[k][nt][1]);
                }
            }
            bool over = false;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
                for (int c = 0; c < 4; ++c) s[nt][c] *= P.scale2;
                if (there != 0xffffu) {
                    if (!((there >> g) & 1u)) s[nt][0] = s[nt][1] = -INFINITY;
                    if (!((there >> (g + 8)) & 1u)) s[nt][2] = s[nt][3] = -INFINITY;
                }
                // (the difference, which is exact where it matters: of logits about 2^27 the sum would round to a reference that is 16 higher, and
                // a weight of 2^16 is no fp16 number)
                over |= fmaxf(s[nt][0], s[nt][2]) - m[nt][0] > kMost || fmaxf(s[nt][1], s[nt][3]) - m[nt][1] > kMost;
            }
            if (__any_sync(0xffffffffu, over)) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        float top = fmaxf(s[nt][c], s[nt][c + 2]);
#pragma unroll
                        for (int d = 4; d < 32; d <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
                        top = fmaxf(top - kHead, m[nt][c]);
                        const float f = fast_exp2(m[nt][c] - top);
                        m[nt][c] = top;
                        l[nt][c] *= f;
#pragma unroll
                        for (int k = 0; k < kMt; ++k) o[k][nt][c] *= f, o[k][nt][c + 2] *= f;
                    }
            }
            uint32_t wh[NT][2], wl[NT][2];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    s[nt][c] = fast_exp2(s[nt][c] - m[nt][c & 1]);
                    l[nt][c & 1] += s[nt][c];
                }
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const uint32_t hi16 = pack16<BF>(s[nt][2 * h], s[nt][2 * h + 1]);
                    const float2 back = unpack16<BF>(hi16);
                    wh[nt][h] = transpose8x8(hi16);
                    wl[nt][h] = transpose8x8(pack16<BF>(kSecond * (s[nt][2 * h] - back.x), kSecond * (s[nt][2 * h + 1] - back.y)));
                }
            }
            {
                const int r = (lane & 7) + ((lane >> 4) << 3);
#pragma unroll
                for (int k = 0; k < kMt; ++k) {
                    uint32_t a[4];
                    ldmatrix4_trans(a, base + G::kTensorBytes + r * G::kRowBytes + (((2 * k + ((lane >> 3) & 1)) ^ (r & 7)) << 4));
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) mma16<BF>(o[k][nt], a, wh[nt][0], wh[nt][1]);
                    if constexpr (!BF) {
#pragma unroll
                        for (int c = 0; c < 4; ++c) a[c] = scaled_half2(a[c], 1.f / kSecond);
                    }
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) mma16<BF>(o[k][nt], a, wl[nt][0], wl[nt][1]);
                }
            }
            if (++at.t == at.tiles || i + 1 == count) {
                sum_lanes();
                const bool ends = at.t == at.tiles;
                if (ends && whole) {
                    write_unit();
                } else if (i + 1 < count) {            // the rest of a unit that an earlier warp began
                    deliver_piece(P.warp_rec + ((size_t)blockIdx.x * kAttnWarps + warp) * attn_record_floats<D, NT>());
                    if (lane == 0) s_piece[2 * warp] = piece_at(at, wlo + i);
                } else {
                    cp_async_wait<0>();
                    __syncwarp();
                    deliver_piece(reinterpret_cast<float*>(ring));
                    if (lane == 0) s_piece[2 * warp + 1] = piece_at(at, wlo + i);
                }
                if (i + 1 < count) {
                    next_unit(at);
                    whole = true;
                    start_unit();
                }
            }
        }
    }
    __syncthreads();

    // ---- pieces of the CTA's units meet.  First every piece's factors 2^(m_k - m) and its unit's sum of weights, a lane per
    // piece; then the outputs, four heads of a channel per thread.
    constexpr int kRec = attn_record_floats<D, NT>(), kPieces = 2 * kAttnWarps, kAtOnce = 32 / kPieces;
    static_assert(kPieces == 16 || kPieces == 32, "a warp holds the pieces");
    // (behind the first warp's piece in its ring)
    struct Factors {
        // factors of the pieces; at a unit's first piece its m, and its sum of weights or, where it is complete, the inverse
        float factor[kPieces][kR], m[kPieces][kR], l[kPieces][kR];
    };
    static_assert(kRec * sizeof(float) + sizeof(Factors) <= G::kRingBytes && (G::kRingBytes - sizeof(Factors)) % 16 == 0, "a ring holds a piece and the factors");
    Factors& s_f = *reinterpret_cast<Factors*>(s_ring_all + G::kRingBytes - sizeof(Factors));
    auto last_piece = [&](int w) { return reinterpret_cast<const float*>(s_ring_all + (size_t)w * G::kRingBytes); };
    auto first_piece = [&](int w) -> const float* { return P.warp_rec + ((size_t)blockIdx.x * kAttnWarps + w) * kRec; };
    struct Place {
        size_t row;                                    // of the block's first head
        int heads;
    };
    auto place_of = [&](int unit) {
        const int b = (int)P.by_units.div((uint32_t)unit), u = unit - b * units_per_row, h0 = (int)P.by_blocks.div((uint32_t)u), hb = u - h0 * P.head_blocks;
        return Place{(size_t)b * P.q_heads + h0 * P.group + hb * kR, min(kR, P.group - hb * kR)};
    };
    auto put_lse = [&](const Place& at, int r, float m, float l) {
        if (P.lse && r < at.heads) P.lse[at.row + r] = l == 0.f ? -INFINITY : m * kLn2 + logf(l);
    };
    auto put = [&](const Place& at, int r, int d, const float4& o, const float* inv) {
        const float x[4] = {o.x, o.y, o.z, o.w};
#pragma unroll
        for (int c = 0; c < 4; ++c)
            if (r + c < at.heads) O[(at.row + r + c) * D + d] = round16<BF>(x[c] * inv[c]);
    };
    const int quads = min(kR, P.group + 3) / 4;        // of heads: at most what the group needs
    if (unit_each) {
        // ---- A unit for the whole cluster: the CTA's part, an equal share of whose channels goes to every CTA of the cluster; then
        // every CTA adds up its channels.  (One CTA that fetched and added up everything took 4 us longer for 16 CTAs.)
        if (hi - lo == 1) return;                      // (its warp has written it)
        const Place at = place_of(group);
        const uint32_t live = __ballot_sync(0xffffffffu, lane < kAttnWarps && s_piece[2 * (lane % kAttnWarps) + 1].unit >= 0);     // warps with a piece
        AttnSent<D, NT>* const sent = reinterpret_cast<AttnSent<D, NT>*>(reinterpret_cast<uint8_t*>(s_place) + attn_place_bytes(P.batch));
        if (C > 1) cg::this_cluster().barrier_wait();
        if (warp < kR * kAttnWarps / 32) {             // kAttnWarps lanes for every head
            const int r = tid / kAttnWarps, w = tid % kAttnWarps;
            const bool in = (live >> w) & 1u;
            const float* p = last_piece(w) + D * kR + r;
            const float m = in ? p[0] : kLowest;
            float top = m;
#pragma unroll
            for (int d = 1; d < kAttnWarps; d <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
            const float f = in ? fast_exp2(m - top) : 0.f;
            float sum = in ? f * p[kR] : 0.f;
#pragma unroll
            for (int d = 1; d < kAttnWarps; d <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
            s_f.factor[w][r] = f;
            if (C > 1) {
                for (int c = w; c < C; c += kAttnWarps) {
                    AttnSent<D, NT>* to = cg::this_cluster().map_shared_rank(sent, c);
                    to->m[rank][r] = top, to->l[rank][r] = sum;
                }
            } else if (w == 0) {
                s_f.l[0][r] = inverse(sum);
                put_lse(at, r, top, sum);
            }
        }
        __syncthreads();
        constexpr int kDLog2 = D == 64 ? 6 : 7;
        const int channels_log2 = kDLog2 - P.cluster_log2, channels = 1 << channels_log2;      // of a CTA
        for (int e = tid; e < quads * D; e += kAttnThreads) {
            const int d = e % D, r = 4 * (e / D);
            float4 so = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (int w = 0; w < kAttnWarps; ++w) {
                if (!((live >> w) & 1u)) continue;
                const float4 y = *reinterpret_cast<const float4*>(last_piece(w) + d * kR + r), f = *reinterpret_cast<const float4*>(&s_f.factor[w][r]);
                so.x += f.x * y.x, so.y += f.y * y.y, so.z += f.z * y.z, so.w += f.w * y.w;
            }
            if (C == 1) put(at, r, d, so, &s_f.l[0][r]);
            else *reinterpret_cast<float4*>(cg::this_cluster().map_shared_rank(sent, d >> channels_log2)->o + (rank * channels + (d & (channels - 1))) * kR + r) = so;
        }
        if (C == 1) return;
        cg::this_cluster().sync();                     // (from here on a CTA reads its own memory only)
        if (warp < kR / 2) {                           // sixteen lanes for every head
            const int r = tid >> 4, c = lane & 15;
            const float m = c < C ? sent->m[c][r] : kLowest, l = c < C ? sent->l[c][r] : 0.f;
            float top = m;
#pragma unroll
            for (int d = 1; d < 16; d <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
            const float f = fast_exp2(m - top);
            float sum = f * l;
#pragma unroll
            for (int d = 1; d < 16; d <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
            s_f.factor[c][r] = f;
            if (c == 0) {
                s_f.l[0][r] = inverse(sum);
                if (rank == 0) put_lse(at, r, top, sum);
            }
        }
        __syncthreads();
        for (int e = tid; e < at.heads * channels; e += kAttnThreads) {
            const int r = e >> channels_log2, d = e & (channels - 1);
            float so = 0.f;
#pragma unroll 8
            for (int c = 0; c < C; ++c) so += s_f.factor[c][r] * sent->o[(c * channels + d) * kR + r];
            O[(at.row + r) * D + rank * channels + d] = round16<BF>(so * s_f.l[0][r]);
        }
        return;
    }
    const int j = lane % kPieces;
    const AttnPiece mine = s_piece[j];
    constexpr uint32_t kAll = kPieces == 32 ? 0xffffffffu : 0xffffu;
    const bool is = mine.unit >= 0;
    const uint32_t live = __ballot_sync(0xffffffffu, is) & kAll, below = live & ((1u << j) - 1);
    const int unit_before = __shfl_sync(0xffffffffu, mine.unit, below ? 31 - __clz((int)below) : j, kPieces);
    const uint32_t leads = __ballot_sync(0xffffffffu, is && (below == 0 || unit_before != mine.unit)) & kAll;     // the units' first pieces
    {
        // the lanes of a unit follow one another: a scan over them, and the unit's last lane has the result
        const uint32_t later = leads & ~((2u << j) - 1), run = live & (later ? (1u << (__ffs((int)later) - 1)) - 1 : kAll);
        const int begin = 31 - __clz((int)(leads & ((2u << j) - 1))), end = run ? 31 - __clz((int)run) : 0;
        const int r = kAtOnce * warp + lane / kPieces; // (a head per warp, or two)
        static_assert(kAtOnce * kAttnWarps >= kR, "every head has its lanes");
        if (kAtOnce * warp < kR) {
            float m = kLowest, l = 0.f;
            if (is) {
                const float* p = (j & 1 ? last_piece(j >> 1) : first_piece(j >> 1)) + D * kR + r;
                m = p[0];
                l = p[kR];
            }
            float top = m;
#pragma unroll
            for (int d = 1; d < kPieces; d <<= 1) {
                const float o = __shfl_up_sync(0xffffffffu, top, d, kPieces);
                if (j - d >= begin) top = fmaxf(top, o);
            }
            top = __shfl_sync(0xffffffffu, top, end, kPieces);
            const float f = fast_exp2(m - top);
            float sum = f * l;
#pragma unroll
            for (int d = 1; d < kPieces; d <<= 1) {
                const float o = __shfl_up_sync(0xffffffffu, sum, d, kPieces);
                if (j - d >= begin) sum += o;
            }
            sum = __shfl_sync(0xffffffffu, sum, end, kPieces);
            s_f.factor[j][r] = f;
            if ((leads >> j) & 1u) {
                const bool closed = mine.begin >= cta_lo && mine.end <= cta_hi;
                s_f.m[j][r] = top;
                s_f.l[j][r] = closed ? inverse(sum) : sum;
                if (closed) put_lse(place_of(mine.unit), r, top, sum);
                else if (r == 0) s_open[2 * ((j >> 1) >> team_log2) + (mine.begin < cta_lo ? 0 : 1)] = j;
            }
        }
    }
    __syncthreads();
    // what goes on in other CTAs of the cluster waits in shared memory (behind the pieces of warps 1 and 2), what goes on in other
    // stretches in the workspace
    auto cluster_rec = [&](int w) { return reinterpret_cast<float*>(s_ring_all + (size_t)(w + 2) * G::kRingBytes) - kRec; };
    auto group_rec = [&](int g, int w) { return P.cta_rec + ((size_t)g * 2 * kAttnAbreast + w) * kRec; };        // (w = 2 member + 0 or 1)
    // threads over the units of the CTA, quads of heads, channels
    for (int e = tid; e < __popc(leads) * quads * D; e += kAttnThreads) {
        const int d = e % D, x = e / D, nth = quads == 1 ? x : quads == 2 ? x / 2 : quads == 3 ? x / 3 : x / 4, r = 4 * (x - nth * quads);
        uint32_t rest = leads;
        for (int k = 0; k < nth; ++k) rest &= rest - 1;
        const int i = __ffs((int)rest) - 1;            // the unit's first piece
        rest &= rest - 1;
        const uint32_t run = live & ~((1u << i) - 1) & (rest ? (1u << (__ffs((int)rest) - 1)) - 1 : kAll);
        // warps that end within the unit, and one at most that ends it and goes on
        const uint32_t lasts = run & 0xaaaaaaaau, firsts = run & 0x55555555u;
        float4 so = make_float4(0.f, 0.f, 0.f, 0.f);
        if (firsts) {
            const int k = __ffs((int)firsts) - 1;
            const float4 f = *reinterpret_cast<const float4*>(&s_f.factor[k][r]), y = *reinterpret_cast<const float4*>(first_piece(k >> 1) + d * kR + r);
            so = make_float4(f.x * y.x, f.y * y.y, f.z * y.z, f.w * y.w);
        }
        auto add = [&](int k) {
            const float4 f = *reinterpret_cast<const float4*>(&s_f.factor[2 * k + 1][r]), y = *reinterpret_cast<const float4*>(last_piece(k) + d * kR + r);
            so.x += f.x * y.x, so.y += f.y * y.y, so.z += f.z * y.z, so.w += f.w * y.w;
        };
        if (__popc(lasts) <= 2) {
            if (lasts) add((__ffs((int)lasts) - 1) >> 1);
            if (lasts & (lasts - 1)) add((31 - __clz((int)lasts)) >> 1);
        } else {
            const int some = (__ffs((int)lasts) - 1) >> 1;
#pragma unroll
            for (int w0 = 0; w0 < kAttnWarps; w0 += 8) {
                float4 y[8], f[8];
#pragma unroll
                for (int w = 0; w < 8; ++w) {          // (no branches: what is not there counts zero times)
                    const bool in = (lasts >> (2 * (w0 + w) + 1)) & 1u;
                    const int k = in ? w0 + w : some;
                    y[w] = *reinterpret_cast<const float4*>(last_piece(k) + d * kR + r);
                    f[w] = *reinterpret_cast<const float4*>(&s_f.factor[2 * k + 1][r]);
                    if (!in) f[w] = make_float4(0.f, 0.f, 0.f, 0.f), y[w] = f[w];
                }
#pragma unroll
                for (int w = 0; w < 8; ++w) so.x += f[w].x * y[w].x, so.y += f[w].y * y[w].y, so.z += f[w].z * y[w].z, so.w += f[w].w * y[w].w;
            }
        }
        if (s_piece[i].begin >= cta_lo && s_piece[i].end <= cta_hi) {
            put(place_of(s_piece[i].unit), r, d, so, &s_f.l[i][r]);
        } else {
            const int which = 2 * ((i >> 1) >> team_log2) + (s_piece[i].begin < cta_lo ? 0 : 1);
            float* rec = C > 1 ? cluster_rec(which) : group_rec(group, which);
            *reinterpret_cast<float4*>(rec + d * kR + r) = so;
            if (d < 2) *reinterpret_cast<float4*>(rec + (D + d) * kR + r) = *reinterpret_cast<const float4*>(d == 0 ? &s_f.m[i][r] : &s_f.l[i][r]);
        }
    }
    if (C > 1) {
        // ---- units that several CTAs of the cluster share: the first of them adds up, lanes and threads as above
        cg::cluster_group cluster = cg::this_cluster();
        cluster.sync();
#pragma unroll 1
        for (int w = 0; w < 2; ++w) {
            const int lead = s_open[w];
            if (lead < 0) continue;                    // (the same for all threads)
            const AttnPiece unit = s_piece[lead];
            const int64_t from = max(unit.begin, lo), to = min(unit.end, hi);
            if (from < cta_lo) {                       // another CTA's
                __syncthreads();
                if (tid == 0) s_open[w] = -1;
                continue;
            }
            const int part = rank + (lane & 15);       // of this lane
            const int64_t p0 = cta_border(min(part, C)), p1 = cta_border(min(part + 1, C));
            const bool in = part < C && p0 < to && p0 < p1;
            const uint32_t parts = __ballot_sync(0xffffffffu, in) & 0xffffu;
            auto record = [&](int r) -> const float* { return cluster.map_shared_rank(cluster_rec(r == rank ? w : 0), r); };
            const bool closed = unit.begin >= lo && unit.end <= hi;
            const Place at = place_of(unit.unit);
            for (int r = 2 * warp + (lane >> 4); r < kR; r += 2 * kAttnWarps) {
                const float* p = record(in ? part : rank) + D * kR + r;
                const float m = in ? p[0] : kLowest, l = in ? p[kR] : 0.f;
                float top = m;
#pragma unroll
                for (int d = 1; d < 16; d <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
                const float f = in ? fast_exp2(m - top) : 0.f;
                float sum = f * l;
#pragma unroll
                for (int d = 1; d < 16; d <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
                s_f.factor[lane & 15][r] = f;
                if ((lane & 15) == 0) {
                    s_f.m[0][r] = top, s_f.l[0][r] = closed ? inverse(sum) : sum;
                    if (closed) put_lse(at, r, top, sum);
                }
            }
            __syncthreads();
            for (int e = tid; e < quads * D; e += kAttnThreads) {
                const int d = e % D, r = 4 * (e / D);
                float4 so = make_float4(0.f, 0.f, 0.f, 0.f);
                for (int k0 = 0; (parts >> k0) != 0; k0 += 8) {    // eight on their way at a time
                    float4 y[8];
#pragma unroll
                    for (int k = 0; k < 8; ++k) y[k] = *reinterpret_cast<const float4*>(record((parts >> (k0 + k)) & 1u ? rank + k0 + k : rank) + d * kR + r);
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        if (!((parts >> (k0 + k)) & 1u)) continue;
                        const float4 f = *reinterpret_cast<const float4*>(&s_f.factor[k0 + k][r]);
                        so.x += f.x * y[k].x, so.y += f.y * y[k].y, so.z += f.z * y[k].z, so.w += f.w * y[k].w;
                    }
                }
                if (closed) {
                    put(at, r, d, so, &s_f.l[0][r]);
                } else {
                    float* rec = group_rec(group, w);
                    *reinterpret_cast<float4*>(rec + d * kR + r) = so;
                    if (d < 2) *reinterpret_cast<float4*>(rec + (D + d) * kR + r) = *reinterpret_cast<const float4*>(d == 0 ? &s_f.m[0][r] : &s_f.l[0][r]);
                }
            }
            __syncthreads();
            if (closed && tid == 0) s_open[w] = -1;
        }
        cluster.sync();                                // (nobody leaves, or uses its rings, while its records may be read)
    }
    // ---- units that several stretches share: the CTA with the last record joins them.  A border inside a unit is more than
    // snap tiles away from both its ends, so the stretches that share it follow from the equal shares alone.
    __syncthreads();                                   // (the records are written)
    const double shares_per_tile = (double)stretches / (double)total;
    auto share_of = [&](int64_t t) {                   // the last stretch whose share begins at or before tile t
        int c = min(stretches - 1, (int)((double)t * shares_per_tile));
        while (c + 1 < stretches && share(c + 1) <= t) ++c;
        while (share(c) > t) --c;
        return c;
    };
    if (tid < 2 * abreast && s_open[tid] >= 0) {
        const AttnPiece unit = s_piece[s_open[tid]];
        const int c0 = share_of(unit.begin + snap), c1 = share_of(unit.end - snap - 1);
        __threadfence();                               // (the whole CTA's records, which the barrier has ordered before)
        const bool last = atomicInc(&P.arrivals[c0 * kAttnAbreast + (tid >> 1)], (uint32_t)(c1 - c0)) == (uint32_t)(c1 - c0);
        __threadfence();
        s_first[tid] = c0;
        s_last[tid] = last ? c1 : -1;
    }
    __syncthreads();
    for (int e = tid; e < 2 * abreast * quads * D; e += kAttnThreads) {
        const int d = e % D, x = e / D, which = quads == 1 ? x : quads == 2 ? x / 2 : quads == 3 ? x / 3 : x / 4, r = 4 * (x - which * quads);
        const int lead = s_open[which];
        if (lead < 0 || s_last[which] < 0) continue;
        // one record after the other, in the order of the axis; only the first begins with the unit
        float m[4] = {kLowest, kLowest, kLowest, kLowest}, l[4] = {0.f, 0.f, 0.f, 0.f}, o[4] = {0.f, 0.f, 0.f, 0.f};
        const int c0 = s_first[which], c1 = s_last[which];
#pragma unroll 4
        for (int c = c0; c <= c1; ++c) {
            const float* rec = group_rec(c, (which & ~1) + (c == c0 ? 1 : 0));
            const float4 m4 = __ldcg(reinterpret_cast<const float4*>(rec + D * kR + r)), l4 = __ldcg(reinterpret_cast<const float4*>(rec + (D + 1) * kR + r));
            const float4 o4 = __ldcg(reinterpret_cast<const float4*>(rec + d * kR + r));
            const float mc[4] = {m4.x, m4.y, m4.z, m4.w}, lc[4] = {l4.x, l4.y, l4.z, l4.w}, oc[4] = {o4.x, o4.y, o4.z, o4.w};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float top = fmaxf(m[k], mc[k]), f0 = fast_exp2(m[k] - top), f1 = fast_exp2(mc[k] - top);
                l[k] = l[k] * f0 + lc[k] * f1;
                o[k] = o[k] * f0 + oc[k] * f1;
                m[k] = top;
            }
        }
        const Place at = place_of(s_piece[lead].unit);
        float inv[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            inv[k] = inverse(l[k]);
            if (d == 0) put_lse(at, r + k, m[k], l[k]);
        }
        put(at, r, d, make_float4(o[0], o[1], o[2], o[3]), inv);
    }
}

}  // namespace kvq
