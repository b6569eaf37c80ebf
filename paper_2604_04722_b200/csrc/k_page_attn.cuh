// Attention of one new token per sequence over a paged 16-bit cache:  o = sum_t w_t v_t / sum_t w_t,  w_t = 2^(c q.k_t - m),
// c the softmax scale in log2 units, m a running reference of the row.  One pass; m moves only when a logit passes it by
// kRescaleSlack, so that the sums are rescaled a few times per unit instead of at every tile.
//
// A UNIT is a (sequence, KV head, block of 8 NT query heads).  The tiles of 16 tokens of all units lie end to end on an axis that
// is cut into equal stretches, one per warp of the launch, whatever the lengths: a warp streams the rows of its stretch through
// a ring of shared-memory stages of its own (16-byte asynchronous copies; page numbers are looked up one tile ahead) and never
// waits for another warp.  The lengths are on the device, so every CTA adds them up for itself.
//
// Heads are the columns of the matrix instructions (m16n8k16): logits = K q^T with the 16 tokens of a tile as rows, and
// o^T = V^T w^T with the channels as rows, so that up to 8 query heads cost the same as one, K and V fragments are read with one
// ldmatrix per 16 x 16 block, and the weights of a tile become the second product's operand with one 8 x 8 transposition per
// eight tokens.  A weight enters as the sum of two 16-bit numbers (what the first loses the second holds): next to the rows'
// bytes the second product costs nothing, and with 8-bit mantissas (bf16) one rounding of the weights would be as large as the
// output's own.  Sums are fp32.
//
// A unit that ends inside a warp's stretch is written by that warp.  Pieces of a unit meet in their CTA, and what is left
// over at the borders of a CTA's stretch meets in records of the workspace: the CTA that delivers a unit's last record joins them,
// in the order of the axis whoever comes last.  Bound: the rows' bytes, 4 D per token and KV head.
#pragma once
#include <cuda_bf16.h>
#include "kvq_common.cuh"
#include "kvq_pages.h"
#include "kvq_ptx.cuh"

namespace kvq {

constexpr int kAttnTile = 16;                          // tokens
constexpr int kAttnWarps = 8, kAttnThreads = 32 * kAttnWarps;
constexpr int kAttnMaxCtas = 1024;                     // arrival counters of a workspace
constexpr int kAttnMinTiles = 1;                       // of a warp, where the work does not fill the launch
constexpr float kLowest = -3.402823466e38f;
constexpr float kLn2 = 0.69314718055994531f;

template <int D>
struct AttnGeom {
    static constexpr int kStages = 3;
    static constexpr int kRowBytes = 2 * D, kTensorBytes = kAttnTile * kRowBytes, kStageBytes = 2 * kTensorBytes;
    static constexpr int kRingBytes = kStages * kStageBytes;               // of a warp
};
template <int D, int NT>
__host__ __device__ constexpr int attn_record_floats() { return 8 * NT * (D + 2); }            // o [D][8 NT], m [8 NT], l [8 NT]

// Shared memory: the rings, and the rows' place on the axis.
template <int D>
inline size_t attn_smem(int batch) {
    return (size_t)kAttnWarps * AttnGeom<D>::kRingBytes + sizeof(int64_t) * ((size_t)batch + 1);
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
template <bool BF>
__device__ __forceinline__ uint16_t round16(float v) {
    return (uint16_t)(pack16<BF>(v, 0.f) & 0xffffu);
}

// A place on the axis: tile t of unit u (head and block) of row b.
struct AttnCursor {
    int b, u, t, tiles, len;
};

// grid: at most kAttnMaxCtas resident CTAs; those that the lengths leave without work return.
template <bool BF, int D, int NT>
__global__ void __launch_bounds__(kAttnThreads, D == 64 ? 2 : 1) k_page_attn(const PageAttnParams P) {
    using G = AttnGeom<D>;
    constexpr int kMt = D / 16, kR = 8 * NT, kStages = G::kStages;
    constexpr int kVecs = D / 8, kRowsAtOnce = 32 / kVecs, kCopies = kAttnTile / kRowsAtOnce;     // 16-byte vectors of a row
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, q = lane & 3;
    extern __shared__ __align__(128) uint8_t s_ring_all[];
    // [batch + 1]: 16 times the tiles before a row, plus the tokens that its last tile lacks
    int64_t* s_place = reinterpret_cast<int64_t*>(s_ring_all + (size_t)kAttnWarps * G::kRingBytes);
    auto tiles_before = [&](int b) -> int64_t { return s_place[b] >> 4; };
    auto tiles_of = [&](int b) -> int { return (int)(tiles_before(b + 1) - tiles_before(b)); };
    auto len_of = [&](int b) -> int { return tiles_of(b) * kAttnTile - (int)(s_place[b] & 15); };
    __shared__ int64_t s_scan[kAttnWarps];
    __shared__ uint32_t s_there[kAttnWarps][kStages];  // tokens of a stage that exist
    __shared__ int s_unit[2 * kAttnWarps];             // unit of a warp's first and last piece, -1: none
    __shared__ uint32_t s_last;

    pdl_launch_dependents();
    pdl_wait();

    // ---- lengths, and tiles before every row
    const int units_per_row = P.kv_heads * P.head_blocks;
    {
        const int per = (P.batch + kAttnThreads - 1) / kAttnThreads;
        const long long room = (long long)P.width * P.page_size;
        auto read_len = [&](int b) { return (int)min((long long)max(P.lens[b], 0), room); };
        auto tiles = [&](int n) { return (n + (long long)kAttnTile - 1) / kAttnTile; };
        int64_t sum = 0;
        for (int k = 0; k < per; ++k) {
            const int b = tid * per + k;
            if (b >= P.batch) break;
            const int n = read_len(b);
            s_place[b] = n;                            // for now
            sum += tiles(n);
        }
        int64_t upto = sum;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int64_t o = __shfl_up_sync(0xffffffffu, upto, d);
            if (lane >= d) upto += o;
        }
        if (lane == 31) s_scan[warp] = upto;
        if (tid < 2 * kAttnWarps) s_unit[tid] = -1;
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
    // rows without a token
    for (int b = blockIdx.x; b < P.batch; b += gridDim.x) {
        if (tiles_of(b) != 0) continue;
        for (int e = tid; e < P.q_heads * D; e += kAttnThreads) O[(size_t)b * P.q_heads * D + e] = 0;
        if (P.lse)
            for (int h = tid; h < P.q_heads; h += kAttnThreads) P.lse[(size_t)b * P.q_heads + h] = -INFINITY;
    }
    const int64_t total = tiles_before(P.batch) * units_per_row;
    const int ctas = (int)min((int64_t)gridDim.x, (total + kAttnWarps * kAttnMinTiles - 1) / (kAttnWarps * kAttnMinTiles));
    if ((int)blockIdx.x >= ctas) return;
    auto cta_begin = [&](int c) -> int64_t { return total * c / ctas; };
    const int64_t lo = cta_begin(blockIdx.x), hi = cta_begin(blockIdx.x + 1);
    const int64_t wlo = lo + (hi - lo) * warp / kAttnWarps, whi = lo + (hi - lo) * (warp + 1) / kAttnWarps;

    auto locate = [&](int64_t at) -> AttnCursor {
        int b0 = 0, b1 = P.batch;
        while (b1 - b0 > 1) {
            const int mid = (b0 + b1) >> 1;
            if (tiles_before(mid) * units_per_row <= at) b0 = mid;
            else b1 = mid;
        }
        AttnCursor c;
        c.b = b0;
        c.tiles = tiles_of(b0);
        c.len = len_of(b0);
        const int64_t rest = at - tiles_before(b0) * units_per_row;
        c.u = (int)(rest / c.tiles);
        c.t = (int)(rest - (int64_t)c.u * c.tiles);
        return c;
    };
    auto next_unit = [&](AttnCursor& c) {
        c.t = 0;
        if (++c.u < units_per_row) return;
        c.u = 0;
        do ++c.b; while (c.b < P.batch && tiles_of(c.b) == 0);
        if (c.b >= P.batch) return;                    // (behind the last tile)
        c.tiles = tiles_of(c.b);
        c.len = len_of(c.b);
    };
    auto unit_id = [&](const AttnCursor& c) { return c.b * units_per_row + c.u; };
    auto unit_begin = [&](int unit) -> int64_t {       // first tile of a unit
        const int b = unit / units_per_row;
        return tiles_before(b) * units_per_row + (int64_t)(unit - b * units_per_row) * tiles_of(b);
    };
    auto unit_end = [&](int unit) -> int64_t {
        return unit_begin(unit) + tiles_of(unit / units_per_row);
    };

    uint8_t* const ring = s_ring_all + (size_t)warp * G::kRingBytes;
    const uint32_t ring_addr = smem_addr(ring);
    const int count = (int)(whi - wlo);
    if (count > 0) {
        // ---- copies: `ahead` is the tile whose page numbers are being looked up
        AttnCursor ahead = locate(wlo);
        int looked = 0;                                // tiles looked up so far
        int page = -1, slot = 0, head = 0;
        auto look_up = [&]() {
            page = -1;
            if (looked >= count) return;
            const int pos = ahead.t * kAttnTile + (lane & 15);
            head = ahead.u / P.head_blocks;
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
            const int h0 = at.u / P.head_blocks, hb = at.u - h0 * P.head_blocks;
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
            const int h0 = at.u / P.head_blocks, hb = at.u - h0 * P.head_blocks;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const float i0 = l[nt][0] > 0.f || l[nt][0] != l[nt][0] ? 1.f / l[nt][0] : 0.f;
                const float i1 = l[nt][1] > 0.f || l[nt][1] != l[nt][1] ? 1.f / l[nt][1] : 0.f;
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
                over |= fmaxf(s[nt][0], s[nt][2]) > m[nt][0] + kRescaleSlack || fmaxf(s[nt][1], s[nt][3]) > m[nt][1] + kRescaleSlack;
            }
            if (__any_sync(0xffffffffu, over)) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        float top = fmaxf(s[nt][c], s[nt][c + 2]);
#pragma unroll
                        for (int d = 4; d < 32; d <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
                        top = fmaxf(top, m[nt][c]);
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
                    wl[nt][h] = transpose8x8(pack16<BF>(s[nt][2 * h] - back.x, s[nt][2 * h + 1] - back.y));
                }
            }
            {
                const int r = (lane & 7) + ((lane >> 4) << 3);
#pragma unroll
                for (int k = 0; k < kMt; ++k) {
                    uint32_t a[4];
                    ldmatrix4_trans(a, base + G::kTensorBytes + r * G::kRowBytes + (((2 * k + ((lane >> 3) & 1)) ^ (r & 7)) << 4));
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        mma16<BF>(o[k][nt], a, wh[nt][0], wh[nt][1]);
                        mma16<BF>(o[k][nt], a, wl[nt][0], wl[nt][1]);
                    }
                }
            }
            if (++at.t == at.tiles || i + 1 == count) {
                sum_lanes();
                const bool ends = at.t == at.tiles;
                if (ends && whole) {
                    write_unit();
                } else if (i + 1 < count) {            // the rest of a unit that an earlier warp began
                    deliver_piece(P.warp_rec + ((size_t)blockIdx.x * kAttnWarps + warp) * attn_record_floats<D, NT>());
                    if (lane == 0) s_unit[2 * warp] = unit_id(at);
                } else {
                    cp_async_wait<0>();
                    __syncwarp();
                    deliver_piece(reinterpret_cast<float*>(ring));
                    if (lane == 0) s_unit[2 * warp + 1] = unit_id(at);
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

    // ---- pieces of the CTA's units meet
    constexpr int kRec = attn_record_floats<D, NT>();
    auto piece = [&](int i) -> const float* {
        return i & 1 ? reinterpret_cast<const float*>(s_ring_all + (size_t)(i >> 1) * G::kRingBytes)
                     : P.warp_rec + ((size_t)blockIdx.x * kAttnWarps + (i >> 1)) * kRec;
    };
    auto put = [&](int unit, int r, int d, float m, float l, float o) {        // of head r of the block, channel d
        const int b = unit / units_per_row, u = unit - b * units_per_row, h0 = u / P.head_blocks;
        const int hr = (u - h0 * P.head_blocks) * kR + r;
        if (hr >= P.group) return;
        const size_t row = (size_t)b * P.q_heads + h0 * P.group + hr;
        O[row * D + d] = round16<BF>(l > 0.f || l != l ? o / l : 0.f);
        if (d == 0 && P.lse) P.lse[row] = l == 0.f ? -INFINITY : m * kLn2 + logf(l);
    };
    int open[2] = {-1, -1};                            // units that go on in other CTAs: one from before, one beyond
    for (int i = 0; i < 2 * kAttnWarps;) {
        const int unit = s_unit[i];
        if (unit < 0) {
            ++i;
            continue;
        }
        int end = i + 1;
        while (end < 2 * kAttnWarps && (s_unit[end] == unit || s_unit[end] < 0)) ++end;
        const int64_t u0 = unit_begin(unit), u1 = unit_end(unit);
        const bool closed = u0 >= lo && u1 <= hi;
        const int which = u0 < lo ? 0 : 1;
        if (!closed) open[which] = unit;
        float* rec = P.cta_rec + ((size_t)blockIdx.x * 2 + which) * kRec;
        for (int e = tid; e < kR * D; e += kAttnThreads) {
            const int r = e % kR, d = e / kR;
            float top = kLowest;
            for (int k = i; k < end; ++k)
                if (s_unit[k] == unit) top = fmaxf(top, piece(k)[D * kR + r]);
            float so = 0.f, sl = 0.f;
            for (int k = i; k < end; ++k)
                if (s_unit[k] == unit) {
                    const float* p = piece(k);
                    const float f = fast_exp2(p[D * kR + r] - top);
                    so += f * p[d * kR + r];
                    sl += f * p[(D + 1) * kR + r];
                }
            if (closed) {
                put(unit, r, d, top, sl, so);
            } else {
                rec[d * kR + r] = so;
                if (d == 0) rec[D * kR + r] = top, rec[(D + 1) * kR + r] = sl;
            }
        }
        i = end;
    }
    // ---- units that several CTAs share: the CTA with the last record joins them
#pragma unroll 1
    for (int which = 0; which < 2; ++which) {
        const int unit = open[which];
        if (unit < 0) continue;                        // (the same for all threads)
        const int64_t u0 = unit_begin(unit), u1 = unit_end(unit);
        auto cta_of = [&](int64_t t) {                 // the CTA whose stretch holds tile t
            int c = (int)(t * ctas / total);
            while (cta_begin(c + 1) <= t) ++c;
            while (cta_begin(c) > t) --c;
            return c;
        };
        const int c0 = cta_of(u0), c1 = cta_of(u1 - 1);
        __threadfence();
        __syncthreads();
        if (tid == 0) s_last = atomicInc(&P.arrivals[c0], (uint32_t)(c1 - c0)) == (uint32_t)(c1 - c0);
        __syncthreads();
        if (!s_last) continue;
        __threadfence();
        auto record = [&](int c) { return P.cta_rec + ((size_t)c * 2 + (cta_begin(c) <= u0 ? 1 : 0)) * kRec; };
        for (int e = tid; e < kR * D; e += kAttnThreads) {
            const int r = e % kR, d = e / kR;
            float top = kLowest, so = 0.f, sl = 0.f;
            for (int c = c0; c <= c1; ++c) top = fmaxf(top, __ldcg(record(c) + D * kR + r));
#pragma unroll 4
            for (int c = c0; c <= c1; ++c) {
                const float* p = record(c);
                const float f = fast_exp2(__ldcg(p + D * kR + r) - top);
                so += f * __ldcg(p + d * kR + r);
                sl += f * __ldcg(p + (D + 1) * kR + r);
            }
            put(unit, r, d, top, sl, so);
        }
    }
}

}  // namespace kvq
