// Attention of several query rows per sequence over the mixed-precision cache (Eq. 5), for speculative decoding and
// for sliding-window layers:
//   kvq_attend_tree         every row belongs to a node of a tree of drafted tokens; it sees the cached tokens (those
//                           of its window and the sinks) and its own ancestors, which are not in the cache
//   kvq_decode_attn_window  one row per query head, which sees the last `window` cached tokens and the sinks
//
// The decode kernel (k_decode.cuh) gives every (sequence, query head) its own walk over the cache, which is right for
// one row.  Here the rows of a tree and the heads of a group share a walk: a unit is (sequence, KV head, block of up
// to 8, 16 or 32 rows), row = node * group + head, and both products run on the fp16 matrix instructions with the rows as
// the 8 columns (mma.sync m16n8k16, fp32 accumulation):
//   S[slot][row] = sum_i c_i q_i            16 rows = the slots of a tile
//   O[channel][row] += sum_slot c w         16 rows = channels, four products for the 64 of a head
// with the packed codes as the 16-row operand of both.  The fragment layout of the store (kvq_common.cuh) has, in lane
// (g, q), the codes of slots g and g + 8, and for V of slots 4q .. 4q + 3: the operand needs exactly those bytes, two
// 16-bit lanes per register.  The weights of a tile leave the softmax with slots as rows and enter the second product
// with slots as columns: one 8x8 transposition (movmatrix) per eight slots.  Eight columns instead of sixteen rows
// keep a decode step of three grouped heads at half the matrix instructions, and the scales belong to slots g and
// g + 8 of a lane alone.
//
// Unpacking K costs one AND per two codes: a field cut out in place at bit k <= 8 of a 16-bit lane IS the fp16 number
// code * 2^(k-24) (a subnormal: that encoding is linear), and the matrix instruction takes subnormals exactly.  The
// power 2^-k is undone on the query's side.  The query is scaled by powers of two only, F (one for the rows of a unit, which
// puts their largest value below 2^15) and down to 2^-6 for k.  That is exact while the rows' largest value is below 512;
// above, values of less than about 2^-22 of it become subnormal, and lose at most 2^-33 of it.  So a logit
//   y = log2(e)/8 * (s_k * sum_i q_i c_i + z_k * sum_i q_i)
// carries, as a rule, only the error of the matrix instruction's sum of 64 products, which it truncates (see below; its tests
// allow 2^-22 per addition of the absolute sum).  V codes are cut out the same way, but as prefixes of their byte (c0, c0 + 4 c1,
// ...), which the accumulators undo when the pool is left.  The weight w = p * s_v is rounded once to fp16 (by at most 2^-11
// of its value: the rounding that the fp16 operand forces).  What that does is made to act on centred codes:
//   sum p (s c + z) = sum w (c - mid) + sum p (z + mid s),   mid = -z / s, inside [0, 2^bits - 1], per token
// with the same rounded w in both terms of (c - mid).  mid is the code of the value zero, so the rounding of w acts on
// the value and not on its distance from the row's minimum, which is far larger for the ordinary channels of a row with
// one large one (values have such).  The sums of p, of p (z + mid s) and of mid w stay in fp32.  With the middle of the codes
// in the place of mid the kernel is 7 % faster and off by 3.0e-4 to 3.5e-4 instead of 2.4e-4 to 2.6e-4 (relative, whole tensors
// of outputs over 2000 to 8000 tokens; the rounding of exact outputs to fp16 is 2.1e-4 of that).
//
// The matrix instruction truncates its sums, towards zero and below the largest possible product of its operands, which for
// subnormal codes is far above the real ones.  Sums of codes 0 .. 2^bits - 1 all lose in the same direction, and next to outputs
// that average out over many tokens that is no small loss: 8000 tokens of 2 bits were off by 6.5e-4 (relative, whole tensors),
// 60000 mixed ones in one CTA by 1.1e-3.  So the codes enter as c - (2^bits - 1) / 2 (rounded down for even slots and up for odd
// ones, which mid takes back): 3.0e-4 at any length.  What is left is about 2^-14 of a token's scale times its weight, which
// shows where one token has nearly all the weight and next to nothing in a channel (a row of 2 bits with values up to 14:
// 0.0356 for 0.0363); in the norm of a row it is far below the rounding of the weights.  The 16
// subtractions per tile take 0 to 5 % of the time (32768 tokens, 16 rows: 399 us against 379 us).
//
// Softmax reference.  p = 2^(y - m), m kept per row and warp.  m is no running maximum: it is moved only when some w
// overflows fp16 (one vote per tile decides), and then to where the row's largest w of the tile is 2^4.  So logits may
// grow by 2^11 or so before anything is rescaled -- with sixteen rows, a reference that followed every new maximum was
// moved on a fifth of all tiles -- and w keeps all its bits down to 2^-18 of the row's largest.
//
// Work split: the units lie end to end on an axis, every unit `ticks` long; a CTA takes `span` ticks of it, in pieces where it
// crosses unit borders.  With as many CTAs as stay resident and equal stretches all SMs finish together, whatever the
// number of units; many units are taken whole.  The tiles of a unit (of its four pools laid end to end, a tile weighted
// by its cost) are cut like the axis, a piece's into four equal shares, one per warp.  A warp streams its share through
// its own ring of bulk copies, as in the decode kernel; the four warps are merged in shared memory.  Up to sixteen CTAs
// of a unit that are resident together are a cluster: each sends its rows to the CTAs that merge them, which is one barrier
// of the cluster (2048 tokens, one sequence: 9.7 us against 14.2 us through global memory).  Other pieces of a unit
// go through global records and are merged by the CTA that arrives last, so that nothing there waits for another CTA.
//
// Window.  Slots of a pool are handed out in position order, so a window is a suffix and the sinks a prefix of every
// pool.  Where they start follows from the per-token index: the first token of class c at or after position p names
// the slot.  One warp per class looks for it, 128 index words per step and round trip, in one or two steps where the
// widths are mixed.  A class that does not occur from p on is looked for up to the end of the sequence: with 16 bits for
// four sinks and 2 to 8 bits behind them a window of 256 takes 9.9 us of 2048 tokens and 68 us of 32768 (6.6 us with
// mixed widths), one of 8192 on 16 sequences x 32 heads 214 us (86 us).  Rows of different depth have different window
// starts; they are told apart only inside the tiles at the edge.
//
// Drafted rows (the tree) are quantized at their bit-width and put back together, rounded to fp16, by the CTA of the
// last piece, as fp16 tiles in shared memory that the fp16 consumer reads under a mask of ancestors.
#pragma once
#include "kvq_common.cuh"
#include "kvq_ptx.cuh"
#include "kvq_rows.h"

namespace kvq {

constexpr int kRowsWarps = 4, kRowsThreads = kRowsWarps * 32;
constexpr int kRowsStages = 2;
constexpr int kRowsStageBytes = 4608;
constexpr int kRowsOutStride = kHeadDim + 4;           // floats per row of the merge buffer
constexpr int kRowsQStride = kHeadDim + 8;             // halves per row of the query block
// Tiles of class c that a chunk holds at most.
__host__ __device__ constexpr int kRowsTps(int c) { return c == 0 ? 6 : c == 1 ? 4 : c == 2 ? 2 : 1; }
static_assert(6 * pool_rec_bytes(0) <= kRowsStageBytes && 4 * pool_rec_bytes(1) <= kRowsStageBytes &&
              2 * pool_rec_bytes(2) <= kRowsStageBytes && pool_rec_bytes(3) <= kRowsStageBytes, "a chunk fits a stage");
constexpr int kDraftTileBytes = 4096;                  // one fp16 tile: K units, then V units
// What a tile of each class costs a warp, for cutting a unit into equal shares.
__device__ constexpr float kRowsTileCost[kNumPools] = {6.f, 7.f, 9.f, 15.f};
constexpr int kWeightTop = 4;                          // log2 of a row's largest weight when its reference is set

// Resident CTAs per SM that the kernel is compiled for (its registers allow; trees of more than 16 nodes take so much shared
// memory that 16 rows per unit keep three).
__host__ __device__ constexpr int rows_ctas_per_sm(int nt) { return nt == 4 ? 2 : 4; }
// NT: blocks of 8 rows per unit.
template <int NT>
__host__ __device__ constexpr size_t rows_smem_bytes(int draft_tiles, uint32_t cluster) {
    return (size_t)kRowsWarps * kRowsStages * kRowsStageBytes + (size_t)kNumPools * NT * 2 * 32 * 16 +
           (size_t)draft_tiles * kDraftTileBytes +
           (cluster > 1 ? (size_t)((8 * NT + cluster - 1) / cluster) * cluster * kRowsOutStride * sizeof(float) : 0);
}
// An upper bound over all clusters.
template <int NT>
__host__ __device__ constexpr size_t rows_smem_limit(int draft_tiles) {
    return rows_smem_bytes<NT>(draft_tiles, 1) + (8 * NT + kRowsMaxCluster - 1) * kRowsOutStride * sizeof(float);
}
static_assert(kRowsWarps * kRowsMaxRows * kRowsOutStride * 4 <= kRowsWarps * kRowsStages * kRowsStageBytes,
              "the merge buffer lives in the rings");

// ---------------------------------------------------------------- small pieces

__device__ __forceinline__ void mma_f16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// d = a b
__device__ __forceinline__ void mma_f16_first(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
}
// 8x8 matrix of 16-bit elements, lane (g, q) holding row g, columns 2q and 2q + 1: its transpose.
__device__ __forceinline__ uint32_t transpose8(uint32_t v) {
    uint32_t d;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(v));
    return d;
}
__device__ __forceinline__ uint32_t prmt(uint32_t a, uint32_t b, uint32_t sel) {
    uint32_t d;
    asm("prmt.b32 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(sel));
    return d;
}
__device__ __forceinline__ void ldsm_x4(uint32_t (&r)[4], const void* p) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
                 : "r"(smem_addr(p))
                 : "memory");
}
// Two fp32 operations as one packed instruction.
__device__ __forceinline__ float2 fma2v(float2 a, float2 b, float2 c) {
    float2 d;
    asm("{ .reg .b64 a, b, c;\n mov.b64 a, {%2, %3};\n mov.b64 b, {%4, %5};\n mov.b64 c, {%6, %7};\n"
        " fma.rn.f32x2 c, a, b, c;\n mov.b64 {%0, %1}, c; }"
        : "=f"(d.x), "=f"(d.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return d;
}
__device__ __forceinline__ float2 mul2v(float2 a, float2 b) {
    float2 d;
    asm("{ .reg .b64 a, b;\n mov.b64 a, {%2, %3};\n mov.b64 b, {%4, %5};\n mul.rn.f32x2 a, a, b;\n mov.b64 {%0, %1}, a; }"
        : "=f"(d.x), "=f"(d.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}
__device__ __forceinline__ float2 add2v(float2 a, float2 b) {
    float2 d;
    asm("{ .reg .b64 a, b;\n mov.b64 a, {%2, %3};\n mov.b64 b, {%4, %5};\n add.rn.f32x2 a, a, b;\n mov.b64 {%0, %1}, a; }"
        : "=f"(d.x), "=f"(d.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}
__device__ __forceinline__ uint32_t pack_half2(float2 v) {
    const __half2 h = __floats2half2_rn(v.x, v.y);
    return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ float2 unpack_half2(uint32_t v) { return __half22float2(*reinterpret_cast<const __half2*>(&v)); }
__device__ __forceinline__ uint32_t max_half2(uint32_t a, uint32_t b) {
    const __half2 m = __hmax2(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b));
    return *reinterpret_cast<const uint32_t*>(&m);
}
__device__ __forceinline__ uint32_t sub_half2(uint32_t a, uint32_t b) {
    const __half2 d = __hsub2(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b));
    return *reinterpret_cast<const uint32_t*>(&d);
}
__device__ __forceinline__ float fast_rcp(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// Stores to the shared memory of CTA `rank` of the cluster, at the address that `at` is in this CTA's.
__device__ __forceinline__ void st_cluster(uint32_t at, uint32_t rank, float4 v) {
    asm volatile("{ .reg .b32 a;\n mapa.shared::cluster.u32 a, %0, %1;\n st.shared::cluster.v4.f32 [a], {%2, %3, %4, %5}; }" ::"r"(at), "r"(rank),
                 "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w)
                 : "memory");
}
// The two halves of a barrier of the cluster.
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ float two_to(int e) { return __int_as_float((127 + e) << 23); }

// The slot of the first token of class c at a position >= p of a sequence of len tokens (n_c if there is none), for the
// whole warp; n_c tokens of that class.
__device__ __forceinline__ uint32_t first_slot_from(const uint32_t* idx, int p, int len, uint32_t c, uint32_t n_c, int lane) {
    if (p <= 0 || n_c == 0) return 0u;
    for (int base = p; base < len; base += 128) {
        uint32_t w[4], hit[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int at = base + 32 * k + lane;
            w[k] = at < len ? idx[at] : ~(c << 30);
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) hit[k] = __ballot_sync(0xffffffffu, (w[k] >> 30) == c);
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (hit[k]) return min(__shfl_sync(0xffffffffu, w[k], __ffs(hit[k]) - 1) & 0x3fffffffu, n_c);
    }
    return n_c;
}

// Chunks of a warp's share are planned 32 at most at a time, a lane each.
struct RowsChunks {
    uint4 chunk[32];               // x, y: source address; z: first tile, class in the top bits; w: bytes | tiles << 16 | mask of edge tiles << 20
    int seg, tile;                 // range of the share and tile that the next plan starts with
};

template <int NT>
struct RowsScratch {
    static constexpr int ROWS = 8 * NT;
    uint64_t bars[kRowsWarps][kRowsStages];
    unsigned long long anc[kMaxTreeNodes];             // a node and its ancestors
    unsigned long long vis[kMaxTreeNodes];             // those of them that it sees (0: the node is not used)
    unsigned long long step_bits[kNumPools];           // class c among the 64 positions after the first window start
    unsigned long long used;                           // nodes that are used
    unsigned long long poison;                         // drafted values that are not finite
    unsigned long long odd_bits;                       // nodes with a bit-width outside {2,4,8,16}
    alignas(16) RowsChunks plan[kRowsWarps];
    uint2 chunk[kRowsWarps][kRowsStages];              // what a stage holds: z, and w >> 16, of its chunk
    int in_sinks[kNumPools], from[kNumPools], full[kNumPools];     // tiles that every row sees whole: [0, in_sinks), [from, full)
    int seg_lo[kRowsWarps][2 * kNumPools], seg_hi[kRowsWarps][2 * kNumPools];   // tile ranges of a warp's share
    uint32_t cnt[kNumPools], sink[kNumPools], start[kNumPools];   // pool fills; slots before the sinks' end; first window slot
    uint32_t lo_row[kNumPools][ROWS];               // first window slot of every row
    float2 ml[kRowsWarps][ROWS];
    float sumq[ROWS];                               // log2(e)/8 * sum_i q_i
    float wmax[kRowsWarps], load[kRowsWarps];
    int16_t node[ROWS];                             // node of a row, -1 behind the last
    int8_t link[kMaxTreeNodes], bad[kMaxTreeNodes];
    uint32_t last;
    int draft_tile[kRowsWarps];
    alignas(16) __half q[ROWS][kRowsQStride];
};

// Softmax state of a warp: per lane rows 2q and 2q + 1 (the two halves of a pair) of every block of eight.
template <int NT>
struct RowsState {
    float2 negm[NT];               // minus the reference m of the row, log2 units
    float2 sumq[NT];               // log2(e)/8 * sum_i q_i
    float2 l[NT], b[NT];           // sum of p, sum of p * (centred zero-point), over the lane's slots
    float acc[NT][4][4];           // output: [j][0, 1] channel 4 g + j, [j][2, 3] channel 32 + 4 g + j, of the two rows
};

// What the K side of a tile leaves for the softmax: products of slots g (s = 0) and g + 8 (s = 1) with rows 2q and 2q + 1 in
// D[nt][2 s], [2 s + 1], and what the two slots carry.
template <int NT>
struct TileLogits {
    float D[NT][4];
    float sk[2], zk[2];            // scale (times the common factor of the K product) and zero-point of K
    float sv[2], zv[2];            // scale and centred zero-point of V
    float mid[2];                  // the code that V is centred on
};

__device__ __forceinline__ float2 both(float v) { return make_float2(v, v); }

// Logits of a tile, relative to the references or as they are.
template <int NT>
__device__ __forceinline__ void logits_of(const RowsState<NT>& st, const TileLogits<NT>& t, bool relative, float2 (&y)[NT][2]) {
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int s = 0; s < 2; ++s)
            y[n][s] = fma2v(make_float2(t.D[n][2 * s], t.D[n][2 * s + 1]), both(t.sk[s]),
                            fma2v(both(t.zk[s]), st.sumq[n], relative ? st.negm[n] : both(0.f)));
}
// From relative logits y to p = 2^y and the fp16 weights; returns their maxima.  (Every scale is at least 2^-24, see k_side, so
// that p itself stays far from the end of fp32.)
template <int NT>
__device__ __forceinline__ uint32_t weigh(const TileLogits<NT>& t, float2 (&y)[NT][2], uint32_t (&w)[NT][2]) {
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            y[n][s] = make_float2(fast_exp2(y[n][s].x), fast_exp2(y[n][s].y));
            w[n][s] = pack_half2(mul2v(y[n][s], both(t.sv[s])));
        }
    uint32_t big = max_half2(w[0][0], w[0][1]);
#pragma unroll
    for (int n = 1; n < NT; ++n) big = max_half2(big, max_half2(w[n][0], w[n][1]));
    return big;
}
// Weights are not negative; a bit pattern of 0x7c00 or above is an overflow.  One vote of the warp.
__device__ __forceinline__ bool overflows(uint32_t big) { return __any_sync(0xffffffffu, (big + 0x04000400u) & 0x80008000u); }
// The tile's part of the sums of p and p (z + mid s) - w mid; w becomes the column operand of the V product.
template <int NT>
__device__ __forceinline__ void add_tile(RowsState<NT>& st, const TileLogits<NT>& t, const float2 (&p)[NT][2], uint32_t (&w)[NT][2]) {
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            st.l[n] = add2v(st.l[n], p[n][s]);
            st.b[n] = fma2v(unpack_half2(w[n][s]), both(-t.mid[s]), fma2v(p[n][s], both(t.zv[s]), st.b[n]));
            w[n][s] = transpose8(w[n][s]);             // (slot g: rows 2q, 2q + 1) -> (row g: slots 2q, 2q + 1)
        }
}
// Where `edge` holds, bit (2 s + x) of seen[nt] says whether row 2q + x sees slot g + 8 s.
template <int NT>
__device__ __forceinline__ void hide(bool edge, const uint32_t (&seen)[NT], float2 (&y)[NT][2]) {
    if (!edge) return;
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            if (!((seen[n] >> (2 * s)) & 1u)) y[n][s].x = -INFINITY;
            if (!((seen[n] >> (2 * s)) & 2u)) y[n][s].y = -INFINITY;
        }
}
// Moves the references of the rows that this tile makes overflow (or nearly: those whose largest weight is above 2^kWeightTop).
template <int NT>
__device__ __forceinline__ void move_references(RowsState<NT>& st, const TileLogits<NT>& t, bool edge, const uint32_t (&seen)[NT]) {
    float2 y[NT][2];
    logits_of(st, t, false, y);
    hide(edge, seen, y);
    const float lg[2] = {__log2f(t.sv[0]), __log2f(t.sv[1])};
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        float2 m = make_float2(fmaxf(y[n][0].x + lg[0], y[n][1].x + lg[1]), fmaxf(y[n][0].y + lg[0], y[n][1].y + lg[1]));
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) {
            m.x = fmaxf(m.x, __shfl_xor_sync(0xffffffffu, m.x, d));
            m.y = fmaxf(m.y, __shfl_xor_sync(0xffffffffu, m.y, d));
        }
        // (a row that sees nothing here has m = -inf and keeps its reference)
        m = make_float2(fmaxf(-st.negm[n].x, m.x - kWeightTop), fmaxf(-st.negm[n].y, m.y - kWeightTop));
        const float2 f = make_float2(fast_exp2(-st.negm[n].x - m.x), fast_exp2(-st.negm[n].y - m.y));
        st.negm[n] = make_float2(-m.x, -m.y);
        st.l[n] = mul2v(st.l[n], f);
        st.b[n] = mul2v(st.b[n], f);
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) st.acc[n][j][e] *= (e & 1) ? f.y : f.x;
    }
}

// ---------------------------------------------------------------- tile consumers (lane = 4 g + q)

// The query as the column operand of step s: qf[nt][s >> 1], words 2 (s & 1) and + 1.
template <int NT>
using RowsQuery = uint4[NT][2];
__device__ __forceinline__ uint32_t query_word(const uint4& v, int k) { return k == 0 ? v.x : k == 1 ? v.y : k == 2 ? v.z : v.w; }

// A quantized class.  kw, va, vb: words of the fragment layout (see kvq_common.cuh).
template <int CLS>
struct RowsQuant {
    static constexpr int BITS = pool_bits(CLS);
    // The middle of the codes for even slots (low half) and odd ones: (2^BITS - 1) / 2 on average.
    static constexpr uint32_t kMiddle = ((1u << (BITS - 1)) - 1u) | ((1u << (BITS - 1)) << 16);
    static constexpr int NW = 2 << CLS;                // words per lane of one tensor: 2, 4, 8
    static constexpr uint32_t MASK = CLS == 0 ? 0x00030003u : CLS == 1 ? 0x000f000fu : 0x00ff00ffu;

    // Register r of step s of the K product holds, in 16-bit lane x, the code of channel
    //   2-bit: 16 q + 2 s + r + 8 x;   4-bit: 8 (q + 4 (s >> 1)) + 2 (s & 1) + r + 4 x;   8-bit: 4 (q + 4 s) + r + 2 x
    // cut out at bit 2 ((2 s + r) & 3), 4 r, 0 (the query's operand is laid out alike, see "column operands" below).
    // The codes of slot g + 8 i for step s, register r.
    __device__ static __forceinline__ uint32_t k_operand(const uint32_t (&kw)[NW], int i, int s, int r) {
        if (CLS == 0) {
            const int e = 2 * s + r;
            return (e < 4 ? kw[i] : kw[i] >> 8) & (MASK << (2 * (e & 3)));
        }
        if (CLS == 1) {
            const uint32_t w = kw[(s >> 1) * 2 + i];
            return ((s & 1) ? w >> 8 : w) & (MASK << (4 * r));
        }
        return prmt(kw[s * 2 + i], 0u, r ? 0x4341u : 0x4240u);
    }
    __device__ static __forceinline__ void load_words(const uint8_t* codes, int lane, uint32_t (&w)[NW]) {
        if (CLS == 0) {
            const uint2 v = *reinterpret_cast<const uint2*>(codes + lane * 8);
            w[0] = v.x; w[1] = v.y;
        } else {
#pragma unroll
            for (int u = 0; u < NW / 4; ++u) {
                const uint4 v = *reinterpret_cast<const uint4*>(codes + (u * 32 + lane) * 16);
                w[4 * u] = v.x; w[4 * u + 1] = v.y; w[4 * u + 2] = v.z; w[4 * u + 3] = v.w;
            }
        }
    }

    template <int NT>
    __device__ static __forceinline__ void k_side(const uint8_t* rec, int lane, const RowsQuery<NT>& qf, float kfactor, TileLogits<NT>& t) {
        const int g = lane >> 2;
        uint32_t kw[NW];
        load_words(rec, lane, kw);
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const float2 km = unpack_half2(*reinterpret_cast<const uint32_t*>(rec + meta_offset(CLS, 0, g + 8 * s)));
            const float2 vm = unpack_half2(*reinterpret_cast<const uint32_t*>(rec + meta_offset(CLS, 1, g + 8 * s)));
            t.sk[s] = km.x * (kfactor * 16777216.0f);
            t.zk[s] = km.y;
            // A constant row has scale zero and codes zero.  It is read with a scale of 2^-24, the smallest there is, which
            // its codes multiply by zero all the same: s (c - mid) + (z + mid s) = z.
            t.sv[s] = fmaxf(vm.x, 5.9604645e-8f);
            t.mid[s] = fminf(fmaxf(-vm.y * fast_rcp(t.sv[s]), 0.f), (float)((1 << BITS) - 1));
            t.zv[s] = fmaf(t.sv[s], t.mid[s], vm.y);
            t.mid[s] -= (g & 1) ? (float)(kMiddle >> 16) : (float)(kMiddle & 0xffffu);
        }
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            const uint32_t a[4] = {k_operand(kw, 0, s, 0), k_operand(kw, 1, s, 0), k_operand(kw, 0, s, 1), k_operand(kw, 1, s, 1)};
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const uint32_t b0 = query_word(qf[n][s >> 1], 2 * (s & 1)), b1 = query_word(qf[n][s >> 1], 2 * (s & 1) + 1);
                if (s == 0) mma_f16_first(t.D[n], a, b0, b1);
                else mma_f16(t.D[n], a, b0, b1);
            }
        }
    }
    // The row operands of the V product: a[j] holds the fields (prefixes, see enter_class) of channels 4 g + j and 32 + 4 g + j.
    __device__ static __forceinline__ void v_operands(const uint8_t* rec, int lane, uint32_t (&a)[4][4], uint32_t) {
        const int g = lane >> 2, q = lane & 3;
        // V words of slots 2q, 2q + 1 (a) and 8 + 2q, 9 + 2q (b): halves of the words of slot quads q >> 1 and 2 + (q >> 1)
        uint32_t va[NW], vb[NW];
        load_words(rec + pool_codes_bytes(CLS), 4 * g + (q >> 1), va);
        load_words(rec + pool_codes_bytes(CLS), 4 * g + 2 + (q >> 1), vb);
        const uint32_t sel = (q & 1) ? 0x4342u : 0x4140u;
        constexpr int PER = 8 / BITS;                              // channels per byte
#pragma unroll
        for (int byte = 0; byte < 4 / PER; ++byte) {               // word of channel group i: CLS 0: i, CLS 1, 2: 2 byte + i
            uint32_t x[4];                             // x0: channel group 0, slots 2q ..; x1: group 1; x2, x3: slots 8 + 2q ..
#pragma unroll
            for (int k = 0; k < 4; ++k) x[k] = prmt((k >> 1) ? vb[2 * byte + (k & 1)] : va[2 * byte + (k & 1)], 0u, sel);
#pragma unroll
            for (int f = 0; f < PER; ++f) {
                const uint32_t prefix = ((1u << (BITS * (f + 1))) - 1u) * 0x00010001u;
                const uint32_t ones = ((1u << (BITS * (f + 1))) - 1u) / ((1u << BITS) - 1u);   // 1 + 2^BITS + ..., a one per field
#pragma unroll
                for (int k = 0; k < 4; ++k) a[byte * PER + f][k] = sub_half2(f + 1 == PER ? x[k] : x[k] & prefix, kMiddle * ones);
            }
        }
    }
};

// fp16 rows: the fp16 pool, and the drafted tokens.
struct RowsFp16 {
    // Register r of step s of the K product: channels 8 (2 s + r) + 2 q + x.

    template <int NT>
    __device__ static __forceinline__ void k_side(const uint8_t* rec, int lane, const RowsQuery<NT>& qf, float kfactor, TileLogits<NT>& t) {
        const int row = lane & 7, mat = lane >> 3;
#pragma unroll
        for (int s = 0; s < 4; ++s) {                  // four 8x8 matrices: (slots 0..7, 8..15) x (unit 2s, 2s + 1)
            uint32_t a[4];
            ldsm_x4(a, rec + ((2 * s + (mat >> 1)) * kTileTokens + 8 * (mat & 1) + row) * 16);
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const uint32_t b0 = query_word(qf[n][s >> 1], 2 * (s & 1)), b1 = query_word(qf[n][s >> 1], 2 * (s & 1) + 1);
                if (s == 0) mma_f16_first(t.D[n], a, b0, b1);
                else mma_f16(t.D[n], a, b0, b1);
            }
        }
        t.sk[0] = t.sk[1] = kfactor;
        t.sv[0] = t.sv[1] = 1.f;
        t.zk[0] = t.zk[1] = t.zv[0] = t.zv[1] = t.mid[0] = t.mid[1] = 0.f;
    }
    // slots: those of the tile that are read (the bytes of the others may be anything, an Inf or NaN pattern included, which
    // a weight of zero would not silence).
    __device__ static __forceinline__ void v_operands(const uint8_t* rec, int lane, uint32_t (&a)[4][4], uint32_t slots) {
        const int g = lane >> 2, q = lane & 3;
        const uint8_t* v = rec + pool_codes_bytes(3) + (g >> 1) * kTileTokens * 16 + (g & 1) * 8;
        uint2 x[2][4];
#pragma unroll
        for (int i = 0; i < 2; ++i)                    // channels 32 i + 4 g .. + 3 of the lane's four slots
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int slot = 2 * q + (k & 1) + 8 * (k >> 1);
                x[i][k] = (slots >> slot) & 1u ? *reinterpret_cast<const uint2*>(v + (i * 4 * kTileTokens + slot) * 16) : make_uint2(0u, 0u);
            }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t sel = (j & 1) ? 0x7632u : 0x5410u;
#pragma unroll
            for (int k = 0; k < 4; ++k) {              // a0, a1: slots 2q, 2q + 1 of channel groups 0, 1; a2, a3: slots 8 + 2q ..
                const uint2 lo = x[k & 1][2 * (k >> 1)], hi = x[k & 1][2 * (k >> 1) + 1];
                a[j][k] = j < 2 ? prmt(lo.x, hi.x, sel) : prmt(lo.y, hi.y, sel);
            }
        }
    }
};
template <int NT>
__device__ __forceinline__ void v_products(RowsState<NT>& st, const uint32_t (&a)[4][4], const uint32_t (&w)[NT][2]) {
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int n = 0; n < NT; ++n) mma_f16(st.acc[n][j], a[j], w[n][0], w[n][1]);
}

// Up to n tiles in a row that every row sees whole; stops in front of one with a weight that overflows.  Returns the tiles
// done.  
template <int NT, class C>
__device__ __forceinline__ uint32_t whole_tiles(const uint8_t* rec, uint32_t n, uint32_t step, int lane, const RowsQuery<NT>& qf,
                                                float kfactor, RowsState<NT>& st) {
    uint32_t i = 0;
#pragma unroll 1
    for (; i < n; ++i, rec += step) {
        TileLogits<NT> t;
        C::template k_side<NT>(rec, lane, qf, kfactor, t);
        uint32_t a[4][4];
        C::v_operands(rec, lane, a, 0xffffu);              // (in front of the vote: it fills the waits of the chain above)
        float2 p[NT][2];
        uint32_t w[NT][2];
        logits_of(st, t, true, p);
        if (__builtin_expect(overflows(weigh(t, p, w)), 0)) break;
        add_tile(st, t, p, w);
        v_products(st, a, w);
    }
    return i;
}

// Accumulators and the units of a class.  V operand j of a byte holds the fields up to that of channels 4 g + j and
// 32 + 4 g + j, as multiples of 2^-24: with b_j the bit of the field inside its byte, the accumulator of operand j is
//   F_j = 2^(b_j - 24) o_j + (b_j > 0 ? F_(j-1) : 0).
// fp16 rows: F_j = o_j.
__device__ __forceinline__ int v_bit(int c, int j) { return c == 0 ? 2 * j : c == 1 ? 4 * (j & 1) : 0; }
template <int NT>
__device__ __forceinline__ void enter_class(RowsState<NT>& st, int c) {
    if (c == 3) return;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float f = two_to(v_bit(c, j) - 24), carry = v_bit(c, j) > 0 ? 1.f : 0.f;
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) st.acc[n][j][e] = fmaf(st.acc[n][j > 0 ? j - 1 : 0][e], carry, st.acc[n][j][e] * f);
    }
}
template <int NT>
__device__ __forceinline__ void leave_class(RowsState<NT>& st, int c) {
    if (c == 3) return;
#pragma unroll
    for (int j = 3; j >= 0; --j) {
        const float f = two_to(24 - v_bit(c, j)), carry = v_bit(c, j) > 0 ? -1.f : 0.f;
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) st.acc[n][j][e] = fmaf(st.acc[n][j > 0 ? j - 1 : 0][e], carry, st.acc[n][j][e]) * f;
    }
}

// ---------------------------------------------------------------- the kernel

__device__ __forceinline__ bool finite_half8(uint4 v) {
    // (an exponent of all ones carries into the sign bit)
    const auto carry = [](uint32_t w) { return (w & 0x7fff7fffu) + 0x04000400u; };
    return !((carry(v.x) | carry(v.y) | carry(v.z) | carry(v.w)) & 0x80008000u);
}
// One drafted row of finite values, eight channels per lane of an eight-lane group, as the store would give it back (the row
// quantizer of Eq. 24, then code * scale + zero-point), rounded to fp16.
__device__ __forceinline__ uint4 draft_row_as_stored(uint4 raw, int c) {
    float x[8];
    const uint32_t rw[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const float2 f = unpack_half2(rw[k]);
        x[2 * k] = f.x;
        x[2 * k + 1] = f.y;
    }
    float mn = x[0], mx = x[0];
#pragma unroll
    for (int k = 1; k < 8; ++k) {
        mn = fminf(mn, x[k]);
        mx = fmaxf(mx, x[k]);
    }
#pragma unroll
    for (int d = 1; d < 8; d <<= 1) {
        mn = fminf(mn, __shfl_xor_sync(0xffffffffu, mn, d));
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, d));
    }
    if (c == 3) return raw;
    if (mn == 0.0f) mn = 0.0f;                         // -0 is stored as +0
    if (mx == 0.0f) mx = 0.0f;
    const float levels = c == 0 ? 3.0f : c == 1 ? 15.0f : 255.0f;
    const float sf = __half2float(__float2half_rn(__fdiv_rn(__fsub_rn(mx, mn), levels)));
    const float inv = sf == 0.0f ? 0.0f : __frcp_rn(sf);
    uint32_t out[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        float v[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const float code = rintf(fminf(__fmul_rn(__fsub_rn(x[2 * k + e], mn), inv), levels));
            v[e] = fminf(fmaxf(__fadd_rn(__fmul_rn(code, sf), mn), -65504.0f), 65504.0f);   // the rounded scale may overshoot the largest fp16
        }
        out[k] = pack_half2(make_float2(v[0], v[1]));
    }
    return make_uint4(out[0], out[1], out[2], out[3]);
}

// The record that CTA j writes for its piece of a unit: a CTA has at most two pieces that are not whole units, its first and
// its last.  (The axis is shorter than 2^32: ticks * units is the number of units, or at most rows_max_units times the CTAs.)
__device__ __forceinline__ uint32_t rows_record(const RowsParams& P, uint32_t j, uint32_t unit) {
    return 2u * j + (j * P.span >= unit * P.ticks ? 0u : 1u);      // (it starts inside the unit, or in front of it)
}

// What bounds it.  Long caches: latency.  A tile is one dependent chain of products, softmax, vote, transposition and
// products, about 240 instructions with 16 rows, which four warps per scheduler (two with 32 rows) do not hide (8192 tokens,
// 16 rows: a scheduler issues in 53 % of its active cycles, ALU 36 %, matrix pipe 28 %, exponentials 23 %).  The 16-row kernel
// is held to 128 registers and spills around its loops (86 bytes stored and 56 loaded with a tree, 60 and 24 without).  16 sequences x 32 heads x 32768 tokens, 1.26 GB of packed rows: 16 rows 401 us (3.1 TB/s of them,
// 0.48 of the copy bandwidth), one row over a window of 8192 87 us (3.6 TB/s); 32 rows over 8192 tokens, 0.42 GB, 235 us, 146
// Tflop/s.  Pools of 16 bits alone are bound by memory.  Short caches: the chain of round trips (fills, index, block table,
// rows, merge) and instructions that are not in the caches yet, 6 to 10 us.  Two tiles at a time, for more independent
// instructions, outgrew the innermost instruction cache (20 % slower on mixed pools).
//
// grid = CTAs of the plan, block = kRowsThreads, dynamic smem = rows_smem_bytes<NT>(draft tiles).
// NT: blocks of eight rows per unit.  TREE: rows belong to drafted nodes (otherwise nodes == 1 and the row is the last
// cached token's).
template <int NT, bool TREE>
__global__ void __launch_bounds__(kRowsThreads, rows_ctas_per_sm(NT)) k_attend_rows(const RowsParams P) {
    constexpr int ROWS = 8 * NT;
    extern __shared__ __align__(128) uint8_t dyn[];
    __shared__ RowsScratch<NT> sc;
    uint8_t* const rings = dyn;
    uint4* const qfrag = reinterpret_cast<uint4*>(dyn + (size_t)kRowsWarps * kRowsStages * kRowsStageBytes);   // [class][NT][2][32]
    const uint32_t draft_at = (uint32_t)((size_t)kRowsWarps * kRowsStages * kRowsStageBytes + (size_t)kNumPools * NT * 2 * 32 * 16);
    uint8_t* const draft = dyn + draft_at;
    float* const inbox = reinterpret_cast<float*>(draft + (size_t)(TREE ? (P.nodes + kTileTokens - 1) / kTileTokens : 0) * kDraftTileBytes);   // [rows of this CTA][CTAs][kRowsOutStride]
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, q = lane & 3;
    const StoreView& S = P.store;

    const int draft_tiles = (P.nodes + kTileTokens - 1) / kTileTokens;
    int cslot = 0;                                     // ring slot that is read next
    uint32_t parity = 0;                               // phase parity of every ring slot (bit s: slot s)
    bool failed = false;

    if (lane == 0) {
        for (int s = 0; s < kRowsStages; ++s) mbar_init(&sc.bars[warp][s], 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncwarp();
    if (P.cluster > 1) cluster_arrive();               // (before another CTA's memory is written, all of them have to be there)
    pdl_launch_dependents();
    pdl_wait();                                        // an append ahead of this launch has stored its tokens

    // This CTA's stretch of the axis, in pieces: ticks [a0, a1) of unit u.  After an expired wait a warp starts no further
    // copy, but every piece is delivered (empty), so that all arrival counters reach their totals.
    uint32_t x = blockIdx.x * P.span;
    const uint32_t x_end = x + P.span;
#pragma unroll 1
    while (x < x_end) {
    const uint32_t unit = x / P.ticks, a0 = x - unit * P.ticks, a1 = min(P.ticks, a0 + (x_end - x));
    x += a1 - a0;
    const uint32_t rb = unit / P.pairs, bh = unit - rb * P.pairs;  // row blocks of a pair lie far apart: CTAs that run at the same time read the same tiles
    const int b = (int)(bh / (uint32_t)S.kv_heads), h = (int)(bh - (uint32_t)b * S.kv_heads);
    const bool has_end = a1 == P.ticks, has_draft = TREE && has_end;

    // ---- what the piece starts from, requested together
    const uint4 fill = *reinterpret_cast<const uint4*>(P.counts + (size_t)b * 4);
    const uint32_t first_id = lane < kNumPools ? stream_table(S, lane, P.layer, b, h)[0] : 0u;     // first block of every stream
    // thread = (row, eight channels), up to 16 rows at a time
    constexpr int RB = ROWS > 16 ? ROWS / 16 : 1;
    const int row16 = tid >> 3, piece8 = tid & 7;
    auto row_of = [&](int k) { return 16 * k + row16; };
    auto place_of = [&](int row, int& node) -> size_t {                // of a row's eight channels in Q and O
        const int R = (int)rb * ROWS + row;
        node = R / P.group;
        return (((size_t)b * P.nodes + node) * S.q_heads + (size_t)h * P.group + (R - node * P.group)) * kHeadDim + piece8 * 8;
    };
    auto row_used = [&](int row) { return row < ROWS && (int)rb * ROWS + row < P.rows; };
    uint4 qv[RB];
    int my_node[RB];
#pragma unroll
    for (int k = 0; k < RB; ++k) {
        const size_t at = place_of(row_of(k), my_node[k]);
        qv[k] = row_used(row_of(k)) ? *reinterpret_cast<const uint4*>(P.Q + at) : make_uint4(0u, 0u, 0u, 0u);
    }
    int par[2] = {-2, -2};
    if (TREE && warp == 0) {
        if (lane < P.nodes) par[0] = P.parents[(size_t)b * P.nodes + lane];
        if (lane + 32 < P.nodes) par[1] = P.parents[(size_t)b * P.nodes + lane + 32];
    }
    const int len = (int)(fill.x + fill.y + fill.z + fill.w);

    // ---- the window: where it and the sinks end in every pool (warp = class)
    int base0 = 0;                                     // first position that the shallowest row's window holds
    if (P.window > 0) {
        base0 = min(max(len - P.window + (TREE ? 1 : 0), 0), len);
        const uint32_t c = (uint32_t)warp;
        const uint32_t n = c == 0 ? fill.x : c == 1 ? fill.y : c == 2 ? fill.z : fill.w;
        const uint32_t* idx = S.index + ((size_t)P.layer * S.batch + b) * S.max_ctx;
        const uint32_t start = first_slot_from(idx, base0, len, c, n, lane);
        const uint32_t sink = P.sinks > 0 ? first_slot_from(idx, min(P.sinks, len), len, c, n, lane) : 0u;
        unsigned long long bits = 0;
        if (TREE) {
            uint32_t m[2];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int at = base0 + 32 * k + lane;
                m[k] = __ballot_sync(0xffffffffu, at < len && (idx[min(at, len - 1)] >> 30) == c);
            }
            bits = ((unsigned long long)m[1] << 32) | m[0];
        }
        if (lane == 0) {
            sc.start[c] = start;
            sc.sink[c] = sink;
            sc.step_bits[c] = bits;
        }
        __syncthreads();
    }
    // ---- this warp's share: tile ranges of the pools, laid end to end [sinks | window] per pool; lane = pool
    const uint32_t ring = (uint32_t)warp * kRowsStages * kRowsStageBytes;          // offset in dyn
    RowsChunks& plan = sc.plan[warp];
    {
        const int c = lane & 3;
        const uint32_t n_c = c == 0 ? fill.x : c == 1 ? fill.y : c == 2 ? fill.z : fill.w;
        const uint32_t start = P.window > 0 ? sc.start[c] : 0u, sink = P.window > 0 ? sc.sink[c] : 0u;
        const int nt = (int)((n_c + kTileTokens - 1) / kTileTokens);
        int ns = (int)((sink + kTileTokens - 1) / kTileTokens), ws = (int)(start / kTileTokens);
        if (ws <= ns) ns = ws = 0;                     // no gap
        const int n = ns + nt - ws;
        const float cost = c == 0 ? kRowsTileCost[0] : c == 1 ? kRowsTileCost[1] : c == 2 ? kRowsTileCost[2] : kRowsTileCost[3], weight = (float)n * cost;
        float before = 0.f, total = 0.f;
#pragma unroll
        for (int k = 0; k < kNumPools; ++k) {
            const float wk = __shfl_sync(0xffffffffu, weight, k);
            before += k < c ? wk : 0.f;
            total += wk;
        }
        // Positions on the pools laid end to end, in units of cost.  Drafted rows cost the last piece of the unit about as much
        // as so many tiles, which stand for them behind the last pool (with an equal share that piece came last: 512 tokens,
        // 8 nodes, 8 parts: 10.1 us against 9.4 us).  The end of a share and the start of the next one are
        // the same expression of the same tick, which does not fall as the tick grows; the last share ends with the last tile.
        // So no tile is lost or taken twice, however this rounds.
        const float drafts = TREE ? 60.f + 20.f * (float)draft_tiles : 0.f, per_tick = (total + drafts) * fast_rcp((float)P.ticks);
        const float x0 = fminf((float)a0 * per_tick, total), x1 = has_end ? total : fminf((float)a1 * per_tick, total);
        const float per_pool = n > 0 ? (float)n * fast_rcp(total) : 0.f, inv = fast_rcp(cost);
        // (where a share is the same fraction of every pool, the last one has the pools' last, ragged tiles, which take longer)
        const float quarter = 0.25f * (x1 - x0 + (P.by_pool && has_end && n > 0 ? total * fast_rcp((float)n) : 0.f));
        auto tiles_before = [&](int share) {           // tiles of the pool in front of warp `share`'s
            if (share == kRowsWarps && has_end) return n;
            const float at = share == kRowsWarps ? x1 : fminf(x0 + quarter * (float)share, x1);
            return min(max((int)(P.by_pool ? at * per_pool : (at - before) * inv), 0), n);
        };
        const int lo = tiles_before(warp), hi = tiles_before(warp + 1);
        if (TREE) {                                    // what the warp's share costs it
            float load = (float)(hi - lo) * cost;
            load += __shfl_xor_sync(0xffffffffu, load, 1);
            load += __shfl_xor_sync(0xffffffffu, load, 2);
            if (lane == 0) sc.load[warp] = load;
        }
        if (lane < kNumPools) {
            sc.seg_lo[warp][2 * c] = lo;
            sc.seg_hi[warp][2 * c] = min(hi, ns);
            sc.seg_lo[warp][2 * c + 1] = max(lo, ns) - ns + ws;
            sc.seg_hi[warp][2 * c + 1] = hi - ns + ws;
            if (warp == 0) {
                const uint32_t lo_last = P.window > 0 ? start + (TREE ? (uint32_t)__popcll(sc.step_bits[c]) : 0u) : 0u;
                sc.cnt[c] = n_c;
                if (P.window == 0) sc.start[c] = sc.sink[c] = 0u;
                sc.in_sinks[c] = (int)(sink / kTileTokens);
                sc.from[c] = (int)((lo_last + kTileTokens - 1) / kTileTokens);
                sc.full[c] = (int)(n_c / kTileTokens);
            }
            if (lane == 0) {
                plan.seg = 0;
                plan.tile = lo;
            }
        }
    }
    auto largest = [](uint4 v) {                       // of eight query values; what is not finite must not set the scale of other rows
        const float2 f0 = unpack_half2(v.x), f1 = unpack_half2(v.y), f2 = unpack_half2(v.z), f3 = unpack_half2(v.w);
        const float top = fmaxf(fmaxf(fmaxf(fabsf(f0.x), fabsf(f0.y)), fmaxf(fabsf(f1.x), fabsf(f1.y))),
                                fmaxf(fmaxf(fabsf(f2.x), fabsf(f2.y)), fmaxf(fabsf(f3.x), fabsf(f3.y))));
        return top <= 65504.f ? top : 0.f;
    };
    float qmax = 0.f;                                  // the query block
#pragma unroll
    for (int k = 0; k < RB; ++k) {
        const float2 f0 = unpack_half2(qv[k].x), f1 = unpack_half2(qv[k].y), f2 = unpack_half2(qv[k].z), f3 = unpack_half2(qv[k].w);
        float sum = ((f0.x + f0.y) + (f1.x + f1.y)) + ((f2.x + f2.y) + (f3.x + f3.y));
        qmax = fmaxf(qmax, largest(qv[k]));
#pragma unroll
        for (int d = 1; d < 8; d <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
        if (row_of(k) < ROWS) {
            *reinterpret_cast<uint4*>(&sc.q[row_of(k)][piece8 * 8]) = qv[k];
            if (piece8 == 0) {
                sc.sumq[row_of(k)] = sum * kLogitScale;
                sc.node[row_of(k)] = (int16_t)(row_used(row_of(k)) ? my_node[k] : -1);
            }
        }
    }
    qmax = warp_max(qmax);
    if (lane == 0) sc.wmax[warp] = qmax;
    if (has_draft && tid == 0) sc.poison = sc.odd_bits = 0ull;
    __syncthreads();

    // ---- the copies: chunks of the share in order; a chunk stays inside one 64 KB block and fits a stage
    int planned = 0, taken = 0;
    auto plan_more = [&]() {                           // (whole warp) the chunks up to the end of the range or of the block
        __syncwarp();
        const int from_seg = plan.seg, my_seg = lane & (2 * kNumPools - 1);
        const int my_lo = my_seg == from_seg ? plan.tile : sc.seg_lo[warp][my_seg], my_hi = sc.seg_hi[warp][my_seg];
        const uint32_t open = __ballot_sync(0xffffffffu, my_seg >= from_seg && my_lo < my_hi) & 0xffu;
        planned = taken = 0;
        if (open == 0) return;
        const int seg = __ffs(open) - 1, tile = __shfl_sync(0xffffffffu, my_lo, seg), hi = __shfl_sync(0xffffffffu, my_hi, seg);
        const int c = seg >> 1, bt = (int)block_tiles(c), tps = kRowsTps(c);
        const uint32_t rec = (uint32_t)(c == 0 ? pool_rec_bytes(0) : c == 1 ? pool_rec_bytes(1) : c == 2 ? pool_rec_bytes(2) : pool_rec_bytes(3));
        int blk = 0, ib = tile;
        uint32_t id = __shfl_sync(0xffffffffu, first_id, c);
        if (tile >= bt) {
            blk = tile / bt;
            ib = tile - blk * bt;
            id = stream_table(S, c, P.layer, b, h)[blk];
        }
        const int in_sinks = sc.in_sinks[c], from = sc.from[c], full = sc.full[c];
        const int piece = min(bt - ib, hi - tile);
        planned = min(c == 3 ? piece : c == 2 ? (piece + 1) >> 1 : c == 1 ? (piece + 3) >> 2 : (piece + 5) / 6, 32);
        const int t0 = tile + lane * tps, n = min(tps, tile + piece - t0);
        uint32_t edge = 0;
#pragma unroll
        for (int i = 0; i < kRowsTps(0); ++i) edge |= i < n && !(t0 + i < full && (t0 + i >= from || t0 + i < in_sinks)) ? 1u << i : 0u;
        const uint8_t* src = S.arena + (size_t)id * kBlockBytes + (uint32_t)(ib + lane * tps) * rec;
        if (lane < planned)
            plan.chunk[lane] = make_uint4((uint32_t)(uintptr_t)src, (uint32_t)((uintptr_t)src >> 32), (uint32_t)t0 | ((uint32_t)c << 30),
                                          (uint32_t)n * rec | ((uint32_t)n << 16) | (edge << 20));
        __syncwarp();
        if (lane == 0) {
            plan.seg = seg;
            plan.tile = tile + min(piece, planned * tps);
        }
        __syncwarp();
    };
    auto feed = [&](int slot) -> int {                 // start the next copy; 0 if there is none
        if (taken == planned) {
            plan_more();
            if (planned == 0) return 0;
        }
        if (lane == 0) {
            const uint4 k = plan.chunk[taken];
            const uint32_t bytes = k.w & 0xffffu;
            mbar_arrive_expect_tx(&sc.bars[warp][slot], bytes);
            bulk_load(dyn + ring + (uint32_t)slot * kRowsStageBytes, reinterpret_cast<const uint8_t*>((uintptr_t)k.x | ((uintptr_t)k.y << 32)), bytes,
                      &sc.bars[warp][slot]);
            sc.chunk[warp][slot] = make_uint2(k.z, k.w >> 16);
        }
        ++taken;
        return 1;
    };
    int in_flight = 0;
#pragma unroll 1
    for (; in_flight < kRowsStages; ++in_flight)
        if (failed || !feed((cslot + in_flight) % kRowsStages)) break;

    // ---- the tree: ancestors by doubling the chain of parents
    if (TREE && warp == 0) {
        unsigned long long a[2];
        int bad[2], link[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int i = lane + 32 * k;
            bad[k] = !(par[k] >= -1 && par[k] < i);
            link[k] = bad[k] ? -1 : par[k];
            a[k] = 1ull << i;
            sc.anc[i] = a[k];
            sc.link[i] = (int8_t)link[k];
            sc.bad[i] = (int8_t)bad[k];
        }
#pragma unroll 1
        while (true) {                                 // (six rounds at most)
            __syncwarp();
            if (!__any_sync(0xffffffffu, link[0] >= 0 || link[1] >= 0)) break;
#pragma unroll
            for (int k = 0; k < 2; ++k)
                if (link[k] >= 0) {
                    a[k] |= sc.anc[link[k]];
                    bad[k] |= sc.bad[link[k]];
                    link[k] = sc.link[link[k]];
                }
            __syncwarp();
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                sc.anc[lane + 32 * k] = a[k];
                sc.bad[lane + 32 * k] = (int8_t)bad[k];
                sc.link[lane + 32 * k] = (int8_t)link[k];
            }
        }
        const uint32_t u0 = __ballot_sync(0xffffffffu, !bad[0]), u1 = __ballot_sync(0xffffffffu, !bad[1]);
        if (lane == 0) sc.used = ((unsigned long long)u1 << 32) | u0;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            unsigned long long v = bad[k] ? 0ull : a[k];
            if (P.window > 0 && v) {                   // drop the ancestors outside the window (unless they are sinks)
                const int d = __popcll(v) - 1;
                unsigned long long rest = v;
                for (int r = 0; r <= d - P.window; ++r) {
                    const unsigned long long bit = rest & (~rest + 1ull);
                    rest ^= bit;
                    if (len + r >= P.sinks) v ^= bit;
                }
            }
            sc.vis[lane + 32 * k] = v;
        }
    }
    // ---- drafted rows as fp16 tiles
    if (has_draft) {
        const int padded = draft_tiles * kTileTokens;
#pragma unroll 1
        for (int k = 0; k < 2 * padded; k += kRowsThreads / 8) {
            const int i = k + row16;
            const bool value = i >= padded;
            const int node = value ? i - padded : i;
            uint4 raw = make_uint4(0u, 0u, 0u, 0u);
            int c = 3;
            if (node < P.nodes) {
                raw = *reinterpret_cast<const uint4*>((value ? P.V : P.K) + (((size_t)b * P.nodes + node) * S.kv_heads + h) * kHeadDim + piece8 * 8);
                if (P.bits) {
                    c = bits_to_class(P.bits[(size_t)b * P.nodes + node]);
                    if (c < 0) {                       // as in an append: kept as fp16, and flagged (if the node is in use, see below)
                        if (piece8 == 0) atomicOr(&sc.odd_bits, 1ull << node);
                        c = 3;
                    }
                }
            }
            uint4 row = draft_row_as_stored(raw, c);
            // What the row quantizer makes of a row that is not finite is asked of the row as it came: its minimum and maximum
            // skip NaN, and its clamp makes numbers of the others.  Such a row has no finite value at 2, 4 or 8 bits (its scale
            // or its zero-point is not finite), so its key is NaN; at 16 it stays what it is.  A value row is left out of the products,
            // where a weight of zero would not silence it for the nodes that do not see it; those that see it become
            // NaN at the end.
            const uint32_t lanes = 0xffu << (lane & 24);
            if (__ballot_sync(0xffffffffu, !finite_half8(raw)) & lanes) {
                if (c != 3) row = make_uint4(0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu, 0x7fff7fffu);
                if (value) {
                    row = make_uint4(0u, 0u, 0u, 0u);
                    if (piece8 == 0 && node < P.nodes) atomicOr(&sc.poison, 1ull << node);
                }
            }
            *reinterpret_cast<uint4*>(draft + (node / kTileTokens) * kDraftTileBytes + (value ? kDraftTileBytes / 2 : 0) +
                                      (piece8 * kTileTokens + node % kTileTokens) * 16) = row;
        }
    }

    // ---- column operands of the K product, one set per class (warp = class): q * F * 2^-k, F a power of two that puts the
    // block's largest query value below 2^15
    float F;
#pragma unroll 1
    for (bool again = false;; again = true) {
        const float block_max = fmaxf(fmaxf(fmaxf(sc.wmax[0], sc.wmax[1]), fmaxf(sc.wmax[2], sc.wmax[3])), 6.103515625e-05f);
        const int e_max = (int)(__float_as_uint(block_max) >> 23) - 127;       // -14 .. 15
        F = two_to(14 - e_max);
        // The channels and bits of the classes' K operands (RowsQuant, RowsFp16) as sums of a part each of q, r, s & 1, s >> 1 and x.
        const int c = warp, at_q = q * (16 >> c), at_r = c == 3 ? 8 : 1, at_x = c == 0 ? 8 : c == 1 ? 4 : c == 2 ? 2 : 1;
        const int at_s1 = c < 2 ? 2 : 16, at_s2 = c == 0 ? 4 : 32;         // of s & 1 and of s >> 1
        const float f1 = c == 0 ? F * 0.25f : c == 1 ? F * 0.0625f : F;    // r = 1
        const float f2 = c == 0 ? 0.0625f : 1.0f;                          // s & 1
#pragma unroll
        for (int n = 0; n < NT; ++n) {                 // column g of block n
            const __half* row = sc.q[8 * n + g] + at_q;
#pragma unroll
            for (int s2 = 0; s2 < 2; ++s2) {
                uint32_t w[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {          // step s = 2 s2 + (k >> 1), register r = k & 1
                    const __half* e = row + s2 * at_s2 + (k >> 1) * at_s1 + (k & 1) * at_r;
                    const float f = ((k & 1) ? f1 : F) * ((k >> 1) ? f2 : 1.0f);
                    w[k] = pack_half2(make_float2(__half2float(e[0]) * f, __half2float(e[at_x]) * f));
                }
                qfrag[((warp * NT + n) * 2 + s2) * 32 + lane] = make_uint4(w[0], w[1], w[2], w[3]);
            }
        }
        __syncthreads();
        if (!TREE || again) break;
        // The rows of nodes that are not in use may hold anything.  Now that these are known: if the block has any, their
        // queries become zeros and everything is laid out once more, so that they neither set F, which costs the others bits,
        // nor make weights overflow.  (512 tokens, 8 nodes: 9.2 us, without this 9.0 us; laid out behind this barrier for every tree
        // 9.4 us.)
        const auto idle = [&](int row) { return sc.node[row] >= 0 && !((sc.used >> sc.node[row]) & 1ull); };
        if (__builtin_expect(!__any_sync(0xffffffffu, lane < ROWS && idle(lane)), 1)) break;
        qmax = 0.f;
#pragma unroll
        for (int k = 0; k < RB; ++k)
            if (row_of(k) < ROWS) {
                uint4* const v = reinterpret_cast<uint4*>(&sc.q[row_of(k)][piece8 * 8]);
                if (idle(row_of(k))) {
                    *v = make_uint4(0u, 0u, 0u, 0u);
                    sc.sumq[row_of(k)] = 0.f;
                }
                qmax = fmaxf(qmax, largest(*v));
            }
        qmax = warp_max(qmax);
        if (lane == 0) sc.wmax[warp] = qmax;
        __syncthreads();
    }
    if (has_draft && tid == 0 && (sc.odd_bits & sc.used)) atomicOr(S.flags, 1u);
    // ---- first window slot of every row, per class
    if (P.window > 0) {
        for (int k = tid; k < kNumPools * ROWS; k += kRowsThreads) {
            const int c = k / ROWS, row = k - c * ROWS;
            uint32_t lo = sc.start[c];
            if (TREE && sc.node[row] >= 0) {
                const int depth = max(__popcll(sc.anc[sc.node[row]]) - 1, 0);
                const int off = min(max(len + depth - P.window + 1, 0), len) - base0;      // 0 .. 63
                lo += (uint32_t)__popcll(sc.step_bits[c] & ((1ull << off) - 1ull));
            }
            sc.lo_row[c][row] = lo;
        }
        __syncthreads();
    }

    // ---- the walk
    RowsState<NT> st;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        st.negm[n] = both(-kNegBig);
        st.l[n] = st.b[n] = both(0.f);
        st.sumq[n] = make_float2(sc.sumq[8 * n + 2 * q], sc.sumq[8 * n + 2 * q + 1]);
#pragma unroll
        for (int j = 0; j < 4; ++j) st.acc[n][j][0] = st.acc[n][j][1] = st.acc[n][j][2] = st.acc[n][j][3] = 0.f;
    }

    auto load_queries = [&](int c, RowsQuery<NT>& qf) {
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int s2 = 0; s2 < 2; ++s2) qf[n][s2] = qfrag[((c * NT + n) * 2 + s2) * 32 + lane];
    };
    const float kfactor = kLogitScale / F;
    RowsQuery<NT> qf;
    // One tile of class c in general.  There is one copy of this code for all classes, and a short loop per class for the
    // tiles in the middle (whole_tiles): the loops have to stay inside the instruction caches.
    bool fresh = true;                                 // no reference has been set yet
    auto any_tile = [&](int c, const uint8_t* rec, bool edge, const uint32_t (&seen)[NT], uint32_t slots) {
        TileLogits<NT> t;
        if (c == 0) RowsQuant<0>::k_side<NT>(rec, lane, qf, kfactor, t);
        else if (c == 1) RowsQuant<1>::k_side<NT>(rec, lane, qf, kfactor, t);
        else if (c == 2) RowsQuant<2>::k_side<NT>(rec, lane, qf, kfactor, t);
        else RowsFp16::k_side<NT>(rec, lane, qf, kfactor, t);
#pragma unroll
        for (int s = 0; s < 2; ++s)
            if (!((slots >> (g + 8 * s)) & 1u)) {      // what a slot carries that is not read may be Inf or NaN
                t.sv[s] = 1.f;
                t.zv[s] = t.mid[s] = 0.f;
            }
        float2 p[NT][2];
        uint32_t w[NT][2];
#pragma unroll 1
        for (bool moved = false;; moved = true) {
            if (moved || fresh) move_references(st, t, edge, seen);
            logits_of(st, t, true, p);
            hide(edge, seen, p);
            if (!overflows(weigh(t, p, w)) || moved || fresh) break;
        }
        fresh = false;
        add_tile(st, t, p, w);
        uint32_t a[4][4];
        if (c == 0) RowsQuant<0>::v_operands(rec, lane, a, slots);
        else if (c == 1) RowsQuant<1>::v_operands(rec, lane, a, slots);
        else if (c == 2) RowsQuant<2>::v_operands(rec, lane, a, slots);
        else RowsFp16::v_operands(rec, lane, a, slots);
        v_products(st, a, w);
    };
    int cls = 3;
    bool draft_left = false;                           // a tile of drafted tokens per warp, at the end: the warps with the least to do first
    if (has_draft) {
        const float load = sc.load[lane & 3], mine = __shfl_sync(0xffffffffu, load, warp);
        const int tile = __popc(__ballot_sync(0xffffffffu, load < mine || (load == mine && (lane & 3) < warp)) & 15u);
        draft_left = tile < draft_tiles;
        if (lane == 0) sc.draft_tile[warp] = tile;
        __syncwarp();
    }
    load_queries(3, qf);
    while ((in_flight > 0 || draft_left) && !failed) {
        const bool drafted = in_flight == 0;
        const uint2 ck = drafted ? make_uint2(3u << 30, 1u | 16u) : sc.chunk[warp][cslot];
        const int c = (int)(ck.x >> 30);
        if (c != cls) {
            leave_class<NT>(st, cls);
            enter_class<NT>(st, c);
            load_queries(c, qf);
            cls = c;
        }
        if (!drafted) {
            failed = !__all_sync(0xffffffffu, mbar_wait(&sc.bars[warp][cslot], (parity >> cslot) & 1u));
            if (failed) break;
        }
        const uint8_t* rec = dyn + (drafted ? draft_at + (uint32_t)sc.draft_tile[warp] * kDraftTileBytes : ring + (uint32_t)cslot * kRowsStageBytes);
        const uint32_t step = (uint32_t)(c == 0 ? pool_rec_bytes(0) : c == 1 ? pool_rec_bytes(1) : c == 2 ? pool_rec_bytes(2) : pool_rec_bytes(3));
        uint32_t left = ck.y & 15u, edges = ck.y >> 4, s0 = (ck.x & 0x3fffffffu) * kTileTokens;
#pragma unroll 1
        while (true) {
            const uint32_t run = edges ? (uint32_t)__ffs(edges) - 1u : left;
            if (run > 0 && !fresh) {
                uint32_t done = 0;
                if (c == 0) done = whole_tiles<NT, RowsQuant<0>>(rec, run, pool_rec_bytes(0), lane, qf, kfactor, st);
                else if (c == 1) done = whole_tiles<NT, RowsQuant<1>>(rec, run, pool_rec_bytes(1), lane, qf, kfactor, st);
                else if (c == 2) done = whole_tiles<NT, RowsQuant<2>>(rec, run, pool_rec_bytes(2), lane, qf, kfactor, st);
                else done = whole_tiles<NT, RowsFp16>(rec, run, pool_rec_bytes(3), lane, qf, kfactor, st);
                left -= done;
                if (left == 0) break;
                rec += done * step;
                s0 += done * kTileTokens;
                edges >>= done;
            }
            uint32_t seen[NT] = {}, slots = 0xffffu;
            const bool edge = edges & 1u;
            if (edge) {                                // the pool's last tile, one where a window starts or the sinks end, a drafted one
                const uint32_t use = drafted ? (uint32_t)(sc.used >> (16 * sc.draft_tile[warp])) : 0u, cnt = sc.cnt[c], sink = sc.sink[c];
                // those that some row sees: up to the end of the pool, from the shallowest row's window on or in the sinks
                const auto below = [&](uint32_t end) { return end <= s0 ? 0u : (1u << min(end - s0, 16u)) - 1u; };
                slots = drafted ? use & 0xffffu : below(cnt) & (~below(sc.start[c]) | below(sink));
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int x = 0; x < 2; ++x) {      // row 2q + x
                        const int row = 8 * n + 2 * q + x, node = sc.node[row];
                        const uint32_t lo = P.window > 0 ? sc.lo_row[c][row] : 0u;
                        const uint32_t vis = drafted && node >= 0 ? (uint32_t)(sc.vis[node] >> (16 * sc.draft_tile[warp])) : 0u;
#pragma unroll
                        for (int s = 0; s < 2; ++s) {
                            const uint32_t at = g + 8 * s, slot = s0 + at;
                            const bool see = drafted ? (vis >> at) & 1u : slot < cnt && (slot >= lo || slot < sink);
                            seen[n] |= see ? 1u << (2 * s + x) : 0u;
                        }
                    }
            }
            any_tile(c, rec, edge, seen, slots);
            if (--left == 0) break;
            rec += step;
            s0 += kTileTokens;
            edges >>= 1;
        }
        if (drafted) {
            draft_left = false;
        } else {
            __syncwarp();                              // every lane is done with the stage before it is refilled
            in_flight += feed(cslot) - 1;
            parity ^= 1u << cslot;
            cslot = cslot + 1 == kRowsStages ? 0 : cslot + 1;
            __syncwarp();                              // (sc.chunk of the refilled stage)
        }
    }
    leave_class<NT>(st, cls);
    if (failed) {                                      // give up: no further copy; those in flight are let land first
        if (lane == 0) atomicOr(S.flags, kFlagWaitTimeout);
        while (in_flight > 0) {
            mbar_wait(&sc.bars[warp][cslot], (parity >> cslot) & 1u);
            parity ^= 1u << cslot;
            cslot = cslot + 1 == kRowsStages ? 0 : cslot + 1;
            --in_flight;
        }
    }

    if (has_draft && sc.poison != 0ull) {              // rows that see a drafted value that is not finite
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            const int n0 = sc.node[8 * n + 2 * q], n1 = sc.node[8 * n + 2 * q + 1];
            if (n0 >= 0 && (sc.vis[n0] & sc.poison)) st.l[n].x = NAN;
            if (n1 >= 0 && (sc.vis[n1] & sc.poison)) st.l[n].y = NAN;
        }
    }

    // ---- merge the four warps: M = max m_w, l = sum l_w 2^(m_w - M), O = sum o_w 2^(m_w - M)
#pragma unroll
    for (int n = 0; n < NT; ++n) {
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) {
            st.l[n].x += __shfl_xor_sync(0xffffffffu, st.l[n].x, d);
            st.l[n].y += __shfl_xor_sync(0xffffffffu, st.l[n].y, d);
            st.b[n].x += __shfl_xor_sync(0xffffffffu, st.b[n].x, d);
            st.b[n].y += __shfl_xor_sync(0xffffffffu, st.b[n].y, d);
        }
        if (g == 0) {
            sc.ml[warp][8 * n + 2 * q] = make_float2(-st.negm[n].x, st.l[n].x);
            sc.ml[warp][8 * n + 2 * q + 1] = make_float2(-st.negm[n].y, st.l[n].y);
        }
    }
    __syncthreads();                                   // also: every warp is done with its ring, which becomes the merge buffer
    float* const out = reinterpret_cast<float*>(rings);             // [warps][ROWS][kRowsOutStride]
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const int row = 8 * n + 2 * q + x;
            float M = kNegBig;
#pragma unroll
            for (int k = 0; k < kRowsWarps; ++k) M = fmaxf(M, sc.ml[k][row].x);
            const float f = fast_exp2(-(x ? st.negm[n].y : st.negm[n].x) - M), fb = f * (x ? st.b[n].y : st.b[n].x);
            float* dst = out + ((size_t)warp * ROWS + row) * kRowsOutStride;
#pragma unroll
            for (int i = 0; i < 2; ++i)                // channels 32 i + 4 g .. + 3
                *reinterpret_cast<float4*>(dst + 32 * i + 4 * g) =
                    make_float4(fmaf(st.acc[n][0][2 * i + x], f, fb), fmaf(st.acc[n][1][2 * i + x], f, fb),
                                fmaf(st.acc[n][2][2 * i + x], f, fb), fmaf(st.acc[n][3][2 * i + x], f, fb));
        }
    __syncthreads();

    // ---- this CTA's rows: thread = (row, eight channels)
    if (P.cluster > 1) cluster_wait();
    auto store_row = [&](int row, const float (&o)[8], float L) {
        if (!row_used(row)) return;
        int node;
        const size_t at = place_of(row, node);
        // nothing seen, or an unused node: zeros (a NaN stays one)
        const float inv = L != 0.f && (!TREE || sc.vis[node]) ? 1.0f / L : 0.f;
        uint32_t v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = inv != 0.f ? pack_half2(make_float2(o[2 * e] * inv, o[2 * e + 1] * inv)) : 0u;
        *reinterpret_cast<uint4*>(P.O + at) = make_uint4(v[0], v[1], v[2], v[3]);
    };
#pragma unroll 1
    for (int k = 0; k < RB; ++k) {
        const int row = row_of(k);
        if (row >= ROWS) break;
        float o[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        float M = kNegBig, L = 0.f;
#pragma unroll
        for (int w = 0; w < kRowsWarps; ++w) M = fmaxf(M, sc.ml[w][row].x);
#pragma unroll
        for (int w = 0; w < kRowsWarps; ++w) {
            L = fmaf(sc.ml[w][row].y, fast_exp2(sc.ml[w][row].x - M), L);
            const float4* src = reinterpret_cast<const float4*>(out + ((size_t)w * ROWS + row) * kRowsOutStride + piece8 * 8);
            const float4 v0 = src[0], v1 = src[1];
            o[0] += v0.x; o[1] += v0.y; o[2] += v0.z; o[3] += v0.w;
            o[4] += v1.x; o[5] += v1.y; o[6] += v1.z; o[7] += v1.w;
        }
        if (a1 - a0 == P.ticks) {
            store_row(row, o, L);
        } else if (P.cluster > 1) {                    // to the CTA that merges this row
            const uint32_t at = smem_addr(inbox + ((size_t)(row / P.cluster) * P.cluster + blockIdx.x % P.cluster) * kRowsOutStride), to = row % P.cluster;
            st_cluster(at + piece8 * 32, to, make_float4(o[0], o[1], o[2], o[3]));
            st_cluster(at + piece8 * 32 + 16, to, make_float4(o[4], o[5], o[6], o[7]));
            if (piece8 == 0) st_cluster(at + kHeadDim * 4, to, make_float4(M, L, 0.f, 0.f));
        } else {
            const size_t rec = (size_t)rows_record(P, blockIdx.x, unit) * ROWS + row;
            float4* dst = reinterpret_cast<float4*>(P.part_o + rec * kHeadDim + piece8 * 8);
            dst[0] = make_float4(o[0], o[1], o[2], o[3]);
            dst[1] = make_float4(o[4], o[5], o[6], o[7]);
            if (piece8 == 0) P.part_ml[rec] = make_float2(M, L);
        }
    }
    if (P.cluster > 1) {
        // ---- the CTAs of a unit are a cluster: each merges the rows that it has been sent
        cluster_arrive();
        cluster_wait();
        const int row = (int)(row16 * P.cluster + blockIdx.x % P.cluster);
        if (row < ROWS) {
            const float* const from = inbox + (size_t)row16 * P.cluster * kRowsOutStride;
            float M = kNegBig, L = 0.f;
            float o[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
            for (uint32_t s = 0; s < P.cluster; ++s) M = fmaxf(M, from[s * kRowsOutStride + kHeadDim]);
#pragma unroll 2
            for (uint32_t s = 0; s < P.cluster; ++s) {
                const float2 ml = *reinterpret_cast<const float2*>(from + s * kRowsOutStride + kHeadDim);
                const float4* src = reinterpret_cast<const float4*>(from + s * kRowsOutStride + piece8 * 8);
                const float4 v0 = src[0], v1 = src[1];
                const float f = fast_exp2(ml.x - M);
                L = fmaf(ml.y, f, L);
                o[0] = fmaf(v0.x, f, o[0]); o[1] = fmaf(v0.y, f, o[1]); o[2] = fmaf(v0.z, f, o[2]); o[3] = fmaf(v0.w, f, o[3]);
                o[4] = fmaf(v1.x, f, o[4]); o[5] = fmaf(v1.y, f, o[5]); o[6] = fmaf(v1.z, f, o[6]); o[7] = fmaf(v1.w, f, o[7]);
            }
            store_row(row, o, L);
        }
    } else if (a1 - a0 < P.ticks) {
        // ---- the CTA that delivers the unit's last piece merges the pieces, in order
        const uint32_t first = unit * P.ticks / P.span, pieces = ((unit + 1) * P.ticks - 1) / P.span - first + 1;
        __syncthreads();
        if (tid == 0) {
            __threadfence();                           // (covers the whole CTA's records, which the barrier has ordered before it)
            sc.last = atomicAdd(P.part_cnt + unit, 1u) + 1u == pieces ? 1u : 0u;
            __threadfence();
        }
        __syncthreads();
        if (sc.last) {
            if (tid == 0) P.part_cnt[unit] = 0u;
#pragma unroll 1
            for (int k = 0; k < RB; ++k) {
                const int row = row_of(k);
                if (row >= ROWS) break;
                float M = kNegBig, L = 0.f;
                float o[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
                for (uint32_t s = 0; s < pieces; ++s) {
                    const size_t rec = (size_t)rows_record(P, first + s, unit) * ROWS + row;
                    const float2 ml = __ldcg(P.part_ml + rec);
                    const float4* src = reinterpret_cast<const float4*>(P.part_o + rec * kHeadDim + piece8 * 8);
                    const float4 v0 = __ldcg(src), v1 = __ldcg(src + 1);
                    const float top = fmaxf(M, ml.x), f = fast_exp2(ml.x - top), r = fast_exp2(M - top);
                    M = top;
                    L = fmaf(L, r, ml.y * f);
                    o[0] = fmaf(o[0], r, v0.x * f); o[1] = fmaf(o[1], r, v0.y * f); o[2] = fmaf(o[2], r, v0.z * f); o[3] = fmaf(o[3], r, v0.w * f);
                    o[4] = fmaf(o[4], r, v1.x * f); o[5] = fmaf(o[5], r, v1.y * f); o[6] = fmaf(o[6], r, v1.z * f); o[7] = fmaf(o[7], r, v1.w * f);
                }
                store_row(row, o, L);
            }
        }
    }
    // the next piece's copies overwrite the merge buffer through the asynchronous proxy
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncthreads();
    }
}

}  // namespace kvq
