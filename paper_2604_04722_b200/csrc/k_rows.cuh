// Attention of several query rows per sequence over the mixed-precision cache (Eq. 5), for speculative decoding and
// for sliding-window layers:
//   kvq_attend_tree         every row belongs to a node of a tree of drafted tokens; it sees the cached tokens (those
//                           of its window and the sinks) and its own ancestors, which are not in the cache
//   kvq_decode_attn_window  one row per query head, which sees the last `window` cached tokens and the sinks
//
// The decode kernel (k_decode.cuh) gives every (sequence, query head) its own walk over the cache, which is right for
// one row.  Here the rows of a tree and the heads of a group share a walk: a unit is (sequence, KV head, block of up
// to 16 or 32 rows), row = node * group + head, and both products run on the fp16 matrix instructions with the rows as
// the 16-row operand (mma.sync m16n8k16, fp32 accumulation):
//   S[row][slot] = sum_i q_i c_i        columns = slots of a 16-slot tile (two column groups of 8)
//   O[row][channel] += sum_slot w c     columns = channels
// with the packed codes as the column operand of both.  The fragment layout of the store (kvq_common.cuh) has, in
// lane (g, q), the codes of slots g and g + 8, and for V of slots 4q .. 4q + 3: a column operand needs exactly those
// bytes, two 16-bit lanes per register.
//
// Unpacking costs one AND per two codes: a field cut out in place at bit k <= 8 of a 16-bit lane IS the fp16 number
// code * 2^(k-24) (a subnormal: that encoding is linear), and the matrix instruction takes subnormals exactly.  The
// power 2^-k is undone on the other operand (K: the query of the channel is scaled by 2^-k when the row operand is
// built) or on the accumulators (V: they move to the class's units when a pool is entered).  Both factors of the K
// product are exact (the query is only scaled by powers of two), so a logit
//   y = log2(e)/8 * (s_k * sum_i q_i c_i + z_k * sum_i q_i)
// carries fp32 accumulation error only.  On the V side the weight w = p * s_v * G is rounded once to fp16 (half a
// step, 2^-11 relative at most: the rounding that the fp16 matrix operand forces; it is smaller than the final
// rounding of the output), G a power of two that the warp picks so that the largest weight sits at 2^13: a weight
// loses bits only when it is 2^27 times smaller than that.  The sums of p and of p * z_v stay in fp32.
//
// The softmax statistics are kept per row and warp with a lazy maximum: a logit may exceed it by 2^8 before the
// accumulators are rescaled, which one vote per tile decides.
//
// Work split: the tiles of a unit (of its four pools laid end to end, a tile weighted by its cost) are cut into
// parts * 4 equal shares, one per warp.  A warp streams its share through its own ring of bulk copies, as in the decode
// kernel; the four warps of a CTA are merged in shared memory, the CTAs of a unit (parts > 1) through global records
// by the CTA that arrives last.  Nothing waits for another CTA.
//
// Window.  Slots of a pool are handed out in position order, so a window is a suffix and the sinks a prefix of every
// pool.  Where they start follows from the per-token index: the first token of class c at or after position p names
// the slot.  One warp per class looks for it (a step reads 128 index words).  Rows of different depth have different
// window starts; they are told apart only inside the tiles at the edge.
//
// Drafted rows (the tree) are quantized at their bit-width and put back together, rounded to fp16, by the CTA of the
// last part, as fp16 tiles in shared memory that the fp16 consumer reads under a mask of ancestors.
#pragma once
#include "kvq_common.cuh"
#include "kvq_ptx.cuh"
#include "kvq_rows.h"
#include <type_traits>

namespace kvq {

constexpr int kRowsWarps = 4, kRowsThreads = kRowsWarps * 32;
constexpr int kRowsStages = 2;
constexpr int kRowsStageBytes = 4352;                  // 6 / 3 / 2 / 1 tiles of the four classes
constexpr int kRowsOutStride = kHeadDim + 4;           // floats per row of the merge buffer
constexpr int kRowsQStride = kHeadDim + 8;             // halves per row of the query block
__host__ __device__ constexpr int kRowsTps(int c) { return kRowsStageBytes / pool_rec_bytes(c); }
constexpr int kDraftTileBytes = 4096;                  // one fp16 tile: K units, then V units
// What a tile of each class costs a warp, for cutting a unit into equal shares.
__device__ constexpr uint32_t kRowsTileCost[kNumPools] = {6u, 7u, 9u, 12u};
constexpr float kWeightTop = 8192.0f;                  // the largest weight of a warp's grid choice, 2^13
constexpr float kGridStart = 1.0995116277760000e12f;   // 2^40: any weight overflows it, so the first tile picks a grid

template <int MT>
__host__ __device__ constexpr size_t rows_smem_bytes(int draft_tiles) {
    return (size_t)kRowsWarps * kRowsStages * kRowsStageBytes + (size_t)kNumPools * MT * 4 * 32 * 16 +
           (size_t)draft_tiles * kDraftTileBytes;
}
static_assert((size_t)kRowsWarps * 2 * 16 * kRowsOutStride * 4 <= (size_t)kRowsWarps * kRowsStages * kRowsStageBytes,
              "the merge buffer lives in the rings");

// ---------------------------------------------------------------- small pieces

__device__ __forceinline__ void mma_f16(float (&d)[4], const uint4& a, uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a.x), "r"(a.y), "r"(a.z), "r"(a.w), "r"(b0), "r"(b1));
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

template <int MT>
struct RowsScratch {
    uint64_t bars[kRowsWarps][kRowsStages];
    unsigned long long anc[kMaxTreeNodes];             // a node and its ancestors
    unsigned long long vis[kMaxTreeNodes];             // those of them that it sees (0: the node is not used)
    unsigned long long step_bits[kNumPools];           // class c among the 64 positions after the first window start
    unsigned long long used;                           // nodes that are used
    int seg_lo[kRowsWarps][2 * kNumPools], seg_hi[kRowsWarps][2 * kNumPools];   // tile ranges of a warp's share
    uint32_t cnt[kNumPools], sink[kNumPools], start[kNumPools];   // pool fills; slots before the sinks' end; first window slot
    uint32_t lo_row[kNumPools][16 * MT];               // first window slot of every row
    float2 ml[kRowsWarps][16 * MT];
    float sumq[16 * MT];                               // log2(e)/8 * sum_i q_i
    float wmax[kRowsWarps];
    int16_t node[16 * MT];                             // node of a row, -1 behind the last
    int8_t link[kMaxTreeNodes], bad[kMaxTreeNodes];
    uint32_t last;
    alignas(16) __half q[16 * MT][kRowsQStride];
};

// Softmax state of a warp: per lane rows g (r = 0) and g + 8 (r = 1) of every 16-row block.
template <int MT>
struct RowsState {
    float m[MT][2];                // running maximum, log2 units
    float2 l2[MT][2], b2[MT][2];   // sum of p, sum of p * zero-point, over the lane's columns (two chains)
    float acc[MT][8][4];           // output accumulators: column group (i, j) = i * 4 + j, channel 4 (column + 8 i) + j
    float grid;                    // G
};

// What the columns of a tile carry, this lane's: column group i, slots 8 i + 2 q and + 1.
struct TileCols {
    float2 sk[2], zk[2];           // scale (times the common factor of the K product) and zero-point of K
    float2 sv[2], zv[2];
};

// From the products D to the fp16 row operand of the V product.  EDGE: `seen` bit (2 i + x) of [mt][r] says whether that
// row sees that slot.
template <int MT, bool PLAIN>
__device__ __forceinline__ void weigh(RowsState<MT>& st, const float (&D)[MT][2][4], const TileCols& tc, const float (&sumq)[MT][2],
                                      bool edge, const uint32_t (&seen)[MT][2], uint4 (&w)[MT]) {
    auto logits = [&](float2 (&y)[MT][2][2], bool relative) {
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int r = 0; r < 2; ++r)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    const float base = relative ? -st.m[mt][r] : 0.f, s = sumq[mt][r];
                    const float2 t = PLAIN ? make_float2(base, base) : fma2v(tc.zk[i], make_float2(s, s), make_float2(base, base));
                    y[mt][r][i] = fma2v(make_float2(D[mt][i][2 * r], D[mt][i][2 * r + 1]), tc.sk[i], t);
                    if (edge) {
                        if (!((seen[mt][r] >> (2 * i)) & 1u)) y[mt][r][i].x = -INFINITY;
                        if (!((seen[mt][r] >> (2 * i)) & 2u)) y[mt][r][i].y = -INFINITY;
                    }
                }
    };
    auto top_of = [&](const float2 (&y)[2]) { return fmaxf(fmaxf(y[0].x, y[0].y), fmaxf(y[1].x, y[1].y)); };
    auto weights = [&](const float2 (&p)[MT][2][2]) {
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            uint32_t h[2][2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const float2 sg = PLAIN ? make_float2(st.grid, st.grid) : mul2v(tc.sv[i], make_float2(st.grid, st.grid));
#pragma unroll
                for (int r = 0; r < 2; ++r) h[r][i] = pack_half2(mul2v(p[mt][r][i], sg));
            }
            w[mt] = make_uint4(h[0][0], h[1][0], h[0][1], h[1][1]);
        }
    };
    float2 p[MT][2][2];
    logits(p, true);
    float top = top_of(p[0][0]);
    uint32_t big = 0;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            top = fmaxf(top, top_of(p[mt][r]));
#pragma unroll
            for (int i = 0; i < 2; ++i) p[mt][r][i] = make_float2(fast_exp2(p[mt][r][i].x), fast_exp2(p[mt][r][i].y));
        }
    weights(p);
    // weights are not negative, so their bit patterns are ordered; 0x7c00 and above is an overflow
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) big = __vmaxu2(__vmaxu2(big, __vmaxu2(w[mt].x, w[mt].y)), __vmaxu2(w[mt].z, w[mt].w));
    if (__builtin_expect(__any_sync(0xffffffffu, top > kRescaleSlack || ((big + 0x04000400u) & 0x80008000u)), 0)) {
        // rare: raise the maxima of all rows, choose the grid anew, do the tile again
        logits(p, false);
        float most = 0.f;
        float f[MT][2];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                float t = top_of(p[mt][r]);
                t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 1));
                t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 2));
                const float m = fmaxf(st.m[mt][r], t);
                f[mt][r] = fast_exp2(st.m[mt][r] - m);
                st.m[mt][r] = m;
                st.l2[mt][r] = mul2v(st.l2[mt][r], make_float2(f[mt][r], f[mt][r]));
                st.b2[mt][r] = mul2v(st.b2[mt][r], make_float2(f[mt][r], f[mt][r]));
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    p[mt][r][i] = make_float2(fast_exp2(p[mt][r][i].x - m), fast_exp2(p[mt][r][i].y - m));
                    const float2 v = PLAIN ? p[mt][r][i] : mul2v(p[mt][r][i], tc.sv[i]);
                    most = fmaxf(most, fmaxf(v.x, v.y));
                }
            }
        most = warp_max(most);
        // G = 2^13 / (the power of two at or below the largest weight); weights of nothing but zeros keep the grid
        float grid = st.grid;
        if (most > 0.f) grid = fminf(kWeightTop / __uint_as_float(__float_as_uint(fmaxf(most, 1e-30f)) & 0x7f800000u), kGridStart);
        const float g = grid / st.grid;                // a power of two
        st.grid = grid;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int n = 0; n < 8; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) st.acc[mt][n][e] *= f[mt][e >> 1] * g;
        weights(p);
    }
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int r = 0; r < 2; ++r)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                st.l2[mt][r] = add2v(st.l2[mt][r], p[mt][r][i]);
                if (!PLAIN) st.b2[mt][r] = fma2v(p[mt][r][i], tc.zv[i], st.b2[mt][r]);
            }
}

// ---------------------------------------------------------------- tile consumers (lane = 4 g + q)

// A quantized class.  kw / vw: words of the fragment layout (see kvq_common.cuh).
template <int CLS>
struct RowsQuant {
    static constexpr int BITS = pool_bits(CLS), REC = pool_rec_bytes(CLS);
    static constexpr int NW = 2 << CLS;                // words per lane of one tensor: 2, 4, 8
    static constexpr uint32_t MASK = CLS == 0 ? 0x00030003u : CLS == 1 ? 0x000f000fu : 0x00ff00ffu;

    // Register r of step s of the K product: channel of 16-bit lane x, and the bit its field is cut out at.
    __device__ static constexpr int k_channel(int s, int r, int q, int x) {
        return CLS == 0   ? 16 * q + (2 * s + r) + 8 * x
               : CLS == 1 ? 8 * (q + 4 * (s >> 1)) + 2 * (s & 1) + r + 4 * x
                          : 4 * (q + 4 * s) + r + 2 * x;
    }
    __device__ static constexpr int k_bit(int s, int r) {
        return CLS == 0 ? 2 * ((2 * s + r) & 3) : CLS == 1 ? 4 * r : 0;
    }
    // The column operand of slot g + 8 i for step s, register r.
    __device__ static __forceinline__ uint32_t k_operand(const uint32_t (&kw)[NW], int i, int s, int r) {
        if (CLS == 0) {
            const int e = 2 * s + r;
            return (e < 4 ? kw[i] : kw[i] >> 8) & (MASK << (2 * (e & 3)));
        }
        if (CLS == 1) {
            const uint32_t w = kw[(s >> 1) * 2 + i];
            return ((s & 1) ? w >> 8 : w) & (MASK << (4 * r));
        }
        const uint32_t w = kw[s * 2 + i];
        return r ? (w >> 8) & MASK : w & MASK;
    }
    // Bit of the V field of column group (i, j).
    __device__ static constexpr int v_bit(int j) { return CLS == 0 ? 2 * j : CLS == 1 ? 4 * (j & 1) : 0; }

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

    template <int MT>
    __device__ static __forceinline__ void tile(const uint8_t* rec, int lane, const uint4 (&qf)[MT][4], float kfactor,
                                                const float (&sumq)[MT][2], RowsState<MT>& st, bool edge,
                                                const uint32_t (&seen)[MT][2], uint32_t) {
        const int g = lane >> 2, q = lane & 3;
        uint32_t kw[NW];
        load_words(rec, lane, kw);
        TileCols tc;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const uint2 km = *reinterpret_cast<const uint2*>(rec + meta_offset(CLS, 0, 8 * i + 2 * q));
            const uint2 vm = *reinterpret_cast<const uint2*>(rec + meta_offset(CLS, 1, 8 * i + 2 * q));
            const float2 k0 = unpack_half2(km.x), k1 = unpack_half2(km.y), v0 = unpack_half2(vm.x), v1 = unpack_half2(vm.y);
            tc.sk[i] = mul2v(make_float2(k0.x, k1.x), make_float2(kfactor, kfactor));
            tc.zk[i] = make_float2(k0.y, k1.y);
            tc.sv[i] = make_float2(v0.x, v1.x);
            tc.zv[i] = make_float2(v0.y, v1.y);
        }
        float D[MT][2][4];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int i = 0; i < 2; ++i) D[mt][i][0] = D[mt][i][1] = D[mt][i][2] = D[mt][i][3] = 0.f;
#pragma unroll
        for (int s = 0; s < 4; ++s)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const uint32_t b0 = k_operand(kw, i, s, 0), b1 = k_operand(kw, i, s, 1);
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) mma_f16(D[mt][i], qf[mt][s], b0, b1);
            }
        // V words of slots 2q, 2q + 1 (a) and 8 + 2q, 9 + 2q (b): halves of the words of slot quads q >> 1 and 2 + (q >> 1)
        uint32_t va[NW], vb[NW];
        load_words(rec + pool_codes_bytes(CLS), 4 * g + (q >> 1), va);
        load_words(rec + pool_codes_bytes(CLS), 4 * g + 2 + (q >> 1), vb);
        uint4 w[MT];
        weigh<MT, false>(st, D, tc, sumq, edge, seen, w);
        const uint32_t sel = (q & 1) ? 0x4342u : 0x4140u;
#pragma unroll
        for (int k = 0; k < NW; ++k) {                 // word k: CLS 0: i = k; CLS 1, 2: (byte of the group) * 2 + i
            const uint32_t xa = prmt(va[k], 0u, sel), xb = prmt(vb[k], 0u, sel);
            const int i = CLS == 0 ? k : k & 1, byte = CLS == 0 ? 0 : k >> 1;
            constexpr int PER = 8 / BITS;              // channels per byte
#pragma unroll
            for (int f = 0; f < PER; ++f) {
                const int n = i * 4 + byte * PER + f;
                const uint32_t b0 = PER == 1 ? xa : xa & (MASK << (BITS * f)), b1 = PER == 1 ? xb : xb & (MASK << (BITS * f));
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) mma_f16(st.acc[mt][n], w[mt], b0, b1);
            }
        }
    }
};

// fp16 rows: the fp16 pool, and the drafted tokens.  valid: bit (2 i + x) says that the lane's slot holds a row (the
// bytes of other slots may be anything, an Inf or NaN pattern included).
struct RowsFp16 {
    static constexpr int REC = pool_rec_bytes(3);
    __device__ static constexpr int k_channel(int s, int r, int q, int x) { return 8 * (2 * s + r) + 2 * q + x; }

    template <int MT>
    __device__ static __forceinline__ void tile(const uint8_t* rec, int lane, const uint4 (&qf)[MT][4], float kfactor,
                                                const float (&sumq)[MT][2], RowsState<MT>& st, bool edge,
                                                const uint32_t (&seen)[MT][2], uint32_t valid) {
        const int g = lane >> 2, q = lane & 3;
        float D[MT][2][4];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int i = 0; i < 2; ++i) D[mt][i][0] = D[mt][i][1] = D[mt][i][2] = D[mt][i][3] = 0.f;
        const int row = lane & 7, mat = lane >> 3;
#pragma unroll
        for (int s = 0; s < 4; ++s) {                  // four 8x8 matrices: (unit 2s, 2s + 1) x (slots 0..7, 8..15)
            uint32_t b[4];
            ldsm_x4(b, rec + ((2 * s + (mat & 1)) * kTileTokens + 8 * (mat >> 1) + row) * 16);
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) mma_f16(D[mt][i], qf[mt][s], b[2 * i], b[2 * i + 1]);
        }
        TileCols tc;
        tc.sk[0] = tc.sk[1] = make_float2(kfactor, kfactor);
        uint4 w[MT];
        weigh<MT, true>(st, D, tc, sumq, edge, seen, w);
        const uint8_t* v = rec + pool_codes_bytes(3) + (g >> 1) * kTileTokens * 16 + (g & 1) * 8;
#pragma unroll
        for (int i = 0; i < 2; ++i) {                  // channels 32 i + 4 g .. + 3 of the lane's four slots
            uint2 x[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int slot = 2 * q + (k & 1) + 8 * (k >> 1);
                x[k] = *reinterpret_cast<const uint2*>(v + (i * 4 * kTileTokens + slot) * 16);
                if (edge && !((valid >> k) & 1u)) x[k] = make_uint2(0u, 0u);
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t sel = (j & 1) ? 0x7632u : 0x5410u;
                const uint32_t b0 = j < 2 ? prmt(x[0].x, x[1].x, sel) : prmt(x[0].y, x[1].y, sel);
                const uint32_t b1 = j < 2 ? prmt(x[2].x, x[3].x, sel) : prmt(x[2].y, x[3].y, sel);
#pragma unroll
                for (int mt = 0; mt < MT; ++mt) mma_f16(st.acc[mt][i * 4 + j], w[mt], b0, b1);
            }
        }
    }
};

// ---------------------------------------------------------------- the kernel

// One drafted row, eight channels per lane of an eight-lane group, as the store would give it back (the row quantizer of
// Eq. 24, then code * scale + zero-point), rounded to fp16.
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

// grid = batch * kv_heads * parts * row_blocks, block = kRowsThreads, dynamic smem = rows_smem_bytes<MT>(draft tiles).
// MT: 16-row blocks per unit.  TREE: rows belong to drafted nodes (otherwise nodes == 1 and the row is the last
// cached token's).
template <int MT, bool TREE>
__global__ void __launch_bounds__(kRowsThreads, MT == 1 ? 4 : 2) k_attend_rows(const RowsParams P) {
    constexpr int ROWS = 16 * MT;
    extern __shared__ __align__(128) uint8_t dyn[];
    __shared__ RowsScratch<MT> sc;
    uint8_t* const rings = dyn;
    uint4* const qfrag = reinterpret_cast<uint4*>(dyn + (size_t)kRowsWarps * kRowsStages * kRowsStageBytes);   // [class][MT][4][32]
    uint8_t* const draft = reinterpret_cast<uint8_t*>(qfrag + kNumPools * MT * 4 * 32);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, q = lane & 3;
    const StoreView& S = P.store;

    uint32_t x = blockIdx.x;
    const uint32_t rb = x % P.row_blocks;
    x /= P.row_blocks;
    const uint32_t part = x % P.parts, bh = x / P.parts;
    const int b = (int)(bh / (uint32_t)S.kv_heads), h = (int)(bh - (uint32_t)b * S.kv_heads);
    const uint32_t unit = bh * P.row_blocks + rb;
    const bool has_draft = TREE && part + 1 == P.parts;
    const int draft_tiles = (P.nodes + kTileTokens - 1) / kTileTokens;

    if (lane == 0) {
        for (int s = 0; s < kRowsStages; ++s) mbar_init(&sc.bars[warp][s], 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    pdl_launch_dependents();
    pdl_wait();                                        // an append ahead of this launch has stored its tokens

    const uint4 fill = *reinterpret_cast<const uint4*>(P.counts + (size_t)b * 4);
    const int len = (int)(fill.x + fill.y + fill.z + fill.w);

    // ---- the query block
    float qmax = 0.f;
#pragma unroll
    for (int k = 0; k < MT; ++k) {
        const int row = 16 * k + (tid >> 3), piece = tid & 7;
        const int R = (int)rb * ROWS + row;
        const int node = R / P.group;
        uint4 v = make_uint4(0u, 0u, 0u, 0u);
        if (R < P.rows)
            v = *reinterpret_cast<const uint4*>(P.Q + (((size_t)b * P.nodes + node) * S.q_heads + (size_t)h * P.group + (R - node * P.group)) * kHeadDim + piece * 8);
        *reinterpret_cast<uint4*>(&sc.q[row][piece * 8]) = v;
        const float2 f0 = unpack_half2(v.x), f1 = unpack_half2(v.y), f2 = unpack_half2(v.z), f3 = unpack_half2(v.w);
        float sum = ((f0.x + f0.y) + (f1.x + f1.y)) + ((f2.x + f2.y) + (f3.x + f3.y));
        qmax = fmaxf(qmax, fmaxf(fmaxf(fmaxf(fabsf(f0.x), fabsf(f0.y)), fmaxf(fabsf(f1.x), fabsf(f1.y))),
                                 fmaxf(fmaxf(fabsf(f2.x), fabsf(f2.y)), fmaxf(fabsf(f3.x), fabsf(f3.y)))));
#pragma unroll
        for (int d = 1; d < 8; d <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
        if (piece == 0) {
            sc.sumq[row] = sum * kLogitScale;
            sc.node[row] = (int16_t)(R < P.rows ? node : -1);
        }
    }
    qmax = warp_max(qmax);
    if (lane == 0) sc.wmax[warp] = qmax;

    // ---- the tree: ancestors by doubling the chain of parents
    if (TREE && warp == 0) {
        unsigned long long a[2];
        int bad[2], link[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int i = lane + 32 * k;
            const int par = i < P.nodes ? P.parents[(size_t)b * P.nodes + i] : -2;
            bad[k] = !(par >= -1 && par < i);
            link[k] = bad[k] ? -1 : par;
            a[k] = 1ull << i;
            sc.anc[i] = a[k];
            sc.link[i] = (int8_t)link[k];
            sc.bad[i] = (int8_t)bad[k];
        }
        for (int round = 0; round < 6; ++round) {
            __syncwarp();
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
    // ---- the window: where it and the sinks end in every pool (warp = class)
    int base0 = 0;                                     // first position that the shallowest row's window holds
    if (P.window > 0) base0 = min(max(len - P.window + (TREE ? 1 : 0), 0), len);
    {
        const uint32_t c = (uint32_t)warp;
        const uint32_t n = c == 0 ? fill.x : c == 1 ? fill.y : c == 2 ? fill.z : fill.w;
        uint32_t start = 0, sink = 0;
        unsigned long long bits = 0;
        if (P.window > 0) {
            const uint32_t* idx = S.index + ((size_t)P.layer * S.batch + b) * S.max_ctx;
            start = first_slot_from(idx, base0, len, c, n, lane);
            sink = P.sinks > 0 ? first_slot_from(idx, min(P.sinks, len), len, c, n, lane) : 0u;
            if (TREE) {
                uint32_t m[2];
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const int at = base0 + 32 * k + lane;
                    m[k] = __ballot_sync(0xffffffffu, at < len && (idx[min(at, len - 1)] >> 30) == c);
                }
                bits = ((unsigned long long)m[1] << 32) | m[0];
            }
        }
        if (lane == 0) {
            sc.cnt[c] = n;
            sc.start[c] = start;
            sc.sink[c] = sink;
            sc.step_bits[c] = bits;
        }
    }
    // ---- drafted rows as fp16 tiles
    if (has_draft) {
        const int padded = draft_tiles * kTileTokens;
        for (int k = 0; k < 2 * padded; k += kRowsThreads / 8) {
            const int i = k + (tid >> 3), piece = tid & 7;
            const bool value = i >= padded;
            const int node = value ? i - padded : i;
            uint4 raw = make_uint4(0u, 0u, 0u, 0u);
            int c = 3;
            if (node < P.nodes) {
                raw = *reinterpret_cast<const uint4*>((value ? P.V : P.K) + (((size_t)b * P.nodes + node) * S.kv_heads + h) * kHeadDim + piece * 8);
                if (P.bits) {
                    c = bits_to_class(P.bits[(size_t)b * P.nodes + node]);
                    if (c < 0) {                       // as in an append: kept as fp16, and flagged
                        atomicOr(S.flags, 1u);
                        c = 3;
                    }
                }
            }
            const uint4 row = draft_row_as_stored(raw, c);
            *reinterpret_cast<uint4*>(draft + (node / kTileTokens) * kDraftTileBytes + (value ? kDraftTileBytes / 2 : 0) +
                                      (piece * kTileTokens + node % kTileTokens) * 16) = row;
        }
    }
    __syncthreads();

    // ---- first window slot of every row, per class
    if (P.window > 0)
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
    // ---- this warp's share: tile ranges of the pools, laid end to end [sinks | window] per pool
    if (lane < kNumPools) {
        const int c = lane;
        const int nt = (int)((sc.cnt[c] + kTileTokens - 1) / kTileTokens);
        int ns = (int)((sc.sink[c] + kTileTokens - 1) / kTileTokens), ws = (int)(sc.start[c] / kTileTokens);
        if (ws <= ns) ns = ws = 0;                     // no gap
        const uint32_t n = (uint32_t)(ns + nt - ws), cost = kRowsTileCost[c];
        uint32_t before = 0, total = 0;
#pragma unroll
        for (int k = 0; k < kNumPools; ++k) {
            const uint32_t wk = __shfl_sync(0xfu, n * cost, k);
            before += k < c ? wk : 0u;
            total += wk;
        }
        const uint32_t shares = P.parts * kRowsWarps, me = part * kRowsWarps + warp;
        const long long r0 = (long long)((unsigned long long)total * me / shares) - before;
        const long long r1 = (long long)((unsigned long long)total * (me + 1) / shares) - before;
        // the same rounding for a share's end and the next one's start
        const int lo = (int)min(max(r0, 0ll) / cost, (long long)n);
        const int hi = me + 1 == shares ? (int)n : (int)min(max(r1, 0ll) / cost, (long long)n);
        sc.seg_lo[warp][2 * c] = lo;
        sc.seg_hi[warp][2 * c] = min(hi, ns);
        sc.seg_lo[warp][2 * c + 1] = max(lo, ns) - ns + ws;
        sc.seg_hi[warp][2 * c + 1] = hi - ns + ws;
    }
    __syncwarp();

    // ---- producer: the chunks of the share in order; a chunk stays inside one 64 KB block and fits a stage
    uint8_t* const ring = rings + (size_t)warp * kRowsStages * kRowsStageBytes;
    int p_seg = -1, p_left = 0, p_tps = 0, p_bt = 0, p_block_left = 0;
    uint32_t p_rec = 0, p_next = 0;
    const uint8_t* p_ptr = nullptr;
    const uint32_t* p_tab = nullptr;                   // entry of the block after the current one
    auto next_segment = [&]() {
        while (p_left <= 0 && ++p_seg < 2 * kNumPools) {
            const int lo = sc.seg_lo[warp][p_seg], c = p_seg >> 1;
            p_left = sc.seg_hi[warp][p_seg] - lo;
            if (p_left <= 0) continue;
            p_rec = (uint32_t)(c == 0 ? pool_rec_bytes(0) : c == 1 ? pool_rec_bytes(1) : c == 2 ? pool_rec_bytes(2) : pool_rec_bytes(3));
            p_tps = c == 0 ? kRowsTps(0) : c == 1 ? kRowsTps(1) : c == 2 ? kRowsTps(2) : kRowsTps(3);
            p_bt = (int)block_tiles(c);
            const int blk = lo / p_bt, ib = lo - blk * p_bt;
            p_tab = stream_table(S, c, P.layer, b, h) + blk;
            p_ptr = S.arena + (size_t)p_tab[0] * kBlockBytes + (size_t)ib * p_rec;
            ++p_tab;
            p_block_left = p_bt - ib;
            if (p_left > p_block_left) p_next = p_tab[0];
        }
    };
    next_segment();
    int pslot = 0, cslot = 0, in_flight = 0;
    uint32_t parity = 0;
    bool failed = false;
    auto issue = [&]() {
        const int n = min(min(p_tps, p_block_left), p_left);
        const uint32_t bytes = (uint32_t)n * p_rec;
        if (lane == 0) {
            mbar_arrive_expect_tx(&sc.bars[warp][pslot], bytes);
            bulk_load(ring + (size_t)pslot * kRowsStageBytes, p_ptr, bytes, &sc.bars[warp][pslot]);
        }
        pslot = pslot + 1 == kRowsStages ? 0 : pslot + 1;
        p_ptr += bytes;
        p_left -= n;
        p_block_left -= n;
        if (p_left == 0) {
            next_segment();
        } else if (p_block_left == 0) {                // on to the stream's next block
            p_ptr = S.arena + (size_t)p_next * kBlockBytes;
            p_block_left = p_bt;
            ++p_tab;
            if (p_left > p_bt) p_next = p_tab[0];
        }
    };
    for (; in_flight < kRowsStages && p_left > 0; ++in_flight) issue();

    // ---- row operands of the K product, one set per class (warp = class): q * F * 2^-k, F a power of two that puts the
    // block's largest query value below 2^15
    const float block_max = fmaxf(fmaxf(fmaxf(sc.wmax[0], sc.wmax[1]), fmaxf(sc.wmax[2], sc.wmax[3])), 6.103515625e-05f);
    const int e_max = (int)(__float_as_uint(block_max) >> 23) - 127;           // -14 .. 15
    const float F = two_to(14 - e_max);
    {
        auto build = [&](auto channel, auto bit) {
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                for (int s = 0; s < 4; ++s) {
                    uint32_t a[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) {      // a0: row g, r = 0; a1: row g + 8, r = 0; a2, a3: r = 1
                        const int r = k >> 1;
                        const __half* row = sc.q[16 * mt + g + 8 * (k & 1)];
                        const float f = F * two_to(-bit(s, r));
                        a[k] = pack_half2(make_float2(__half2float(row[channel(s, r, q, 0)]) * f, __half2float(row[channel(s, r, q, 1)]) * f));
                    }
                    qfrag[((warp * MT + mt) * 4 + s) * 32 + lane] = make_uint4(a[0], a[1], a[2], a[3]);
                }
        };
        if (warp == 0) build(RowsQuant<0>::k_channel, RowsQuant<0>::k_bit);
        else if (warp == 1) build(RowsQuant<1>::k_channel, RowsQuant<1>::k_bit);
        else if (warp == 2) build(RowsQuant<2>::k_channel, RowsQuant<2>::k_bit);
        else build(RowsFp16::k_channel, [](int, int) { return 0; });
    }
    __syncthreads();

    // ---- the walk
    RowsState<MT> st;
    float sumq[MT][2];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            st.m[mt][r] = kNegBig;
            st.l2[mt][r] = st.b2[mt][r] = make_float2(0.f, 0.f);
            sumq[mt][r] = sc.sumq[16 * mt + g + 8 * r];
        }
#pragma unroll
        for (int n = 0; n < 8; ++n) st.acc[mt][n][0] = st.acc[mt][n][1] = st.acc[mt][n][2] = st.acc[mt][n][3] = 0.f;
    }
    st.grid = kGridStart;

    auto load_queries = [&](int c, uint4 (&qf)[MT][4]) {
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int s = 0; s < 4; ++s) qf[mt][s] = qfrag[((c * MT + mt) * 4 + s) * 32 + lane];
    };
    auto scale_acc = [&](auto factor) {                // per column group j
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int n = 0; n < 8; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) st.acc[mt][n][e] *= factor(n & 3);
    };
    auto walk = [&](auto cls_tag, auto consumer) {
        constexpr int CLS = decltype(cls_tag)::value;
        using C = decltype(consumer);
        constexpr int TPS = kRowsTps(CLS), BT = (int)block_tiles(CLS);
        if (sc.seg_lo[warp][2 * CLS] >= sc.seg_hi[warp][2 * CLS] && sc.seg_lo[warp][2 * CLS + 1] >= sc.seg_hi[warp][2 * CLS + 1]) return;
        uint4 qf[MT][4];
        load_queries(CLS, qf);
        const float kfactor = kLogitScale * (CLS == 3 ? 1.0f : 16777216.0f) / F;
        if constexpr (CLS < 3) scale_acc([](int j) { return two_to(RowsQuant<CLS == 3 ? 0 : CLS>::v_bit(j) - 24); });
        const uint32_t cnt = sc.cnt[CLS], sink = sc.sink[CLS];
        const uint32_t lo_last = P.window > 0 ? sc.start[CLS] + (TREE ? (uint32_t)__popcll(sc.step_bits[CLS]) : 0u) : 0u;
#pragma unroll 1
        for (int part_of_pool = 0; part_of_pool < 2; ++part_of_pool) {
            int tile0 = sc.seg_lo[warp][2 * CLS + part_of_pool];
            const int hi = sc.seg_hi[warp][2 * CLS + part_of_pool];
            int block_left = BT - tile0 % BT;
            while (tile0 < hi && !failed) {
                failed = !__all_sync(0xffffffffu, mbar_wait(&sc.bars[warp][cslot], (parity >> cslot) & 1u));
                if (failed) break;
                const int n = min(min(TPS, block_left), hi - tile0);
                const uint8_t* buf = ring + (size_t)cslot * kRowsStageBytes;
#pragma unroll 1
                for (int i = 0; i < n; ++i) {
                    const uint32_t s0 = (uint32_t)(tile0 + i) * kTileTokens;
                    uint32_t seen[MT][2], valid = 0;
                    // at an edge: the pool's last tile, or one where the window starts or the sinks end
                    const bool edge = s0 + kTileTokens > cnt || (s0 < lo_last && s0 + kTileTokens > sink);
                    if (edge) {
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            const uint32_t slot = s0 + 8 * (k >> 1) + 2 * q + (k & 1);
                            valid |= slot < cnt ? 1u << k : 0u;
                        }
#pragma unroll
                        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                            for (int r = 0; r < 2; ++r) {
                                const uint32_t lo = P.window > 0 ? sc.lo_row[CLS][16 * mt + g + 8 * r] : 0u;
                                seen[mt][r] = 0;
#pragma unroll
                                for (int k = 0; k < 4; ++k) {
                                    const uint32_t slot = s0 + 8 * (k >> 1) + 2 * q + (k & 1);
                                    seen[mt][r] |= slot >= lo || slot < sink ? 1u << k : 0u;
                                }
                                seen[mt][r] &= valid;
                            }
                    }
                    C::template tile<MT>(buf + (size_t)i * C::REC, lane, qf, kfactor, sumq, st, edge, seen, valid);
                }
                tile0 += n;
                block_left -= n;
                if (block_left == 0) block_left = BT;
                --in_flight;
                __syncwarp();                          // every lane is done with the stage before it is refilled
                if (p_left > 0) {
                    issue();
                    ++in_flight;
                }
                parity ^= 1u << cslot;
                cslot = cslot + 1 == kRowsStages ? 0 : cslot + 1;
            }
        }
        if constexpr (CLS < 3) scale_acc([](int j) { return two_to(24 - RowsQuant<CLS == 3 ? 0 : CLS>::v_bit(j)); });
    };
    walk(std::integral_constant<int, 0>{}, RowsQuant<0>{});
    walk(std::integral_constant<int, 1>{}, RowsQuant<1>{});
    walk(std::integral_constant<int, 2>{}, RowsQuant<2>{});
    walk(std::integral_constant<int, 3>{}, RowsFp16{});
    if (has_draft && warp < draft_tiles) {             // a tile of drafted tokens per warp, under the mask of ancestors
        uint4 qf[MT][4];
        load_queries(3, qf);
        const uint32_t use = (uint32_t)(sc.used >> (16 * warp));
        const uint32_t valid = ((use >> (2 * q)) & 3u) | (((use >> (8 + 2 * q)) & 3u) << 2);
        uint32_t seen[MT][2];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const int node = sc.node[16 * mt + g + 8 * r];
                const uint32_t v = node >= 0 ? (uint32_t)(sc.vis[node] >> (16 * warp)) : 0u;
                seen[mt][r] = ((v >> (2 * q)) & 3u) | (((v >> (8 + 2 * q)) & 3u) << 2);
            }
        RowsFp16::tile<MT>(draft + (size_t)warp * kDraftTileBytes, lane, qf, kLogitScale / F, sumq, st, true, seen, valid);
    }
    if (failed) {                                      // give up: no further copy; those in flight are let land first
        if (lane == 0) atomicOr(S.flags, kFlagWaitTimeout);
        while (in_flight > 0) {
            mbar_wait(&sc.bars[warp][cslot], (parity >> cslot) & 1u);
            parity ^= 1u << cslot;
            cslot = cslot + 1 == kRowsStages ? 0 : cslot + 1;
            --in_flight;
        }
    }

    // ---- merge the four warps: M = max m_w, l = sum l_w 2^(m_w - M), O = sum o_w 2^(m_w - M)
    float bsum[MT][2];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            float l = st.l2[mt][r].x + st.l2[mt][r].y, z = st.b2[mt][r].x + st.b2[mt][r].y;
#pragma unroll
            for (int d = 1; d < 4; d <<= 1) {
                l += __shfl_xor_sync(0xffffffffu, l, d);
                z += __shfl_xor_sync(0xffffffffu, z, d);
            }
            bsum[mt][r] = z;
            if (q == 0) sc.ml[warp][16 * mt + g + 8 * r] = make_float2(st.m[mt][r], l);
        }
    __syncthreads();                                   // also: every warp is done with its ring, which becomes the merge buffer
    float* const out = reinterpret_cast<float*>(rings);             // [warps][ROWS][kRowsOutStride]
    const float ungrid = 1.0f / st.grid;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            const int row = 16 * mt + g + 8 * r;
            float M = kNegBig;
#pragma unroll
            for (int k = 0; k < kRowsWarps; ++k) M = fmaxf(M, sc.ml[k][row].x);
            const float f = fast_exp2(st.m[mt][r] - M), fg = f * ungrid, fb = f * bsum[mt][r];
            float* dst = out + ((size_t)warp * ROWS + row) * kRowsOutStride;
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int e = 0; e < 2; ++e) {          // column 2q + e of the groups (i, 0..3): channels 4 (2q + e + 8i) ..
                    const float4 v = make_float4(fmaf(st.acc[mt][4 * i][2 * r + e], fg, fb), fmaf(st.acc[mt][4 * i + 1][2 * r + e], fg, fb),
                                                 fmaf(st.acc[mt][4 * i + 2][2 * r + e], fg, fb), fmaf(st.acc[mt][4 * i + 3][2 * r + e], fg, fb));
                    *reinterpret_cast<float4*>(dst + 4 * (2 * q + e + 8 * i)) = v;
                }
        }
    __syncthreads();

    // ---- this CTA's rows: thread = (row, eight channels)
    auto store_row = [&](int row, const float (&o)[8], float L) {
        const int R = (int)rb * ROWS + row;
        if (R >= P.rows) return;
        const int node = R / P.group;
        const float inv = L > 0.f && (!TREE || sc.vis[node]) ? 1.0f / L : 0.f;     // nothing seen, or an unused node: zeros
        uint32_t v[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = inv != 0.f ? pack_half2(make_float2(o[2 * k] * inv, o[2 * k + 1] * inv)) : 0u;
        *reinterpret_cast<uint4*>(P.O + (((size_t)b * P.nodes + node) * S.q_heads + (size_t)h * P.group + (R - node * P.group)) * kHeadDim + (tid & 7) * 8) =
            make_uint4(v[0], v[1], v[2], v[3]);
    };
#pragma unroll
    for (int k = 0; k < MT; ++k) {
        const int row = 16 * k + (tid >> 3);
        float o[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        float M = kNegBig, L = 0.f;
#pragma unroll
        for (int w = 0; w < kRowsWarps; ++w) M = fmaxf(M, sc.ml[w][row].x);
#pragma unroll
        for (int w = 0; w < kRowsWarps; ++w) {
            L = fmaf(sc.ml[w][row].y, fast_exp2(sc.ml[w][row].x - M), L);
            const float4* src = reinterpret_cast<const float4*>(out + ((size_t)w * ROWS + row) * kRowsOutStride + (tid & 7) * 8);
            const float4 v0 = src[0], v1 = src[1];
            o[0] += v0.x; o[1] += v0.y; o[2] += v0.z; o[3] += v0.w;
            o[4] += v1.x; o[5] += v1.y; o[6] += v1.z; o[7] += v1.w;
        }
        if (P.parts == 1) {
            store_row(row, o, L);
        } else {
            const size_t rec = ((size_t)unit * P.parts + part) * ROWS + row;
            float4* dst = reinterpret_cast<float4*>(P.part_o + rec * kHeadDim + (tid & 7) * 8);
            dst[0] = make_float4(o[0], o[1], o[2], o[3]);
            dst[1] = make_float4(o[4], o[5], o[6], o[7]);
            if ((tid & 7) == 0) P.part_ml[rec] = make_float2(M, L);
        }
    }
    if (P.parts == 1) return;

    // ---- the CTA that delivers the unit's last part merges the parts, in part order
    __threadfence();
    __syncthreads();
    if (tid == 0) sc.last = atomicAdd(P.part_cnt + unit, 1u) + 1u == P.parts ? 1u : 0u;
    __syncthreads();
    if (!sc.last) return;
    __threadfence();
    if (tid == 0) P.part_cnt[unit] = 0u;
#pragma unroll
    for (int k = 0; k < MT; ++k) {
        const int row = 16 * k + (tid >> 3);
        const size_t rec0 = (size_t)unit * P.parts * ROWS + row;
        float M = kNegBig, L = 0.f;
        for (uint32_t s = 0; s < P.parts; ++s) M = fmaxf(M, __ldcg(P.part_ml + rec0 + (size_t)s * ROWS).x);
        float o[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
        for (uint32_t s = 0; s < P.parts; ++s) {
            const size_t rec = rec0 + (size_t)s * ROWS;
            const float2 ml = __ldcg(P.part_ml + rec);
            const float4* src = reinterpret_cast<const float4*>(P.part_o + rec * kHeadDim + (tid & 7) * 8);
            const float4 v0 = __ldcg(src), v1 = __ldcg(src + 1);
            const float f = fast_exp2(ml.x - M);
            L = fmaf(ml.y, f, L);
            o[0] = fmaf(v0.x, f, o[0]); o[1] = fmaf(v0.y, f, o[1]); o[2] = fmaf(v0.z, f, o[2]); o[3] = fmaf(v0.w, f, o[3]);
            o[4] = fmaf(v1.x, f, o[4]); o[5] = fmaf(v1.y, f, o[5]); o[6] = fmaf(v1.z, f, o[6]); o[7] = fmaf(v1.w, f, o[7]);
        }
        store_row(row, o, L);
    }
}

}  // namespace kvq
