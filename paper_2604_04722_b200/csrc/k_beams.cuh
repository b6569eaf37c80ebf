// One step of beam search: of all candidates (beam w, token v) with the score  s_w + z_wv - log sum_u exp(z_wu)  the n best,
// ties to the lowest (w, v).
//
// A cluster of CTAs serves a request.  Every row is cut into slices, one warp each; the cut does not depend on the row or its
// address, so that equal rows have equal sums and tie as they should.  Reading its slice, a warp keeps nothing but the sum of
// exponentials (fp32 within 16 entries of a lane, fp64 beyond: what is compared between beams must not depend on their order)
// and the largest entry of every group of chunks: one exponential, a maximum and two or three more instructions per logit.
//
// The slices' sums are exchanged (a cluster barrier).  Then the scores of the groups' largest entries are known, and the n-th
// best of a CTA's bounds its n best candidates from below: only groups whose largest entry reaches it are read again, and of
// those only the entries that reach it are kept, a few more than n in all.  A CTA ranks its own, sends its n best to the first
// CTA (a second barrier), and that ranks them.  Scores are compared in fp64.
//
// Bound: of many requests instructions and the barriers between the phases: 64 requests of 16 beams over 32000 bf16 logits take 25.5 us,
// the bytes alone 10; over 32003, where rows are not aligned and every load becomes two, 32, of which the loop over the logits is 17 (five to six
// instructions a logit; with what lies behind it 20, issue slots half busy).  Of few requests the chain of the rows' loads, two cluster barriers, the bound, a second read and two rankings: 9.1 us for
// one request of 4 beams over 49152 logits.  Keeping the slices' best entries in the first pass took 94 us where this takes 32.
#pragma once
#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <cfloat>
#include <type_traits>
#include "kvq_common.cuh"
#include "kvq_pages.h"
#include "kvq_ptx.cuh"

namespace kvq {

constexpr int kBeamThreads = 512, kBeamWarps = kBeamThreads / 32;
constexpr int kBeamMaxCluster = 16;
constexpr int kBeamChunk = 512;                        // entries that a warp works on at a time, 16 per lane
constexpr int kBeamBuffer = 128;                       // entries of a warp's buffer, 4 per lane: at least n + 32
constexpr int kBeamRounds = 2;                         // slices of a warp at most: where there are more rows than warps
static_assert(kMaxBeams <= kBeamRounds * kBeamWarps, "every row has its warp");
constexpr int kBeamMaxSlices = kBeamMaxCluster * kBeamWarps;
constexpr int kBeamGroups = 16;                        // groups of chunks of a warp's slices at most
constexpr float kBeamLowest = -FLT_MAX;
constexpr float kBeamSlack = 4.f;                      // how far a lane's entries may pass the one that its sum is relative to

// Order-preserving keys of scores (-0 counts as 0); none is 0 or the largest number.
__device__ __forceinline__ uint64_t score_key(double x) {
    const uint64_t b = (uint64_t)__double_as_longlong(x + 0.0);
    return b >> 63 ? ~b : b | (1ull << 63);
}
__device__ __forceinline__ double key_score(uint64_t k) {
    return __longlong_as_double((long long)(k >> 63 ? k ^ (1ull << 63) : ~k));
}

// A candidate: its score (score_key; 0: none) and its place.
struct BeamPick {
    uint64_t score;
    uint32_t row, token;
    __device__ bool before(const BeamPick& o) const {
        return score != o.score ? score > o.score : row != o.row ? row < o.row : token < o.token;
    }
};
__device__ __forceinline__ BeamPick no_pick() { return BeamPick{0, 0xffffffffu, 0xffffffffu}; }

// Dynamic shared memory: the warps' buffers, the CTA's picks and, in the first CTA, those of all CTAs.
inline size_t beam_smem(int n) { return ((size_t)kBeamWarps * kBeamBuffer + kBeamThreads + (size_t)kBeamMaxCluster * n) * sizeof(BeamPick); }

// Cuts a warp's buffer back to its n best entries, in order; it holds n or more.
__device__ __noinline__ void warp_best(BeamPick* buffer, int count, int n) {
    const int lane = threadIdx.x & 31;
    BeamPick e[kBeamBuffer / 32];
#pragma unroll
    for (int k = 0; k < kBeamBuffer / 32; ++k) e[k] = lane + 32 * k < count ? buffer[lane + 32 * k] : no_pick();
    __syncwarp();
#pragma unroll 1
    for (int i = 0; i < n; ++i) {
        BeamPick best = e[0];
#pragma unroll
        for (int k = 1; k < kBeamBuffer / 32; ++k)
            if (e[k].before(best)) best = e[k];
        const uint32_t hi = __reduce_max_sync(0xffffffffu, (uint32_t)(best.score >> 32));
        bool in = (uint32_t)(best.score >> 32) == hi;
        const uint32_t lo = __reduce_max_sync(0xffffffffu, in ? (uint32_t)best.score : 0u);
        in = in && (uint32_t)best.score == lo;
        const uint32_t row = __reduce_min_sync(0xffffffffu, in ? best.row : 0xffffffffu);
        in = in && best.row == row;
        const uint32_t token = __reduce_min_sync(0xffffffffu, in ? best.token : 0xffffffffu);
        in = in && best.token == token;
#pragma unroll
        for (int k = 0; k < kBeamBuffer / 32; ++k)
            if (in && e[k].row == row && e[k].token == token) e[k] = no_pick();
        if (lane == 0) buffer[i] = BeamPick{((uint64_t)hi << 32) | lo, row, token};
    }
    __syncwarp();
}

// The n-th largest of the lanes' numbers: a bitonic sort, descending.
__device__ __forceinline__ float warp_nth(float v, int n) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int size = 2; size <= 32; size <<= 1)
#pragma unroll
        for (int d = size >> 1; d > 0; d >>= 1) {
            const float o = __shfl_xor_sync(0xffffffffu, v, d);
            v = ((lane & d) == 0) == ((lane & size) == 0) ? fmaxf(v, o) : fminf(v, o);
        }
    return __shfl_sync(0xffffffffu, v, n - 1);
}
// A score that n of a warp's candidates (0: none, K per lane) reach, and not many more: the n-th best of the lanes' best ones, rounded down to
// fp32; 0 if fewer than n lanes have one.  (256 candidates, n = 4 / 16 / 32: about 4 / 21 / 90 reach it if they lie as they please; an
// exact bound took 1.8 us, this one 0.4.)
template <int K>
__device__ __forceinline__ uint64_t warp_bound(const uint64_t (&mine)[K], int n) {
    uint64_t top = mine[0];
#pragma unroll
    for (int k = 1; k < K; ++k) top = mine[k] > top ? mine[k] : top;
    const float v = warp_nth(top ? __double2float_rd(key_score(top)) : -INFINITY, n);
    return v > -INFINITY ? score_key((double)v) : 0ull;
}

// Two fp32 operations in one instruction.
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
    float2 r;
    asm("{\n\t.reg .b64 x, y, z;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tadd.rn.f32x2 z, x, y;\n\tmov.b64 {%0, %1}, z;\n\t}"
        : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return r;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
    float2 r;
    asm("{\n\t.reg .b64 x, y, z;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tmul.rn.f32x2 z, x, y;\n\tmov.b64 {%0, %1}, z;\n\t}"
        : "=f"(r.x), "=f"(r.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return r;
}

// The 16 bytes that begin `off` bytes (the same for all lanes) into u, which w follows in memory.
__device__ __forceinline__ uint4 shifted(const uint4& u, const uint4& w, uint32_t off) {
    uint32_t x0 = u.x, x1 = u.y, x2 = u.z, x3 = u.w, x4 = w.x, x5 = w.y, x6 = w.z;
    if (off & 8u) x0 = x2, x1 = x3, x2 = x4, x3 = x5, x4 = x6, x5 = w.w;
    if (off & 4u) x0 = x1, x1 = x2, x2 = x3, x3 = x4, x4 = x5;
    const uint32_t bits = (off & 3u) * 8u;
    return make_uint4(__funnelshift_r(x0, x1, bits), __funnelshift_r(x1, x2, bits), __funnelshift_r(x2, x3, bits), __funnelshift_r(x3, x4, bits));
}
// Eight neighbouring 16-bit entries of a row as they lie in memory, one by one, for the ends of the tensor: `n` of them, the rest is zero.
template <class T>
__device__ __noinline__ uint4 load_few(const T* src, int n) {
    uint32_t out[4] = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if (i >= n) break;
        out[i / 2] |= (uint32_t)(*reinterpret_cast<const uint16_t*>(src + i)) << (16 * (i & 1));
    }
    return make_uint4(out[0], out[1], out[2], out[3]);
}

template <class T>
__device__ __forceinline__ void widen(const uint4& v, float* x) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(T) == 4) {
            x[i] = __uint_as_float(w[i]);
        } else if constexpr (std::is_same<T, __nv_bfloat16>::value) {
            x[2 * i] = __uint_as_float(w[i] << 16);
            x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
        } else {
            const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[i]));
            x[2 * i] = f.x;
            x[2 * i + 1] = f.y;
        }
    }
}

// The eight 16-bit entries that begin OFF bytes into two neighbouring vectors, from where they lie.
template <class T, int OFF>
__device__ __forceinline__ void widen_at(const uint4& u, const uint4& v, float* x) {
    const uint32_t w[8] = {u.x, u.y, u.z, u.w, v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int at = OFF + 2 * i;
        const uint32_t word = w[at / 4];
        if constexpr (std::is_same<T, __nv_bfloat16>::value) x[i] = __uint_as_float(at % 4 ? word & 0xffff0000u : word << 16);
        else x[i] = __half2float(__ushort_as_half((unsigned short)(at % 4 ? word >> 16 : word & 0xffffu)));
    }
}

// grid = batch clusters, block = kBeamThreads.  ALIGNED: every row starts on a 16-byte border.
template <class T, bool ALIGNED>
__global__ void __launch_bounds__(kBeamThreads, 2) k_beam_select(const BeamParams P) {
    namespace cg = cooperative_groups;
    cg::cluster_group cluster = cg::this_cluster();
    const int ctas = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    const int b = (int)blockIdx.x / ctas;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    constexpr int kVec = 16 / (int)sizeof(T), kLoads = 16 / kVec;          // entries of a load, loads of a lane per chunk
    __shared__ float s_top[kBeamMaxSlices];            // of all slices of the request: a logit at most kBeamSlack below the largest ...
    __shared__ double s_sum[kBeamMaxSlices];           // ... and sum of exponentials relative to it
    __shared__ float s_row_top[kMaxBeams];
    __shared__ double s_row_off[kMaxBeams];            // score - log of the sum
    __shared__ uint8_t s_alive[kMaxBeams], s_over[kMaxBeams];
    __shared__ float s_score[kMaxBeams];
    __shared__ float s_group_top[kBeamWarps * kBeamGroups];
    __shared__ uint64_t s_group_best[kBeamWarps * kBeamGroups];            // score of that logit, 0 without candidates
    __shared__ uint64_t s_bound;
    __shared__ int s_picked, s_listed, s_counts[kBeamWarps];
    __shared__ uint16_t s_list[kBeamThreads];
    extern __shared__ __align__(16) uint8_t s_dyn[];
    const int n = P.n_out;
    const int tasks = P.beams * P.slices, warps = ctas * kBeamWarps, gwarp = rank * kBeamWarps + warp;
    const int rounds = P.rounds, group_len = P.group_len, per_slice = P.per_slice, groups = kBeamWarps * rounds * per_slice;       // groups of the CTA
    auto slice_no = [&](int task) { return (int)P.by_beams.div((uint32_t)task); };
    auto row_no = [&](int task) { return task - slice_no(task) * P.beams; };
    BeamPick* s_buffers = reinterpret_cast<BeamPick*>(s_dyn);              // [warps][kBeamBuffer]
    BeamPick* s_picks = s_buffers + kBeamWarps * kBeamBuffer;              // [threads]
    BeamPick* s_sent = s_picks + kBeamThreads;                             // [CTAs][n]
    if (tid == 0) s_picked = s_listed = 0;
    if (tid < kBeamWarps * kBeamGroups) s_group_top[tid] = -INFINITY;
    static_assert(kBeamWarps * kBeamGroups <= kBeamThreads, "a thread per group");
    __syncthreads();

    cluster.barrier_arrive();                          // (before another CTA's memory is written, all of them have to be there)
    pdl_launch_dependents();
    pdl_wait();
    if (tid < P.beams) {
        const size_t r = (size_t)b * P.beams + tid;
        s_score[tid] = P.scores[r];
        s_over[tid] = P.finished && P.finished[r] != 0;
    }

    // a warp's view of a slice
    struct Slice {
        int lo, hi;
        const T* z;                                    // its row
        const uint4* vecs;                             // (kPairs) the row from the 16-byte border before its start
        uint32_t off;
        bool inside;                                   // whole vectors lie within the tensor
    };
    // A chunk on its way: a vector for every 16 bytes.  Where rows are not aligned a 16-bit entry lies in a lane's vector or in the one after
    // it; both are loaded, and entries taken from where they lie when they are used (64 x 16 beams over 32003 bf16 logits 32 us, loaded one
    // by one 45).  fp32 entries are loaded one by one, neighbours by neighbouring lanes: two vectors would take twice the registers, and
    // shifted as they arrive every chunk is waited for (15 x 15 beams over 42689 logits 42 us, so 30).
    constexpr bool kPairs = !ALIGNED && sizeof(T) == 2, kSingle = !ALIGNED && sizeof(T) == 4;
    auto place = [&](int k) { return kSingle ? k * 32 + lane : (k / kVec * 32 + lane) * kVec + k % kVec; };      // of a lane's k-th entry in its chunk
    struct Raw {
        uint4 v[kLoads][kPairs ? 2 : 1];
    };
    auto ends_inside = [&](const uint4* vecs, uint32_t off, int from, int to) {
        return reinterpret_cast<uintptr_t>(vecs + from / kVec) >= reinterpret_cast<uintptr_t>(P.logits) &&
               reinterpret_cast<uintptr_t>(vecs + (to + kVec - 1) / kVec + (off ? 1 : 0)) <= reinterpret_cast<uintptr_t>(P.logits_end);
    };
    auto slice_of = [&](int task) {
        Slice v;
        const int slice = slice_no(task), row = task - slice * P.beams;
        v.lo = (int)min((long long)slice * P.slice_len, (long long)P.vocab);
        v.hi = (int)min((long long)v.lo + P.slice_len, (long long)P.vocab);
        v.z = static_cast<const T*>(P.logits) + ((size_t)b * P.beams + row) * (size_t)P.vocab;
        if constexpr (kPairs) {
            const uintptr_t at = reinterpret_cast<uintptr_t>(v.z);
            v.off = (uint32_t)(at & 15u);
            v.vecs = reinterpret_cast<const uint4*>(at - v.off);
            v.inside = ends_inside(v.vecs, v.off, v.lo, v.hi);
        }
        return v;
    };
    auto load = [&](const Slice& v, int c0, Raw& raw) {
        if constexpr (kSingle) {
            uint32_t w[16];
#pragma unroll
            for (int k = 0; k < 16; ++k) w[k] = c0 + place(k) < v.hi ? __float_as_uint(__ldg(reinterpret_cast<const float*>(v.z) + c0 + place(k))) : 0u;
#pragma unroll
            for (int k = 0; k < kLoads; ++k) raw.v[k][0] = make_uint4(w[4 * k], w[4 * k + 1], w[4 * k + 2], w[4 * k + 3]);
        } else if constexpr (kPairs) {
            const bool inside = v.inside || ends_inside(v.vecs, v.off, c0, min(v.hi, c0 + kBeamChunk));    // (only the tensor's first and last chunk are not)
#pragma unroll
            for (int k = 0; k < kLoads; ++k) {
                const int t = c0 + (k * 32 + lane) * kVec;
                if (t >= v.hi) continue;
                if (inside) {
                    raw.v[k][0] = __ldg(v.vecs + t / kVec);
                    if (v.off) raw.v[k][1] = __ldg(v.vecs + t / kVec + 1);
                } else {                               // as if it had been read behind the border
                    const uint4 few = load_few<T>(v.z + t, P.vocab - t);
                    raw.v[k][0] = v.off ? shifted(make_uint4(0, 0, 0, 0), few, 16u - v.off) : few;
                    raw.v[k][1] = shifted(few, make_uint4(0, 0, 0, 0), 16u - v.off);
                }
            }
        } else {                                       // (a row is whole vectors)
#pragma unroll
            for (int k = 0; k < kLoads; ++k)
                if (c0 + place(k * kVec) < v.hi) raw.v[k][0] = __ldg(reinterpret_cast<const uint4*>(v.z + c0 + place(k * kVec)));
        }
    };
    auto values = [&](const Slice& v, int c0, const Raw& raw, float (&x)[16]) {
        if constexpr (kPairs) {
            auto at = [&](auto off) {
#pragma unroll
                for (int k = 0; k < kLoads; ++k) widen_at<T, decltype(off)::value>(raw.v[k][0], raw.v[k][1], x + k * kVec);
            };
            switch (v.off) {
            case 0: at(std::integral_constant<int, 0>()); break;
            case 2: at(std::integral_constant<int, 2>()); break;
            case 4: at(std::integral_constant<int, 4>()); break;
            case 6: at(std::integral_constant<int, 6>()); break;
            case 8: at(std::integral_constant<int, 8>()); break;
            case 10: at(std::integral_constant<int, 10>()); break;
            case 12: at(std::integral_constant<int, 12>()); break;
            default: at(std::integral_constant<int, 14>()); break;
            }
        } else {
#pragma unroll
            for (int k = 0; k < kLoads; ++k) widen<T>(raw.v[k][0], x + k * kVec);
        }
        if (c0 + kBeamChunk > v.hi) {
#pragma unroll
            for (int k = 0; k < 16; ++k)
                if (c0 + place(k) >= v.hi) x[k] = -INFINITY;
        }
    };
#pragma unroll 1
    for (int j = 0, task = gwarp; j < rounds; ++j, task += warps) {
        float top = kBeamLowest;
        double sum = 0.0;
        if (task < tasks) {
            const int row = row_no(task);
            const size_t r = (size_t)b * P.beams + row;
            float* tops = s_group_top + (warp * rounds + j) * per_slice;
            const Slice v = slice_of(task);
            Raw raw;
            load(v, v.lo, raw);                        // (of rows that are out no more than this is read)
            const bool over = P.finished && P.finished[r] != 0, alive = isfinite(P.scores[r]);
            if (over) {                                // one candidate: the end token at the score as it is
                if (task < P.beams) top = 0.f, sum = lane == 0 ? 1.0 : 0.0, tops[0] = 0.f;
            } else if (alive) {
                float most = -INFINITY;
                int g = 0, next = v.lo + group_len;
#pragma unroll 1
                for (int c0 = v.lo; c0 < v.hi; c0 += kBeamChunk) {
                    float x[16];
                    values(v, c0, raw, x);
                    load(v, c0 + kBeamChunk, raw);     // (on their way while this chunk is worked on)
                    float here = x[0];
#pragma unroll
                    for (int k = 1; k < 16; ++k) here = fmaxf(here, x[k]);
                    // (Not for every new largest entry: over the chunks of a row that rises the errors of the factors add up.  32 rows of 2^20 that rise
                    // by 4 in all: 110 x 2^-24, so none that shows.  What weighs anything sees a few of these.)
                    if (here - top > kBeamSlack) {
                        sum *= (double)fast_exp2((top - here) * kLog2e);
                        top = here;
                    }
                    // (x - top) log2 e: the difference first, so that the type's lowest value next to itself is zero, and what is near
                    // the largest loses nothing
                    float2 part = make_float2(0.f, 0.f);
#pragma unroll
                    for (int k = 0; k < 16; k += 2) {
                        const float2 t = mul2(add2(make_float2(x[k], x[k + 1]), make_float2(-top, -top)), make_float2(kLog2e, kLog2e));
                        part = add2(part, make_float2(fast_exp2(t.x), fast_exp2(t.y)));
                    }
                    sum += (double)(part.x + part.y);
                    most = fmaxf(most, here);
                    if (c0 + kBeamChunk >= min(next, v.hi)) {
                        most = warp_max(most);
                        if (lane == 0) tops[g] = most;
                        ++g;
                        next += group_len;
                        most = -INFINITY;
                    }
                }
                // the lanes' sums relative to the largest of theirs
                const float all = warp_max(top);
                sum *= (double)fast_exp2((top - all) * kLog2e);
                top = all;
            }
#pragma unroll
            for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
        }
        if (j == 0) cluster.barrier_wait();
        if (task < tasks && lane < ctas) {
            cluster.map_shared_rank(s_top, lane)[task] = top;
            cluster.map_shared_rank(s_sum, lane)[task] = sum;
        }
    }
    cluster.sync();

    // ---- rows: a warp each
    for (int row = warp; row < P.beams; row += kBeamWarps) {
        float top = kBeamLowest;
        for (int s = lane; s < P.slices; s += 32) top = fmaxf(top, s_top[s * P.beams + row]);
        top = warp_max(top);
        double sum = 0.0;
        for (int s = lane; s < P.slices; s += 32) sum += s_sum[s * P.beams + row] * exp((double)s_top[s * P.beams + row] - (double)top);
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
        if (lane == 0) {
            const float score = s_score[row];
            s_row_top[row] = top;
            s_row_off[row] = (double)score - log(sum);
            s_alive[row] = isfinite(score) && isfinite(sum) && sum > 0.0 && isfinite(top);
        }
    }
    __syncthreads();
    // ---- a bound: the n-th best of the CTA's groups' largest entries, which n of its candidates reach
    auto slice_of_group = [&](int group, int& g) {     // the slice (task) of a group and its number there
        const int slot = (int)P.by_groups.div((uint32_t)group), w = rounds == 1 ? slot : slot >> 1;
        g = group - slot * per_slice;
        return rank * kBeamWarps + w + (slot - w * rounds) * warps;
    };
    uint64_t best = 0;                                 // of this thread's group
    if (tid < kBeamWarps * kBeamGroups) {
        int g;
        const int task = slice_of_group(min(tid, groups - 1), g), row = row_no(task);
        const float top = s_group_top[tid];
        if (tid < groups && task < tasks && s_alive[row] && top > -INFINITY) best = score_key(s_row_off[row] + ((double)top - (double)s_row_top[row]));
        s_group_best[tid] = best;
    }
    __syncthreads();
    if (warp == 0) {
        uint64_t some[kBeamWarps * kBeamGroups / 32];
#pragma unroll
        for (int k = 0; k < kBeamWarps * kBeamGroups / 32; ++k) some[k] = s_group_best[32 * k + lane];
        const uint64_t of_groups = warp_bound(some, n);
        if (lane == 0) s_bound = of_groups;
    }
    __syncthreads();
    const uint64_t bound = s_bound;
    if (best != 0 && best >= bound) s_list[atomicAdd(&s_listed, 1)] = (uint16_t)tid;
    __syncthreads();
    // ---- the groups that reach it are read again, one warp each, and the entries that reach it kept; more than n of a warp never
    // count
    {
        BeamPick* buffer = s_buffers + warp * kBeamBuffer;
        BeamPick worst = no_pick();                    // once the buffer was full: what has to be beaten
        uint64_t reach = bound;                        // what has to be reached
        float lane_top = -INFINITY;                    // score of the best entry that this lane has seen
        int count = 0;
        {
            const int listed = s_listed;
#pragma unroll 1
            for (int i = warp; i < listed; i += kBeamWarps) {
                int g;
                const int task = slice_of_group(s_list[i], g), row = row_no(task);
                const double off = s_row_off[row];
                const float row_top = s_row_top[row];
                auto score_of = [&](float x) { return score_key(off + ((double)x - (double)row_top)); };
                auto keep = [&](bool mine_in, BeamPick p) {
                    uint32_t in = __ballot_sync(0xffffffffu, mine_in);
                    if (count + __popc(in) > kBeamBuffer) {
                        __syncwarp();
                        warp_best(buffer, count, n);
                        count = n;                     // (at least n + 1 were in it)
                        worst = buffer[n - 1];
                        mine_in = mine_in && p.before(worst);
                        in = __ballot_sync(0xffffffffu, mine_in);
                    }
                    if (mine_in) buffer[count + __popc(in & ((1u << lane) - 1))] = p;
                    count += __popc(in);
                };
                if (s_over[row]) {
                    keep(lane == 0, BeamPick{score_of(0.f), (uint32_t)row, (uint32_t)P.end_token});
                    continue;
                }
                // Logits below this do not reach it (or what has to be beaten; exactly: below).  A score was rounded when the logit was added to
                // `off`, by up to 2^-53 of its size, which is more than all logits where beams have scores like -1e30; so are the
                // differences here, and 2^-51 of both is more than all of these.
                auto least_logit = [&]() {
                    const uint64_t key = worst.score > reach ? worst.score : reach;
                    if (key == 0) return -FLT_MAX;
                    const double score = key_score(key), rounded = (fabs(score) + fabs(off)) * 0x1p-51;
                    return fmaxf(-FLT_MAX, nextafterf(__double2float_rd((score - off - rounded) + (double)row_top), -INFINITY));
                };
                float least = least_logit();
                const Slice v = slice_of(task);
                const int begin = v.lo + g * group_len;
#pragma unroll 1
                for (int c0 = begin; c0 < min(v.hi, begin + group_len); c0 += kBeamChunk) {
                    Raw raw;
                    float x[16];
                    load(v, c0, raw);
                    values(v, c0, raw, x);
                    auto hits_of = [&]() {             // entries of this lane that may count
                        uint32_t hits = 0;
#pragma unroll
                        for (int k = 0; k < 16; ++k)
                            if (x[k] >= least) hits |= 1u << k;
                        return hits;
                    };
                    uint32_t hits = hits_of();
                    // Where the bound is weak (one beam is far ahead, or has all the candidates) many reach it.  The n-th best of the lanes'
                    // best entries so far is one that n of this warp's reach.
                    float most = x[0];
#pragma unroll
                    for (int k = 1; k < 16; ++k) most = fmaxf(most, x[k]);
                    if (most > -INFINITY) lane_top = fmaxf(lane_top, __double2float_rd(off + ((double)most - (double)row_top)));
                    if (__reduce_add_sync(0xffffffffu, __popc(hits)) > 2 * n) {
                        const float nth = warp_nth(lane_top, n);
                        if (nth > -INFINITY && score_key((double)nth) > reach) {
                            reach = score_key((double)nth);
                            least = least_logit();
                            hits = hits_of();
                        }
                    }
                    while (__any_sync(0xffffffffu, hits != 0)) {           // one of every lane at a time
                        const int k = __ffs((int)hits) - 1;
                        float z = x[0];
#pragma unroll
                        for (int c = 1; c < 16; ++c) z = k == c ? x[c] : z;
                        BeamPick p;
                        p.score = score_of(z);
                        p.row = (uint32_t)row;
                        p.token = (uint32_t)(c0 + place(k));
                        keep(k >= 0 && p.score >= reach && (worst.score == 0 || p.before(worst)), p);
                        hits &= hits - 1;
                    }
                }
            }
        }
        // (all that was kept, if there is room for it; otherwise the n best of every warp)
        if (lane == 0) s_counts[warp] = count;
        __syncthreads();
        int kept = 0;
#pragma unroll
        for (int w = 0; w < kBeamWarps; ++w) kept += s_counts[w];
        if (kept > kBeamThreads && count > n) {
            warp_best(buffer, count, n);
            count = n;
        }
        int at = 0;
        if (lane == 0) at = atomicAdd(&s_picked, count);
        at = __shfl_sync(0xffffffffu, at, 0);
        for (int i = lane; i < count; i += 32) s_picks[at + i] = buffer[i];
    }
    __syncthreads();
    // Ranks `count` candidates, one per thread at most, and calls put(rank, candidate) in one lane for each of the n best: those
    // that reach the bound are listed, then the better ones of each are counted.  (The order in which they lie does not matter.)
    auto rank_all = [&](const BeamPick* list, int count, auto put) {
        const bool few = count <= 96;                  // (looking for the bound takes as long as ranking so many)
        int listed = count;
        if (!few) {
            if (warp == 0) {
                uint64_t some[kBeamThreads / 32];
#pragma unroll
                for (int k = 0; k < kBeamThreads / 32; ++k) some[k] = 32 * k + lane < count ? list[32 * k + lane].score : 0ull;
                const uint64_t least = warp_bound(some, n);
                if (lane == 0) s_bound = least, s_listed = 0;
            }
            __syncthreads();
            const uint64_t mine = tid < count ? list[tid].score : 0ull;
            if (mine != 0 && mine >= s_bound) s_list[atomicAdd(&s_listed, 1)] = (uint16_t)tid;
            __syncthreads();
            listed = s_listed;
        }
        for (int i0 = 0; i0 < listed; i0 += kBeamThreads / 8) {            // eight threads per candidate
            const int i = i0 + (tid >> 3);
            const BeamPick p = i < listed ? list[few ? i : s_list[i]] : no_pick();
            int better = 0;
#pragma unroll 4
            for (int o = tid & 7; o < listed; o += 8) better += list[few ? o : s_list[o]].before(p);
#pragma unroll
            for (int d = 1; d < 8; d <<= 1) better += __shfl_xor_sync(0xffffffffu, better, d);
            if (p.score != 0 && better < n && (tid & 7) == 0) put(better, p);
        }
    };
    static_assert(kBeamWarps * kMaxBeams <= kBeamThreads && kBeamMaxCluster * kMaxBeams <= kBeamThreads, "a thread per candidate");
    // ---- the CTA's n best go to the first CTA, which joins those of all
    {
        BeamPick* to = cluster.map_shared_rank(s_sent, 0) + rank * n;
        rank_all(s_picks, s_picked, [&](int i, const BeamPick& p) { to[i] = p; });
        for (int i = s_picked + tid; i < n; i += kBeamThreads) to[i] = no_pick();
    }
    cluster.sync();
    if (rank != 0) return;
    rank_all(s_sent, ctas * n, [&](int i, const BeamPick& p) {
        const size_t at = (size_t)b * n + i, from = (size_t)b * P.beams + p.row;
        P.parents[at] = (int32_t)from;
        P.tokens[at] = (int32_t)p.token;
        P.scores_out[at] = (float)key_score(p.score);
        if (P.finished_out) P.finished_out[at] = (int32_t)p.token == P.end_token || s_over[p.row];
    });
    const int found = __syncthreads_count(tid < ctas * n && s_sent[tid].score != 0);   // candidates in all
    for (int i = found + tid; i < n; i += kBeamThreads) {
        const size_t at = (size_t)b * n + i;
        P.parents[at] = P.tokens[at] = -1;
        P.scores_out[at] = -INFINITY;
        if (P.finished_out) P.finished_out[at] = 1;
    }
}

}  // namespace kvq
