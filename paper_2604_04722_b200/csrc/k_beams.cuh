// One step of beam search: of all candidates (beam w, token v) with the score  s_w + z_wv - log sum_u exp(z_wu)  the n best,
// ties to the lowest (w, v).
//
// A cluster of CTAs serves a request, and reads its logits once.  Every row is cut into slices, one warp each; the cut does not
// depend on the row or its address, so that equal rows have equal sums and tie as they should.  A warp keeps, over its slice, the
// largest logit and the sum of exponentials (fp32 within 16 entries of a lane, fp64 beyond: what is compared between beams
// must not depend on their order), and the entries that can still be among the n best of the row: those above a
// threshold, which starts as the n-th largest of the 32 lanes' maxima (n entries are at least as large, so nothing smaller can
// be among the n best) and rises whenever the buffer is full and cut back to its n best.  After the first 512 entries hardly any logit
// passes, so the loop is one exponential and a comparison per entry.
//
// Then the slices' sums are exchanged (one cluster barrier), every CTA merges its warps' sorted lists to its n best, a warp per CTA, by score in
// fp64, and the first CTA merges those.  Bound: the logits' bytes for many requests; for few of them the chain of the
// row's loads, two cluster barriers and two merges.
#pragma once
#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <type_traits>
#include "kvq_common.cuh"
#include "kvq_pages.h"
#include "kvq_ptx.cuh"

namespace kvq {

constexpr int kBeamThreads = 512, kBeamWarps = kBeamThreads / 32;
constexpr int kBeamMaxCluster = 16;
constexpr int kBeamChunk = 512;                        // entries that a warp works on at a time, 16 per lane
constexpr int kBeamBuffer = 128;                       // entries of a warp's buffer, 4 per lane: at least n + 32
constexpr int kBeamTasks = (kMaxBeams + kBeamWarps - 1) / kBeamWarps;      // slices of a warp at most
constexpr int kBeamMaxSlices = kBeamMaxCluster * kBeamWarps;
constexpr float kBeamLowest = -3.402823466e38f;

// Order-preserving 32-bit keys of logits (-0 counts as 0); no logit has the key 0.
__device__ __forceinline__ uint32_t logit_key(float x) {
    const uint32_t b = __float_as_uint(x + 0.f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float key_logit(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k); }
__device__ __forceinline__ uint64_t score_key(double x) {
    const uint64_t b = (uint64_t)__double_as_longlong(x + 0.0);
    return b >> 63 ? ~b : b | (1ull << 63);
}
__device__ __forceinline__ double key_score(uint64_t k) {
    return __longlong_as_double((long long)(k >> 63 ? k ^ (1ull << 63) : ~k));
}

struct BeamEntry {
    uint32_t key, token;                               // logit (0: none)
};
struct BeamPick {
    uint64_t score;                                    // score_key (0: none)
    uint32_t row, token;
};

// Dynamic shared memory: the lists of a CTA's slices, then the CTAs' picks (used by the first CTA).
inline size_t beam_smem(int n_out) {
    return (size_t)kBeamWarps * kBeamTasks * n_out * sizeof(BeamEntry) + (size_t)kBeamMaxCluster * n_out * sizeof(BeamPick);
}

// The n best entries of a warp's buffer, in order (value descending, token ascending), to `list`; missing ones have the key 0.
__device__ __forceinline__ void warp_best(const BeamEntry* buffer, int count, int n, BeamEntry* list) {
    const int lane = threadIdx.x & 31;
    BeamEntry e[kBeamBuffer / 32];
#pragma unroll
    for (int k = 0; k < kBeamBuffer / 32; ++k) {
        e[k].key = 0, e[k].token = 0xffffffffu;
        if (lane + 32 * k < count) e[k] = buffer[lane + 32 * k];
    }
    __syncwarp();                                      // (the list may be the buffer itself)
#pragma unroll 1
    for (int i = 0; i < n; ++i) {
        uint32_t key = 0, token = 0xffffffffu;
#pragma unroll
        for (int k = 0; k < kBeamBuffer / 32; ++k)
            if (e[k].key > key || (e[k].key == key && e[k].token < token)) key = e[k].key, token = e[k].token;
        const uint32_t best = __reduce_max_sync(0xffffffffu, key);
        const uint32_t at = __reduce_min_sync(0xffffffffu, key == best ? token : 0xffffffffu);
#pragma unroll
        for (int k = 0; k < kBeamBuffer / 32; ++k)
            if (e[k].key == best && e[k].token == at) e[k].key = 0, e[k].token = 0xffffffffu;
        if (lane == 0) list[i].key = best, list[i].token = at;
    }
    __syncwarp();
}

// Merges up to 32 sorted lists, one per lane: head(i) gives a lane's i-th pick (score 0 behind its last).  take(i, pick) is
// called by all lanes with the picks in order.
template <class Head, class Take>
__device__ __forceinline__ void merge_lists(int n, Head head, Take take) {
    int mine = 0;
    BeamPick h = head(0);
#pragma unroll 1
    for (int i = 0; i < n; ++i) {
        const uint32_t hi = (uint32_t)(h.score >> 32), lo = (uint32_t)h.score;
        const uint32_t best_hi = __reduce_max_sync(0xffffffffu, hi);
        bool in = hi == best_hi;
        const uint32_t best_lo = __reduce_max_sync(0xffffffffu, in ? lo : 0u);
        in = in && lo == best_lo;
        const uint32_t row = __reduce_min_sync(0xffffffffu, in ? h.row : 0xffffffffu);
        in = in && h.row == row;
        const uint32_t token = __reduce_min_sync(0xffffffffu, in ? h.token : 0xffffffffu);
        BeamPick pick;
        pick.score = ((uint64_t)best_hi << 32) | best_lo;
        pick.row = row;
        pick.token = token;
        take(i, pick);
        if (in && h.token == token && pick.score != 0) h = head(++mine);
    }
}

// Eight (16-bit) or four (fp32) neighbouring entries of a row as they lie in memory, from any address that is a multiple of
// their size: two aligned 16-byte loads and a shift where the row is not aligned.  Bytes outside [begin, end) are not read.
template <class T>
__device__ __forceinline__ uint4 load_entries(const T* src, const void* begin, const void* end) {
    const uintptr_t a = reinterpret_cast<uintptr_t>(src);
    const uint32_t off = (uint32_t)(a & 15u);
    if (off == 0 && a + 16 <= reinterpret_cast<uintptr_t>(end)) return __ldg(reinterpret_cast<const uint4*>(src));
    const uint4* p = reinterpret_cast<const uint4*>(a - off);
    if (reinterpret_cast<uintptr_t>(p) >= reinterpret_cast<uintptr_t>(begin) && reinterpret_cast<uintptr_t>(p + 2) <= reinterpret_cast<uintptr_t>(end)) {
        const uint4 u = __ldg(p), w = __ldg(p + 1);
        uint32_t x0 = u.x, x1 = u.y, x2 = u.z, x3 = u.w, x4 = w.x, x5 = w.y, x6 = w.z;
        if (off & 8u) x0 = x2, x1 = x3, x2 = x4, x3 = x5, x4 = x6, x5 = w.w;
        if (off & 4u) x0 = x1, x1 = x2, x2 = x3, x3 = x4, x4 = x5;
        const uint32_t bits = (off & 3u) * 8u;
        return make_uint4(__funnelshift_r(x0, x1, bits), __funnelshift_r(x1, x2, bits), __funnelshift_r(x2, x3, bits), __funnelshift_r(x3, x4, bits));
    }
    constexpr int kN = 16 / sizeof(T);
    uint32_t out[4] = {0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < kN; ++i) {                     // at the ends of the tensor: one by one
        if (reinterpret_cast<uintptr_t>(src + i + 1) > reinterpret_cast<uintptr_t>(end)) break;
        if constexpr (sizeof(T) == 2) out[i / 2] |= (uint32_t)(*reinterpret_cast<const uint16_t*>(src + i)) << (16 * (i & 1));
        else out[i] = *reinterpret_cast<const uint32_t*>(src + i);
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

// grid = batch clusters, block = kBeamThreads.
template <class T>
__global__ void __launch_bounds__(kBeamThreads, 2) k_beam_select(const BeamParams P) {
    namespace cg = cooperative_groups;
    cg::cluster_group cluster = cg::this_cluster();
    const int ctas = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    const int b = (int)blockIdx.x / ctas;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    constexpr int kVec = 16 / (int)sizeof(T), kLoads = 16 / kVec;          // entries of a load, loads of a lane per chunk
    __shared__ BeamEntry s_buffer[kBeamWarps][kBeamBuffer];
    __shared__ float s_top[kBeamMaxSlices];            // of all slices of the request: largest logit ...
    __shared__ double s_sum[kBeamMaxSlices];           // ... and sum of exponentials relative to it
    __shared__ float s_row_top[kMaxBeams];
    __shared__ double s_row_off[kMaxBeams];            // score - log of the sum
    __shared__ uint8_t s_alive[kMaxBeams];
    extern __shared__ __align__(16) uint8_t s_dyn[];
    const int n = P.n_out;
    BeamPick* s_picks = reinterpret_cast<BeamPick*>(s_dyn);                // [CTAs][n]
    BeamEntry* s_lists = reinterpret_cast<BeamEntry*>(s_picks + kBeamMaxCluster * n);      // [warps * kBeamTasks][n]

    cluster.barrier_arrive();                          // (before another CTA's memory is written, all of them have to be there)
    pdl_launch_dependents();
    pdl_wait();

    const int tasks = P.beams * P.slices, warps = ctas * kBeamWarps, gwarp = rank * kBeamWarps + warp;
    constexpr float kLog2eF = 1.4426950408889634f;
#pragma unroll 1
    for (int j = 0, task = gwarp; j < kBeamTasks; ++j, task += warps) {
        BeamEntry* list = s_lists + (warp * kBeamTasks + j) * n;
        float top = kBeamLowest;
        double sum = 0.0;
        int count = 0;
        BeamEntry* buffer = s_buffer[warp];
        if (task < tasks) {
            const int row = task % P.beams, slice = task / P.beams;
            const size_t r = (size_t)b * P.beams + row;
            const bool over = P.finished && P.finished[r] != 0, alive = isfinite(P.scores[r]);
            if (over) {                                // one candidate: the end token at the score as it is
                if (slice == 0) {
                    if (lane == 0) buffer[0].key = logit_key(0.f), buffer[0].token = (uint32_t)P.end_token;
                    count = 1;
                    top = 0.f;
                    sum = 1.0;
                }
            } else if (alive) {
                const int lo = min((long long)slice * P.slice_len, (long long)P.vocab), hi = min((long long)lo + P.slice_len, (long long)P.vocab);
                const T* z = static_cast<const T*>(P.logits) + r * (size_t)P.vocab;
                // threshold: an entry stays in the running if it is larger, or as large and its token is below `above`
                float least = -INFINITY;
                uint32_t above = 0;
                uint4 raw[kLoads];
                auto load = [&](int c0) {
#pragma unroll
                    for (int k = 0; k < kLoads; ++k) {
                        const int v = c0 + (k * 32 + lane) * kVec;
                        if (v < hi) raw[k] = load_entries<T>(z + v, P.logits, P.logits_end);
                    }
                };
                load(lo);
#pragma unroll 1
                for (int c0 = lo; c0 < hi; c0 += kBeamChunk) {
                    float x[16];
#pragma unroll
                    for (int k = 0; k < kLoads; ++k) widen<T>(raw[k], x + k * kVec);
                    if (c0 + kBeamChunk > hi) {
#pragma unroll
                        for (int k = 0; k < 16; ++k)
                            if (c0 + ((k / kVec) * 32 + lane) * kVec + k % kVec >= hi) x[k] = -INFINITY;
                    }
                    load(c0 + kBeamChunk);             // (on their way while this chunk is worked on)
                    float most = x[0];
#pragma unroll
                    for (int k = 1; k < 16; ++k) most = fmaxf(most, x[k]);
                    if (most > top) {
                        sum *= (double)fast_exp2((top - most) * kLog2eF);
                        top = most;
                    }
                    float part = 0.f;
#pragma unroll
                    for (int k = 0; k < 16; ++k) part += fast_exp2((x[k] - top) * kLog2eF);
                    sum += (double)part;
                    if (c0 == lo) {                    // the n-th largest of the lanes' maxima: a bitonic sort, descending
                        float v = most;
#pragma unroll
                        for (int size = 2; size <= 32; size <<= 1)
#pragma unroll
                            for (int d = size >> 1; d > 0; d >>= 1) {
                                const float o = __shfl_xor_sync(0xffffffffu, v, d);
                                const bool keep_max = ((lane & d) == 0) == ((lane & size) == 0);
                                v = keep_max ? fmaxf(v, o) : fminf(v, o);
                            }
                        least = __shfl_sync(0xffffffffu, v, n - 1);
                        above = least > -INFINITY ? 0xffffffffu : 0u;      // (masked entries are no candidates)
                    }
                    if (!__any_sync(0xffffffffu, most >= least)) continue;
#pragma unroll
                    for (int k = 0; k < 16; ++k) {
                        const uint32_t v = (uint32_t)(c0 + ((k / kVec) * 32 + lane) * kVec + k % kVec);
                        uint32_t in = __ballot_sync(0xffffffffu, x[k] > least || (x[k] == least && v < above));
                        if (in == 0) continue;
                        if (count + __popc(in) > kBeamBuffer) {
                            __syncwarp();
                            warp_best(buffer, count, n, buffer);
                            count = n;                 // (at least n + 1 were in it)
                            least = key_logit(buffer[n - 1].key);
                            above = buffer[n - 1].token;
                            in = __ballot_sync(0xffffffffu, x[k] > least || (x[k] == least && v < above));
                        }
                        if ((in >> lane) & 1u) {
                            BeamEntry& e = buffer[count + __popc(in & ((1u << lane) - 1))];
                            e.key = logit_key(x[k]);
                            e.token = v;
                        }
                        count += __popc(in);
                    }
                }
                // the lanes' sums relative to the slice's largest
                const float all = warp_max(top);
                sum *= exp((double)top - (double)all);
                top = all;
#pragma unroll
                for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
            }
            __syncwarp();
        }
        warp_best(buffer, count, n, list);
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
            const float score = P.scores[(size_t)b * P.beams + row];
            s_row_top[row] = top;
            s_row_off[row] = (double)score - log(sum);
            s_alive[row] = isfinite(score) && isfinite(sum) && sum > 0.0 && isfinite(top);
        }
    }
    __syncthreads();
    // ---- the CTA's lists, then the CTAs' picks
    if (warp == 0) {
        const int task = rank * kBeamWarps + lane % kBeamWarps + (lane / kBeamWarps) * warps, row = task % P.beams;
        const bool live = lane < kBeamWarps * kBeamTasks && task < tasks && s_alive[row];
        const BeamEntry* list = s_lists + ((lane % kBeamWarps) * kBeamTasks + lane / kBeamWarps) * n;
        BeamPick* to = cluster.map_shared_rank(s_picks, 0) + rank * n;
        merge_lists(
            n,
            [&](int i) {
                BeamPick p = {0, 0xffffffffu, 0xffffffffu};
                if (live && i < n && list[i].key != 0) {
                    p.score = score_key(s_row_off[row] + ((double)key_logit(list[i].key) - (double)s_row_top[row]));
                    p.row = (uint32_t)row;
                    p.token = list[i].token;
                }
                return p;
            },
            [&](int i, const BeamPick& p) {
                if (lane == 0) to[i] = p;
            });
    }
    cluster.sync();
    if (rank == 0 && warp == 0) {
        merge_lists(
            n,
            [&](int i) {
                BeamPick p = {0, 0xffffffffu, 0xffffffffu};
                if (lane < ctas && i < n) p = s_picks[lane * n + i];
                return p;
            },
            [&](int i, const BeamPick& p) {
                if (lane != 0) return;
                const size_t at = (size_t)b * n + i;
                const bool there = p.score != 0;
                const size_t from = (size_t)b * P.beams + p.row;
                P.parents[at] = there ? (int32_t)from : -1;
                P.tokens[at] = there ? (int32_t)p.token : -1;
                P.scores_out[at] = there ? (float)key_score(p.score) : -INFINITY;
                if (P.finished_out) P.finished_out[at] = !there || (int32_t)p.token == P.end_token || (P.finished && P.finished[from] != 0);
            });
    }
}

}  // namespace kvq
