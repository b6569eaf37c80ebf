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
    uint64_t score;                                    // score_key
    uint32_t row, token;
    __device__ bool before(const BeamPick& o) const {
        return score != o.score ? score > o.score : row != o.row ? row < o.row : token < o.token;
    }
};

// Dynamic shared memory: the buffers of a CTA's slices, and in every CTA room for the picks that are left over (those of the
// first CTA are used): of n slices at most n + 32 each.
__host__ __device__ constexpr int beam_max_picks(int n) { return n * (n + 32); }
inline size_t beam_smem(int tasks, int n) {
    return (size_t)kBeamWarps * tasks * kBeamBuffer * sizeof(BeamEntry) + (size_t)beam_max_picks(n) * sizeof(BeamPick);
}

// Cuts a warp's buffer back to its n best entries, in order (value descending, token ascending); it holds n or more.
__device__ __noinline__ void warp_best(BeamEntry* buffer, int count, int n) {
    const int lane = threadIdx.x & 31;
    BeamEntry e[kBeamBuffer / 32];
#pragma unroll
    for (int k = 0; k < kBeamBuffer / 32; ++k) {
        e[k].key = 0, e[k].token = 0xffffffffu;
        if (lane + 32 * k < count) e[k] = buffer[lane + 32 * k];
    }
    __syncwarp();
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
        if (lane == 0) buffer[i].key = best, buffer[i].token = at;
    }
    __syncwarp();
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

__device__ __forceinline__ float widen_one(float x) { return x; }
__device__ __forceinline__ float widen_one(__half x) { return __half2float(x); }
__device__ __forceinline__ float widen_one(__nv_bfloat16 x) { return __bfloat162float(x); }

// grid = batch clusters, block = kBeamThreads.
template <class T>
__global__ void __launch_bounds__(kBeamThreads, 2) k_beam_select(const BeamParams P) {
    namespace cg = cooperative_groups;
    cg::cluster_group cluster = cg::this_cluster();
    const int ctas = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    const int b = (int)blockIdx.x / ctas;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    constexpr int kVec = 16 / (int)sizeof(T), kLoads = 16 / kVec;          // entries of a load, loads of a lane per chunk
    __shared__ float s_top[kBeamMaxSlices];            // of all slices of the request: largest logit ...
    __shared__ double s_sum[kBeamMaxSlices];           // ... and sum of exponentials relative to it
    __shared__ uint64_t s_best[kBeamMaxSlices];        // by row, then slice: score of that logit, 0 for a slice without candidates
    __shared__ uint8_t s_in[kBeamMaxSlices];           // ... and whether it is among the n best
    __shared__ float s_row_top[kMaxBeams];
    __shared__ double s_row_off[kMaxBeams];            // score - log of the sum
    __shared__ uint8_t s_alive[kMaxBeams];
    __shared__ int s_count[kBeamWarps * kBeamTasks];
    __shared__ uint64_t s_least;
    __shared__ int s_picked;                           // (of the first CTA)
    extern __shared__ __align__(16) uint8_t s_dyn[];
    const int n = P.n_out;
    const int tasks = P.beams * P.slices, warps = ctas * kBeamWarps, gwarp = rank * kBeamWarps + warp;
    const int rounds = (tasks + warps - 1) / warps;    // slices of a warp, at most kBeamTasks
    BeamPick* s_picks = reinterpret_cast<BeamPick*>(s_dyn);
    BeamEntry* s_buffers = reinterpret_cast<BeamEntry*>(s_picks + beam_max_picks(n));      // [warps * rounds][kBeamBuffer]
    if (tid == 0) s_picked = 0, s_least = 0;

    cluster.barrier_arrive();                          // (before another CTA's memory is written, all of them have to be there)
    pdl_launch_dependents();
    pdl_wait();

#pragma unroll 1
    for (int j = 0, task = gwarp; j < rounds; ++j, task += warps) {
        float top = kBeamLowest;
        double sum = 0.0;
        int count = 0;
        BeamEntry* buffer = s_buffers + (warp * rounds + j) * kBeamBuffer;
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
                uint32_t above = 0, chunk = 0;
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
                        sum *= (double)fast_exp2((top - most) * kLog2e);
                        top = most;
                    }
                    float part = 0.f;
#pragma unroll
                    for (int k = 0; k < 16; ++k) part += fast_exp2((x[k] - top) * kLog2e);
                    sum += (double)part;
                    ++chunk;
                    if ((chunk & (chunk - 1)) == 0) {  // the n-th largest of the lanes' maxima so far: a bitonic sort, descending
                        float v = top;
#pragma unroll
                        for (int size = 2; size <= 32; size <<= 1)
#pragma unroll
                            for (int d = size >> 1; d > 0; d >>= 1) {
                                const float o = __shfl_xor_sync(0xffffffffu, v, d);
                                const bool keep_max = ((lane & d) == 0) == ((lane & size) == 0);
                                v = keep_max ? fmaxf(v, o) : fminf(v, o);
                            }
                        v = __shfl_sync(0xffffffffu, v, n - 1);
                        if (v > least) least = v, above = 0xffffffffu;
                    }
                    if (!__any_sync(0xffffffffu, most >= least)) continue;
                    uint32_t hits = 0;                 // entries of this lane that may stay
#pragma unroll
                    for (int k = 0; k < 16; ++k)
                        if (x[k] >= least) hits |= 1u << k;
                    for (;;) {                         // one of every lane at a time, read again
                        const int k = __ffs((int)hits) - 1;
                        const uint32_t v = (uint32_t)(c0 + (k / kVec * 32 + lane) * kVec + k % kVec);
                        const float z_v = k >= 0 ? widen_one(z[v]) : 0.f;
                        bool mine = k >= 0 && (z_v > least || (z_v == least && v < above));
                        uint32_t in = __ballot_sync(0xffffffffu, mine);
                        if (count + __popc(in) > kBeamBuffer) {
                            __syncwarp();
                            warp_best(buffer, count, n);
                            count = n;                 // (at least n + 1 were in it)
                            least = key_logit(buffer[n - 1].key);
                            above = buffer[n - 1].token;
                            mine = mine && (z_v > least || (z_v == least && v < above));
                            in = __ballot_sync(0xffffffffu, mine);
                        }
                        if (mine) {
                            BeamEntry& e = buffer[count + __popc(in & ((1u << lane) - 1))];
                            e.key = logit_key(z_v);
                            e.token = v;
                        }
                        count += __popc(in);
                        hits &= hits - 1;
                        if (!__any_sync(0xffffffffu, hits != 0)) break;
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
        if (count > n + 32) {
            warp_best(buffer, count, n);
            count = n;
        }
        if (lane == 0) s_count[warp * rounds + j] = count;
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
    // ---- a bound: the n-th best of the slices' largest entries (every CTA for itself; ties by row and slice, which is their
    // candidates' order).  n candidates are at least as good, so neither what is worse nor any other slice holds one of the n best.
    for (int t = tid; t < tasks; t += kBeamThreads) {
        const int row = t % P.beams;
        const bool some = s_alive[row] && s_sum[t] > 0.0;
        s_best[row * P.slices + t / P.beams] = some ? score_key(s_row_off[row] + ((double)s_top[t] - (double)s_row_top[row])) : 0ull;
    }
    __syncthreads();
    for (int t = tid; t < tasks; t += kBeamThreads) {
        const uint64_t mine = s_best[t];
        int better = 0;
        for (int o = 0; o < tasks; ++o) better += s_best[o] > mine || (s_best[o] == mine && o < t);
        s_in[t] = better < n;
        if (better == n - 1) s_least = mine;
    }
    __syncthreads();
    // ---- the candidates that reach it go to the first CTA ...
    {
        const uint64_t least = s_least;
        BeamPick* to = cluster.map_shared_rank(s_picks, 0);
        int* picked = cluster.map_shared_rank(&s_picked, 0);
        for (int j = 0, task = gwarp; j < rounds && task < tasks; ++j, task += warps) {
            const int row = task % P.beams, count = s_count[warp * rounds + j];
            if (!s_alive[row] || !s_in[row * P.slices + task / P.beams]) continue;
            for (int i = lane; i < count; i += 32) {
                const BeamEntry e = s_buffers[(warp * rounds + j) * kBeamBuffer + i];
                BeamPick p;
                p.score = score_key(s_row_off[row] + ((double)key_logit(e.key) - (double)s_row_top[row]));
                p.row = (uint32_t)row;
                p.token = e.token;
                if (p.score < least) continue;
                const int at = atomicAdd(picked, 1);
                if (at < beam_max_picks(n)) to[at] = p;
            }
        }
    }
    cluster.sync();
    if (rank != 0) return;
    // ---- ... which ranks them: the order in which they came does not matter
    const int picked = min(s_picked, beam_max_picks(n));
    auto put = [&](int i, bool there, const BeamPick& p) {
        const size_t at = (size_t)b * n + i, from = (size_t)b * P.beams + p.row;
        P.parents[at] = there ? (int32_t)from : -1;
        P.tokens[at] = there ? (int32_t)p.token : -1;
        P.scores_out[at] = there ? (float)key_score(p.score) : -INFINITY;
        if (P.finished_out) P.finished_out[at] = !there || (int32_t)p.token == P.end_token || (P.finished && P.finished[from] != 0);
    };
    for (int i = tid; i < picked; i += kBeamThreads) {
        const BeamPick p = s_picks[i];
        int better = 0;
        for (int o = 0; o < picked && better < n; ++o) better += s_picks[o].before(p);
        if (better < n) put(better, true, p);
    }
    for (int i = picked + tid; i < n; i += kBeamThreads) put(i, false, BeamPick{0, 0, 0});
}

}  // namespace kvq
