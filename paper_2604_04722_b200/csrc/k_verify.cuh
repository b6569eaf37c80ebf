// Verification of drafted tokens against the target's probabilities from given random numbers (speculative sampling on
// a tree).  Row r = 0 of the probabilities is the distribution after the last cached token, row i + 1 the one after
// node i.  From the root, the children of the node reached so far are tested in index order; child i with token x is
// accepted when
//   u_i Z q(x) < r(x),   r = max(p - c q, 0),  Z = sum_v r(v)   (no child turned down yet: c = 0 and Z = 1)
// p, q the target's and the draft's row of that node.  A rejection replaces the target by the normalised residual
// max(r / Z - q, 0); because max(max(p - a q, 0) - b q, 0) = max(p - (a + b) q, 0), that is c += Z and one sum over the
// row.  When no child is left the next token is drawn from r by inverse transform.  Without a draft distribution
// (fixed guesses) q is one at the child's token and zero elsewhere: a rejection takes the token out of r.
//
// The answers are whole numbers, so sums are kept in fp64 (their order then does not matter in practice) and the
// products of the acceptance test are exact or off by one fp64 rounding.
//
// A cluster of CTAs serves a sequence, each with a contiguous slice of the vocabulary, every warp with a contiguous part of
// the slice.  p(x) and q(x) of every node are gathered at once (they do not depend on the walk), so the walk itself is a
// few ballots per tested node, the same in every warp; only a rejection with a sibling behind it, and the final draw, sum
// over a row.  A lane keeps its entries of the row it has last summed over in registers (all loads of a pass are in flight
// at once, row 0 is requested before anything else), so that more rejections at a node, and the draw, cost no memory pass;
// what does not fit (a vocabulary of more than kVerifyKeep * 4096 entries at the full cluster width) is read again.  Every
// warp hands its sum to every CTA of the cluster through distributed shared memory: one cluster barrier per pass and no
// other.  The kernel is a chain of memory round trips (parents and tokens, their probabilities, a row) and exchanges: 9 us for one
// sequence of 8 nodes over 49152 entries, 15 us for 16 sequences of 64 nodes,
// 8 us for 8 of 31 fixed guesses over 32003 entries; the rows alone, 8 bytes per entry, would take 0.1, 1.0 and 0.2 us.
#pragma once
#include <cooperative_groups.h>
#include "kvq_common.cuh"
#include "kvq_rows.h"

namespace kvq {

constexpr int kVerifyThreads = 512, kVerifyWarps = kVerifyThreads / 32;
constexpr int kVerifyMaxCluster = 8;
constexpr int kVerifyKeep = 16;            // vocabulary entries of a row (of each distribution) that a lane keeps

__device__ __forceinline__ double warp_sum_f64(double v) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    return v;
}

// grid = batch * cluster CTAs, block = kVerifyThreads.
__global__ void __launch_bounds__(kVerifyThreads) k_verify_tree(const VerifyParams P) {
    namespace cg = cooperative_groups;
    cg::cluster_group cluster = cg::this_cluster();
    const int ctas = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    const int b = (int)blockIdx.x / ctas;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    __shared__ int s_tok[kMaxTreeNodes];
    __shared__ float s_u[kMaxTreeNodes], s_p[kMaxTreeNodes], s_q[kMaxTreeNodes];
    __shared__ double s_sums[2][kVerifyMaxCluster * kVerifyWarps];         // sums of all warps of the cluster, in vocabulary order; two passes alternate
    __shared__ double s_r[32 * kVerifyKeep];                               // the final draw's part of the row

    cluster.barrier_arrive();                          // (before another CTA's memory is written, all of them have to be there)
    pdl_launch_dependents();
    pdl_wait();                                        // the kernel ahead in the stream may be the one that wrote the probabilities

    const size_t row0 = (size_t)b * (P.nodes + 1);
    // this warp's part of the vocabulary (a multiple of 32 entries, so that the parts of a row read whole lines)
    const int per_warp = (int)(((uint32_t)P.vocab + ctas * kVerifyWarps - 1) / (ctas * kVerifyWarps) + 31) & ~31;
    const long long first = (long long)per_warp * (rank * kVerifyWarps + warp);
    const int lo = (int)min(first, (long long)P.vocab), hi = (int)min(first + per_warp, (long long)P.vocab);

    float pk[kVerifyKeep], qk[kVerifyKeep];                                // entries lo + lane + 32 k of the row `kept`
    int kept = -1;
    auto keep_row = [&](int row) {
        const float* p = P.target + (row0 + row) * P.vocab + lo + lane;
        const float* q = P.draft + (row0 + row) * P.vocab + lo + lane;
#pragma unroll
        for (int k = 0; k < kVerifyKeep; ++k) {
            const bool in = lo + lane + 32 * k < hi;
            pk[k] = in ? __ldg(p + 32 * k) : 0.f;
            qk[k] = in && P.draft ? __ldg(q + 32 * k) : 0.f;
        }
        kept = row;
    };
    auto forget = [&](int token) {                     // a fixed guess that was turned down leaves the kept row
        const int d = token - lo - lane;
#pragma unroll
        for (int k = 0; k < kVerifyKeep; ++k) pk[k] = d == 32 * k ? 0.f : pk[k];
    };

    // every warp holds the parents of nodes `lane` and `lane + 32`; the rest of a node's data is gathered once per CTA
    int par[2] = {-2, -2};
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int i = lane + 32 * k;
        if (i < P.nodes) par[k] = P.parents[(size_t)b * P.nodes + i];
        if (par[k] < -1 || par[k] >= i) par[k] = -2;   // not in use
    }
    const int tok = tid < P.nodes ? P.tokens[(size_t)b * P.nodes + tid] : -1;
    const float u = tid < P.nodes ? P.u_accept[(size_t)b * P.nodes + tid] : 0.f, u_next = P.u_next[b];
    keep_row(0);
    if (tid < P.nodes) {
        const int mine = warp == 0 ? par[0] : par[1];  // (tid = lane + 32 warp, warp < 2)
        float p = 0.f, q = P.draft ? 0.f : 1.f;
        if (mine >= -1 && tok >= 0 && tok < P.vocab) {
            const size_t e = (row0 + mine + 1) * P.vocab + tok;
            p = P.target[e];
            if (P.draft) q = P.draft[e];
        }
        s_tok[tid] = tok;
        s_u[tid] = u;
        s_p[tid] = p;
        s_q[tid] = q;
    }
    __syncthreads();

    int cur = 0;                                       // row of the node reached
    double c = 0.0, Z = 1.0;
    unsigned long long tried = 0;                      // its children that were turned down
    int n_accepted = 0;
    bool pending = false;                              // Z is out of date: a rejection has not been followed by its sum yet
    uint32_t pass = 0;
    // r(v) of the current row from p(v) and q(v) (zero for fixed guesses), as far as fixed guesses were not turned down.  Where no
    // child was turned down q takes no part: a node without children has no draft distribution, and its row may hold anything
    // (zero times what is not finite would be NaN).
    auto residual = [&](float p, float q) -> double { return fmax((double)p - (c != 0.0 ? c * (double)q : 0.0), 0.0); };
    auto turned_down = [&](int v) -> bool {
        if (P.draft) return false;
        for (unsigned long long m = tried; m; m &= m - 1ull)
            if (s_tok[__ffsll((long long)m) - 1] == v) return true;
        return false;
    };
    auto far_entry = [&](int v) -> double {            // of an entry that no lane keeps
        const size_t e = (row0 + cur) * P.vocab + v;
        return turned_down(v) ? 0.0 : residual(P.target[e], P.draft ? P.draft[e] : 0.f);
    };
    const int sums = ctas * kVerifyWarps, per_lane = (sums + 31) / 32;     // sums of a pass, and of them per lane
    double total = 0.0;
    bool plain = false;                                // the residual had no mass: the target itself
#pragma unroll 1
    for (;;) {
        bool wanted = false;                           // a sibling waits for Z
#pragma unroll 1
        for (;;) {
            const uint32_t k0 = __ballot_sync(0xffffffffu, par[0] + 1 == cur), k1 = __ballot_sync(0xffffffffu, par[1] + 1 == cur);
            const unsigned long long left = (((unsigned long long)k1 << 32) | k0) & ~tried;
            if (left == 0 || plain) break;
            if (pending) {
                wanted = true;
                break;
            }
            const int i = __ffsll((long long)left) - 1;            // the children in index order
            const double r = turned_down(s_tok[i]) ? 0.0 : residual(s_p[i], P.draft ? s_q[i] : 0.f);
            if ((double)s_u[i] * Z * (double)s_q[i] < r) {
                if (rank == 0 && tid == 0) P.path[(size_t)b * P.nodes + n_accepted] = i;
                ++n_accepted;
                cur = i + 1;
                c = 0.0;
                Z = 1.0;
                tried = 0;
            } else {
                tried |= 1ull << i;
                if (P.draft) {
                    c += Z;
                    pending = true;
                } else {
                    Z -= r;
                    if (kept == cur) forget(s_tok[i]);
                }
            }
        }
        // the sum of r over the row; every warp's is handed to every CTA
        if (kept != cur) {
            keep_row(cur);
            if (!P.draft)
                for (unsigned long long m = tried; m; m &= m - 1ull) forget(s_tok[__ffsll((long long)m) - 1]);
        }
        double part[2] = {0.0, 0.0};
#pragma unroll
        for (int k = 0; k < kVerifyKeep; ++k) part[k & 1] += residual(pk[k], qk[k]);
        double sum = part[0] + part[1];
#pragma unroll 1
        for (int v = lo + lane + 32 * kVerifyKeep; v < hi; v += 32) sum += far_entry(v);
        sum = warp_sum_f64(sum);
        if (pass == 0) cluster.barrier_wait();
        ++pass;
        if (lane < ctas) *cluster.map_shared_rank(&s_sums[pass & 1][rank * kVerifyWarps + warp], lane) = sum;
        cluster.sync();
        sum = 0.0;
        for (int k = 0; k < per_lane; ++k) {
            const int e = lane * per_lane + k;
            if (e < sums) sum += s_sums[pass & 1][e];
        }
        total = warp_sum_f64(sum);
        if (wanted) {
            Z = total;
            pending = false;
            continue;
        }
        if (total > 0.0 || plain) break;
        plain = true;
        c = 0.0;
        tried = 0;
        kept = -1;
    }
    if (rank == 0) {
        if (tid == 0) P.n_accepted[b] = n_accepted;
        for (int i = n_accepted + tid; i < P.nodes; i += kVerifyThreads) P.path[(size_t)b * P.nodes + i] = -1;
    }

    // ---- the next token: the first v with sum_{w <= v} r(w) > u R.  The warp whose part holds it, from the warps' sums ...
    const double t = (double)u_next * total;
    double upto = 0.0;
    for (int k = 0; k < per_lane; ++k) {
        const int e = lane * per_lane + k;
        if (e < sums) upto += s_sums[pass & 1][e];
    }
    const double own = upto;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const double o = __shfl_up_sync(0xffffffffu, upto, d);
        if (lane >= d) upto += o;
    }
    const uint32_t over = __ballot_sync(0xffffffffu, own > 0.0 && upto > t), some = __ballot_sync(0xffffffffu, own > 0.0);
    if (some == 0) {                                   // no mass at all
        if (rank == 0 && tid == 0) P.next_token[b] = -1;
        return;
    }
    const int at = over ? __ffs(over) - 1 : 31 - __clz(some);      // (u R may reach R by rounding: the last part with mass)
    double before = __shfl_sync(0xffffffffu, upto - own, at);
    int owner = -1;
    for (int k = 0; k < per_lane; ++k) {
        const int e = at * per_lane + k;
        const double s = e < sums ? s_sums[pass & 1][e] : 0.0;
        if (s <= 0.0) continue;
        if (owner >= 0) before += s_sums[pass & 1][owner];
        owner = e;
        if (before + s > t) break;
    }
    if (owner != rank * kVerifyWarps + warp) return;
    // ... and in that part 32 entries at a time: an inclusive scan over the lanes finds the one that passes t
#pragma unroll
    for (int k = 0; k < kVerifyKeep; ++k) s_r[32 * k + lane] = residual(pk[k], qk[k]);
    __syncwarp();
    int token = -1, last_v = -1;
#pragma unroll 1
    for (int v0 = lo; v0 < hi && token < 0; v0 += 32) {
        const int v = v0 + lane, k = v - lo;
        const double r = k < 32 * kVerifyKeep ? s_r[k] : v < hi ? far_entry(v) : 0.0;
        double run = r;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const double o = __shfl_up_sync(0xffffffffu, run, d);
            if (lane >= d) run += o;
        }
        const uint32_t passed = __ballot_sync(0xffffffffu, r > 0.0 && before + run > t), mass = __ballot_sync(0xffffffffu, r > 0.0);
        if (passed) token = v0 + __ffs(passed) - 1;
        if (mass) last_v = v0 + 31 - __clz(mass);
        before += __shfl_sync(0xffffffffu, run, 31);
    }
    if (lane == 0) P.next_token[b] = token >= 0 ? token : last_v;
}

}  // namespace kvq
