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
// A cluster of CTAs serves a sequence, each with a contiguous slice of the vocabulary, every warp with a contiguous
// part of the slice.  p(x) and q(x) of every node are gathered at once (they do not depend on the walk), so the walk
// itself runs in registers, the same in every thread; only a rejection with a sibling behind it, and the final draw,
// read a whole row: 8 bytes per vocabulary entry, one pass, one exchange of the CTAs' sums through distributed shared
// memory.  The kernel is a chain of such passes, latency-bound for few sequences and bound by HBM for many.
#pragma once
#include <cooperative_groups.h>
#include "kvq_common.cuh"
#include "kvq_rows.h"

namespace kvq {

constexpr int kMaxVerifyNodes = 64;
constexpr int kVerifyThreads = 512, kVerifyWarps = kVerifyThreads / 32;
constexpr int kVerifyMaxCluster = 8;
constexpr int kVerifyLoads = 4;            // vocabulary entries a lane has in flight (of each distribution)

__device__ __forceinline__ double warp_sum_f64(double v) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    return v;
}

// grid = batch * cluster CTAs, block = kVerifyThreads.
__global__ void __launch_bounds__(kVerifyThreads) k_verify_tree(const VerifyParams P) {
    namespace cg = cooperative_groups;
    cg::cluster_group cluster = cg::this_cluster();
    const uint32_t ctas = cluster.num_blocks(), rank = cluster.block_rank();
    const int b = (int)(blockIdx.x / ctas);
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    __shared__ int s_par[kMaxVerifyNodes], s_tok[kMaxVerifyNodes], s_gone[kMaxVerifyNodes];
    __shared__ float s_u[kMaxVerifyNodes], s_p[kMaxVerifyNodes], s_q[kMaxVerifyNodes];
    __shared__ double s_warp[kVerifyWarps];                        // sums of the warps' parts of the last pass
    __shared__ double s_total[2][kVerifyMaxCluster];               // sums of the CTAs' slices, two passes alternate

    const size_t row0 = (size_t)b * (P.nodes + 1);
    if (tid < P.nodes) {
        const size_t at = (size_t)b * P.nodes + tid;
        int par = P.parents[at];
        const int tok = P.tokens[at];
        if (par < -1 || par >= tid) par = -2;                      // not in use
        float p = 0.f, q = P.draft ? 0.f : 1.f;
        if (par >= -1 && tok >= 0 && tok < P.vocab) {
            const size_t e = (row0 + par + 1) * P.vocab + tok;
            p = P.target[e];
            if (P.draft) q = P.draft[e];
        }
        s_par[tid] = par;
        s_tok[tid] = tok;
        s_u[tid] = P.u_accept[at];
        s_p[tid] = p;
        s_q[tid] = q;
    }
    __syncthreads();

    // this warp's part of the vocabulary (a multiple of 32 entries, so that the parts of a row read whole lines)
    const int per_warp = (int)(((uint32_t)P.vocab + ctas * kVerifyWarps - 1) / (ctas * kVerifyWarps) + 31) & ~31;
    const long long first = (long long)per_warp * (long long)(rank * kVerifyWarps + warp);
    const int lo = (int)min(first, (long long)P.vocab), hi = (int)min(first + per_warp, (long long)P.vocab);

    int cur = 0;                   // row of the node reached
    double c = 0.0, Z = 1.0;
    int gone = 0;                  // fixed guesses: tokens turned down at this node (s_gone)
    int n_accepted = 0;
    bool pending = false;          // Z is out of date: a rejection has not been followed by its sum yet
    uint32_t pass = 0;

    auto value = [&](double p, double q, int v, double cc) -> double {
        if (P.draft) return fmax(p - cc * q, 0.0);
        for (int k = 0; k < gone; ++k)
            if (s_gone[k] == v) return 0.0;
        return p;
    };
    // Sum of r over the whole row; leaves the warps' and the CTAs' sums in s_warp and s_total[pass & 1].
    auto sum_row = [&](double cc) -> double {
        const float* p = P.target + (row0 + cur) * P.vocab;
        const float* q = P.draft ? P.draft + (row0 + cur) * P.vocab : nullptr;
        double sum = 0.0;
        for (int v0 = lo + lane; v0 < hi; v0 += 32 * kVerifyLoads) {
            float pv[kVerifyLoads], qv[kVerifyLoads];
#pragma unroll
            for (int k = 0; k < kVerifyLoads; ++k) {
                const int v = v0 + 32 * k;
                pv[k] = v < hi ? p[v] : 0.f;
                qv[k] = q && v < hi ? q[v] : 0.f;
            }
#pragma unroll
            for (int k = 0; k < kVerifyLoads; ++k) sum += value(pv[k], qv[k], v0 + 32 * k, cc);
        }
        sum = warp_sum_f64(sum);
        ++pass;
        __syncthreads();                               // the last pass's s_warp is not needed any more
        if (lane == 0) s_warp[warp] = sum;
        __syncthreads();
        double mine = 0.0;
        for (int w = 0; w < kVerifyWarps; ++w) mine += s_warp[w];
        if (tid < (int)ctas) *cluster.map_shared_rank(&s_total[pass & 1][rank], tid) = mine;
        cluster.sync();
        double all = 0.0;
        for (uint32_t k = 0; k < ctas; ++k) all += s_total[pass & 1][k];
        return all;
    };

    for (int i = 0; i < P.nodes; ++i) {                // a child comes behind its parent: one walk in index order
        if (s_par[i] + 1 != cur) continue;
        if (pending && P.draft) {
            Z = sum_row(c);
            pending = false;
        }
        const double r = value(s_p[i], s_q[i], s_tok[i], c);
        if ((double)s_u[i] * Z * (double)s_q[i] < r) {
            if (rank == 0 && tid == 0) P.path[(size_t)b * P.nodes + n_accepted] = i;
            ++n_accepted;
            cur = i + 1;
            c = 0.0;
            Z = 1.0;
            gone = 0;
            __syncthreads();                           // s_gone starts again
        } else if (P.draft) {
            c += Z;
            pending = true;
        } else {
            Z -= r;
            if (tid == 0) s_gone[gone] = s_tok[i];
            __syncthreads();
            ++gone;
        }
    }
    if (rank == 0) {
        if (tid == 0) P.n_accepted[b] = n_accepted;
        for (int i = n_accepted + tid; i < P.nodes; i += kVerifyThreads) P.path[(size_t)b * P.nodes + i] = -1;
    }

    // ---- the next token: the first v with sum_{w <= v} r(w) > u R
    double total = sum_row(c);
    if (!(total > 0.0)) {                              // the residual has no mass: the target itself
        c = 0.0;
        gone = 0;
        total = sum_row(c);
    }
    const double t = (double)P.u_next[b] * total;
    double before = 0.0;
    int owner = -1, last = -1;
    double owner_before = 0.0;
    for (int k = 0; k < (int)ctas; ++k) {
        const double s = s_total[pass & 1][k];
        if (s > 0.0) {
            last = k;
            if (owner < 0 && before + s > t) {
                owner = k;
                owner_before = before;
            }
        }
        before += s;
    }
    if (owner < 0) {                                   // u R reached R by rounding: the last entry that has any mass
        owner = last;
        owner_before = before;
    }
    if (owner < 0) {
        if (rank == 0 && tid == 0) P.next_token[b] = -1;           // no mass at all
        return;
    }
    if ((int)rank != owner) return;
    before = owner_before;
    int mine = -1;
    last = -1;
    double mine_before = 0.0;
    for (int w = 0; w < kVerifyWarps; ++w) {
        const double s = s_warp[w];
        if (s > 0.0) {
            last = w;
            if (mine < 0 && before + s > t) {
                mine = w;
                mine_before = before;
            }
        }
        before += s;
    }
    if (mine < 0) {
        mine = last;
        mine_before = before;
    }
    if (warp != mine) return;
    // every lane takes a contiguous piece of the part
    const float* p = P.target + (row0 + cur) * P.vocab;
    const float* q = P.draft ? P.draft + (row0 + cur) * P.vocab : nullptr;
    const int per_lane = (hi - lo + 31) / 32, l0 = min(lo + lane * per_lane, hi), l1 = min(l0 + per_lane, hi);
    double sum = 0.0;
    int last_v = -1;
    for (int v = l0; v < l1; ++v) {
        const double r = value(p[v], q ? q[v] : 0.f, v, c);
        sum += r;
        if (r > 0.0) last_v = v;
    }
    double upto = sum;                                 // inclusive scan over the lanes
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const double o = __shfl_up_sync(0xffffffffu, upto, d);
        if (lane >= d) upto += o;
    }
    const uint32_t over = __ballot_sync(0xffffffffu, last_v >= 0 && mine_before + upto > t);
    const uint32_t some = __ballot_sync(0xffffffffu, last_v >= 0);
    if (over) {
        if (lane != __ffs(over) - 1) return;
        double run = mine_before + (upto - sum);
        int token = last_v;
        for (int v = l0; v < l1; ++v) {
            const double r = value(p[v], q ? q[v] : 0.f, v, c);
            run += r;
            if (r > 0.0 && run > t) {
                token = v;
                break;
            }
        }
        P.next_token[b] = token;
    } else if (some && lane == 31 - __clz(some)) {
        P.next_token[b] = last_v;
    }
}

}  // namespace kvq
