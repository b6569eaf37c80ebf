// Block tables, slot maps and row storage of the paged 16-bit cache.
//
// k_page_step is a function of its inputs alone: the pages in use are the ones that the rows list, so there is no free list
// and there are no reference counts that could go stale.  Row b takes over the pages of row p_b (its own without parents),
// of which n_b tokens are used.  A page that is not full has one owner: with several children of a row the first keeps it, each of the
// others gets a page of its own for it, and the copy is listed for the kernel that moves rows.  Then
//   pages wanted by row b:  w_b = ceil((n_b + m_b) / S) - kept_b,   kept_b = floor(n_b / S) for a copy, ceil(n_b / S) otherwise
// and the pages wanted, in row order, are the free ones in ascending order.
//
// One cluster does it all; every CTA computes what concerns rows for itself (lengths, prefix sums: no exchange), and marks
// in a bitmap of its own (one bit a page, shared memory) the pages that its part of the tables lists.  After a cluster barrier CTA r joins
// slice r of all bitmaps; the free pages of the slices are counted, one more barrier, and a warp hands out the free pages of a
// word with one bit per lane.  The last barrier makes the tables visible to the threads that write the slots.  The kernel is a chain of
// round trips (lengths, tables, three cluster barriers, slots): see the figures at kPageStepCluster.
#pragma once
#include <cooperative_groups.h>
#include "kvq_common.cuh"
#include "kvq_pages.h"

namespace kvq {

constexpr int kPageStepThreads = 1024, kPageStepWarps = kPageStepThreads / 32;
constexpr int kPageStepCluster = 8;

constexpr uint32_t kPageFull = 1u, kPageLong = 2u, kPageSlots = 4u, kPageBad = 8u;

// Shared memory: five words per row (old length, parent, kept | copy flag, first page wanted, first new token), the bitmap,
// and one word for each of a slice of it.
inline size_t page_step_smem(int batch, int n_pages, int ctas) {
    const size_t words = ((size_t)n_pages + 31) / 32;
    return sizeof(int32_t) * (5 * ((size_t)batch + 1) + words + (words + ctas - 1) / ctas);
}

// Inclusive sums over the block of three values per thread; totals are returned to every thread.
struct Sum3 {
    long long a, b;
    int m;                                             // (a maximum)
};
__device__ __forceinline__ Sum3 block_scan(Sum3 v, Sum3* s_warp, Sum3& total) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const long long a = __shfl_up_sync(0xffffffffu, v.a, d), b = __shfl_up_sync(0xffffffffu, v.b, d);
        const int m = __shfl_up_sync(0xffffffffu, v.m, d);
        if (lane >= d) v.a += a, v.b += b, v.m = max(v.m, m);
    }
    if (lane == 31) s_warp[warp] = v;
    __syncthreads();
    Sum3 w = s_warp[lane];                             // (one warp total per lane: 32 warps)
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const long long a = __shfl_up_sync(0xffffffffu, w.a, d), b = __shfl_up_sync(0xffffffffu, w.b, d);
        const int m = __shfl_up_sync(0xffffffffu, w.m, d);
        if (lane >= d) w.a += a, w.b += b, w.m = max(w.m, m);
    }
    const int before = max(warp - 1, 0);
    const long long a = __shfl_sync(0xffffffffu, w.a, before), b = __shfl_sync(0xffffffffu, w.b, before);
    if (warp > 0) v.a += a, v.b += b;
    total.a = __shfl_sync(0xffffffffu, w.a, 31);
    total.b = __shfl_sync(0xffffffffu, w.b, 31);
    total.m = __shfl_sync(0xffffffffu, w.m, 31);
    return v;
}

// The last row whose first item is at or before `item` (first[0] = 0; rows without items are passed over).
__device__ __forceinline__ int row_of(const int32_t* first, int rows, int item) {
    int lo = 0, hi = rows;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (first[mid] <= item) lo = mid;
        else hi = mid;
    }
    return lo;
}

// grid = one cluster, block = kPageStepThreads.
__global__ void __launch_bounds__(kPageStepThreads, 1) k_page_step(const PageStepParams P) {
    namespace cg = cooperative_groups;
    cg::cluster_group cluster = cg::this_cluster();
    const int ctas = (int)cluster.num_blocks(), rank = (int)cluster.block_rank();
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    extern __shared__ __align__(16) int32_t s_mem[];
    const int B = P.batch, S = P.page_size;
    int32_t* s_old = s_mem;                            // [B] tokens taken over
    int32_t* s_par = s_old + B;                        // [B]
    int32_t* s_kept = s_par + B;                       // [B] entries taken over; bit 31: the page behind them is copied
    int32_t* s_want = s_kept + B;                      // [B + 1] pages wanted by the rows before
    int32_t* s_cu = s_want + B + 1;                    // [B + 1] new tokens of the rows before
    const int words = (P.n_pages + 31) / 32;
    uint32_t* s_map = reinterpret_cast<uint32_t*>(s_cu + B + 1);   // [words] pages listed, by this CTA's part of the tables
    uint32_t* s_before = s_map + words;                // [w1 - w0] free pages of this slice before a word
    const int per_cta = (words + ctas - 1) / ctas, w0 = min(words, rank * per_cta), w1 = min(words, w0 + per_cta);
    __shared__ Sum3 s_scan[32];
    __shared__ uint32_t s_flags;
    __shared__ int s_free[kPageStepCluster];           // free pages of every slice
    __shared__ int s_warp_free[kPageStepWarps];

    pdl_launch_dependents();
    if (tid == 0) s_flags = 0;
    for (int w = tid; w < words; w += kPageStepThreads) s_map[w] = 0;
    pdl_wait();

    // ---- rows: every CTA for itself
    for (int b = tid; b < B; b += kPageStepThreads) {
        s_old[b] = P.lens_in[b];
        s_kept[b] = 0x7fffffff;                        // first child, for now
        s_par[b] = P.parents ? P.parents[b] : b;
    }
    __syncthreads();
    uint32_t flags = 0;
    const long long room = (long long)P.width * S;
    for (int b = tid; b < B; b += kPageStepThreads) {
        const int p = s_par[b];
        if (p < -1 || p >= B) flags |= kPageBad;
        else if (p >= 0) {
            atomicMin(&s_kept[p], b);
            if (s_old[p] < 0 || (long long)s_old[p] > room) flags |= kPageBad;
        }
    }
    __syncthreads();
    const int per = (B + kPageStepThreads - 1) / kPageStepThreads;         // at most kMaxPageRows / kPageStepThreads
    constexpr int kPer = kMaxPageRows / kPageStepThreads;
    int old[kPer], kept[kPer], want[kPer], more[kPer];
    Sum3 mine = {0, 0, 0}, total;
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
        const int b = tid * per + k;
        old[k] = kept[k] = want[k] = more[k] = 0;
        if (k >= per || b >= B) continue;
        const int p = s_par[b];
        if (p >= 0 && p < B && s_old[p] >= 0 && (long long)s_old[p] <= room) {
            old[k] = s_old[p];
            const int full = (int)P.by_page.div((uint32_t)old[k]);
            const bool part = full * (long long)S != old[k], copy = part && s_kept[p] != b;
            kept[k] = copy ? full | (int)0x80000000u : full + (part ? 1 : 0);
        }
        more[k] = P.new_lens[b];
        if (more[k] < 0) {
            flags |= kPageBad;
            more[k] = 0;
        }
        const long long after = (long long)old[k] + more[k];
        if (after > room || after > 0x7fffffffll) flags |= kPageLong;
        else want[k] = (int)((after + S - 1) / S) - (kept[k] & 0x7fffffff);
        mine.a += want[k];
        mine.b += more[k];
        mine.m = max(mine.m, kept[k] & 0x7fffffff);
    }
    if (flags) atomicOr(&s_flags, flags);
    const Sum3 upto = block_scan(mine, s_scan, total); // (its barrier: s_old and s_kept have been read)
    const bool fits = total.a <= P.n_pages && total.b <= P.max_new;
    if (tid == 0 && total.a > P.n_pages) atomicOr(&s_flags, kPageFull);
    if (tid == 0 && total.b > P.max_new) atomicOr(&s_flags, kPageSlots);
    {
        long long a = upto.a - mine.a, t = upto.b - mine.b;
#pragma unroll
        for (int k = 0; k < kPer; ++k) {
            const int b = tid * per + k;
            if (k >= per || b >= B) continue;
            s_old[b] = old[k];
            s_kept[b] = kept[k];
            s_want[b] = fits ? (int)a : 0;
            s_cu[b] = fits ? (int)t : 0;
            a += want[k];
            t += more[k];
        }
        if (tid == 0) {
            s_want[B] = fits ? (int)total.a : 0;
            s_cu[B] = fits ? (int)total.b : 0;
        }
    }
    __syncthreads();

    // ---- the pages that the rows list: stretches of 256 entries, one per warp of the cluster at a time
    const int gwarp = rank * kPageStepWarps + warp, warps = ctas * kPageStepWarps;
    const long long stretches = (long long)((total.m + 255) / 256) * B;
    flags = 0;
    for (long long i = gwarp; i < stretches; i += warps) {
        const int b = (int)(i % B), j0 = (int)(i / B) * 256, n = min(s_kept[b] & 0x7fffffff, j0 + 256);
        if (j0 >= n) continue;
        const int32_t* row = P.tables_in + (size_t)s_par[b] * P.width;
        int page[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) page[k] = j0 + 32 * k + lane < n ? row[j0 + 32 * k + lane] : 0;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            if (j0 + 32 * k + lane >= n) continue;
            if ((uint32_t)page[k] < (uint32_t)P.n_pages) atomicOr(&s_map[page[k] >> 5], 1u << (page[k] & 31));
            else flags = kPageBad;
        }
    }
    // a page to be copied has to be one, too
    for (int b = rank * kPageStepThreads + tid; b < B; b += ctas * kPageStepThreads)
        if (s_kept[b] < 0) {
            const int page = P.tables_in[(size_t)s_par[b] * P.width + (s_kept[b] & 0x7fffffff)];
            if ((uint32_t)page >= (uint32_t)P.n_pages) flags = kPageBad;
        }
    if (flags) atomicOr(&s_flags, flags);
    // the pages of this CTA's slice that are held by somebody else, one bit each
    for (int w = w0 + warp; w < w1; w += kPageStepWarps) {
        const int page = w * 32 + lane;
        const uint32_t bits = __ballot_sync(0xffffffffu, page >= P.n_pages || (P.held && P.held[page] != 0));
        if (lane == 0) s_before[w - w0] = bits;
    }
    cluster.sync();

    // ---- free pages of the slice: their bits replace this CTA's own map of it, which no other CTA reads; s_before becomes
    // their number before each word
    const int per_thread = (w1 - w0 + kPageStepThreads - 1) / kPageStepThreads;
    int count = 0;
    for (int k = 0; k < per_thread; ++k) {
        const int w = w0 + tid * per_thread + k;
        if (w >= w1) break;
        uint32_t used = s_before[w - w0];
        for (int c = 0; c < ctas; ++c) used |= cluster.map_shared_rank(s_map, c)[w];
        s_map[w] = ~used;
        count += __popc(~used);
    }
    flags = 0;
    for (int c = 0; c < ctas; ++c) flags |= *cluster.map_shared_rank(&s_flags, c);
    int upto_me = count;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int o = __shfl_up_sync(0xffffffffu, upto_me, d);
        if (lane >= d) upto_me += o;
    }
    if (lane == 31) s_warp_free[warp] = upto_me;
    __syncthreads();
    int upto_warp = s_warp_free[lane];
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int o = __shfl_up_sync(0xffffffffu, upto_warp, d);
        if (lane >= d) upto_warp += o;
    }
    int first_free = upto_me - count;
    const int warps_before = __shfl_sync(0xffffffffu, upto_warp, max(warp - 1, 0)), slice_free = __shfl_sync(0xffffffffu, upto_warp, 31);
    if (warp > 0) first_free += warps_before;
    for (int k = 0; k < per_thread; ++k) {
        const int w = w0 + tid * per_thread + k;
        if (w >= w1) break;
        s_before[w - w0] = (uint32_t)first_free;
        first_free += __popc(s_map[w]);
    }
    if (tid < ctas) cluster.map_shared_rank(s_free, tid)[rank] = slice_free;
    cluster.sync();

    // ---- the pages wanted are handed out, and the entries taken over move where the tables do
    int slice0 = 0, all_free = 0;
    for (int c = 0; c < ctas; ++c) {
        if (c < rank) slice0 += s_free[c];
        all_free += s_free[c];
    }
    const int wanted = s_want[B];
    if (wanted > all_free) flags |= kPageFull;
    const bool ok = flags == 0;
    if (ok) {
        for (int w = w0 + warp; w < w1; w += kPageStepWarps) {
            const int i0 = slice0 + (int)s_before[w - w0];
            if (i0 >= wanted) break;                   // (the words of a slice are in order)
            const uint32_t bits = s_map[w];
            const int i = i0 + __popc(bits & ((1u << lane) - 1));
            if (((bits >> lane) & 1u) == 0 || i >= wanted) continue;
            const int b = row_of(s_want, B, i);
            P.tables_out[(size_t)b * P.width + (s_kept[b] & 0x7fffffff) + (i - s_want[b])] = w * 32 + lane;
        }
    }
    if (P.tables_out != P.tables_in) {                 // (without a step the rows stay as they were)
        for (int b = gwarp; b < B; b += warps) {
            const int len = ok ? 0 : P.lens_in[b];
            const int n = ok ? s_kept[b] & 0x7fffffff : len < 0 || (long long)len > room ? 0 : (int)(((long long)len + S - 1) / S);
            const int32_t* from = P.tables_in + (size_t)(ok ? s_par[b] : b) * P.width;
            int32_t* to = P.tables_out + (size_t)b * P.width;
#pragma unroll 8
            for (int j = lane; j < n; j += 32) to[j] = from[j];
        }
    }
    cluster.sync();

    // ---- slots of the new tokens, lengths, copies
    const int thread = rank * kPageStepThreads + tid, threads = ctas * kPageStepThreads;
    const int fresh = ok ? s_cu[B] : 0;
    for (long long t = thread; t < P.max_new; t += threads) {
        long long slot = -1;
        int pos = -1;
        if (t < fresh) {
            const int b = row_of(s_cu, B, (int)t);
            pos = s_old[b] + (int)t - s_cu[b];
            const int entry = (int)P.by_page.div((uint32_t)pos);
            slot = (long long)__ldcg(P.tables_out + (size_t)b * P.width + entry) * S + (pos - entry * S);
        }
        P.slots[t] = slot;
        if (P.positions) P.positions[t] = pos;
    }
    for (int b = thread; b < B; b += threads) {
        P.lens_out[b] = ok ? s_old[b] + s_cu[b + 1] - s_cu[b] : P.lens_in[b];
        if (!P.copies) continue;
        int32_t* c = P.copies + 3 * (size_t)b;
        const bool copy = ok && s_kept[b] < 0;
        const int full = s_kept[b] & 0x7fffffff;
        c[0] = copy ? P.tables_in[(size_t)s_par[b] * P.width + full] : -1;
        c[1] = copy ? __ldcg(P.tables_out + (size_t)b * P.width + full) : -1;
        c[2] = copy ? s_old[b] - full * S : 0;
    }
    for (int b = thread; b <= B; b += threads) P.cu_new[b] = ok ? s_cu[b] : 0;
    if (thread == 0) *P.status = flags;
}

// Rows to their slots, and the used part of the pages that a step copied: 16-byte vectors, no row is touched twice.  The first
// copy_blocks CTAs take a copy each.  Bound by the rows' bytes, once in and once out.
constexpr int kPageAppendThreads = 256, kPageAppendVecs = 4;

__global__ void __launch_bounds__(kPageAppendThreads) k_page_append(const PageAppendParams P) {
    pdl_launch_dependents();
    pdl_wait();
    auto place = [&](int page, int slot, int vec) -> int64_t {     // byte offset in either cache
        const int head = (int)P.by_head.div((uint32_t)vec);
        return page * P.page_stride + slot * P.slot_stride + head * P.head_stride + (vec - head * P.head_vecs) * 16;
    };
    if (blockIdx.x < P.copy_blocks) {
        const int32_t* c = P.copies + 3 * (size_t)blockIdx.x;
        const int src = c[0], dst = c[1], rows = c[2];
        if ((uint32_t)src >= (uint32_t)P.n_pages || (uint32_t)dst >= (uint32_t)P.n_pages || rows <= 0 || rows > P.page_size) return;
        const int64_t n = (int64_t)rows * P.row_vecs;
#pragma unroll 4
        for (int64_t i = threadIdx.x; i < n; i += kPageAppendThreads) {
            const int r = (int)(i / P.row_vecs), vec = (int)(i - (int64_t)r * P.row_vecs);
            const int64_t from = place(src, r, vec), to = place(dst, r, vec);
            const uint4 k = *reinterpret_cast<const uint4*>(P.Kc + from), v = *reinterpret_cast<const uint4*>(P.Vc + from);
            *reinterpret_cast<uint4*>(P.Kc + to) = k;
            *reinterpret_cast<uint4*>(P.Vc + to) = v;
        }
        return;
    }
    const int tokens = max(1, kPageAppendThreads * kPageAppendVecs / P.row_vecs);      // of this CTA
    const int t0 = (int)(blockIdx.x - P.copy_blocks) * tokens;
    const int n = min(tokens, P.n_new - t0) * P.row_vecs;
    for (int base = threadIdx.x; base < n; base += kPageAppendThreads * kPageAppendVecs) {
        uint4 k[kPageAppendVecs], v[kPageAppendVecs];
        int64_t at[kPageAppendVecs];
#pragma unroll
        for (int u = 0; u < kPageAppendVecs; ++u) {
            const int i = base + u * kPageAppendThreads;
            at[u] = -1;
            if (i >= n) continue;
            const int t = (int)P.by_row.div((uint32_t)i), vec = i - t * P.row_vecs;
            const int64_t slot = P.slots[t0 + t];
            if (slot < 0 || slot >= P.n_slots) continue;           // padding
            const int64_t e = (int64_t)t0 * P.row_vecs + i;
            k[u] = __ldg(P.K + e);
            v[u] = __ldg(P.V + e);
            const int page = (int)(slot / P.page_size);
            at[u] = place(page, (int)(slot - (int64_t)page * P.page_size), vec);
        }
#pragma unroll
        for (int u = 0; u < kPageAppendVecs; ++u)
            if (at[u] >= 0) {
                *reinterpret_cast<uint4*>(P.Kc + at[u]) = k[u];
                *reinterpret_cast<uint4*>(P.Vc + at[u]) = v[u];
            }
    }
}

}  // namespace kvq
