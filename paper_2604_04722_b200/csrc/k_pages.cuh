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
// word with one bit per lane.  The last barrier makes the tables visible to the threads that write the slots.
//
// Bound: a chain of round trips (lengths, tables, three cluster barriers, slots) and scans: 7 us for 8 rows of 2048 tokens, 10 us for 256
// rows of 4 beams and up to 4096, 11 us for 36096 slots; what it reads and writes would take 0.1.
#pragma once
#include <cooperative_groups.h>
#include "kvq_common.cuh"
#include "kvq_pages.h"

namespace kvq {

// 512 rows of 8192 tokens take 18 us, with 4 CTAs 26 and with 2 39; 8 rows 7 us with any of them.  1024 threads a CTA: 8 rows 10 us, 256: 512 rows 25 us.
constexpr int kPageStepThreads = 512, kPageStepWarps = kPageStepThreads / 32;
constexpr int kPageStepCluster = 8;

constexpr uint32_t kPageFull = 1u, kPageLong = 2u, kPageSlots = 4u, kPageBad = 8u;

// Shared memory: five words per row (old length, parent, kept | copy flag, first page wanted, first new token), the bitmap,
// and one word for each of a slice of it.
inline size_t page_step_smem(int batch, int n_pages) {
    const size_t words = ((size_t)n_pages + 31) / 32;
    return sizeof(int32_t) * (5 * ((size_t)batch + 1) + words + (words + kPageStepCluster - 1) / kPageStepCluster);
}

// Sums that stay at 2^32 - 1 instead of passing it: pages and tokens are counted up to limits far below.
__device__ __forceinline__ uint32_t add_sat(uint32_t a, uint32_t b) { return a + b < a ? 0xffffffffu : a + b; }

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
    constexpr int kCtas = kPageStepCluster, kWarps = kPageStepWarps, kThreads = kPageStepThreads;
    const int rank = (int)cluster.block_rank(), tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
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
    const int per_cta = (words + kCtas - 1) / kCtas, w0 = min(words, rank * per_cta), w1 = min(words, w0 + per_cta);
    __shared__ uint32_t s_scan[2][kWarps];
    __shared__ int s_most[kWarps], s_warp_free[kWarps];
    __shared__ uint32_t s_flags;                       // the same in all CTAs after the first exchange
    __shared__ int s_free[kCtas];                      // free pages of every slice

    if (tid == 0) s_flags = 0;
    cluster.barrier_arrive();                          // (before another CTA's memory is written, all of them have to be there)
    pdl_launch_dependents();
    for (int w = tid; w < words; w += kThreads) s_map[w] = 0;
    pdl_wait();

    // ---- rows: every CTA for itself
    for (int b = tid; b < B; b += kThreads) {
        const int len = P.lens_in[b], parent = P.parents ? P.parents[b] : b, more = P.new_lens[b];
        s_old[b] = len;
        s_par[b] = parent;
        s_cu[b] = more;                                // for now
        s_kept[b] = P.parents ? 0x7fffffff : b;        // first child, for now
    }
    // meanwhile the pages of this CTA's slice that are held by somebody else, one bit each: sixteen pages a thread
    for (int h = tid; h < 2 * (w1 - w0); h += kThreads) {
        const int page = w0 * 32 + 16 * h;
        uint32_t bits = 0;
        if (page + 16 > P.n_pages || (P.held && (reinterpret_cast<uintptr_t>(P.held) & 15u))) {
            uint8_t v[16];
#pragma unroll
            for (int k = 0; k < 16; ++k) v[k] = page + k >= P.n_pages ? 1 : P.held ? P.held[page + k] : 0;
#pragma unroll
            for (int k = 0; k < 16; ++k) bits |= (v[k] ? 1u : 0u) << k;
        } else if (P.held) {
            const uint4 v = *reinterpret_cast<const uint4*>(P.held + page);
            const uint32_t word[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int k = 0; k < 16; ++k)
                if ((word[k / 4] >> (8 * (k & 3))) & 0xffu) bits |= 1u << k;
        }
        reinterpret_cast<uint16_t*>(s_before)[h] = (uint16_t)bits;
    }
    __syncthreads();
    uint32_t flags = 0;
    const long long room = (long long)P.width * S;
    if (P.parents) {
        for (int b = tid; b < B; b += kThreads) {
            const int p = s_par[b];
            if (p < -1 || p >= B) flags |= kPageBad;
            else if (p >= 0) atomicMin(&s_kept[p], b);
        }
        __syncthreads();
    }
    const int per = (B + kThreads - 1) / kThreads;     // at most kPer
    constexpr int kPer = kMaxPageRows / kThreads;
    int old[kPer], kept[kPer], more[kPer];
    uint32_t want[kPer], sum_want = 0, sum_more = 0;
    int most = 0;
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
        if (k >= per) break;
        const int b = tid * per + k;
        old[k] = kept[k] = more[k] = 0;
        want[k] = 0;
        if (b >= B) continue;
        const int p = s_par[b];
        if (p >= 0 && p < B) {
            const int n = s_old[p];
            if (n < 0 || (long long)n > room) flags |= kPageBad;
            else {
                const int full = (int)P.by_page.div((uint32_t)n);
                const bool part = full * (long long)S != n, copy = part && s_kept[p] != b;
                old[k] = n;
                kept[k] = copy ? full | (int)0x80000000u : full + (part ? 1 : 0);
            }
        }
        more[k] = s_cu[b];
        if (more[k] < 0) {
            flags |= kPageBad;
            more[k] = 0;
        }
        const long long after = (long long)old[k] + more[k];
        if (after > room || after > 0x7fffffffll) flags |= kPageLong;
        else want[k] = P.by_page.div((uint32_t)after) + (P.by_page.div((uint32_t)after) * (long long)S != after ? 1u : 0u) - (uint32_t)(kept[k] & 0x7fffffff);
        sum_want = add_sat(sum_want, want[k]);
        sum_more = add_sat(sum_more, (uint32_t)more[k]);
        most = max(most, kept[k] & 0x7fffffff);
    }
    if (flags) atomicOr(&s_flags, flags);
    uint32_t upto_want = sum_want, upto_more = sum_more;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const uint32_t a = __shfl_up_sync(0xffffffffu, upto_want, d), t = __shfl_up_sync(0xffffffffu, upto_more, d);
        if (lane >= d) upto_want = add_sat(upto_want, a), upto_more = add_sat(upto_more, t);
    }
    most = __reduce_max_sync(0xffffffffu, most);
    if (lane == 31) s_scan[0][warp] = upto_want, s_scan[1][warp] = upto_more, s_most[warp] = most;
    __syncthreads();                                   // (and all have read s_old, s_kept and s_cu of other rows)
    uint32_t all_want = 0, all_more = 0, before_want = 0, before_more = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
        if (w == warp) before_want = all_want, before_more = all_more;
        all_want = add_sat(all_want, s_scan[0][w]);
        all_more = add_sat(all_more, s_scan[1][w]);
        most = max(most, s_most[w]);
    }
    const bool fits = all_want <= (uint32_t)P.n_pages && all_more <= (uint32_t)P.max_new;
    if (tid == 0 && all_want > (uint32_t)P.n_pages) atomicOr(&s_flags, kPageFull);
    if (tid == 0 && all_more > (uint32_t)P.max_new) atomicOr(&s_flags, kPageSlots);
    before_want += upto_want - sum_want;               // (what is used below did not reach the limit)
    before_more += upto_more - sum_more;
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
        if (k >= per) break;
        const int b = tid * per + k;
        if (b >= B) continue;
        s_old[b] = old[k];
        s_kept[b] = kept[k];
        s_want[b] = fits ? (int)before_want : 0;
        s_cu[b] = fits ? (int)before_more : 0;
        before_want += want[k];
        before_more += (uint32_t)more[k];
    }
    if (tid == 0) {
        s_want[B] = fits ? (int)all_want : 0;
        s_cu[B] = fits ? (int)all_more : 0;
    }
    __syncthreads();

    // ---- the pages that the rows list, stretches of 256 entries to a warp of the cluster at a time: marked, and on their way to
    // where the tables go
    const int gwarp = rank * kWarps + warp;
    const bool moves = P.tables_out != P.tables_in;
    const long long stretches = (long long)((most + 255) / 256) * B;
    flags = 0;
    for (long long i = gwarp; i < stretches; i += kCtas * kWarps) {
        const int b = i < B ? (int)i : (int)(i % B), j0 = i < B ? 0 : (int)(i / B) * 256, n = min(s_kept[b] & 0x7fffffff, j0 + 256);
        if (j0 >= n) continue;
        const int32_t* row = P.tables_in + (size_t)s_par[b] * P.width + j0;
        int page[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) page[k] = j0 + 32 * k + lane < n ? row[32 * k + lane] : 0;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            if (j0 + 32 * k + lane >= n) continue;
            if ((uint32_t)page[k] < (uint32_t)P.n_pages) atomicOr(&s_map[page[k] >> 5], 1u << (page[k] & 31));
            else flags = kPageBad;
            if (moves) P.tables_out[(size_t)b * P.width + j0 + 32 * k + lane] = page[k];
        }
    }
    // a page to be copied has to be one, too
    for (int b = rank * kThreads + tid; b < B; b += kCtas * kThreads)
        if (s_kept[b] < 0) {
            const int page = P.tables_in[(size_t)s_par[b] * P.width + (s_kept[b] & 0x7fffffff)];
            if ((uint32_t)page >= (uint32_t)P.n_pages) flags = kPageBad;
        }
    cluster.barrier_wait();                            // (all CTAs are there)
    if (flags)
        for (int c = 0; c < kCtas; ++c) atomicOr(cluster.map_shared_rank(&s_flags, c), flags);
    cluster.sync();

    // ---- free pages of the slice: their bits replace this CTA's own map of it, which no other CTA reads; s_before becomes
    // their number before each word
    const int per_thread = (w1 - w0 + kThreads - 1) / kThreads;
    int count = 0;
    for (int k = 0; k < per_thread; ++k) {
        const int w = w0 + tid * per_thread + k;
        if (w >= w1) break;
        uint32_t used = s_before[w - w0];
#pragma unroll
        for (int c = 0; c < kCtas; ++c) used |= cluster.map_shared_rank(s_map, c)[w];
        s_map[w] = ~used;
        count += __popc(~used);
    }
    flags = s_flags;
    int upto = count;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int o = __shfl_up_sync(0xffffffffu, upto, d);
        if (lane >= d) upto += o;
    }
    if (lane == 31) s_warp_free[warp] = upto;
    __syncthreads();
    int first_free = upto - count, slice_free = 0;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
        if (w == warp) first_free += slice_free;
        slice_free += s_warp_free[w];
    }
    if (tid < kCtas) cluster.map_shared_rank(s_free, tid)[rank] = slice_free;
    for (int k = 0; k < per_thread; ++k) {
        const int w = w0 + tid * per_thread + k;
        if (w >= w1) break;
        s_before[w - w0] = (uint32_t)first_free;
        first_free += __popc(s_map[w]);
    }
    cluster.sync();

    // ---- the pages wanted are handed out
    int slice0 = 0, all_free = 0;
#pragma unroll
    for (int c = 0; c < kCtas; ++c) {
        if (c < rank) slice0 += s_free[c];
        all_free += s_free[c];
    }
    const int wanted = s_want[B];
    if (wanted > all_free) flags |= kPageFull;
    const bool ok = flags == 0;
    if (ok) {
        for (int w = w0 + warp; w < w1; w += kWarps) {
            const int i0 = slice0 + (int)s_before[w - w0];
            if (i0 >= wanted) break;                   // (the words of a slice are in order)
            const uint32_t bits = s_map[w];
            const int i = i0 + __popc(bits & ((1u << lane) - 1));
            if (((bits >> lane) & 1u) == 0 || i >= wanted) continue;
            const int b = row_of(s_want, B, i);
            P.tables_out[(size_t)b * P.width + (s_kept[b] & 0x7fffffff) + (i - s_want[b])] = w * 32 + lane;
        }
    } else if (moves) {                                // without a step the rows are those that came in
        for (int b = gwarp; b < B; b += kCtas * kWarps) {
            const int len = P.lens_in[b];
            const int n = len < 0 || (long long)len > room ? 0 : (int)(((long long)len + S - 1) / S);
            for (int j = lane; j < n; j += 32) P.tables_out[(size_t)b * P.width + j] = P.tables_in[(size_t)b * P.width + j];
        }
    }
    cluster.sync();

    // ---- slots of the new tokens, four neighbours a thread, and lengths and copies, by other CTAs if there are few tokens
    const int thread = rank * kThreads + tid, threads = kCtas * kThreads, fresh = ok ? s_cu[B] : 0;
    for (int b = (kCtas - 1 - rank) * kThreads + tid; b <= B; b += threads) {
        P.cu_new[b] = ok ? s_cu[b] : 0;
        if (b == B) break;
        P.lens_out[b] = ok ? s_old[b] + s_cu[b + 1] - s_cu[b] : P.lens_in[b];
        if (!P.copies) continue;
        int32_t* c = P.copies + 3 * (size_t)b;
        const bool copy = ok && s_kept[b] < 0;
        const int full = s_kept[b] & 0x7fffffff;
        c[0] = copy ? P.tables_in[(size_t)s_par[b] * P.width + full] : -1;
        c[1] = copy ? __ldcg(P.tables_out + (size_t)b * P.width + full) : -1;
        c[2] = copy ? s_old[b] - full * S : 0;
    }
    if (thread == 0) *P.status = flags;
    const bool vectors = ((reinterpret_cast<uintptr_t>(P.slots) | reinterpret_cast<uintptr_t>(P.positions)) & 15u) == 0;
    for (long long t0 = 4ll * thread; t0 < P.max_new; t0 += 4ll * threads) {
        int pos[4], offset[4], page[4];
        int b = t0 < fresh ? row_of(s_cu, B, (int)t0) : B;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const long long t = t0 + k;
            pos[k] = page[k] = -1;
            offset[k] = 0;
            if (t >= fresh) continue;
            while (s_cu[b + 1] <= (int)t) ++b;         // (there is a row with this token)
            pos[k] = s_old[b] + (int)t - s_cu[b];
            const int entry = (int)P.by_page.div((uint32_t)pos[k]);
            offset[k] = pos[k] - entry * S;
            page[k] = __ldcg(P.tables_out + (size_t)b * P.width + entry);
        }
        long long slot[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) slot[k] = pos[k] < 0 ? -1ll : (long long)page[k] * S + offset[k];
        if (t0 + 4 <= P.max_new && vectors) {
            *reinterpret_cast<longlong2*>(P.slots + t0) = make_longlong2(slot[0], slot[1]);
            *reinterpret_cast<longlong2*>(P.slots + t0 + 2) = make_longlong2(slot[2], slot[3]);
            if (P.positions) *reinterpret_cast<int4*>(P.positions + t0) = make_int4(pos[0], pos[1], pos[2], pos[3]);
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if (t0 + k >= P.max_new) break;
                P.slots[t0 + k] = slot[k];
                if (P.positions) P.positions[t0 + k] = pos[k];
            }
        }
    }
}

// Rows to their slots, and the used part of the pages that a step copied: 16-byte vectors, no row is touched twice.  The first
// copy_blocks CTAs take a copy each.  Bound by the rows' bytes, once in and once out: 15000 rows of 32 heads (246 MB) take 38.9 us, 6.3 TB/s or
// 0.97 of the copy rate; a few rows 2 us.
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
