// The paged 16-bit cache and beam search: argument checks and launches of the entry points that need no handle
// (include/kvq.h).  Compiled apart from the rest of the library.
#include "../../include/kvq.h"

#include <algorithm>
#include <cmath>

#include "k_beams.cuh"
#include "k_page_attn.cuh"
#include "k_pages.cuh"
#include "once_per_device.h"

using namespace kvq;

namespace {

static_assert(KVQ_MAX_PAGE_ROWS == kMaxPageRows && KVQ_MAX_PAGES == kMaxPages && KVQ_MAX_BEAMS == kMaxBeams, "the header states what the kernels hold");
static_assert(KVQ_PAGE_FULL == kPageFull && KVQ_PAGE_LONG == kPageLong && KVQ_PAGE_SLOTS == kPageSlots && KVQ_PAGE_BAD == kPageBad, "status bits");

bool aligned(const void* p, size_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) == 0; }
bool overlap(const void* a, size_t a_bytes, const void* b, size_t b_bytes) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return x < y + b_bytes && y < x + a_bytes;
}

// What a device allows, asked for once; the kernels' shared-memory limits and cluster sizes are set on the way.
struct PagesDevice {
    int sm_count = 0, sm_smem = 0;                     // shared memory of an SM, bytes
    int beam_clusters[5] = {};                         // resident clusters of 2^i CTAs of the selection ...
    int attn_clusters[6][5] = {};                      // ... and of the attention: see attn_variant
};
int log2_of(int c) { return c <= 1 ? 0 : 1 + log2_of(c / 2); }

OncePerDevice<PagesDevice> g_device;

template <class Kernel>
cudaError_t allow_smem(Kernel kernel, bool cluster) {
    int most = 0, device = 0;
    cudaFuncAttributes a;
    cudaError_t e = cudaGetDevice(&device);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&most, cudaDevAttrMaxSharedMemoryPerBlockOptin, device);
    if (e == cudaSuccess) e = cudaFuncGetAttributes(&a, kernel);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, most - (int)a.sharedSizeBytes);
    if (e == cudaSuccess && cluster) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    return e;
}

template <class Kernel>
cudaError_t ask_clusters(Kernel kernel, int threads, size_t smem, int (&clusters)[5]) {
    cudaError_t e = cudaSuccess;
    for (int i = 1; i < 5 && e == cudaSuccess; ++i) {
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3(1u << i);
        cfg.blockDim = dim3((unsigned)threads);
        cfg.dynamicSmemBytes = smem;
        cudaLaunchAttribute attr;
        attr.id = cudaLaunchAttributeClusterDimension;
        attr.val.clusterDim.x = 1u << i;
        attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
        cfg.attrs = &attr;
        cfg.numAttrs = 1;
        e = cudaOccupancyMaxActiveClusters(&clusters[i], kernel, &cfg);
    }
    return e;
}

// (All of them have the same threads, registers and shared memory.)
template <class T>
cudaError_t set_up_beams(int (&clusters)[5]) {
    cudaError_t e = allow_smem(k_beam_select<T, true>, true);
    if (e == cudaSuccess) e = allow_smem(k_beam_select<T, false>, true);
    return e == cudaSuccess ? ask_clusters(k_beam_select<T, false>, kBeamThreads, beam_smem(kMaxBeams), clusters) : e;
}

// Both types of a shape are the same to the device; the batch's share of the shared memory is small.
template <int D, int NT, int W>
cudaError_t set_up_attn(int (&clusters)[5]) {
    cudaError_t e = allow_smem(k_page_attn<true, D, NT, W>, true);
    if (e == cudaSuccess) e = allow_smem(k_page_attn<false, D, NT, W>, true);
    return e == cudaSuccess ? ask_clusters(k_page_attn<false, D, NT, W>, AttnGeom<D, W>::kThreads, attn_smem<D, NT, W>(64, true), clusters) : e;
}

const PagesDevice* device_of_call() {
    int device = 0;
    if (cudaGetDevice(&device) != cudaSuccess) return nullptr;
    if (const PagesDevice* d = g_device.of(device)) return d;
    const cudaError_t e = g_device.make(device, [&](PagesDevice& d) {
        cudaError_t err = cudaDeviceGetAttribute(&d.sm_count, cudaDevAttrMultiProcessorCount, device);
        if (err == cudaSuccess) err = cudaDeviceGetAttribute(&d.sm_smem, cudaDevAttrMaxSharedMemoryPerMultiprocessor, device);
        if (err == cudaSuccess) err = allow_smem(k_page_step, false);
        if (err == cudaSuccess) err = set_up_beams<__half>(d.beam_clusters);
        if (err == cudaSuccess) err = set_up_beams<__nv_bfloat16>(d.beam_clusters);
        if (err == cudaSuccess) err = set_up_beams<float>(d.beam_clusters);
        if (err == cudaSuccess) err = set_up_attn<64, 1, 8>(d.attn_clusters[0]);
        if (err == cudaSuccess) err = set_up_attn<64, 2, 8>(d.attn_clusters[1]);
        if (err == cudaSuccess) err = set_up_attn<64, 1, 16>(d.attn_clusters[2]);
        if (err == cudaSuccess) err = set_up_attn<64, 2, 16>(d.attn_clusters[3]);
        if (err == cudaSuccess) err = set_up_attn<128, 1, 8>(d.attn_clusters[4]);
        if (err == cudaSuccess) err = set_up_attn<128, 2, 8>(d.attn_clusters[5]);
        return err;
    });
    if (e != cudaSuccess) cudaGetLastError();          // (reported by the call's return code)
    return g_device.of(device);
}

// May be scheduled behind the kernel ahead of it in the stream (see pdl_wait); in clusters of `cluster` CTAs.
template <class Kernel, class Params>
int launch(Kernel kernel, uint64_t ctas, int threads, size_t smem, int cluster, const Params& p, void* stream) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)ctas);
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = static_cast<cudaStream_t>(stream);
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 0 ? 2 : 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, p);
    if (e == cudaSuccess) return KVQ_OK;
    cudaGetLastError();                                // (nothing was queued; the code says so)
    return KVQ_ERR_CUDA;
}

bool cache_ok(const kvq_page_cache* c) {
    if (!c || !c->K || !c->V || !aligned(c->K, 16) || !aligned(c->V, 16)) return false;
    if (c->n_pages < 1 || c->page_size < 1 || c->kv_heads < 1 || c->kv_heads > 1024) return false;
    if (c->head_dim < 8 || c->head_dim % 8 != 0 || c->head_dim > 1024) return false;
    for (int64_t s : {c->page_stride, c->slot_stride, c->head_stride})
        if (s < 0 || s % 8 != 0) return false;
    return c->dtype == KVQ_FP16 || c->dtype == KVQ_BF16;
}

// The kernel's variants: 64 channels with 8 or 16 warps a CTA, 128 with 8; one or two blocks of eight heads.
int attn_variant(int head_dim, int nt, int warps) { return (head_dim == 128 ? 4 : warps == 16 ? 2 : 0) + nt - 1; }
int attn_resident(int sm_count, int head_dim, int warps) { return std::min(kAttnMaxCtas, sm_count * (1024 / (head_dim * warps))); }

// What the attention keeps in the workspace: arrival counters, then two kinds of records.
struct AttnSpace {
    int nt;
    size_t warp_at, cta_at, bytes;
};
AttnSpace attn_space(int sm_count, int group, int head_dim) {
    AttnSpace s;
    s.nt = group <= 8 ? 1 : 2;
    const size_t record = (size_t)8 * s.nt * (head_dim + 2) * sizeof(float), ctas = (size_t)attn_resident(sm_count, head_dim, 8);
    s.warp_at = (size_t)kAttnCounters * sizeof(uint32_t);
    s.cta_at = s.warp_at + ctas * 8 * record;          // (half as many CTAs of 16 warps need as much)
    s.bytes = s.cta_at + ctas * 2 * kAttnAbreast * record;
    return s;
}
bool attn_shape_ok(int batch, int q_heads, int kv_heads, int head_dim) {
    return batch >= 0 && batch <= KVQ_MAX_PAGE_ROWS && kv_heads >= 1 && kv_heads <= 1024 && q_heads >= kv_heads && q_heads <= 16384 &&
           q_heads % kv_heads == 0 && (head_dim == 64 || head_dim == 128);
}

template <bool BF, int D, int W>
int launch_attn(const PageAttnParams& p, int nt, uint64_t ctas, void* stream) {
    const int threads = AttnGeom<D, W>::kThreads, cluster = p.cluster_log2 > 0 ? 1 << p.cluster_log2 : 0;
    return nt == 1 ? launch(k_page_attn<BF, D, 1, W>, ctas, threads, attn_smem<D, 1, W>(p.batch, cluster > 0), cluster, p, stream)
                   : launch(k_page_attn<BF, D, 2, W>, ctas, threads, attn_smem<D, 2, W>(p.batch, cluster > 0), cluster, p, stream);
}

template <class T>
int launch_beams(const BeamParams& p, bool rows_aligned, int ctas, void* stream) {
    const uint64_t grid = (uint64_t)p.batch * ctas;
    return rows_aligned ? launch(k_beam_select<T, true>, grid, kBeamThreads, beam_smem(p.n_out), ctas, p, stream)
                        : launch(k_beam_select<T, false>, grid, kBeamThreads, beam_smem(p.n_out), ctas, p, stream);
}

}  // namespace

extern "C" {

int kvq_page_step(const int32_t* tables_in, int32_t* tables_out, int table_width, const int32_t* lens_in, int32_t* lens_out,
                  const int32_t* parents_opt, const int32_t* new_lens, int batch, const uint8_t* held_opt, int n_pages,
                  int page_size, int max_new, int32_t* cu_new, int64_t* slots, int32_t* positions_opt, int32_t* copies_opt,
                  uint32_t* status, void* stream) {
    if (batch < 0 || batch > KVQ_MAX_PAGE_ROWS || n_pages < 1 || n_pages > KVQ_MAX_PAGES || page_size < 1 || table_width < 1 || max_new < 0)
        return KVQ_ERR_ARG;
    if (!cu_new || !status || (max_new > 0 && !slots) || (parents_opt && !copies_opt)) return KVQ_ERR_ARG;
    if (batch > 0 && (!tables_in || !tables_out || !lens_in || !lens_out || !new_lens)) return KVQ_ERR_ARG;
    for (const void* p : {(const void*)tables_in, (const void*)tables_out, (const void*)lens_in, (const void*)lens_out, (const void*)parents_opt,
                          (const void*)new_lens, (const void*)cu_new, (const void*)positions_opt, (const void*)copies_opt, (const void*)status})
        if (!aligned(p, 4)) return KVQ_ERR_ARG;
    if (!aligned(slots, 8)) return KVQ_ERR_ARG;
    const size_t bytes = (size_t)batch * table_width * sizeof(int32_t);
    if (batch > 0 && overlap(tables_in, bytes, tables_out, bytes) && (parents_opt || tables_in != tables_out)) return KVQ_ERR_ARG;
    const size_t len_bytes = batch * sizeof(int32_t);
    if (batch > 0 && overlap(lens_in, len_bytes, lens_out, len_bytes) && lens_in != lens_out) return KVQ_ERR_ARG;
    if (!device_of_call()) return KVQ_ERR_CUDA;
    PageStepParams p{};
    p.tables_in = tables_in;
    p.tables_out = tables_out;
    p.lens_in = lens_in;
    p.lens_out = lens_out;
    p.parents = parents_opt;
    p.new_lens = new_lens;
    p.held = held_opt;
    p.cu_new = cu_new;
    p.slots = slots;
    p.positions = positions_opt;
    p.copies = copies_opt;
    p.status = status;
    p.width = table_width;
    p.batch = batch;
    p.n_pages = n_pages;
    p.page_size = page_size;
    p.max_new = max_new;
    p.by_page = FastDiv((uint32_t)page_size);
    return launch(k_page_step, kPageStepCluster, kPageStepThreads, page_step_smem(batch, n_pages), kPageStepCluster, p, stream);
}

int kvq_page_append(const kvq_page_cache* cache, const void* K, const void* V, const int64_t* slots, int n_new,
                    const int32_t* copies_opt, int batch, void* stream) {
    if (!cache_ok(cache) || n_new < 0 || batch < 0) return KVQ_ERR_ARG;
    if (n_new > 0 && (!K || !V || !slots || !aligned(K, 16) || !aligned(V, 16) || !aligned(slots, 8))) return KVQ_ERR_ARG;
    if (copies_opt && (!aligned(copies_opt, 4) || batch > KVQ_MAX_PAGE_ROWS)) return KVQ_ERR_ARG;
    PageAppendParams p{};
    p.copy_blocks = copies_opt ? (uint32_t)batch : 0u;
    if (n_new == 0 && p.copy_blocks == 0) return KVQ_OK;
    p.Kc = static_cast<uint8_t*>(cache->K);
    p.Vc = static_cast<uint8_t*>(cache->V);
    p.page_stride = 2 * cache->page_stride;
    p.slot_stride = 2 * cache->slot_stride;
    p.head_stride = 2 * cache->head_stride;
    p.K = static_cast<const uint4*>(K);
    p.V = static_cast<const uint4*>(V);
    p.slots = slots;
    p.copies = copies_opt;
    p.n_slots = (int64_t)cache->n_pages * cache->page_size;
    p.n_new = n_new;
    p.batch = batch;
    p.n_pages = cache->n_pages;
    p.page_size = cache->page_size;
    p.head_vecs = cache->head_dim / 8;
    p.row_vecs = cache->kv_heads * p.head_vecs;
    p.by_row = FastDiv((uint32_t)p.row_vecs);
    p.by_head = FastDiv((uint32_t)p.head_vecs);
    const int tokens = std::max(1, kPageAppendThreads * kPageAppendVecs / p.row_vecs);
    const uint64_t ctas = (uint64_t)p.copy_blocks + ((uint64_t)n_new + tokens - 1) / tokens;
    if (ctas > 0x7fffffffull) return KVQ_ERR_ARG;
    return launch(k_page_append, ctas, kPageAppendThreads, 0, 0, p, stream);
}

int kvq_page_attn_workspace_bytes(int batch, int q_heads, int kv_heads, int head_dim, uint64_t* bytes_out) {
    if (!bytes_out || !attn_shape_ok(batch, q_heads, kv_heads, head_dim)) return KVQ_ERR_ARG;
    const PagesDevice* d = device_of_call();
    if (!d) return KVQ_ERR_CUDA;
    *bytes_out = attn_space(d->sm_count, q_heads / kv_heads, head_dim).bytes;
    return KVQ_OK;
}

int kvq_page_attn(const kvq_page_cache* cache, const void* Q, void* O, float* lse_opt, const int32_t* tables, int table_width,
                  const int32_t* lens, int batch, int q_heads, float scale, void* workspace, uint64_t workspace_bytes,
                  void* stream) {
    if (!cache_ok(cache) || !attn_shape_ok(batch, q_heads, cache->kv_heads, cache->head_dim) || table_width < 1) return KVQ_ERR_ARG;
    const float scale2 = scale * kLog2e;               // (Inf times a product of zero would be NaN)
    if (!std::isfinite(scale2)) return KVQ_ERR_ARG;
    if (batch == 0) return KVQ_OK;
    if (!Q || !O || !tables || !lens || !workspace || !aligned(Q, 16) || !aligned(O, 16) || !aligned(tables, 4) || !aligned(lens, 4) ||
        !aligned(lse_opt, 4) || !aligned(workspace, 16))
        return KVQ_ERR_ARG;
    const PagesDevice* d = device_of_call();
    if (!d) return KVQ_ERR_CUDA;
    const int D = cache->head_dim;
    PageAttnParams p{};
    p.group = q_heads / cache->kv_heads;
    const AttnSpace space = attn_space(d->sm_count, p.group, D);
    if (workspace_bytes < space.bytes) return KVQ_ERR_NOMEM;
    p.Kc = static_cast<const uint8_t*>(cache->K);
    p.Vc = static_cast<const uint8_t*>(cache->V);
    p.page_stride = 2 * cache->page_stride;
    p.slot_stride = 2 * cache->slot_stride;
    p.head_stride = 2 * cache->head_stride;
    p.Q = Q;
    p.O = O;
    p.lse = lse_opt;
    p.tables = tables;
    p.lens = lens;
    uint8_t* const w = static_cast<uint8_t*>(workspace);
    p.arrivals = reinterpret_cast<uint32_t*>(w);
    p.warp_rec = reinterpret_cast<float*>(w + space.warp_at);
    p.cta_rec = reinterpret_cast<float*>(w + space.cta_at);
    p.width = table_width;
    p.batch = batch;
    p.n_pages = cache->n_pages;
    p.page_size = cache->page_size;
    p.q_heads = q_heads;
    p.kv_heads = cache->kv_heads;
    p.head_blocks = (p.group + 8 * space.nt - 1) / (8 * space.nt);
    p.scale2 = scale2;
    p.by_page = FastDiv((uint32_t)cache->page_size);
    p.by_units = FastDiv((uint32_t)(p.kv_heads * p.head_blocks));
    p.by_blocks = FastDiv((uint32_t)p.head_blocks);
    // Clusters as wide as leaves one for every unit, with two tiles for every warp of the longest that the table could hold.  CTAs
    // of 8 warps, two to an SM, where that is enough (1 x 3000 tokens of 3 heads: 6.7 us, with 16 warps 7.9); of 16, so that a cluster
    // has more warps, where the longest unit would give more than eight tiles to a warp of the widest (1 x 32768 of 5 heads: 13.7 us,
    // with 8 15.9), unless there would be narrower ones (4 of up to 30000 of 2 heads: 15.9 us with 8, 18.2 with 16).
    const double units = (double)batch * p.kv_heads * p.head_blocks, longest = std::ceil((double)table_width * cache->page_size / kAttnTile);
    auto widest = [&](int warps) {
        const int* clusters = d->attn_clusters[attn_variant(D, space.nt, warps)];
        int c = 1;
        while (c < kAttnMaxCluster && longest >= 2.0 * warps * (2 * c) && units <= clusters[log2_of(2 * c)]) c *= 2;
        return c;
    };
    int warps = 8, cluster = widest(warps);
    if (D == 64 && cluster == kAttnMaxCluster && longest > 8.0 * warps * cluster && widest(16) == cluster) warps = 16;
    p.cluster_log2 = log2_of(cluster);
    // Of very many rows the table of their places leaves no room for two CTAs of 8 warps (2 KB for what else a CTA has): one of 16 then
    // (4096 rows of 122 tokens of 8 heads, 1.05 GB: 179 us, with 8 warps 214).
    if (D == 64 && 2 * (attn_smem<64, 1, 8>(batch, false) + 2048) > (size_t)d->sm_smem) warps = 16;
    // Where CTAs take equal shares of many units, two heads side by side in memory are read at the same time: 128 bytes of a row here and
    // there cost DRAM more than 256 (16 x 8192 tokens of 32 heads, slot by slot: 174 us, with one at a time 199, four 175, sixteen 180).
    p.abreast_log2 = cluster == 1 && p.slot_stride > p.head_stride && D == 64 && p.kv_heads * p.head_blocks % 2 == 0 ? kAttnAbreastLog2 : 0;
    // as many CTAs as the tables could give a tile to every warp of, as far as they are resident together
    const int resident = attn_resident(d->sm_count, D, warps);
    const int most = cluster > 1 ? std::min(resident, cluster * d->attn_clusters[attn_variant(D, space.nt, warps)][p.cluster_log2]) : resident;
    const double wanted = std::max(units, std::ceil(units * longest / (warps * cluster)));       // clusters
    const uint64_t ctas = (uint64_t)std::max(1.0, std::min((double)(most / cluster), wanted)) * cluster;
    if (cache->dtype == KVQ_BF16) {
        if (D == 128) return launch_attn<true, 128, 8>(p, space.nt, ctas, stream);
        return warps == 8 ? launch_attn<true, 64, 8>(p, space.nt, ctas, stream) : launch_attn<true, 64, 16>(p, space.nt, ctas, stream);
    }
    if (D == 128) return launch_attn<false, 128, 8>(p, space.nt, ctas, stream);
    return warps == 8 ? launch_attn<false, 64, 8>(p, space.nt, ctas, stream) : launch_attn<false, 64, 16>(p, space.nt, ctas, stream);
}

int kvq_beam_select(const void* logits, int dtype, const float* scores, const uint8_t* finished_opt, int batch, int beams,
                    int vocab, int n_out, int end_token, int32_t* parents, int32_t* tokens, float* scores_out,
                    uint8_t* finished_out_opt, void* stream) {
    if (batch < 0 || batch > (1 << 24) || beams < 1 || beams > KVQ_MAX_BEAMS || vocab < 1 || vocab > (1 << 30) || n_out < 1 || n_out > KVQ_MAX_BEAMS ||
        end_token < -1 || end_token >= vocab || (dtype != KVQ_FP16 && dtype != KVQ_BF16 && dtype != KVQ_FP32))
        return KVQ_ERR_ARG;
    if (batch == 0) return KVQ_OK;
    const size_t size = dtype == KVQ_FP32 ? 4 : 2;
    if (!logits || !scores || !parents || !tokens || !scores_out || (finished_opt && end_token < 0)) return KVQ_ERR_ARG;
    if (!aligned(logits, size) || !aligned(scores, 4) || !aligned(parents, 4) || !aligned(tokens, 4) || !aligned(scores_out, 4)) return KVQ_ERR_ARG;
    // a request's scores and ends are read before its results are written, but other requests' may not be read yet
    const size_t in = (size_t)batch * beams, out = (size_t)batch * n_out;
    auto clash = [&](const void* from, void* to, size_t each) {
        return from && to && !(from == to && n_out == beams) && overlap(from, in * each, to, out * each);
    };
    if (clash(scores, scores_out, sizeof(float)) || clash(finished_opt, finished_out_opt, 1)) return KVQ_ERR_ARG;
    const PagesDevice* d = device_of_call();
    if (!d) return KVQ_ERR_CUDA;
    // a cluster per request, as wide as leaves all of them resident together
    int ctas = kBeamMaxCluster;
    while (ctas > 1 && batch > d->beam_clusters[log2_of(ctas)]) ctas /= 2;
    BeamParams p{};
    p.logits = logits;
    p.logits_end = static_cast<const uint8_t*>(logits) + size * (size_t)batch * beams * vocab;
    p.scores = scores;
    p.finished = finished_opt;
    p.parents = parents;
    p.tokens = tokens;
    p.scores_out = scores_out;
    p.finished_out = finished_out_opt;
    p.batch = batch;
    p.beams = beams;
    p.vocab = vocab;
    p.n_out = n_out;
    p.end_token = end_token;
    // slices of at least a chunk, at most as many as there are warps (a row each where there are more rows)
    p.slices = std::max(1, std::min(ctas * kBeamWarps / beams, (vocab + kBeamChunk - 1) / kBeamChunk));
    p.slice_len = (int)((((int64_t)vocab + p.slices - 1) / p.slices + 255) / 256 * 256);
    p.rounds = (beams * p.slices + ctas * kBeamWarps - 1) / (ctas * kBeamWarps);
    const int most_groups = kBeamGroups / p.rounds, slice_chunks = (p.slice_len + kBeamChunk - 1) / kBeamChunk;
    p.group_len = (slice_chunks + most_groups - 1) / most_groups * kBeamChunk;
    p.per_slice = (p.slice_len + p.group_len - 1) / p.group_len;
    p.by_beams = FastDiv((uint32_t)beams);
    p.by_groups = FastDiv((uint32_t)p.per_slice);
    const bool rows_aligned = aligned(logits, 16) && (size_t)vocab * size % 16 == 0;
    if (dtype == KVQ_FP32) return launch_beams<float>(p, rows_aligned, ctas, stream);
    return dtype == KVQ_BF16 ? launch_beams<__nv_bfloat16>(p, rows_aligned, ctas, stream) : launch_beams<__half>(p, rows_aligned, ctas, stream);
}

}  // extern "C"
