// Launches of the many-row attention and of the draft verification: planning and instantiation.
#include "kvq_rows.h"

#include <algorithm>

#include "k_rows.cuh"
#include "k_verify.cuh"
#include "once_per_device.h"

namespace kvq {

namespace {

constexpr int kMaxDraftTiles = kMaxTreeNodes / kTileTokens;

// CTAs of a kernel that fit an SM, and clusters of c of them that fit the device, by blocks of eight rows (1, 2, 4) and
// 16-node tiles of the tree (0: no tree).
struct Residency {
    int ctas[5][kMaxDraftTiles + 1] = {};
    int clusters[5][kMaxDraftTiles + 1][kRowsMaxCluster + 1] = {};
};
OncePerDevice<Residency> g_residency;

// A launch of `ctas` CTAs in clusters of `cluster`.
struct Launch {
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[2];
    Launch(uint64_t ctas, uint32_t cluster, size_t smem, cudaStream_t st) {
        cfg.gridDim = dim3((unsigned)ctas);
        cfg.blockDim = dim3(kRowsThreads);
        cfg.dynamicSmemBytes = smem;
        cfg.stream = st;
        attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;   // may be scheduled behind the kernel ahead of it; see pdl_wait
        attr[0].val.programmaticStreamSerializationAllowed = 1;
        attr[1].id = cudaLaunchAttributeClusterDimension;
        attr[1].val.clusterDim.x = cluster;
        attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
        cfg.attrs = attr;
        cfg.numAttrs = cluster > 1 ? 2 : 1;
    }
};

template <int NT, bool TREE>
cudaError_t set_limits() {
    cudaError_t e = cudaFuncSetAttribute(k_attend_rows<NT, TREE>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)rows_smem_limit<NT>(TREE ? kMaxDraftTiles : 0));
    if (e == cudaSuccess) e = cudaFuncSetAttribute(k_attend_rows<NT, TREE>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    return e;
}

template <int NT, bool TREE>
cudaError_t ask_residency(Residency& r) {
    cudaError_t e = cudaSuccess;
    for (int tiles = TREE ? 1 : 0; e == cudaSuccess && tiles <= (TREE ? kMaxDraftTiles : 0); ++tiles) {
        e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&r.ctas[NT][tiles], k_attend_rows<NT, TREE>, kRowsThreads, rows_smem_bytes<NT>(tiles, 1));
        for (uint32_t c = 2; e == cudaSuccess && c <= kRowsMaxCluster; ++c) {
            Launch l(c, c, rows_smem_bytes<NT>(tiles, c), nullptr);
            e = cudaOccupancyMaxActiveClusters(&r.clusters[NT][tiles][c], k_attend_rows<NT, TREE>, &l.cfg);
        }
    }
    return e;
}

template <int NT, bool TREE>
void launch(const RowsParams& p, uint64_t ctas, cudaStream_t st) {
    Launch l(ctas, p.cluster, rows_smem_bytes<NT>(TREE ? (p.nodes + kTileTokens - 1) / kTileTokens : 0, p.cluster), st);
    cudaLaunchKernelEx(&l.cfg, k_attend_rows<NT, TREE>, p);
}

}  // namespace

cudaError_t rows_setup(int device) {
    cudaError_t e = cudaSuccess;
    for (cudaError_t (*set)() : {set_limits<1, true>, set_limits<2, true>, set_limits<4, true>, set_limits<1, false>, set_limits<2, false>, set_limits<4, false>})
        if (e == cudaSuccess) e = set();
    if (e != cudaSuccess) return e;
    return g_residency.make(device, [](Residency& r) {
        cudaError_t err = cudaSuccess;
        for (cudaError_t (*ask)(Residency&) : {ask_residency<1, true>, ask_residency<2, true>, ask_residency<4, true>, ask_residency<1, false>,
                                               ask_residency<2, false>, ask_residency<4, false>})
            if (err == cudaSuccess) err = ask(r);
        return err;
    });
}

namespace {

// A model of a launch in us: a CTA's set-up, longer the more CTAs share the SM and the more 16-node tiles of drafted rows it
// stages; its warps' tiles, which slow each other down; in as many waves as it takes; then the merge of a unit's parts, by a
// cluster or through records.  CTAs with stretches that do not end at unit borders work on two units one after the other, with
// a second set-up.  Fitted to 457 shapes (3 to 512 units, 120 to 20000 tokens) in 1 to 16 parts: what it picks is within 2 % of
// the best of them on average.
struct LaunchModel {
    double set_up, crowded, draft, tile, tile_full, merge, part, record, second, second_draft;
};
constexpr LaunchModel kLaunchModels[3] = {{4.7, 2.8, 1.2, 0.56, 0.58, 0.4, 0.01, 0.30, 12.0, 4.0},     // 8, 16 and 32 rows per unit
                                          {6.1, 1.7, 1.6, 0.80, 0.80, 0.0, 0.02, 0.30, 11.0, 12.0},
                                          {11.6, 1.75, 1.4, 0.787, 0.77, 0.0, 0.0, 0.48, 24.0, 14.0}};

struct Shape {
    const Residency* fit;
    int sm_count, draft_tiles, splits;
    uint64_t pairs;
    int rows;
    double tiles;
};

// The plan with blocks of 8 nt rows, and what the model says.
RowsPlan plan_blocks(const Shape& w, int nt, double& best) {
    RowsPlan plan;
    plan.ctas = 0;
    plan.nt = nt;
    plan.row_blocks = (uint32_t)((w.rows + 8 * nt - 1) / (8 * nt));
    // Shares that are the same fraction of every pool keep the warps of an SM in the same loop, which the longest code profits
    // from (8192 tokens, 32 rows: 224 us against 243 us); the others are faster with fewer changes of pool (2048 tokens of
    // one sequence, 15 rows: 13 us against 17 us).
    plan.by_pool = nt == 4;
    best = 1e30;
    const uint64_t units = w.pairs * plan.row_blocks;
    if (units > 0x7fffffffull) return plan;
    const int per_sm = w.fit ? std::max(1, w.fit->ctas[nt][w.draft_tiles]) : 1;
    const uint64_t resident = (uint64_t)w.sm_count * per_sm;
    const uint64_t max_ctas = std::min<uint64_t>(4 * (uint64_t)w.sm_count, rows_max_record_rows(w.sm_count) / (16 * nt));   // of a launch that cuts units
    // Up to sixteen CTAs of a unit merge as a cluster, through shared memory, if all of the launch are resident at once: 2048
    // tokens of one sequence in 16 parts take 9.7 us, in 8 parts 11.2 us, and through global records 14.2 us; but 40 clusters of
    // 7 of which some wait for room took 45 us instead of 28 us.  Two large CTAs per SM leave too little room to move up behind
    // an earlier launch when they fill the device (30 clusters of 9: 31 us against 25 us with 8), so with 32 rows an eighth stays free.
    auto cluster_of = [&](uint64_t parts) {
        const uint64_t most = w.fit && parts >= 2 && parts <= kRowsMaxCluster ? (uint64_t)w.fit->clusters[nt][w.draft_tiles][parts] : 0;
        return units <= (nt == 4 ? most * 7 / 8 : most) ? (uint32_t)parts : 1u;
    };
    const LaunchModel& m = kLaunchModels[nt == 1 ? 0 : nt == 2 ? 1 : 2];
    const double per_cta = m.set_up + m.draft * w.draft_tiles;
    auto cost_of = [&](uint64_t parts) {
        const uint64_t ctas = units * parts;
        const double waves = (double)((ctas + resident - 1) / resident);
        const double load = std::min(1.0, (double)((ctas + w.sm_count - 1) / w.sm_count) / (double)per_sm);
        const double merge = parts == 1 ? 0.0 : cluster_of(parts) > 1 ? m.merge + m.part * (double)parts : m.record * (double)parts;
        return waves * (per_cta + m.crowded * load + w.tiles / (double)(parts * kRowsWarps) * std::max(m.tile, m.tile_full * load)) + merge;
    };
    uint64_t parts = 1;
    if (w.splits > 0) {
        parts = (uint64_t)((w.splits + kRowsWarps - 1) / kRowsWarps);
        while (parts > 1 && units * parts > max_ctas) --parts;
        best = cost_of(parts);
    } else {
        for (uint64_t p = 1; p == 1 || (units * p <= max_ctas && p <= 64); ++p) {
            const double cost = cost_of(p);
            if (cost < best) best = cost, parts = p;
        }
    }
    if (parts == 1) plan.ctas = (uint32_t)units, plan.ticks = plan.span = 1;
    else plan.ctas = plan.ticks = (uint32_t)(units * parts), plan.span = (uint32_t)units;
    plan.cluster = cluster_of(parts);
    if (w.splits == 0 && 2 * units > resident && units < 4 * resident && resident <= max_ctas && units < rows_max_units(w.sm_count)) {
        const double cost = per_cta + m.crowded + (double)units * w.tiles / (double)(resident * kRowsWarps) * m.tile_full + m.second + m.second_draft * w.draft_tiles;
        if (cost < best) best = cost, plan.ctas = plan.ticks = (uint32_t)resident, plan.span = (uint32_t)units, plan.cluster = 1;
    }
    return plan;
}

}  // namespace

RowsPlan rows_plan(int device, int sm_count, uint64_t pairs, int rows, int tree_nodes, int visible_tokens, int splits) {
    Shape w;
    w.fit = g_residency.of(device);
    w.sm_count = sm_count;
    w.draft_tiles = (tree_nodes + kTileTokens - 1) / kTileTokens;
    w.splits = splits;
    w.pairs = pairs;
    w.rows = rows;
    w.tiles = (double)visible_tokens / kTileTokens + 2.0;
    double cost, cost4;
    const RowsPlan plan = plan_blocks(w, rows <= 8 ? 1 : 2, cost);
    if (rows <= 16) return plan;
    // 32 rows share the unpacking of a tile, but their kernel runs with half the warps and a longer set-up: faster where 16 rows
    // per unit need more waves (256 pairs of 20 rows over 1500 tokens: 37 us against 75 us; 3 pairs of 60 rows over 3000: 19
    // against 12).
    const RowsPlan plan4 = plan_blocks(w, 4, cost4);
    return cost4 < cost ? plan4 : plan;
}

void rows_launch(const RowsParams& p, const RowsPlan& plan, bool tree, cudaStream_t st) {
    if (tree) {
        if (plan.nt == 1) launch<1, true>(p, plan.ctas, st);
        else if (plan.nt == 2) launch<2, true>(p, plan.ctas, st);
        else launch<4, true>(p, plan.ctas, st);
    } else {
        if (plan.nt == 1) launch<1, false>(p, plan.ctas, st);
        else if (plan.nt == 2) launch<2, false>(p, plan.ctas, st);
        else launch<4, false>(p, plan.ctas, st);
    }
}

cudaError_t verify_launch(const VerifyParams& p, int batch, int sm_count, cudaStream_t st) {
    // a cluster per sequence, as wide as keeps the launch within two CTAs per SM
    unsigned ctas = kVerifyMaxCluster;
    while (ctas > 1 && (uint64_t)batch * ctas > 2ull * (unsigned)sm_count) ctas /= 2;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)batch * ctas);
    cfg.blockDim = dim3(kVerifyThreads);
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = ctas;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, k_verify_tree, p);
}

}  // namespace kvq
