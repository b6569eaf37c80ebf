// Launches of the many-row attention and of the draft verification: planning and instantiation.
#include "kvq_rows.h"

#include "k_rows.cuh"
#include "k_verify.cuh"

namespace kvq {

namespace {

template <int NT, bool TREE>
cudaError_t set_smem() {
    const int draft_tiles = TREE ? kMaxTreeNodes / kTileTokens : 0;
    return cudaFuncSetAttribute(k_attend_rows<NT, TREE>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)rows_smem_bytes<NT>(draft_tiles));
}

template <int NT, bool TREE>
void launch(const RowsParams& p, uint64_t ctas, cudaStream_t st) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)ctas);
    cfg.blockDim = dim3(kRowsThreads);
    cfg.dynamicSmemBytes = rows_smem_bytes<NT>(TREE ? (p.nodes + kTileTokens - 1) / kTileTokens : 0);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];                       // may be scheduled behind the kernel ahead of it; see pdl_wait
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    cudaLaunchKernelEx(&cfg, k_attend_rows<NT, TREE>, p);
}

}  // namespace

cudaError_t rows_setup() {
    cudaError_t e = set_smem<1, true>();
    if (e == cudaSuccess) e = set_smem<2, true>();
    if (e == cudaSuccess) e = set_smem<1, false>();
    if (e == cudaSuccess) e = set_smem<2, false>();
    return e;
}

// pairs = (sequence, KV head) pairs.
RowsPlan rows_plan(int sm_count, uint64_t pairs, int rows, int visible_tokens, int splits) {
    RowsPlan plan;
    plan.nt = rows <= 8 ? 1 : 2;
    plan.row_blocks = (uint32_t)((rows + 8 * plan.nt - 1) / (8 * plan.nt));
    const uint64_t units = pairs * plan.row_blocks;
    if (splits > 0) {
        plan.parts = (uint32_t)((splits + kRowsWarps - 1) / kRowsWarps);
        while (plan.parts > 1 && units * plan.parts > rows_max_records(sm_count)) --plan.parts;
        return plan;
    }
    const double tiles = (double)visible_tokens / kTileTokens + 2.0;
    const uint64_t resident = (uint64_t)sm_count * rows_ctas_per_sm(plan.nt);
    // Time of a launch in tiles of one warp: waves of CTAs, each a set-up of about twelve tiles and its warps' shares;
    // parts merged through global records cost about another twelve.
    double best = 0.0;
    for (uint32_t parts = 1; parts <= 64 && (parts == 1 || units * parts <= rows_max_records(sm_count)); ++parts) {
        const double waves = (double)((units * parts + resident - 1) / resident);
        const double share = tiles / (double)(parts * kRowsWarps);
        const double cost = waves * (12.0 + share) + (parts > 1 ? 12.0 : 0.0);
        if (parts == 1 || cost < best) {
            best = cost;
            plan.parts = parts;
        }
    }
    return plan;
}

void rows_launch(const RowsParams& p, const RowsPlan& plan, bool tree, uint64_t pairs, cudaStream_t st) {
    const uint64_t ctas = pairs * plan.row_blocks * plan.parts;
    if (tree) {
        if (plan.nt == 1) launch<1, true>(p, ctas, st);
        else launch<2, true>(p, ctas, st);
    } else {
        if (plan.nt == 1) launch<1, false>(p, ctas, st);
        else launch<2, false>(p, ctas, st);
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
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = ctas;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, k_verify_tree, p);
}

}  // namespace kvq
