// Launch side of the many-row attention (k_rows.cuh) and of the draft verification (k_verify.cuh), which are compiled
// apart from the rest of the library.
#pragma once
#include <cstddef>
#include <cstdint>
#include "kvq_common.cuh"

namespace kvq {

constexpr int kMaxTreeNodes = 64;

struct RowsParams {
    StoreView store;
    const uint32_t* counts;        // [batch][4] pool fills of this layer
    const __half* Q;               // [batch][nodes][q_heads][64]
    __half* O;                     // [batch][nodes][q_heads][64]
    const __half* K;               // [batch][nodes][kv_heads][64]   drafted rows (tree only)
    const __half* V;
    const uint8_t* bits;           // [batch][nodes] or nullptr: fp16 rows (tree only)
    const int32_t* parents;        // [batch][nodes] (tree only)
    float* part_o;                 // [2 * CTAs][8 NT][64] unnormalised
    float2* part_ml;               // [2 * CTAs][8 NT]     (m in log2 units, l)
    uint32_t* part_cnt;            // [units] pieces delivered so far; zero between launches
    int layer, group, nodes, rows; // rows = nodes * group
    uint32_t pairs;                // (sequence, KV head) pairs; unit = row block * pairs + pair
    uint32_t ticks, span;          // ticks per unit and per CTA of the axis on which the units lie end to end
    uint32_t cluster;              // > 1: the CTAs of a unit, in exact parts, are a cluster and merge through shared memory
    bool by_pool;                  // a share is the same fraction of every pool (otherwise a stretch of the pools laid end to end)
    int window, sinks;             // window == 0: everything is visible
};

struct VerifyParams {
    const float* target;           // [batch][nodes + 1][vocab]
    const float* draft;            // the same, or nullptr: fixed guesses
    const int32_t* tokens;         // [batch][nodes]
    const int32_t* parents;        // [batch][nodes]
    const float* u_accept;         // [batch][nodes]
    const float* u_next;           // [batch]
    int32_t* n_accepted;           // [batch]
    int32_t* path;                 // [batch][nodes], -1 behind the last accepted node
    int32_t* next_token;           // [batch]
    int nodes, vocab;
};

// How a launch is cut: blocks of eight rows per unit (1, 2 or 4), units per (sequence, KV head), CTAs, and the axis of RowsParams.
struct RowsPlan {
    int nt = 1;
    uint32_t row_blocks = 1, ctas = 1, ticks = 1, span = 1, cluster = 1;
    bool by_pool = false;
};
constexpr uint32_t kRowsMaxCluster = 16;               // CTAs of a unit that merge through shared memory at most
constexpr int kRowsMaxRows = 32;                       // rows of a unit at most

// What a handle keeps for launches that cut units: rows of partial records, two records for each CTA (at most four CTAs of
// 8 or 16 rows per SM, two of 32), and arrival counters, for at most four times as many units as there are CTAs.
inline size_t rows_max_record_rows(int sm_count) { return 128 * (size_t)sm_count; }
inline size_t rows_max_units(int sm_count) { return 16 * (size_t)sm_count; }

// For every handle with one scale group per row: shared-memory limits of the kernels on this device, and how many of their CTAs fit an SM.
cudaError_t rows_setup(int device);
// pairs: (sequence, KV head) pairs; tree_nodes: 0 without a tree; splits > 0: as many warps per unit as that (rounded up to
// whole CTAs, and down to what the records hold).  ctas == 0: too many units for a launch.
RowsPlan rows_plan(int device, int sm_count, uint64_t pairs, int rows, int tree_nodes, int visible_tokens, int splits);
void rows_launch(const RowsParams& p, const RowsPlan& plan, bool tree, cudaStream_t st);
cudaError_t verify_launch(const VerifyParams& p, int batch, int sm_count, cudaStream_t st);

}  // namespace kvq
