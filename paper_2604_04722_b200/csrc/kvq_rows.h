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
    float* part_o;                 // [units * parts][8 NT][64] unnormalised
    float2* part_ml;               // [units * parts][8 NT]     (m in log2 units, l)
    uint32_t* part_cnt;            // [units] parts delivered so far; zero between launches
    int layer, group, nodes, rows; // rows = nodes * group
    uint32_t row_blocks, parts;
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

// How a launch is cut: blocks of eight rows per unit (1 or 2), units per (sequence, KV head), parts per unit.
struct RowsPlan {
    int nt = 1;
    uint32_t row_blocks = 1, parts = 1;
};
constexpr int kRowsMaxRows = 16;                       // rows of a partial record

// Partial records (of kRowsMaxRows rows) and arrival counters a handle keeps.
inline size_t rows_max_records(int sm_count) { return 8 * (size_t)sm_count; }

// Once per device and process image: shared-memory limits of the kernels.
cudaError_t rows_setup();
// splits > 0: as many warps per unit as that (rounded up to whole CTAs, and down to what the records hold).
RowsPlan rows_plan(int sm_count, uint64_t pairs, int rows, int visible_tokens, int splits);
void rows_launch(const RowsParams& p, const RowsPlan& plan, bool tree, uint64_t pairs, cudaStream_t st);
cudaError_t verify_launch(const VerifyParams& p, int batch, int sm_count, cudaStream_t st);

}  // namespace kvq
