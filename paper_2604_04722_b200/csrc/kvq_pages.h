// Parameters of the kernels for the paged 16-bit cache (k_pages.cuh, k_page_attn.cuh) and for beam search (k_beams.cuh).
#pragma once
#include <cstddef>
#include <cstdint>
#include "kvq_common.cuh"

namespace kvq {

constexpr int kMaxPageRows = 4096;                     // rows of a batch of tables
constexpr int kMaxPages = 1 << 20;                     // pages of a cache: one bit each in shared memory
constexpr int kMaxBeams = 32;

// n / d for 0 <= n < 2^31 by a multiplication (d >= 1): with s = ceil(log2 d), q = floor(n m / 2^(31+s)) is exact for
// m = floor(2^(31+s) / d) + 1, because m d exceeds 2^(31+s) by at most d <= 2^s (Granlund and Montgomery 1994).
struct FastDiv {
    uint32_t d = 1, m = 0, s = 0;
    FastDiv() = default;
    explicit FastDiv(uint32_t div) : d(div) {
        while ((1ull << s) < div) ++s;
        m = (uint32_t)((1ull << (31 + s)) / div + 1);
    }
    __device__ __forceinline__ uint32_t div(uint32_t n) const { return (uint32_t)(((uint64_t)n * m) >> (31 + s)); }
};

struct PageStepParams {
    const int32_t* tables_in;      // [batch][width]
    int32_t* tables_out;           // the same (may be tables_in without parents)
    const int32_t* lens_in;        // [batch]
    int32_t* lens_out;             // [batch] (may be lens_in)
    const int32_t* parents;        // [batch] or nullptr: every row goes on with its own pages
    const int32_t* new_lens;       // [batch]
    const uint8_t* held;           // [n_pages] or nullptr
    int32_t* cu_new;               // [batch + 1]
    int64_t* slots;                // [max_new]
    int32_t* positions;            // [max_new] or nullptr
    int32_t* copies;               // [batch][3] or nullptr
    uint32_t* status;              // [1]
    int width, batch, n_pages, page_size, max_new;
    FastDiv by_page;
};

struct PageAppendParams {
    uint8_t *Kc, *Vc;              // caches
    int64_t page_stride, slot_stride, head_stride;     // bytes
    const uint4 *K, *V;            // [n_new][row_vecs]
    const int64_t* slots;          // [n_new]
    const int32_t* copies;         // [batch][3] or nullptr
    int64_t n_slots;
    int n_new, batch, n_pages, page_size, row_vecs, head_vecs;     // 16-byte vectors of a token's row and of a head's part
    uint32_t copy_blocks;
    FastDiv by_row, by_head;       // row_vecs and head_vecs
};

struct PageAttnParams {
    const uint8_t *Kc, *Vc;
    int64_t page_stride, slot_stride, head_stride;     // bytes
    const void* Q;                 // [batch][q_heads][D]
    void* O;
    float* lse;                    // [batch][q_heads] or nullptr
    const int32_t* tables;         // [batch][width]
    const int32_t* lens;           // [batch]
    uint32_t* arrivals;            // [CTAs][2], zero between launches
    float* warp_rec;               // [CTAs][warps] records of R (D + 2) floats
    float* cta_rec;                // [CTAs][2 abreast][2] records
    int width, batch, n_pages, page_size, q_heads, kv_heads, group, head_blocks;
    int abreast_log2;              // of the units of a row that a CTA's warps may take side by side: 0 or 1, divides kv_heads * head_blocks
    int cluster_log2;              // of the CTAs that share a stretch of the axis and meet through shared memory (0: no clusters)
    float scale2;                  // softmax scale in log2 units
    FastDiv by_page, by_units, by_blocks;              // page_size, kv_heads * head_blocks, head_blocks
};

struct BeamParams {
    const void* logits;            // [batch][beams][vocab]
    const float* scores;           // [batch][beams]
    const uint8_t* finished;       // [batch][beams] or nullptr
    int32_t *parents, *tokens;     // [batch][n_out]
    float* scores_out;             // [batch][n_out]
    uint8_t* finished_out;         // [batch][n_out] or nullptr
    const void* logits_end;        // first byte behind the logits
    int batch, beams, vocab, n_out, end_token;
    int slices, slice_len;         // pieces of a row, entries of a piece (a multiple of 256)
    int rounds;                    // slices of a warp
    int group_len, per_slice;      // entries of a group of chunks, groups of a slice
    FastDiv by_beams, by_groups;   // beams, per_slice
};

}  // namespace kvq
