// What the attention's front end (uq_api.cu) hands to its kernels.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/uq_api.h"

namespace uq {

struct AttnArgs {
    uq_kv_cache c;
    const void* q;
    void* out;
    float* lse;                        // NULL: not wanted
    const int32_t* table;
    const int32_t* seq_lens;
    float* work;
    int64_t q_batch, q_head, out_batch, out_head, table_stride;
    int batch, heads, dtype, page_shift;
    int max_tokens;                    // positions the table has room for, 2^30 at most
    int window;                        // 0: every position
    float scale;
    uint64_t nonce;                    // marks this launch's flags in the workspace
};

namespace attn {
// Columns of the products: query heads of a key/value head that are worked on together.  16 for more than 8, as far as
// registers allow; else the rows are read once for every 8, from L2 but for the first.  16 x 4096 positions of 16 heads
// a key/value head, 16 columns / 8: 64 channels, bf16 rows, fp32 queries 25.4 / 27.5 us; 128 channels, bf16 queries:
// rows of bf16 34.9 / 44.0, 8 bits 30.8 / 34.6; fp32 queries: bf16 56.2 / 45.6, 8 bits 41.3 / 38.6, 4 bits 42.4 / 38.8;
// 256 channels, bf16 queries: bf16 37.2 / 27.0, 8 bits 43.8 / 36.9, 4 bits 53.4 / 36.0.
constexpr int query_columns(int heads_per_kv, int head_dim) { return heads_per_kv > 8 && head_dim <= 128 ? 16 : 8; }
}  // namespace attn

}  // namespace uq
