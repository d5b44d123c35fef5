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
// registers allow; else the rows are read once for every 8, from L2 but for the first.  16 x 4096 positions of 4 key/value
// heads that 16 heads share each, 16 columns / 8, us: 64 channels: rows of bf16 22.6 / 24.4, fp32 queries 25.2 / 27.4; of 8
// bits 19.5 / 22.3, 22.7 / 25.7; of 4 bits 19.9 / 21.4, 23.0 / 24.2.  128 channels, bf16 queries: rows of bf16 34.5 / 44.1, of 8 bits
// 29.8 / 32.9, of 4 bits 31.0 / 32.7; fp32 queries take 8 (by_head): bf16 56.2 / 45.6, 8 bits 41.3 / 38.6, 4 bits 42.4 /
// 38.8.  256 channels, bf16 queries: bf16 37.2 / 27.0, 8 bits 43.8 / 36.9, 4 bits 53.4 / 36.0.  The workspace, whose size
// does not depend on the queries' type, has room for what is returned here.
constexpr int query_columns(int heads_per_kv, int head_dim) { return heads_per_kv > 8 && head_dim <= 128 ? 16 : 8; }
}  // namespace attn

}  // namespace uq
