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
// Columns of the products: query heads of a key/value head that are worked on together.
constexpr int query_columns(int heads_per_kv) { return heads_per_kv > 8 ? 16 : 8; }
}  // namespace attn

}  // namespace uq
