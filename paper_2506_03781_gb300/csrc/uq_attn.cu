// Attention over the paged key-value cache: the workspace, and the kernels by
// format (uq_attn_bf16.cu, uq_attn_int8.cu, uq_attn_int4.cu).
#include <chrono>

#include "uq_attn.cuh"

namespace uq {

cudaError_t attn_bf16(const AttnArgs& a, cudaStream_t st);
cudaError_t attn_int8(const AttnArgs& a, cudaStream_t st);
cudaError_t attn_int4(const AttnArgs& a, cudaStream_t st);
cudaError_t attn_sinks_bf16(const AttnArgs& a, cudaStream_t st);
cudaError_t attn_sinks_int8(const AttnArgs& a, cudaStream_t st);
cudaError_t attn_sinks_int4(const AttnArgs& a, cudaStream_t st);

int64_t attn_workspace_bytes(int heads, int kv_heads, int head_dim) {
    // flags; per block two partials of its own, and one of each warp
    const int blocks = sm_count(), cols = attn::query_columns(heads / kv_heads, head_dim);
    return 4 * (attn::flag_floats(blocks) + (int64_t)blocks * (2 + attn::most_warps(head_dim)) * cols * (head_dim + 2));
}

cudaError_t launch_attn(const AttnArgs& args, cudaStream_t st) {
    // What a raised flag of the workspace holds: anything else counts as not raised, so nobody has to clear it.
    // Another number for each launch, never 0; a replayed graph finds the flags at 0 again.
    static std::atomic<uint64_t> launches{(uint64_t)std::chrono::steady_clock::now().time_since_epoch().count() * 0x9e3779b97f4a7c15ull};
    AttnArgs a = args;
    a.nonce = launches.fetch_add(1, std::memory_order_relaxed) | 1ull << 63;
    if (a.sinks > 0)
        return a.c.format == UQ_KV_BF16 ? attn_sinks_bf16(a, st) : a.c.format == UQ_KV_INT8 ? attn_sinks_int8(a, st) : attn_sinks_int4(a, st);
    return a.c.format == UQ_KV_BF16 ? attn_bf16(a, st) : a.c.format == UQ_KV_INT8 ? attn_int8(a, st) : attn_int4(a, st);
}

}  // namespace uq
