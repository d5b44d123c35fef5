// Attention over a key-value cache of bf16 rows (uq_attn.cuh).
#include "uq_attn.cuh"

namespace uq {

cudaError_t attn_bf16(const AttnArgs& a, cudaStream_t st) { return attn::by_head<UQ_KV_BF16>(a, st); }

}  // namespace uq
