// Attention over a key-value cache of 8-bit codes (uq_attn.cuh).
#include "uq_attn.cuh"

namespace uq {

cudaError_t attn_int8(const AttnArgs& a, cudaStream_t st) { return attn::by_head<UQ_KV_INT8, false>(a, st); }

}  // namespace uq
