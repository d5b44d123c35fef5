// Attention over a key-value cache of 4-bit codes (uq_attn.cuh).
#include "uq_attn.cuh"

namespace uq {

cudaError_t attn_int4(const AttnArgs& a, cudaStream_t st) { return attn::by_head<UQ_KV_INT4, false>(a, st); }

}  // namespace uq
