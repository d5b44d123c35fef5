// Attention with sinks over a key-value cache of int8 rows (uq_attn.cuh).
#include "uq_attn.cuh"

namespace uq {

cudaError_t attn_sinks_int8(const AttnArgs& a, cudaStream_t st) { return attn::by_head<UQ_KV_INT8, true>(a, st); }

}  // namespace uq
