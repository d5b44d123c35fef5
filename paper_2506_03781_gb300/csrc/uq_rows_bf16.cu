// Attention of several new tokens over a key-value cache of bf16 rows (uq_rows.cuh).
#include "uq_rows.cuh"

namespace uq {

cudaError_t rows_bf16(const RowsArgs& a, cudaStream_t st) { return rows::by_head<UQ_KV_BF16>(a, st); }

cudaError_t rows_bf16_error(bool clear, unsigned int* flag) { return rows::error(clear, flag); }

}  // namespace uq
