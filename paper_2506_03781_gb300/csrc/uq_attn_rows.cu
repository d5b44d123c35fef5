// Attention of several new tokens of each sequence over the paged key-value
// cache, its last ones: chunks of prompts, trees of drafts (see uq_api.h).  On the
// tensor cores (uq_rows.cuh); fp32 results of 256 channels, whose sums have no room in
// a thread's registers there, with a warp for a token and head (uq_rows_plain.cuh): a
// prompt of 2048 tokens of 32 heads over 8 of bf16 rows 10 ms, of 64 tokens 36 us.
#include "uq_launch.h"
#include "uq_rows_plain.cuh"

namespace uq {
namespace {

constexpr int kWarpsOf = 8;

template <int FMT>
__global__ void __launch_bounds__(32 * kWarpsOf) plain_kernel(const RowsArgs a) {
    constexpr int HD = 256;
    __shared__ float qs[kWarpsOf][HD];
    const int warp = threadIdx.x >> 5;
    inputs_ready();
    const int64_t id = (int64_t)blockIdx.x * kWarpsOf + warp, token = id / a.heads;
    const int head = (int)(id - token * a.heads);
    if (a.starts != nullptr) {
        if (token >= a.tokens) return;
        int b = 0, hi = a.batch;                       // the last one that starts at or before it
        while (hi - b > 1) {
            const int mid = (b + hi) / 2;
            if (__ldg(a.starts + mid) <= token) b = mid;
            else hi = mid;
        }
        const int s0 = __ldg(a.starts + b), s1 = __ldg(a.starts + b + 1);
        if (token < s0 || token >= s1) return;
        plain::attend<FMT, HD, UQ_W_F32>(a, b, (int)token - s0, s1 - s0, head, token * a.q_row, token * a.out_row, token, qs[warp]);
    } else {
        if (token >= (int64_t)a.batch * a.most) return;
        const int b = (int)(token / a.most), i = (int)(token - (int64_t)b * a.most);
        const int c = a.counts != nullptr ? min(max(__ldg(a.counts + b), 0), a.most) : a.most;
        if (i >= c) return;
        plain::attend<FMT, HD, UQ_W_F32>(a, b, i, c, head, b * a.q_batch + i * a.q_row, b * a.out_batch + i * a.out_row, token, qs[warp]);
    }
}

template <int FMT>
cudaError_t go(const RowsArgs& a, cudaStream_t st) {
    const int64_t rows = (a.starts != nullptr ? a.tokens : (int64_t)a.batch * a.most) * a.heads;
    return launch_dependent(plain_kernel<FMT>, dim3((unsigned)((rows + kWarpsOf - 1) / kWarpsOf)), dim3(32 * kWarpsOf), 0, st, a);
}

}  // namespace

cudaError_t rows_bf16(const RowsArgs& a, cudaStream_t st);
cudaError_t rows_int8(const RowsArgs& a, cudaStream_t st);
cudaError_t rows_int4(const RowsArgs& a, cudaStream_t st);

int64_t attn_rows_workspace_bytes(int, int, int head_dim) {
    // per block what is open (Open), and two partials of 256 rows (256 channels: 128)
    return sm_count() * (64 + (int64_t)2 * 4 * (head_dim == 256 ? 128 : 256) * (head_dim + 2));
}

cudaError_t launch_attn_rows(const RowsArgs& a, cudaStream_t st) {
    if (a.dtype == UQ_W_F32 && a.c.head_dim == 256)
        return a.c.format == UQ_KV_BF16 ? go<UQ_KV_BF16>(a, st) : a.c.format == UQ_KV_INT8 ? go<UQ_KV_INT8>(a, st) : go<UQ_KV_INT4>(a, st);
    return a.c.format == UQ_KV_BF16 ? rows_bf16(a, st) : a.c.format == UQ_KV_INT8 ? rows_int8(a, st) : rows_int4(a, st);
}

}  // namespace uq
