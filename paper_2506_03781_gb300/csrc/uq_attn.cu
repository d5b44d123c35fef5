// Attention of one new token of each sequence over the paged key-value cache
// (see uq_api.h), the plain way: a block per sequence and head, a warp per
// cached token, a running maximum and sum per warp, the warps joined at the end.
#include "uq_kv.cuh"
#include "uq_attn.h"
#include "uq_launch.h"

namespace uq {
namespace {

template <int FMT, int HD>
__device__ __forceinline__ float kv_value(const void* rows, const void* scales, int64_t row, int d) {
    using R = KvRow<FMT, HD>;
    const uint8_t* src = static_cast<const uint8_t*>(rows) + row * R::kBytes;
    if constexpr (FMT == UQ_KV_BF16) {
        return __uint_as_float((uint32_t)reinterpret_cast<const uint16_t*>(src)[d] << 16);
    } else if constexpr (FMT == UQ_KV_INT8) {
        return __fmul_rn((float)(int8_t)src[d], static_cast<const float*>(scales)[row]);
    } else {
        const uint32_t w = static_cast<const uint32_t*>(scales)[row * R::kWords + d / kKvGroup];
        return __fmaf_rn((float)((src[d / 2] >> (4 * (d & 1))) & 15), bf16_low(w), bf16_high(w));
    }
}

template <int FMT, int HD, int WD>
__global__ void __launch_bounds__(kThreads) attn_kernel(AttnArgs a) {
    constexpr int NV = HD / 32;
    __shared__ float sm_m[kWarps], sm_l[kWarps], sm_o[kWarps][HD];
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    inputs_ready();
    const int b = blockIdx.y, h = blockIdx.x, kvh = h / (a.heads / a.c.kv_heads);
    const int64_t cap = a.max_pages << a.page_shift;
    const int64_t n = min((int64_t)a.seq_lens[b], cap);
    const int64_t first = a.window > 0 ? max((int64_t)0, n - a.window) : 0;
    float q[NV], o[NV], m = -INFINITY, l = 0.0f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int64_t e = b * a.q_batch + h * a.q_head + lane + 32 * i;
        q[i] = WD == UQ_W_F32 ? static_cast<const float*>(a.q)[e]
                              : __uint_as_float((uint32_t)static_cast<const uint16_t*>(a.q)[e] << 16);
        o[i] = 0.0f;
    }
    for (int64_t t = first + warp; t < n; t += kWarps) {
        const int64_t page = a.table[b * a.table_stride + (t >> a.page_shift)];
        if (page < 0 || page >= a.c.pages) continue;
        const int64_t row = ((page * a.c.kv_heads + kvh) << a.page_shift) + (t & ((1 << a.page_shift) - 1));
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < NV; ++i) s = fmaf(q[i], kv_value<FMT, HD>(a.c.k, a.c.k_scale, row, lane + 32 * i), s);
        s = warp_sum(s) * a.scale;
        const float m2 = fmaxf(m, s), mm = m2 == -INFINITY ? 0.0f : m2;
        const float f = expf(m - mm), p = expf(s - mm);
        l = fmaf(l, f, p);
#pragma unroll
        for (int i = 0; i < NV; ++i) o[i] = fmaf(p, kv_value<FMT, HD>(a.c.v, a.c.v_scale, row, lane + 32 * i), o[i] * f);
        m = m2;
    }
    if (lane == 0) {
        sm_m[warp] = m;
        sm_l[warp] = l;
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) sm_o[warp][lane + 32 * i] = o[i];
    __syncthreads();
    float top = -INFINITY, sum = 0.0f;
    for (int w = 0; w < kWarps; ++w) top = fmaxf(top, sm_m[w]);
    const float base = top == -INFINITY ? 0.0f : top;
    for (int w = 0; w < kWarps; ++w) sum = fmaf(sm_l[w], expf(sm_m[w] - base), sum);
    for (int d = threadIdx.x; d < HD; d += kThreads) {
        float acc = 0.0f;
        for (int w = 0; w < kWarps; ++w) acc = fmaf(sm_o[w][d], expf(sm_m[w] - base), acc);
        acc = sum == 0.0f ? 0.0f : acc / sum;
        const int64_t e = b * a.out_batch + h * a.out_head + d;
        if (WD == UQ_W_F32) static_cast<float*>(a.out)[e] = acc;
        else static_cast<uint16_t*>(a.out)[e] = (uint16_t)bf16_pair(acc, 0.0f);
    }
    if (threadIdx.x == 0 && a.lse != nullptr) a.lse[(int64_t)b * a.heads + h] = logf(sum) + base;
}

template <int FMT, int HD>
cudaError_t go(const AttnArgs& a, cudaStream_t st) {
    const dim3 grid(a.heads, (unsigned)a.batch);
    return launch_dependent(a.dtype == UQ_W_F32 ? attn_kernel<FMT, HD, UQ_W_F32> : attn_kernel<FMT, HD, UQ_W_BF16>, grid,
                            dim3(kThreads), 0, st, a);
}

template <int FMT>
cudaError_t by_head(const AttnArgs& a, cudaStream_t st) {
    return a.c.head_dim == 64 ? go<FMT, 64>(a, st) : a.c.head_dim == 128 ? go<FMT, 128>(a, st) : go<FMT, 256>(a, st);
}

}  // namespace

int64_t attn_workspace_bytes(int heads, int kv_heads, int head_dim) { return 16; }

cudaError_t launch_attn(const AttnArgs& a, cudaStream_t st) {
    return a.c.format == UQ_KV_BF16   ? by_head<UQ_KV_BF16>(a, st)
           : a.c.format == UQ_KV_INT8 ? by_head<UQ_KV_INT8>(a, st)
                                      : by_head<UQ_KV_INT4>(a, st);
}

}  // namespace uq
