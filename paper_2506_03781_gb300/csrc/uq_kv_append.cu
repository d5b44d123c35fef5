// New tokens' keys and values into the paged cache, keys (and queries) rotated
// by their positions on the way (see uq_api.h).
//
// Rotation.  Channels (j, j + rot / 2) of a query or key are turned by (c, s) =
// rope[position, j]: (a c - b s, a s + b c), every product, sum and difference
// rounded to fp32, and keys are quantised from that (uq_kv_rows.cuh).
//
// One pass over the data: queries are read and written once, keys and values read
// once and written as the cache keeps them.  Queries: a thread has 8 channels and
// the 8 that they are turned with, of kHeads heads of one token, so that its part
// of the table is read once for all of them and q_out may be q itself.  Keys and
// values: a thread has 16 channels of a row of each, as in uq_kv.cu; what its
// channels are turned with it loads too (from L1 for the most part), because a
// row's codes are made from 16 channels a lane.  20011 tokens of 32 and 8 heads of 128
// into 4 bits, a thirteenth of them padding, and back again (uq_kv_read): 104 us, 4.9
// TB/s of the bytes that have to move, 72 % of the copy rate; 2048 tokens into 8 bits
// 14.6 us on the device, one token 4.4, both launches and the reading counted in.
#include "uq_kv_rows.cuh"
#include "uq_attn.h"
#include "uq_launch.h"

namespace uq {
namespace {

constexpr int kHeads = 4;                          // heads of a thread's queries

// (c, s) of 8 channels; NaN where the table has no such position.
struct Turn {
    float c[8], s[8];
    __device__ __forceinline__ void load(const float* __restrict__ rope, bool there) {
        const float nan = kKvNan;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float4 w = there ? __ldg(reinterpret_cast<const float4*>(rope) + i) : make_float4(nan, nan, nan, nan);
            c[2 * i] = w.x;
            s[2 * i] = w.y;
            c[2 * i + 1] = w.z;
            s[2 * i + 1] = w.w;
        }
    }
    __device__ __forceinline__ float low(float a, float b, int i) const { return __fsub_rn(__fmul_rn(a, c[i]), __fmul_rn(b, s[i])); }
    __device__ __forceinline__ float high(float a, float b, int i) const { return __fadd_rn(__fmul_rn(a, s[i]), __fmul_rn(b, c[i])); }
};

template <int WD>
__device__ __forceinline__ void put8(void* p, int64_t e, const float x[8]) {
    if constexpr (WD == UQ_W_F32) {
        float4* d = reinterpret_cast<float4*>(static_cast<float*>(p) + e);
        d[0] = make_float4(x[0], x[1], x[2], x[3]);
        d[1] = make_float4(x[4], x[5], x[6], x[7]);
    } else {
        *reinterpret_cast<uint4*>(static_cast<uint16_t*>(p) + e) = pack8(x);
    }
}

template <int FMT, int HD, int WD>
__global__ void __launch_bounds__(kThreads) kv_append_kernel(const AppendArgs a, const uint32_t kv_blocks, const uint32_t n_rows,
                                                             const uint32_t q_items, const uint32_t q_groups) {
    constexpr int LPR = HD / kWriteCh, RPB = kThreads / LPR;
    const int lane = threadIdx.x % LPR, half = a.rot / 2;
    inputs_ready();
    if (blockIdx.x < kv_blocks) {
        // --- a row of keys and one of values
        const uint32_t r = blockIdx.x * RPB + threadIdx.x / LPR, i = r / a.c.kv_heads, h = r - i * a.c.kv_heads;
        const int64_t slot = r < n_rows ? __ldg(a.slots + i) : -1;
        const bool there = slot >= 0 && slot < (a.c.pages << a.page_shift);
        const int64_t row = there ? (((slot >> a.page_shift) * a.c.kv_heads + h) << a.page_shift) + (slot & ((1 << a.page_shift) - 1)) : 0;
        float x[kWriteCh], y[kWriteCh];
#pragma unroll
        for (int j = 0; j < kWriteCh; ++j) x[j] = y[j] = 0.0f;
        if (there) {
            const int64_t p = __ldg(a.positions + i);
            const int64_t ke = (int64_t)i * a.k_token + (int64_t)h * a.k_head, ve = (int64_t)i * a.v_token + (int64_t)h * a.v_head;
            Raw own[2], other[2], val[2];
            Turn turn[2];
#pragma unroll
            for (int g = 0; g < 2; ++g) {
                const int ch = lane * kWriteCh + 8 * g;
                own[g] = load8<WD>(a.k, ke + ch);
                val[g] = load8<WD>(a.v, ve + ch);
                other[g] = own[g];
                if (ch < a.rot) {
                    other[g] = load8<WD>(a.k, ke + (ch < half ? ch + half : ch - half));
                    turn[g].load(a.rope + (p * half + (ch < half ? ch : ch - half)) * 2, p >= 0 && p < a.rope_rows);
                }
            }
#pragma unroll
            for (int g = 0; g < 2; ++g) {
                const int ch = lane * kWriteCh + 8 * g;
                unpack8<WD>(own[g], x + 8 * g);
                unpack8<WD>(val[g], y + 8 * g);
                if (ch < a.rot) {
                    float z[8];
                    unpack8<WD>(other[g], z);
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        float& own_x = x[8 * g + j];
                        own_x = ch < half ? turn[g].low(own_x, z[j], j) : turn[g].high(z[j], own_x, j);
                    }
                }
            }
        }
        put_row<FMT, HD>(x, a.c.k, a.c.k_scale, row, lane, there);
        put_row<FMT, HD>(y, a.c.v, a.c.v_scale, row, lane, there);
        return;
    }
    // --- queries: 8 channels and the 8 they are turned with, or 16 that are not
    const uint32_t item = (blockIdx.x - kv_blocks) * RPB + threadIdx.x / LPR;
    if (item >= q_items) return;
    const uint32_t i = item / q_groups, h0 = (item - i * q_groups) * kHeads;
    const bool turned = lane < half / 8;
    const int c0 = turned ? 8 * lane : 16 * lane, c1 = c0 + (turned ? half : 8);
    Raw raw[kHeads][2];
#pragma unroll
    for (int u = 0; u < kHeads; ++u)
        if ((int)h0 + u < a.heads) {
            const int64_t e = (int64_t)i * a.q_token + (int64_t)(h0 + u) * a.q_head;
            raw[u][0] = load8_any<WD>(a.q, e + c0);
            raw[u][1] = load8_any<WD>(a.q, e + c1);
        }
    Turn turn;
    if (turned) {
        const int64_t p = __ldg(a.positions + i);
        turn.load(a.rope + (p * half + c0) * 2, p >= 0 && p < a.rope_rows);
    }
#pragma unroll
    for (int u = 0; u < kHeads; ++u)
        if ((int)h0 + u < a.heads) {
            const int64_t e = (int64_t)i * a.out_token + (int64_t)(h0 + u) * a.out_head;
            float x[8], y[8];
            unpack8<WD>(raw[u][0], x);
            unpack8<WD>(raw[u][1], y);
            if (turned) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float lo = turn.low(x[j], y[j], j);
                    y[j] = turn.high(x[j], y[j], j);
                    x[j] = lo;
                }
            }
            put8<WD>(a.q_out, e + c0, x);
            put8<WD>(a.q_out, e + c1, y);
        }
}

template <int FMT, int HD, int WD>
cudaError_t go(const AppendArgs& a, cudaStream_t st) {
    constexpr uint32_t rpb = kThreads / (HD / kWriteCh);
    const uint32_t n_rows = (uint32_t)(a.tokens * a.c.kv_heads), groups = (uint32_t)((a.heads + kHeads - 1) / kHeads);
    const uint32_t items = a.q == nullptr ? 0 : (uint32_t)a.tokens * groups;
    const uint32_t kv_blocks = (n_rows + rpb - 1) / rpb, blocks = kv_blocks + (items + rpb - 1) / rpb;
    return launch_dependent(kv_append_kernel<FMT, HD, WD>, dim3(blocks), dim3(kThreads), 0, st, a, kv_blocks, n_rows, items,
                            groups);
}

template <int FMT>
cudaError_t by_head(const AppendArgs& a, cudaStream_t st) {
    const bool f32 = a.dtype == UQ_W_F32;
    switch (a.c.head_dim) {
        case 64: return f32 ? go<FMT, 64, UQ_W_F32>(a, st) : go<FMT, 64, UQ_W_BF16>(a, st);
        case 128: return f32 ? go<FMT, 128, UQ_W_F32>(a, st) : go<FMT, 128, UQ_W_BF16>(a, st);
        default: return f32 ? go<FMT, 256, UQ_W_F32>(a, st) : go<FMT, 256, UQ_W_BF16>(a, st);
    }
}

}  // namespace

cudaError_t launch_kv_append(const AppendArgs& a, cudaStream_t st) {
    switch (a.c.format) {
        case UQ_KV_BF16: return by_head<UQ_KV_BF16>(a, st);
        case UQ_KV_INT8: return by_head<UQ_KV_INT8>(a, st);
        default: return by_head<UQ_KV_INT4>(a, st);
    }
}

}  // namespace uq
