// Attention of one new token and head over the paged key-value cache, by a warp:
// what the tensor cores' kernel (uq_rows.cuh) is not for.
//
// 32 positions at a time a lane has one of them: its score q . k_t, by which the
// warp moves on its running maximum and sum; then the lanes share out the channels
// and add up p_t v_t.  Everything is fp32, and nothing of a position that the token
// does not see is touched.
#pragma once

#include "uq_attn.h"
#include "uq_kv.cuh"

namespace uq {
namespace plain {

// Channels 8 g .. 8 g + 7 of a row.
template <int FMT, int HD>
__device__ __forceinline__ void row8(const void* rows, const void* scales, int64_t row, int g, float x[8]) {
    using R = KvRow<FMT, HD>;
    const uint8_t* const src = static_cast<const uint8_t*>(rows) + row * R::kBytes;
    if constexpr (FMT == UQ_KV_BF16) {
        const uint4 w = __ldg(reinterpret_cast<const uint4*>(src) + g);
        const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = bf16_low(u[i]);
            x[2 * i + 1] = bf16_high(u[i]);
        }
    } else if constexpr (FMT == UQ_KV_INT8) {
        const uint2 w = __ldg(reinterpret_cast<const uint2*>(src) + g);
        const float s = __ldg(static_cast<const float*>(scales) + row);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = __fmul_rn((float)(int8_t)((i < 4 ? w.x : w.y) >> (8 * (i & 3))), s);
    } else {
        const uint32_t w = __ldg(reinterpret_cast<const uint32_t*>(src) + g);
        const uint32_t p = __ldg(static_cast<const uint32_t*>(scales) + row * R::kWords + g / 8);
        const float s = bf16_low(p), m = bf16_high(p);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = __fmaf_rn((float)((w >> (4 * i)) & 15), s, m);
    }
}

// Token i of the c new ones of sequence b; q_row and out_row: rows of q and out, in elements but for the head; qs: HD floats.
// d0 >= 0: channels d0 .. d0 + 31 only, and no lse.
template <int FMT, int HD, int WD>
__device__ __forceinline__ void attend(const RowsArgs& a, int b, int i, int c, int head, int64_t q_row, int64_t out_row, int64_t lse_row, float* qs, int d0 = -1) {
    constexpr int CH = HD / 32;                        // channels of a lane
    const int lane = threadIdx.x & 31;
    const int n = min(max(__ldg(a.seq_lens + b), 0), a.max_tokens), ctx = n - c;
    const uint64_t drafts = c >= 64 ? ~0ull : (1ull << c) - 1;
    const uint64_t mine = a.tree != nullptr ? __ldg(reinterpret_cast<const unsigned long long*>(a.tree) + b * a.tree_stride + i) & drafts : 0;
    const int p = a.tree != nullptr ? ctx + __popcll(mine) - 1 : ctx + i;
    const int low = a.window > 0 ? p - a.window + 1 : 0;                  // first position of the window
    const int end = a.tree != nullptr ? n : p + 1;
    auto sees = [&](int t) {
        if (t < 0 || t >= end) return false;
        int at = t;
        if (a.tree != nullptr && t >= ctx) {
            if (!((mine >> (t - ctx)) & 1)) return false;
            const uint64_t m = __ldg(reinterpret_cast<const unsigned long long*>(a.tree) + b * a.tree_stride + (t - ctx)) & drafts;
            at = ctx + __popcll(m) - 1;
        }
        return a.window == 0 || at >= low || at < a.sinks;
    };
    // --- the query
    const int kvh = head / (a.heads / a.c.kv_heads);
    q_row += (int64_t)head * a.q_head;
    for (int d = lane; d < HD; d += 32)
        qs[d] = WD == UQ_W_F32 ? __ldg(static_cast<const float*>(a.q) + q_row + d)
                                     : __uint_as_float((uint32_t)__ldg(static_cast<const uint16_t*>(a.q) + q_row + d) << 16);
    __syncwarp();
    float top = -INFINITY, sum = 0.0f, o[CH];
#pragma unroll
    for (int k = 0; k < CH; ++k) o[k] = 0.0f;
    const float to_log2 = a.scale * 1.4426950408889634f;
    const int pmask = (1 << a.page_shift) - 1;
    // blocks of 32 positions: those of the sinks, then from the window's on (a draft's position may lie before its place)
    const int from = a.window > 0 ? max(min(low, ctx), 0) & ~31 : 0, lead = a.window > 0 ? min(a.sinks, from) : 0;
    for (int t0 = lead > 0 ? 0 : from; t0 < end; t0 = t0 + 32 >= lead && t0 < from ? from : t0 + 32) {
        const int t = t0 + lane;
        bool there = sees(t);
        int64_t row = 0;
        if (there) {
            const int page = __ldg(a.table + (int64_t)b * a.table_stride + (t >> a.page_shift));
            there = (uint32_t)page < (uint64_t)a.c.pages;
            row = there ? (((int64_t)page * a.c.kv_heads + kvh) << a.page_shift) + (t & pmask) : 0;
        }
        if (!__any_sync(kFull, there)) continue;
        float x = -INFINITY;
        if (there) {
            float s = 0.0f;
#pragma unroll 4
            for (int g = 0; g < HD / 8; ++g) {
                float k[8];
                row8<FMT, HD>(a.c.k, a.c.k_scale, row, g, k);
#pragma unroll
                for (int j = 0; j < 8; ++j) s = fmaf(qs[8 * g + j], k[j], s);
            }
            x = s * to_log2;
        }
        float m = x;
#pragma unroll
        for (int off = 16; off >= 1; off >>= 1) m = fmaxf(m, __shfl_xor_sync(kFull, m, off));
        m = fmaxf(m, top);
        const float base = m == -INFINITY ? 0.0f : m, f = exp2f(top - base);
        top = m;
        const float w = there ? exp2f(x - base) : 0.0f;
        sum = sum * f + warp_sum(w);
#pragma unroll
        for (int k = 0; k < CH; ++k) o[k] *= f;
        uint32_t left = __ballot_sync(kFull, there);
        while (left) {
            const int from_lane = __ffs(left) - 1;
            left &= left - 1;
            const float pt = __shfl_sync(kFull, w, from_lane);
            const int64_t r = __shfl_sync(kFull, row, from_lane);
            float v[8];
            row8<FMT, HD>(a.c.v, a.c.v_scale, r, lane * CH / 8, v);
#pragma unroll
            for (int k = 0; k < CH; ++k) {
                float mine_v = 0.0f;
#pragma unroll
                for (int e = 0; e < 8 / CH; ++e)
                    if (lane % (8 / CH) == e) mine_v = v[e * CH + k];
                o[k] = fmaf(pt, mine_v, o[k]);
            }
        }
    }
    const float inv = sum == 0.0f ? 0.0f : __fdiv_rn(1.0f, sum);
    if (d0 >= 0 && (lane * CH < d0 || lane * CH >= d0 + 32)) return;
    out_row += (int64_t)head * a.out_head + lane * CH;
#pragma unroll
    for (int k = 0; k < CH; ++k)
        if constexpr (WD == UQ_W_F32) static_cast<float*>(a.out)[out_row + k] = o[k] * inv;
        else static_cast<uint16_t*>(a.out)[out_row + k] = (uint16_t)bf16_pair(o[k] * inv, 0.0f);
    if (a.lse != nullptr && lane == 0 && d0 < 0)
        a.lse[lse_row * a.heads + head] = sum == 0.0f ? -INFINITY : ((top == -INFINITY ? 0.0f : top) + log2f(sum)) * 0.6931471805599453f;
}

}  // namespace plain
}  // namespace uq
