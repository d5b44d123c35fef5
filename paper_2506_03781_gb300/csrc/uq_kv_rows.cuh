// Rows of the key-value cache as threads hold them: loads and stores of the
// caller's rows and the arithmetic that quantises them (see uq_api.h), shared by
// the kernels that write the cache.
#pragma once

#include "uq_kv.cuh"

namespace uq {
namespace {

constexpr int kWriteCh = 16;                    // channels of a lane that quantises

struct Rows {                          // the caller's rows (i, h); strides in elements
    void* base;
    int64_t token_stride, head_stride;
};

struct Raw {                           // 8 channels as they are stored
    uint4 a, b;                        // bf16: a only
};

// rint(v) of |v| < 2^21 in the low bits (two's complement), above them the pattern of 1.5 * 2^23.
__device__ __forceinline__ uint32_t rounded(float v) { return __float_as_uint(__fadd_rn(v, 12582912.0f)); }

template <int WD>
__device__ __forceinline__ Raw load8(const void* p, int64_t e) {
    Raw r;
    if constexpr (WD == UQ_W_F32) {
        const uint4* s = reinterpret_cast<const uint4*>(static_cast<const float*>(p) + e);
        r.a = __ldg(s);
        r.b = __ldg(s + 1);
    } else {
        r.a = __ldg(reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p) + e));
    }
    return r;
}

// The same of rows that this kernel may write too (q_out may be q): not through the read-only path.
template <int WD>
__device__ __forceinline__ Raw load8_any(const void* p, int64_t e) {
    Raw r;
    if constexpr (WD == UQ_W_F32) {
        const uint4* s = reinterpret_cast<const uint4*>(static_cast<const float*>(p) + e);
        r.a = s[0];
        r.b = s[1];
    } else {
        r.a = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(p) + e);
    }
    return r;
}

template <int WD>
__device__ __forceinline__ void unpack8(const Raw& r, float x[8]) {
    const uint32_t w[8] = {r.a.x, r.a.y, r.a.z, r.a.w, r.b.x, r.b.y, r.b.z, r.b.w};
#pragma unroll
    for (int i = 0; i < 8; ++i)
        x[i] = WD == UQ_W_F32 ? __uint_as_float(w[i]) : (i & 1) ? bf16_high(w[i >> 1]) : bf16_low(w[i >> 1]);
}

__device__ __forceinline__ uint4 pack8(const float x[8]) {
    return make_uint4(bf16_pair(x[0], x[1]), bf16_pair(x[2], x[3]), bf16_pair(x[4], x[5]), bf16_pair(x[6], x[7]));
}

// Stores channels 8 lane .. 8 lane + 7 of a row at element e.  fp32: neighbours halve their parts, so that lanes store 16
// bytes next to each other (a lane its 32 bytes: half a sector at a time); all lanes of the warp take part.
template <int WD>
__device__ __forceinline__ void store8(void* p, int64_t e, int lane, const float x[8], bool in) {
    if constexpr (WD == UQ_W_F32) {
        const bool odd = lane & 1;
        float y[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] = __shfl_xor_sync(kFull, odd ? x[i] : x[4 + i], 1);
        if (!in) return;
        float4* d = reinterpret_cast<float4*>(static_cast<float*>(p) + e + 8 * (lane & ~1)) + (lane & 1);
        d[0] = odd ? make_float4(y[0], y[1], y[2], y[3]) : make_float4(x[0], x[1], x[2], x[3]);
        d[2] = odd ? make_float4(x[4], x[5], x[6], x[7]) : make_float4(y[0], y[1], y[2], y[3]);
    } else if (in) {
        *reinterpret_cast<uint4*>(static_cast<uint16_t*>(p) + e + 8 * lane) = pack8(x);
    }
}

// Quantises a row of which this lane holds channels 16 chunk .. 16 chunk + 15; all
// lanes of the warp take part in the shuffles, those of a row with `keep`
// store it as row `row` of the pool.
template <int FMT, int HD>
__device__ __forceinline__ void put_row(const float x[kWriteCh], void* rows, void* scales, int64_t row, int chunk, bool keep) {
    constexpr int LPR = HD / kWriteCh;
    using R = KvRow<FMT, HD>;
    uint8_t* dst = static_cast<uint8_t*>(rows) + row * R::kBytes;
    if constexpr (FMT == UQ_KV_BF16) {
        if (keep) {
            reinterpret_cast<uint4*>(dst)[2 * chunk] = pack8(x);
            reinterpret_cast<uint4*>(dst)[2 * chunk + 1] = pack8(x + 8);
        }
    } else if constexpr (FMT == UQ_KV_INT8) {
        float a = fabsf(x[0]);
#pragma unroll
        for (int i = 1; i < kWriteCh; ++i) a = max_nan(a, fabsf(x[i]));
#pragma unroll
        for (int off = LPR / 2; off >= 1; off >>= 1) a = max_nan(a, __shfl_xor_sync(kFull, a, off));
        const bool fine = finite(a), some = fine && a >= kKvTiny;
        const float inv = some ? __fdiv_rn(127.0f, a) : 0.0f;
        uint32_t w[4];
#pragma unroll
        for (int h = 0; h < 4; ++h) {
            uint32_t c[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) c[i] = rounded(__fmul_rn(x[4 * h + i], inv));
            w[h] = some ? __byte_perm(__byte_perm(c[0], c[1], 0x0040), __byte_perm(c[2], c[3], 0x0040), 0x5410) : 0;
        }
        if (keep) {
            reinterpret_cast<uint4*>(dst)[chunk] = make_uint4(w[0], w[1], w[2], w[3]);
            if (chunk == 0) static_cast<float*>(scales)[row] = some ? __fdiv_rn(a, 127.0f) : fine ? 0.0f : kKvNan;
        }
    } else {
        float lo = x[0], hi = x[0];
#pragma unroll
        for (int i = 1; i < kWriteCh; ++i) {
            lo = min_nan(lo, x[i]);
            hi = max_nan(hi, x[i]);
        }
#pragma unroll
        for (int off = kKvGroup / kWriteCh / 2; off >= 1; off >>= 1) {
            lo = min_nan(lo, __shfl_xor_sync(kFull, lo, off));
            hi = max_nan(hi, __shfl_xor_sync(kFull, hi, off));
        }
        // the pair as it is kept decides the codes, so that they fit the values read back
        const uint32_t pair = bf16_pair(__fdiv_rn(__fsub_rn(hi, lo), 15.0f), lo);
        const float s = bf16_low(pair), m = bf16_high(pair);
        const bool fine = finite(s) && finite(m), some = fine && s >= kKvTiny;
        const float inv = some ? __fdiv_rn(1.0f, s) : 0.0f;
        uint32_t w[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            // sum of 16^i (pattern of 1.5 * 2^23 + code), less what the patterns add up to
            w[h] = 0u - 0x4b400000u * 0x11111111u;
#pragma unroll
            for (int i = 0; i < 8; ++i)
                w[h] += rounded(fminf(fmaxf(__fmul_rn(__fsub_rn(x[8 * h + i], m), inv), 0.0f), 15.0f)) << (4 * i);
            if (!some) w[h] = 0;
        }
        if (keep) {
            reinterpret_cast<uint2*>(dst)[chunk] = make_uint2(w[0], w[1]);
            if (chunk % (kKvGroup / kWriteCh) == 0)
                static_cast<uint32_t*>(scales)[row * R::kWords + chunk / (kKvGroup / kWriteCh)] =
                    some ? pair : fine ? pair & 0xffff0000u : kKvNanPair;
        }
    }
}

}  // namespace
}  // namespace uq
