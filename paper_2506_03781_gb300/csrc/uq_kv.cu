// Writing rows into the paged key-value cache and reading them back.
//
// Both are one pass over the data, bound by memory as long as few instructions go
// to a value: a bf16 row of 128 channels into 8 bits moves 256 + 132 bytes, an fp32
// one into 4 bits 512 + 72.  Writing, a lane has 16 channels, so that the quotients
// of a row, its shuffles and its place are few for a value (8 to a lane: 60000 tokens
// from bf16 into 4 bits 89 us); reading, 8, so that lanes store next to each other.
// A thread has K and V of one row, reading of two (one: 62 us for 60000 tokens back
// from 4 bits, two 51); all are loaded before the first is worked on, with one
// division for their places.  Codes are made by adding 1.5 * 2^23, whose sum is
// rounded to an integer in its low bits (to even, as rint), and become
// floating-point numbers as 16-bit patterns: conversions run at a quarter of the
// rate.
#include "uq_kv.cuh"
#include "uq_launch.h"

namespace uq {
namespace {

constexpr int kReadCh = 8, kWriteCh = 16;       // channels per lane
constexpr int kReadRows = 2, kWriteRows = 1;    // rows per thread, K's and V's each

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

// Quantises a row of which this lane holds channels 16 lane .. 16 lane + 15; all
// lanes of the warp take part in the shuffles, those of a row with `keep`
// store it as row `row` of the pool.
template <int FMT, int HD>
__device__ __forceinline__ void put_row(const float x[kWriteCh], void* rows, void* scales, int64_t row, int lane, bool keep) {
    constexpr int LPR = HD / kWriteCh;
    using R = KvRow<FMT, HD>;
    uint8_t* dst = static_cast<uint8_t*>(rows) + row * R::kBytes;
    if constexpr (FMT == UQ_KV_BF16) {
        if (keep) {
            reinterpret_cast<uint4*>(dst)[2 * lane] = pack8(x);
            reinterpret_cast<uint4*>(dst)[2 * lane + 1] = pack8(x + 8);
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
            reinterpret_cast<uint4*>(dst)[lane] = make_uint4(w[0], w[1], w[2], w[3]);
            if (lane == 0) static_cast<float*>(scales)[row] = some ? __fdiv_rn(a, 127.0f) : fine ? 0.0f : kKvNan;
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
            reinterpret_cast<uint2*>(dst)[lane] = make_uint2(w[0], w[1]);
            if (lane % (kKvGroup / kWriteCh) == 0)
                static_cast<uint32_t*>(scales)[row * R::kWords + lane / (kKvGroup / kWriteCh)] =
                    some ? pair : fine ? pair & 0xffff0000u : kKvNanPair;
        }
    }
}

// The stored bytes of this lane's 8 channels, and their scale word.
template <int FMT, int HD>
struct Kept {
    uint4 code;
    uint32_t word;
    __device__ __forceinline__ void load(const void* rows, const void* scales, int64_t row, int lane) {
        using R = KvRow<FMT, HD>;
        const uint8_t* src = static_cast<const uint8_t*>(rows) + row * R::kBytes;
        if constexpr (FMT == UQ_KV_BF16) {
            code = __ldg(reinterpret_cast<const uint4*>(src) + lane);
        } else if constexpr (FMT == UQ_KV_INT8) {
            const uint2 c = __ldg(reinterpret_cast<const uint2*>(src) + lane);
            code = make_uint4(c.x, c.y, 0, 0);
            word = __ldg(static_cast<const uint32_t*>(scales) + row);
        } else {
            code.x = __ldg(reinterpret_cast<const uint32_t*>(src) + lane);
            word = __ldg(static_cast<const uint32_t*>(scales) + row * R::kWords + lane / 8);
        }
    }
    __device__ __forceinline__ void values(float x[8]) const {
        if constexpr (FMT == UQ_KV_BF16) {
            Raw r;
            r.a = code;
            unpack8<UQ_W_BF16>(r, x);
        } else if constexpr (FMT == UQ_KV_INT8) {
            const float s = __uint_as_float(word);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t p = bf16_of_int8(__byte_perm(i < 2 ? code.x : code.y, 0, i & 1 ? 0x4342 : 0x4140), kKvBf16_128);
                x[2 * i] = __fmul_rn(bf16_low(p), s);
                x[2 * i + 1] = __fmul_rn(bf16_high(p), s);
            }
        } else {
            // a code has 4 bits and the scale 8: their product is exact, so there is one rounding in all
            const float s = bf16_low(word), m = bf16_high(word);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t p = bf16_of_int4(code.x >> (4 * i), kKvBf16_128, 0x43004300u);
                x[i] = __fmaf_rn(bf16_low(p), s, m);
                x[i + 4] = __fmaf_rn(bf16_high(p), s, m);
            }
        }
    }
};

// Row r = i * kv + h of the caller's: its place in the pool, counted in rows, and whether it has one.
struct Place {
    uint32_t i, h;
    int64_t row;
    bool in, there;                    // one of the caller's rows; its slot is in the pool
    __device__ __forceinline__ void find(const uq_kv_cache& c, int page_shift, const int64_t* __restrict__ slots) {
        const int64_t slot = in ? __ldg(slots + i) : -1;
        there = slot >= 0 && slot < (c.pages << page_shift);
        row = there ? (((slot >> page_shift) * c.kv_heads + h) << page_shift) + (slot & ((1 << page_shift) - 1)) : 0;
    }
};

// The rows r0, r0 + step, ... of a thread, from one division.
template <int ROWS>
__device__ __forceinline__ void places_of(Place (&p)[ROWS], uint32_t r0, uint32_t step, uint32_t n_rows,
                                          const uq_kv_cache& c, int page_shift, const int64_t* __restrict__ slots) {
    const uint32_t kv = c.kv_heads, di = step / kv, dh = step - di * kv;
    p[0].i = r0 / kv;
    p[0].h = r0 - p[0].i * kv;
#pragma unroll
    for (int u = 0; u < ROWS; ++u) {
        if (u > 0) {
            p[u].i = p[u - 1].i + di;
            p[u].h = p[u - 1].h + dh;
            if (p[u].h >= kv) {
                p[u].h -= kv;
                ++p[u].i;
            }
        }
        p[u].in = r0 + u * step < n_rows;
        p[u].find(c, page_shift, slots);
    }
}

__device__ __forceinline__ int64_t element_of(const Rows& x, const Place& p, int channel) {
    return p.i * x.token_stride + p.h * x.head_stride + channel;
}

template <int FMT, int HD, int WD>
__global__ void __launch_bounds__(kThreads) kv_write_kernel(uq_kv_cache c, int page_shift, Rows k, Rows v,
                                                            uint32_t n_rows, const int64_t* __restrict__ slots) {
    constexpr int LPR = HD / kWriteCh, RPB = kThreads / LPR;
    const int lane = threadIdx.x % LPR;
    inputs_ready();
    Place p[kWriteRows];
    places_of(p, blockIdx.x * (RPB * kWriteRows) + threadIdx.x / LPR, RPB, n_rows, c, page_shift, slots);
    Raw raw[2][kWriteRows][2];
#pragma unroll
    for (int u = 0; u < kWriteRows; ++u)
#pragma unroll
        for (int h = 0; h < 2; ++h)
            if (p[u].there) {
                raw[0][u][h] = load8<WD>(k.base, element_of(k, p[u], lane * kWriteCh + 8 * h));
                raw[1][u][h] = load8<WD>(v.base, element_of(v, p[u], lane * kWriteCh + 8 * h));
            } else {
                raw[0][u][h].a = raw[0][u][h].b = raw[1][u][h].a = raw[1][u][h].b = make_uint4(0, 0, 0, 0);
            }
#pragma unroll
    for (int u = 0; u < kWriteRows; ++u)
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            float x[kWriteCh];
            unpack8<WD>(raw[t][u][0], x);
            unpack8<WD>(raw[t][u][1], x + 8);
            put_row<FMT, HD>(x, t ? c.v : c.k, t ? c.v_scale : c.k_scale, p[u].row, lane, p[u].there);
        }
}

template <int FMT, int HD, int WD>
__global__ void __launch_bounds__(kThreads) kv_read_kernel(uq_kv_cache c, int page_shift, Rows k, Rows v,
                                                           uint32_t n_rows, const int64_t* __restrict__ slots) {
    constexpr int LPR = HD / kReadCh, RPB = kThreads / LPR;
    const int lane = threadIdx.x % LPR;
    inputs_ready();
    Place p[kReadRows];
    places_of(p, blockIdx.x * (RPB * kReadRows) + threadIdx.x / LPR, RPB, n_rows, c, page_shift, slots);
    Kept<FMT, HD> kept[2][kReadRows];
#pragma unroll
    for (int u = 0; u < kReadRows; ++u) {
        kept[0][u].load(c.k, c.k_scale, p[u].row, lane);
        kept[1][u].load(c.v, c.v_scale, p[u].row, lane);
    }
#pragma unroll
    for (int u = 0; u < kReadRows; ++u) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            float x[8];
            kept[t][u].values(x);
            if (!p[u].there) {
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = 0.0f;
            }
            store8<WD>(t ? v.base : k.base, element_of(t ? v : k, p[u], 0), lane, x, p[u].in);
        }
    }
}

template <int FMT, int HD, int WD>
cudaError_t go(bool write, const uq_kv_cache& c, Rows k, Rows v, uint32_t n_rows, const int64_t* slots, cudaStream_t st) {
    const uint32_t rpb = write ? kThreads / (HD / kWriteCh) * kWriteRows : kThreads / (HD / kReadCh) * kReadRows;
    const dim3 grid((n_rows + rpb - 1) / rpb);
    return launch_dependent(write ? kv_write_kernel<FMT, HD, WD> : kv_read_kernel<FMT, HD, WD>, grid, dim3(kThreads), 0,
                            st, c, __builtin_ctz((unsigned)c.page_size), k, v, n_rows, slots);
}

template <int FMT, int HD>
cudaError_t by_type(bool write, const uq_kv_cache& c, Rows k, Rows v, int dtype, uint32_t n_rows, const int64_t* slots,
                    cudaStream_t st) {
    return dtype == UQ_W_F32 ? go<FMT, HD, UQ_W_F32>(write, c, k, v, n_rows, slots, st)
                             : go<FMT, HD, UQ_W_BF16>(write, c, k, v, n_rows, slots, st);
}

template <int FMT>
cudaError_t by_head(bool write, const uq_kv_cache& c, Rows k, Rows v, int dtype, uint32_t n_rows, const int64_t* slots,
                    cudaStream_t st) {
    switch (c.head_dim) {
        case 64: return by_type<FMT, 64>(write, c, k, v, dtype, n_rows, slots, st);
        case 128: return by_type<FMT, 128>(write, c, k, v, dtype, n_rows, slots, st);
        default: return by_type<FMT, 256>(write, c, k, v, dtype, n_rows, slots, st);
    }
}

}  // namespace

cudaError_t launch_kv_copy(bool write, const uq_kv_cache& c, const int64_t* slots, int64_t tokens, void* k, void* v,
                           int dtype, const int64_t strides[4], cudaStream_t st) {
    const Rows kr{k, strides[0], strides[1]}, vr{v, strides[2], strides[3]};
    const uint32_t n = (uint32_t)(tokens * c.kv_heads);
    switch (c.format) {
        case UQ_KV_BF16: return by_head<UQ_KV_BF16>(write, c, kr, vr, dtype, n, slots, st);
        case UQ_KV_INT8: return by_head<UQ_KV_INT8>(write, c, kr, vr, dtype, n, slots, st);
        default: return by_head<UQ_KV_INT4>(write, c, kr, vr, dtype, n, slots, st);
    }
}

}  // namespace uq
