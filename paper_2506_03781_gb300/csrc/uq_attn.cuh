// Attention of one new token of each sequence over the paged key-value cache
// (see uq_api.h).
//
// Per key/value head the r query heads that share it are the columns of two
// small products, with t the cached positions:
//     X^T [t, r] = K [t, hd] Q^T      O^T [hd, r] = V^T [hd, t] P^T,  P = exp2(X - m)
// bound by reading K and V once.  A warp does both on the tensor cores for a
// tile of kTok positions (m16n8k16: positions, then channels, are the 16 rows; 8
// query heads the columns), keeps a running maximum m, sum and O^T in registers
// and never exchanges anything with other warps until its sequence is done.
//
// Shares.  The tiles of all sequences and heads, in order, are cut into one
// contiguous share of equal size per block, whatever the lengths, so a block ends
// up with the end of one (sequence, head), some whole ones and the start of
// another.  A (sequence, head) that lies in several blocks is joined by the one
// that finishes last: partial m, sum and O^T go to the workspace, a counter says
// who is last, and that block adds the partials in their order.
//
// Copies.  Every warp has a ring of kStages tiles in shared memory that it fills
// with 16-byte asynchronous copies, through shares and sequences without a stop; a
// position that does not count is filled with zeros.  128-byte lines are permuted
// so that neither product's loads meet in a bank.
//
// Codes.  8- and 4-bit codes become exact bf16 integers with two to four logic
// operations per pair (128 + low bits as a bf16 pattern, less 128, 256 or 136).
// A row's scale multiplies its score, and its weight before P V.  fp32 queries and
// weights enter as the sum of three bf16, weights of bf16 results as two: products
// and sums lose nothing that the result's type shows.
#pragma once

#include <atomic>

#include "uq_attn.h"
#include "uq_kv.cuh"
#include "uq_launch.h"

namespace uq {
namespace attn {

constexpr int kAttnWarps = 4, kAttnThreads = 32 * kAttnWarps, kMaxBlocksPerSm = 4;

// Shapes of a tile: 4 KB of rows or more, and room for a warp's O^T.
template <int FMT, int HD, int NT>
struct Tile {
    static constexpr int RB = KvRow<FMT, HD>::kBytes;             // bytes of a row
    static constexpr int W = KvRow<FMT, HD>::kWords;              // scale words of a row
    static constexpr int kNeed = 8 * NT * HD * 4 > 4096 ? 8 * NT * HD * 4 : 4096;
    static constexpr int kTok = kNeed / (2 * RB) > 16 ? kNeed / (2 * RB) : 16;
    static constexpr int kStages = 3;
    static constexpr int NSB = kTok / 16;                         // blocks of 16 positions: each in one page
    static constexpr int CPR = RB / 16;                           // 16-byte chunks of a row
    static constexpr int kRows = kTok * RB;                       // bytes of K, and of V
    static constexpr int kScales = kTok * W * 4;
    static constexpr int kSlot = 2 * kRows + 2 * kScales;
    static constexpr int kGroups = FMT == UQ_KV_INT4 ? HD / kKvGroup : 1;
};

template <int FMT, int HD, int WD, int NT>
struct Plan {
    using T = Tile<FMT, HD, NT>;
    static constexpr int NQ = WD == UQ_W_F32 ? 3 : 1;             // bf16 terms of a query
    static constexpr int NP = WD == UQ_W_F32 ? 3 : 2;             // and of a weight
    static constexpr int kCols = 8 * NT;
    static constexpr int kQStride = HD * 2 + (FMT == UQ_KV_BF16 ? 64 : 16);
    static constexpr int kRing = kAttnWarps * T::kStages * T::kSlot;
    static constexpr int kMask = kRing;                           // 64-bit masks of the ring's tiles
    static constexpr int kQ = kMask + kAttnWarps * T::kStages * 8;
    static constexpr int kQSum = kQ + NQ * kCols * kQStride;      // int4: sums of a query's groups
    static constexpr int kStats = kQSum + kCols * T::kGroups * 4; // m and sum of each warp, column
    static constexpr int kBias = kStats + kAttnWarps * kCols * 8; // int4: weighted minima of each warp, column, group
    static constexpr int kMisc = kBias + kAttnWarps * kCols * T::kGroups * 4;
    static constexpr int kBytes = kMisc + 64;
    static_assert(kCols * HD * 4 <= T::kSlot, "a slot holds a warp's O^T");
};

__device__ __forceinline__ uint32_t smem_at(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void copy16(uint32_t dst, const void* src, bool there) {
    const int n = there ? 16 : 0;
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(n) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ uint4 lds128(uint32_t a) {
    uint4 r;
    asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "r"(a));
    return r;
}
__device__ __forceinline__ uint2 lds64(uint32_t a) {
    uint2 r;
    asm volatile("ld.shared.v2.b32 {%0,%1}, [%2];" : "=r"(r.x), "=r"(r.y) : "r"(a));
    return r;
}
__device__ __forceinline__ uint32_t lds32(uint32_t a) {
    uint32_t r;
    asm volatile("ld.shared.b32 %0, [%1];" : "=r"(r) : "r"(a));
    return r;
}
__device__ __forceinline__ void mma(float d[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// An 8 x 8 matrix of 16-bit values, a row of pairs on four lanes, transposed.
__device__ __forceinline__ uint32_t transposed(uint32_t x) {
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
    return r;
}
__device__ __forceinline__ float exp2_fast(float x) {
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
__device__ __forceinline__ uint32_t sub_bf16x2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
// Two int8 codes in the low bytes of x's halves (the high bytes are ignored) as
// bf16: 128 + the low seven bits, less 128, or 256 where the sign bit is set.
__device__ __forceinline__ uint32_t bf16_of_int8(uint32_t x) {
    return sub_bf16x2((x & 0x007f007fu) | 0x43004300u, (x & 0x00800080u) | 0x43004300u);
}
// Two int4 codes in the low bits of x's halves as bf16, less 8: 128 + c - 136.
__device__ __forceinline__ uint32_t bf16_of_int4(uint32_t x) {
    return sub_bf16x2((x & 0x000f000fu) | 0x43004300u, 0x43084308u);
}

// The pair (x0, x1) as N pairs of bf16 whose sums are x0, x1: all but the last
// are cut off (so that no value overflows), the last is rounded.
template <int N>
__device__ __forceinline__ void split_pair(float x0, float x1, uint32_t part[N]) {
#pragma unroll
    for (int i = 0; i < N - 1; ++i) {
        part[i] = __byte_perm(__float_as_uint(x0), __float_as_uint(x1), 0x7632);
        x0 -= bf16_low(part[i]);
        x1 -= bf16_high(part[i]);
    }
    part[N - 1] = bf16_pair(x0, x1);
}

// Byte offset of 16-byte chunk `chunk` of row t of a tile.  Rows of K are read
// by 8-row blocks, 16 or 8 bytes a lane; rows of V by positions 2c (and 2c + 1), c
// = 0..3, 16, 8 or 4 bytes a lane: both meet no bank twice.
template <int RB>
__device__ __forceinline__ uint32_t line_swizzle(int t) {
    return RB >= 128 ? (t & 6) ^ ((t & 1) << 2) : RB == 64 ? t & 6 : (t >> 1) & 2;
}
template <int RB>
__device__ __forceinline__ uint32_t chunk_at(int t, int chunk, uint32_t swizzle) {
    if (RB >= 128) return t * RB + (chunk >> 3) * 128 + (((chunk & 7) ^ swizzle) << 4);
    constexpr int RPL = RB >= 128 ? 1 : 128 / RB;
    return (t / RPL) * 128 + ((((t % RPL) * (RB / 16) + chunk) ^ swizzle) << 4);
}

// First channel of row tile i of O^T for lane group g (rows g and g + 8 are this channel and the next).
template <int FMT, int HD>
__device__ __forceinline__ int channel_of(int i, int g) {
    if (FMT == UQ_KV_INT8 && HD >= 128) return 128 * (i / 8) + 16 * g + 2 * (i % 8);
    return 64 * (i / 4) + 8 * g + 2 * (i % 4);
}

// A place in the order of tiles: sequence b, unit u (a key/value head and its
// query heads), tile of its positions.
struct Cursor {
    int b, u, tile, tiles, n, first;   // of sequence b: tiles, positions first .. n - 1
    template <int TOK>
    __device__ __forceinline__ void sequence(const AttnArgs& a, int seq) {
        b = seq;
        const int64_t cap = a.max_pages << a.page_shift;
        n = (int)min((int64_t)max(__ldg(a.seq_lens + seq), 0), cap);
        first = a.window > 0 && a.window < n ? n - (int)a.window : 0;
        tiles = max(1, (n - (first & ~15) + TOK - 1) / TOK);
    }
    template <int TOK>
    __device__ __forceinline__ void advance(const AttnArgs& a, int units, int step) {
        tile += step;
        while (tile >= tiles) {
            tile -= tiles;
            if (++u == units) {
                u = 0;
                if (b + 1 >= a.batch) { tile = 0; return; }
                sequence<TOK>(a, b + 1);
            }
        }
    }
};

// The share of a block: `total` tiles over `blocks` blocks, the first
// total % blocks of them one tile more.
struct Shares {
    int64_t per, more;
    __device__ __forceinline__ Shares(int64_t total, int blocks) {
        if (total <= 0x7fffffff) {
            per = (uint32_t)total / (uint32_t)blocks;
            more = (uint32_t)total - (uint32_t)per * (uint32_t)blocks;
        } else {
            per = total / blocks;
            more = total - per * blocks;
        }
    }
    __device__ __forceinline__ int64_t start(int i) const { return per * i + min((int64_t)i, more); }
    __device__ __forceinline__ int owner(int64_t t) const {
        const int64_t big = more * (per + 1);
        return (int)(t < big ? t / (per + 1) : more + (t - big) / per);
    }
};

// Floats of the counters, one of 64 bits a block, ahead of the partials.
__host__ __device__ constexpr int counter_floats(int blocks) { return 2 * blocks + 2 * (blocks & 1); }

// Four channels of a finished row: acc / sum (nothing counted: 0), and its logarithm, from base 2.
template <int WD>
__device__ __forceinline__ void put_out(const AttnArgs& a, int b, int head, int d, const float4& acc, float low, float sum) {
    const float inv = sum == 0.0f ? 0.0f : __fdiv_rn(1.0f, sum);
    const int64_t e = b * a.out_batch + head * a.out_head + d;
    if (WD == UQ_W_F32) {
        *reinterpret_cast<float4*>(static_cast<float*>(a.out) + e) = make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv);
    } else {
        *reinterpret_cast<uint2*>(static_cast<uint16_t*>(a.out) + e) =
            make_uint2(bf16_pair(acc.x * inv, acc.y * inv), bf16_pair(acc.z * inv, acc.w * inv));
    }
    if (d == 0 && a.lse != nullptr) a.lse[(int64_t)b * a.heads + head] = sum == 0.0f ? -INFINITY : (low + log2f(sum)) * 0.6931471805599453f;
}

template <int FMT, int HD, int WD, int NT>
__global__ void __launch_bounds__(kAttnThreads) attn_kernel(const AttnArgs a, const int units, const int chunks) {
    using T = Tile<FMT, HD, NT>;
    using P = Plan<FMT, HD, WD, NT>;
    constexpr int TOK = T::kTok, ST = T::kStages, MT = TOK / 16, OT = HD / 16, RB = T::RB, W = T::W, NG = T::kGroups;
    constexpr int CO = P::kCols, NQ = P::NQ, NP = P::NP;
    extern __shared__ __align__(128) uint8_t smem[];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, c = lane & 3;
    float* const stats = reinterpret_cast<float*>(smem + P::kStats);
    float* const bias_sm = reinterpret_cast<float*>(smem + P::kBias);
    int64_t* const misc = reinterpret_cast<int64_t*>(smem + P::kMisc);
    const uint32_t ring = smem_at(smem) + warp * ST * T::kSlot, masks = smem_at(smem) + P::kMask + warp * ST * 8;
    const uint32_t qs = smem_at(smem) + P::kQ;
    inputs_ready();

    // --- this block's share
    Cursor cur;
    int64_t total;
    {
        const int per = (a.batch + kAttnThreads - 1) / kAttnThreads, b0 = min(a.batch, tid * per), b1 = min(a.batch, b0 + per);
        int64_t sum = 0;
        for (int b = b0; b < b1; ++b) {
            cur.sequence<TOK>(a, b);
            sum += cur.tiles;
        }
        int64_t incl = sum;
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
            const int64_t x = __shfl_up_sync(kFull, incl, off);
            if (lane >= off) incl += x;
        }
        if (lane == 31) misc[warp] = incl;
        __syncthreads();
        int64_t excl = incl - sum;
        total = 0;
#pragma unroll
        for (int w = 0; w < kAttnWarps; ++w) {
            const int64_t x = misc[w];
            if (w < warp) excl += x;
            total += x;
        }
        total *= units;
        excl *= units;
        __syncthreads();
        const int blocks = (int)min((int64_t)gridDim.x, (total + kAttnWarps - 1) / kAttnWarps);
        if ((int)blockIdx.x >= blocks) return;
        const int64_t at = Shares(total, blocks).start(blockIdx.x);
        if (at >= excl && at < excl + sum * units) {
            int64_t t = at - excl;
            int b = b0;
            for (;; ++b) {
                cur.sequence<TOK>(a, b);
                if (t < (int64_t)cur.tiles * units) break;
                t -= (int64_t)cur.tiles * units;
            }
            misc[4] = b;
            misc[5] = t;
        }
        __syncthreads();
        const int64_t t = misc[5];
        cur.sequence<TOK>(a, (int)misc[4]);
        cur.u = (int)(t / cur.tiles);
        cur.tile = (int)(t - (int64_t)cur.u * cur.tiles);
    }
    const int blocks = (int)min((int64_t)gridDim.x, (total + kAttnWarps - 1) / kAttnWarps);
    const Shares shares(total, blocks);
    const int64_t share0 = shares.start(blockIdx.x);
    const int64_t share_n = shares.start(blockIdx.x + 1) - share0;

    // --- the ring: `load` is the next tile to be copied
    const int pmask = (1 << a.page_shift) - 1;
    Cursor load = cur;
    int64_t to_load = share_n > warp ? (share_n - warp + kAttnWarps - 1) / kAttnWarps : 0;
    if (to_load > 0 && warp > 0) load.advance<TOK>(a, units, warp);
    int page = -1;                                     // lane i < NSB: page of the next tile's block i, -1: none
    auto find_page = [&] {
        const int t = (load.first & ~15) + load.tile * TOK + 16 * lane;
        page = -1;
        if (lane < T::NSB && to_load > 0 && t < load.n) {
            page = __ldg(a.table + load.b * a.table_stride + (t >> a.page_shift));
            if ((uint32_t)page >= (uint64_t)a.c.pages) page = -1;
        }
    };
    auto issue = [&](int slot) {
        if (to_load > 0) {
            const int t0 = (load.first & ~15) + load.tile * TOK, kvh = load.u / chunks;
            const uint32_t dst = ring + slot * T::kSlot;
            int64_t row[T::NSB];                       // first row of each block in the pool
            int pg[T::NSB];
#pragma unroll
            for (int s = 0; s < T::NSB; ++s) {
                pg[s] = __shfl_sync(kFull, page, s);
                row[s] = (((int64_t)max(pg[s], 0) * a.c.kv_heads + kvh) << a.page_shift) + ((t0 + 16 * s) & pmask);
            }
            uint32_t mask[2] = {0, 0};
#pragma unroll
            for (int h = 0; h < (TOK + 31) / 32; ++h) {
                const int t = t0 + 32 * h + lane;
                const int p = T::NSB == 1 ? pg[0] : lane < 16 ? pg[2 * h] : pg[(2 * h + 1) % T::NSB];
                mask[h] = __ballot_sync(kFull, (TOK >= 32 || lane < TOK) && t >= load.first && t < load.n && p >= 0);
            }
            if (lane == 0) asm volatile("st.shared.v2.b32 [%0], {%1,%2};" ::"r"(masks + slot * 8), "r"(mask[0]), "r"(mask[1]));
#pragma unroll
            for (int i = 0; i < T::kRows / 512; ++i) {
                const int id = 32 * i + lane, t = id / T::CPR, s = 32 * i / (16 * T::CPR);
                const bool there = (mask[(32 * i / T::CPR) >> 5] >> (t & 31)) & 1;
                const int64_t off = row[s] * RB + (id - s * 16 * T::CPR) * 16;
                const uint32_t at = dst + chunk_at<RB>(t, id % T::CPR, line_swizzle<RB>(t));
                copy16(at, static_cast<const uint8_t*>(a.c.k) + off, there);
                copy16(at + T::kRows, static_cast<const uint8_t*>(a.c.v) + off, there);
            }
            if constexpr (W > 0) {
                constexpr int SC = T::kScales / 16;    // chunks of K's scales, and of V's; 4 W of a block
#pragma unroll
                for (int i = 0; i < (2 * SC + 31) / 32; ++i) {
                    const int id = 32 * i + lane, local = id % SC, s = local / (4 * W);
                    int64_t r = row[0];
                    int p = pg[0];
#pragma unroll
                    for (int k = 1; k < T::NSB; ++k)
                        if (s == k) { r = row[k]; p = pg[k]; }
                    const uint8_t* from = static_cast<const uint8_t*>(id < SC ? a.c.k_scale : a.c.v_scale);
                    if (id < 2 * SC) copy16(dst + 2 * T::kRows + id * 16, from + r * (4 * W) + (local % (4 * W)) * 16, p >= 0);
                }
            }
            if (--to_load > 0) load.advance<TOK>(a, units, kAttnWarps);
            find_page();
        }
        copies_commit();
    };
    find_page();
#pragma unroll
    for (int s = 0; s < ST; ++s) issue(s);
    int slot = 0;                                      // of the tile that comes next

    const float to_log2 = a.scale * 1.4426950408889634f;
    const uint32_t k_swz = line_swizzle<RB>(g), v_swz0 = line_swizzle<RB>(2 * c), v_swz1 = line_swizzle<RB>(2 * c + 1);

    // --- the parts of (sequence, head)s in this share
    for (int64_t done = 0; done < share_n;) {
        const int64_t part = min((int64_t)(cur.tiles - cur.tile), share_n - done);
        const int kvh = cur.u / chunks, r = a.heads / a.c.kv_heads, col0 = (cur.u - kvh * chunks) * CO;
        const int head0 = kvh * r + col0, cols = min(CO, r - col0);

        // queries: 8 channels a thread, rows beyond the heads are zero
        for (int i = tid; i < CO * (HD / 8); i += kAttnThreads) {
            const int n = i / (HD / 8), d = (i % (HD / 8)) * 8;
            float x[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = 0.0f;
            if (n < cols) {
                const int64_t e = cur.b * a.q_batch + (head0 + n) * a.q_head + d;
                if (WD == UQ_W_F32) {
                    f4_to(ldg4(static_cast<const float*>(a.q) + e), x);
                    f4_to(ldg4(static_cast<const float*>(a.q) + e + 4), x + 4);
                } else {
                    const uint4 w = __ldg(reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(a.q) + e));
                    const uint32_t ww[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                    for (int j = 0; j < 8; ++j) x[j] = (j & 1) ? bf16_high(ww[j >> 1]) : bf16_low(ww[j >> 1]);
                }
            }
            if constexpr (FMT == UQ_KV_INT4) {
                float s = ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
#pragma unroll
                for (int off = 4; off >= 1; off >>= 1) s += __shfl_xor_sync(kFull, s, off);
                if ((i & 7) == 0) reinterpret_cast<float*>(smem + P::kQSum)[n * NG + d / kKvGroup] = s;
            }
            uint32_t part_of[4][NQ];
#pragma unroll
            for (int j = 0; j < 4; ++j)                // codes of 4 bits come as pairs (i, i + 4)
                split_pair<NQ>(FMT == UQ_KV_INT4 ? x[j] : x[2 * j], FMT == UQ_KV_INT4 ? x[j + 4] : x[2 * j + 1], part_of[j]);
#pragma unroll
            for (int q = 0; q < NQ; ++q)
                *reinterpret_cast<uint4*>(smem + P::kQ + (q * CO + n) * P::kQStride + d * 2) =
                    make_uint4(part_of[0][q], part_of[1][q], part_of[2][q], part_of[3][q]);
        }
        __syncthreads();

        float m[NT][2], l[NT][2], o[OT][NT][4], bias[NG][NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                m[nt][j] = -INFINITY;
                l[nt][j] = 0.0f;
#pragma unroll
                for (int k = 0; k < NG; ++k) bias[k][nt][j] = 0.0f;
            }
#pragma unroll
        for (int i = 0; i < OT; ++i)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int j = 0; j < 4; ++j) o[i][nt][j] = 0.0f;

        const int64_t mine0 = done + ((warp - (int)(done & 3)) & 3);
        bool held = false;                             // the last tile's slot is not refilled yet
        for (int64_t j = mine0; j < done + part; j += kAttnWarps) {
            if (held) {
                __syncwarp();
                issue(slot == 0 ? ST - 1 : slot - 1);
            }
            copies_wait<ST - 1>();
            __syncwarp();
            const uint32_t at = ring + slot * T::kSlot, sk = at + 2 * T::kRows, sv = sk + T::kScales;
            const uint2 mk = lds64(masks + slot * 8);
            const uint64_t mask = (uint64_t)mk.y << 32 | mk.x;

            // scores, to base 2: rows of a tile are positions 16 mt + g and + 8
            float x[MT][NT][4];
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                float acc[NT][4];
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        acc[nt][e] = 0.0f;
                        x[mt][nt][e] = 0.0f;
                    }
                const int t0 = 16 * mt + g, t1 = t0 + 8;
                if constexpr (FMT == UQ_KV_BF16) {
#pragma unroll
                    for (int kk = 0; kk < HD / 32; ++kk) {
                        const uint4 lo = lds128(at + chunk_at<RB>(t0, 4 * kk + c, k_swz));
                        const uint4 hi = lds128(at + chunk_at<RB>(t1, 4 * kk + c, k_swz));
#pragma unroll
                        for (int q = 0; q < NQ; ++q)
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt) {
                                const uint4 b = lds128(qs + (q * CO + 8 * nt + g) * P::kQStride + (32 * kk + 8 * c) * 2);
                                mma(acc[nt], lo.x, hi.x, lo.y, hi.y, b.x, b.y);
                                mma(acc[nt], lo.z, hi.z, lo.w, hi.w, b.z, b.w);
                            }
                    }
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int e = 0; e < 4; ++e) x[mt][nt][e] = acc[nt][e] * to_log2;
                } else if constexpr (FMT == UQ_KV_INT8) {
#pragma unroll
                    for (int kk = 0; kk < HD / 64; ++kk) {
                        const uint4 lo4 = lds128(at + chunk_at<RB>(t0, 4 * kk + c, k_swz));
                        const uint4 hi4 = lds128(at + chunk_at<RB>(t1, 4 * kk + c, k_swz));
                        const uint32_t lo[4] = {lo4.x, lo4.y, lo4.z, lo4.w}, hi[4] = {hi4.x, hi4.y, hi4.z, hi4.w};
#pragma unroll
                        for (int s = 0; s < 4; s += 2) {
                            uint32_t av[2][4];
#pragma unroll
                            for (int k = 0; k < 2; ++k) {
                                av[k][0] = bf16_of_int8(__byte_perm(lo[s + k], 0, 0x4140));
                                av[k][1] = bf16_of_int8(__byte_perm(hi[s + k], 0, 0x4140));
                                av[k][2] = bf16_of_int8(__byte_perm(lo[s + k], 0, 0x4342));
                                av[k][3] = bf16_of_int8(__byte_perm(hi[s + k], 0, 0x4342));
                            }
#pragma unroll
                            for (int q = 0; q < NQ; ++q)
#pragma unroll
                                for (int nt = 0; nt < NT; ++nt) {
                                    const uint4 b = lds128(qs + (q * CO + 8 * nt + g) * P::kQStride + (64 * kk + 16 * c + 4 * s) * 2);
                                    mma(acc[nt], av[0][0], av[0][1], av[0][2], av[0][3], b.x, b.y);
                                    mma(acc[nt], av[1][0], av[1][1], av[1][2], av[1][3], b.z, b.w);
                                }
                        }
                    }
                    const float s0 = __uint_as_float(lds32(sk + 4 * t0)) * to_log2, s1 = __uint_as_float(lds32(sk + 4 * t1)) * to_log2;
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int e = 0; e < 4; ++e) x[mt][nt][e] = acc[nt][e] * (e < 2 ? s0 : s1);
                } else {
#pragma unroll
                    for (int kk = 0; kk < NG; ++kk) {
                        const uint2 lo2 = lds64(at + chunk_at<RB>(t0, 2 * kk + (c >> 1), k_swz) + (c & 1) * 8);
                        const uint2 hi2 = lds64(at + chunk_at<RB>(t1, 2 * kk + (c >> 1), k_swz) + (c & 1) * 8);
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                            for (int e = 0; e < 4; ++e) acc[nt][e] = 0.0f;
#pragma unroll
                        for (int w = 0; w < 2; ++w) {
                            const uint32_t lo = w ? lo2.y : lo2.x, hi = w ? hi2.y : hi2.x;
                            uint32_t av[2][4];
#pragma unroll
                            for (int k = 0; k < 2; ++k) {
                                av[k][0] = bf16_of_int4(lo >> (8 * k));
                                av[k][1] = bf16_of_int4(hi >> (8 * k));
                                av[k][2] = bf16_of_int4(lo >> (8 * k + 4));
                                av[k][3] = bf16_of_int4(hi >> (8 * k + 4));
                            }
#pragma unroll
                            for (int q = 0; q < NQ; ++q)
#pragma unroll
                                for (int nt = 0; nt < NT; ++nt) {
                                    const uint4 b = lds128(qs + (q * CO + 8 * nt + g) * P::kQStride + (64 * kk + 16 * c + 8 * w) * 2);
                                    mma(acc[nt], av[0][0], av[0][1], av[0][2], av[0][3], b.x, b.y);
                                    mma(acc[nt], av[1][0], av[1][1], av[1][2], av[1][3], b.z, b.w);
                                }
                        }
                        // value = scale (c - 8) + (minimum + 8 scale): the second part meets the sum of the query's group
                        const uint32_t p0 = lds32(sk + 4 * (t0 * W + kk)), p1 = lds32(sk + 4 * (t1 * W + kk));
                        const float s0 = bf16_low(p0), s1 = bf16_low(p1);
                        const float z0 = fmaf(8.0f, s0, bf16_high(p0)), z1 = fmaf(8.0f, s1, bf16_high(p1));
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const float qsum = reinterpret_cast<const float*>(smem + P::kQSum)[(8 * nt + 2 * c + (e & 1)) * NG + kk];
                                x[mt][nt][e] = fmaf(acc[nt][e], e < 2 ? s0 : s1, fmaf(e < 2 ? z0 : z1, qsum, x[mt][nt][e]));
                            }
                    }
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int e = 0; e < 4; ++e) x[mt][nt][e] *= to_log2;
                }
            }
            constexpr uint64_t kAll = TOK == 64 ? ~0ull : (1ull << (TOK & 63)) - 1;
            const bool whole = mask == kAll;
            if (!whole) {
#pragma unroll
                for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const bool in = (mask >> (16 * mt + g + (e < 2 ? 0 : 8))) & 1;
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
                            if (!in) x[mt][nt][e] = -INFINITY;
                    }
            }

            // running maximum, weights
            float base[NT][2];
            bool grew = false;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    float top = fmaxf(x[0][nt][j], x[0][nt][j + 2]);
#pragma unroll
                    for (int mt = 1; mt < MT; ++mt) top = fmaxf(top, fmaxf(x[mt][nt][j], x[mt][nt][j + 2]));
#pragma unroll
                    for (int off = 4; off <= 16; off <<= 1) top = fmaxf(top, __shfl_xor_sync(kFull, top, off));
                    base[nt][j] = fmaxf(m[nt][j], top);
                    grew |= base[nt][j] > m[nt][j];
                }
            if (__any_sync(kFull, grew)) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const float f = base[nt][j] == -INFINITY ? 0.0f : exp2_fast(m[nt][j] - base[nt][j]);
                        m[nt][j] = base[nt][j];
                        l[nt][j] *= f;
#pragma unroll
                        for (int k = 0; k < NG; ++k) bias[k][nt][j] *= f;
#pragma unroll
                        for (int i = 0; i < OT; ++i) {
                            o[i][nt][j] *= f;
                            o[i][nt][j + 2] *= f;
                        }
                    }
            }
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const float low = m[nt][j] == -INFINITY ? 0.0f : m[nt][j];
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt) {
                        x[mt][nt][j] = exp2_fast(x[mt][nt][j] - low);
                        x[mt][nt][j + 2] = exp2_fast(x[mt][nt][j + 2] - low);
                        l[nt][j] += x[mt][nt][j] + x[mt][nt][j + 2];
                    }
                }

            // O^T += V^T P^T, 16 positions at a time
            const uint32_t av = at + T::kRows;
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                const int ta[4] = {16 * mt + 2 * c, 16 * mt + 2 * c + 1, 16 * mt + 2 * c + 8, 16 * mt + 2 * c + 9};
                const bool in0 = whole || ((mask >> (16 * mt + g)) & 1), in1 = whole || ((mask >> (16 * mt + g + 8)) & 1);
#pragma unroll
                for (int kk = 0; kk < NG; ++kk) {
                    float s0 = 1.0f, s1 = 1.0f;
                    if constexpr (FMT == UQ_KV_INT8) {
                        s0 = in0 ? __uint_as_float(lds32(sv + 4 * (16 * mt + g))) : 0.0f;
                        s1 = in1 ? __uint_as_float(lds32(sv + 4 * (16 * mt + g + 8))) : 0.0f;
                    } else if constexpr (FMT == UQ_KV_INT4) {
                        const uint32_t p0 = in0 ? lds32(sv + 4 * ((16 * mt + g) * W + kk)) : 0u;
                        const uint32_t p1 = in1 ? lds32(sv + 4 * ((16 * mt + g + 8) * W + kk)) : 0u;
                        s0 = bf16_low(p0);
                        s1 = bf16_low(p1);
                        const float z0 = fmaf(8.0f, s0, bf16_high(p0)), z1 = fmaf(8.0f, s1, bf16_high(p1));
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                            for (int j = 0; j < 2; ++j)
                                bias[kk][nt][j] = fmaf(x[mt][nt][j], z0, fmaf(x[mt][nt][j + 2], z1, bias[kk][nt][j]));
                    }
                    uint32_t b[NT][NP][2];
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        uint32_t p0[NP], p1[NP];
                        split_pair<NP>(x[mt][nt][0] * s0, x[mt][nt][1] * s0, p0);
                        split_pair<NP>(x[mt][nt][2] * s1, x[mt][nt][3] * s1, p1);
#pragma unroll
                        for (int p = 0; p < NP; ++p) {
                            b[nt][p][0] = transposed(p0[p]);
                            b[nt][p][1] = transposed(p1[p]);
                        }
                    }
                    auto add = [&](int i, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3) {
#pragma unroll
                        for (int p = 0; p < NP; ++p)
#pragma unroll
                            for (int nt = 0; nt < NT; ++nt) mma(o[i][nt], a0, a1, a2, a3, b[nt][p][0], b[nt][p][1]);
                    };
                    if constexpr (FMT == UQ_KV_BF16) {
#pragma unroll
                        for (int jj = 0; jj < HD / 64; ++jj) {
                            uint32_t v[4][4];
#pragma unroll
                            for (int k = 0; k < 4; ++k) {
                                const uint4 w = lds128(av + chunk_at<RB>(ta[k], 8 * jj + g, (k & 1) ? v_swz1 : v_swz0));
                                v[k][0] = w.x; v[k][1] = w.y; v[k][2] = w.z; v[k][3] = w.w;
                            }
#pragma unroll
                            for (int i = 0; i < 4; ++i)
                                add(4 * jj + i, __byte_perm(v[0][i], v[1][i], 0x5410), __byte_perm(v[0][i], v[1][i], 0x7632),
                                    __byte_perm(v[2][i], v[3][i], 0x5410), __byte_perm(v[2][i], v[3][i], 0x7632));
                        }
                    } else if constexpr (FMT == UQ_KV_INT8) {
                        constexpr int NW = HD >= 128 ? 4 : 2;     // words of a lane's part of a row
#pragma unroll
                        for (int jj = 0; jj < HD / (32 * NW); ++jj) {
                            uint32_t v[4][4];
#pragma unroll
                            for (int k = 0; k < 4; ++k) {
                                const uint32_t swz = (k & 1) ? v_swz1 : v_swz0;
                                if constexpr (NW == 4) {
                                    const uint4 w = lds128(av + chunk_at<RB>(ta[k], 8 * jj + g, swz));
                                    v[k][0] = w.x; v[k][1] = w.y; v[k][2] = w.z; v[k][3] = w.w;
                                } else {
                                    const uint2 w = lds64(av + chunk_at<RB>(ta[k], g >> 1, swz) + (g & 1) * 8);
                                    v[k][0] = w.x; v[k][1] = w.y;
                                }
                            }
#pragma unroll
                            for (int w = 0; w < NW; ++w)
#pragma unroll
                                for (int h = 0; h < 2; ++h) {
                                    const int s0x = h ? 0x6662 : 0x4440, s1x = h ? 0x7773 : 0x5551;
                                    add(2 * NW * jj + 2 * w + h, bf16_of_int8(__byte_perm(v[0][w], v[1][w], s0x)),
                                        bf16_of_int8(__byte_perm(v[0][w], v[1][w], s1x)),
                                        bf16_of_int8(__byte_perm(v[2][w], v[3][w], s0x)),
                                        bf16_of_int8(__byte_perm(v[2][w], v[3][w], s1x)));
                                }
                        }
                    } else {
                        uint32_t v[4];
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            v[k] = lds32(av + chunk_at<RB>(ta[k], 2 * kk + (g >> 2), (k & 1) ? v_swz1 : v_swz0) + (g & 3) * 4);
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const uint32_t w0 = __byte_perm(v[0], v[1], h ? 0x7632 : 0x5410);
                            const uint32_t w1 = __byte_perm(v[2], v[3], h ? 0x7632 : 0x5410);
#pragma unroll
                            for (int i = 0; i < 2; ++i)
                                add(4 * kk + 2 * h + i, bf16_of_int4(w0 >> (8 * i)), bf16_of_int4(w0 >> (8 * i + 4)),
                                    bf16_of_int4(w1 >> (8 * i)), bf16_of_int4(w1 >> (8 * i + 4)));
                        }
                    }
                }
            }
            slot = slot + 1 == ST ? 0 : slot + 1;
            held = true;
        }

        // --- join the warps: the last tile's slot takes O^T [column][channel]; one that had no tile has sum 0
        const int spare = slot == 0 ? ST - 1 : slot - 1;
        float* const mine = reinterpret_cast<float*>(smem + (warp * ST + spare) * T::kSlot);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int off = 4; off <= 16; off <<= 1) {
                    l[nt][j] += __shfl_xor_sync(kFull, l[nt][j], off);
#pragma unroll
                    for (int k = 0; k < NG; ++k)
                        if (FMT == UQ_KV_INT4) bias[k][nt][j] += __shfl_xor_sync(kFull, bias[k][nt][j], off);
                }
        if (g == 0) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const int col = 8 * nt + 2 * c + j;
                    stats[(warp * CO + col) * 2] = m[nt][j];
                    stats[(warp * CO + col) * 2 + 1] = l[nt][j];
#pragma unroll
                    for (int k = 0; k < NG; ++k) bias_sm[(warp * CO + col) * NG + k] = bias[k][nt][j];
                }
        }
        __syncwarp();
        if (held) {
#pragma unroll
            for (int i = 0; i < OT; ++i)
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int j = 0; j < 2; ++j)
                        *reinterpret_cast<float2*>(mine + (8 * nt + 2 * c + j) * HD + channel_of<FMT, HD>(i, g)) =
                            make_float2(o[i][nt][j], o[i][nt][j + 2]);
        }
        // warps that hold a slot have it at the ring's place of their own
        if (lane == 0) misc[warp] = held ? spare : -1;
        __syncthreads();

        const bool all = cur.tile == 0 && part == cur.tiles;
        const int64_t seg0 = share0 + done - cur.tile;           // first tile of this (sequence, head)
        const int own0 = all ? 0 : shares.owner(seg0), own1 = all ? 0 : shares.owner(seg0 + cur.tiles - 1);
        constexpr int kPart = CO * (HD + 2);                      // floats of a partial: O^T, then m and sum of each column
        float* const parts = a.work + counter_floats(gridDim.x);
        float* const to = parts + (int64_t)(2 * blockIdx.x + (done > 0 ? 1 : 0)) * kPart;
        for (int i = tid; i < CO * (HD / 4); i += kAttnThreads) {
            const int col = i / (HD / 4), d = (i % (HD / 4)) * 4;
            float top = -INFINITY, sum = 0.0f;
#pragma unroll
            for (int w = 0; w < kAttnWarps; ++w) top = fmaxf(top, stats[(w * CO + col) * 2]);
            const float low = top == -INFINITY ? 0.0f : top;
            float4 acc = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
            for (int w = 0; w < kAttnWarps; ++w) {
                const int s = (int)misc[w];
                if (s < 0) continue;
                const float f = exp2_fast(stats[(w * CO + col) * 2] - low);
                const float4 v = *reinterpret_cast<const float4*>(smem + (w * ST + s) * T::kSlot + (col * HD + d) * 4);
                const float z = FMT == UQ_KV_INT4 ? bias_sm[(w * CO + col) * NG + d / kKvGroup] : 0.0f;
                sum = fmaf(stats[(w * CO + col) * 2 + 1], f, sum);
                acc.x = fmaf(v.x + z, f, acc.x);
                acc.y = fmaf(v.y + z, f, acc.y);
                acc.z = fmaf(v.z + z, f, acc.z);
                acc.w = fmaf(v.w + z, f, acc.w);
            }
            if (all) {
                if (col < cols) put_out<WD>(a, cur.b, head0 + col, d, acc, low, sum);
            } else {
                *reinterpret_cast<float4*>(to + col * HD + d) = acc;
                if (d == 0) *reinterpret_cast<float2*>(to + CO * HD + 2 * col) = make_float2(top, sum);
            }
        }
        if (!all) {
            // --- join the blocks: the last to arrive adds the partials in order
            __threadfence();
            __syncthreads();
            if (tid == 0) {
                unsigned long long* const word = reinterpret_cast<unsigned long long*>(a.work) + own0;
                unsigned long long was = *reinterpret_cast<volatile unsigned long long*>(word), next;
                for (;;) {
                    next = was >> 16 == a.nonce ? was + 1 : (unsigned long long)a.nonce << 16 | 1;
                    const unsigned long long now = atomicCAS(word, was, next);
                    if (now == was) break;
                    was = now;
                }
                const bool last = (int)(next & 0xffff) == own1 - own0 + 1;
                if (last) *word = 0;
                misc[6] = last;
            }
            __syncthreads();
            if (misc[6]) {
                __threadfence();
                const bool first_here = shares.start(own0) == seg0;       // the first block's slot
                for (int i = tid; i < cols * (HD / 4); i += kAttnThreads) {
                    const int col = i / (HD / 4), d = (i % (HD / 4)) * 4;
                    float top = -INFINITY, sum = 0.0f;
                    float4 acc = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
                    for (int o1 = own0; o1 <= own1; ++o1) {
                        const float* p = parts + (int64_t)(2 * o1 + (o1 == own0 && !first_here ? 1 : 0)) * kPart;
                        const float2 ms = __ldcg(reinterpret_cast<const float2*>(p + CO * HD + 2 * col));
                        const float4 v = __ldcg(reinterpret_cast<const float4*>(p + col * HD + d));
                        const float t2 = fmaxf(top, ms.x), low = t2 == -INFINITY ? 0.0f : t2;
                        const float f0 = exp2_fast(top - low), f1 = exp2_fast(ms.x - low);
                        top = t2;
                        sum = fmaf(sum, f0, ms.y * f1);
                        acc.x = fmaf(acc.x, f0, v.x * f1);
                        acc.y = fmaf(acc.y, f0, v.y * f1);
                        acc.z = fmaf(acc.z, f0, v.z * f1);
                        acc.w = fmaf(acc.w, f0, v.w * f1);
                    }
                    put_out<WD>(a, cur.b, head0 + col, d, acc, top == -INFINITY ? 0.0f : top, sum);
                }
            }
        }
        __syncthreads();
        if (held) issue(spare);
        done += part;
        cur.advance<TOK>(a, units, (int)part);
    }
    copies_wait<0>();
}

// Blocks per SM of a kernel, asked for once per device, and its shared memory allowed.
template <int FMT, int HD, int WD, int NT>
cudaError_t blocks_per_sm(int* blocks) {
    constexpr int kDevices = 64;
    static std::atomic<int> known[kDevices];
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    const bool keep = dev < kDevices;
    if (keep && (*blocks = known[dev].load(std::memory_order_acquire)) > 0) return cudaSuccess;
    auto kern = attn_kernel<FMT, HD, WD, NT>;
    constexpr int bytes = Plan<FMT, HD, WD, NT>::kBytes;
    e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == cudaSuccess) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(blocks, kern, kAttnThreads, bytes);
    if (e != cudaSuccess) return e;
    *blocks = *blocks < 1 ? 1 : *blocks > kMaxBlocksPerSm ? kMaxBlocksPerSm : *blocks;
    if (keep) known[dev].store(*blocks, std::memory_order_release);
    return cudaSuccess;
}

template <int FMT, int HD, int WD, int NT>
cudaError_t go(const AttnArgs& a, cudaStream_t st) {
    using T = Tile<FMT, HD, NT>;
    int per_sm = 0;
    const cudaError_t e = blocks_per_sm<FMT, HD, WD, NT>(&per_sm);
    if (e != cudaSuccess) return e;
    const int r = a.heads / a.c.kv_heads, chunks = (r + 8 * NT - 1) / (8 * NT), units = a.c.kv_heads * chunks;
    // no more blocks than the table has room for tiles
    const int64_t tiles = ((a.max_pages << a.page_shift) + T::kTok - 1) / T::kTok * units;
    const int64_t most = (tiles + kAttnWarps - 1) / kAttnWarps, full = (int64_t)sm_count() * per_sm;
    const int grid = (int)(most > full / a.batch ? full : most * a.batch);
    return launch_dependent(attn_kernel<FMT, HD, WD, NT>, dim3(grid), dim3(kAttnThreads),
                            Plan<FMT, HD, WD, NT>::kBytes, st, a, units, chunks);
}

template <int FMT, int HD, int NT>
cudaError_t by_type(const AttnArgs& a, cudaStream_t st) {
    return a.dtype == UQ_W_F32 ? go<FMT, HD, UQ_W_F32, NT>(a, st) : go<FMT, HD, UQ_W_BF16, NT>(a, st);
}

template <int FMT>
cudaError_t by_head(const AttnArgs& a, cudaStream_t st) {
    const bool two = query_columns(a.heads / a.c.kv_heads, a.c.head_dim) == 16;
    switch (a.c.head_dim) {
        case 64: return two ? by_type<FMT, 64, 2>(a, st) : by_type<FMT, 64, 1>(a, st);
        case 128: return two ? by_type<FMT, 128, 2>(a, st) : by_type<FMT, 128, 1>(a, st);
        default: return by_type<FMT, 256, 1>(a, st);
    }
}

}  // namespace attn
}  // namespace uq
