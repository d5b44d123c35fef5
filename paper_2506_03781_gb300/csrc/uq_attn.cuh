// Attention of one new token of each sequence over the paged key-value cache
// (see uq_api.h).
//
// Per key/value head the r query heads that share it are the columns of two
// small products, with t the cached positions:
//     X^T [t, r] = K [t, hd] Q^T      O^T [hd, r] = V^T [hd, t] P^T,  P = exp2(X - m)
// A warp does both on the tensor cores for a tile of kTok positions (m16n8k16:
// positions, then channels, are the 16 rows; 8 query heads the columns) and keeps a
// running maximum m, sum and O^T in registers.
//
// What bounds it.  Reading K and V once: 64 sequences of up to 8192 tokens in bf16
// (224 MB) take 45.3 us, 4.9 TB/s, 74 % of the copy rate, of which the median warp's
// share 29 and the ends and the joins 11.  With codes it is the chain of a warp's own
// instructions, with two or three warps a scheduler to hide it: 131000 tokens in 8
// bits, fp32 queries (277 MB) 60.4 us, 4.6 TB/s, 990 instructions a tile of 32
// positions, 0.45 issued a cycle and scheduler; 128 x 4096 tokens in 4 bits, 8 heads a
// key/value head (608 MB) 166 us, 3.7 TB/s, 927 and 0.62, no pipe above 48 %.
// Calls of a few microseconds are bound by the chain of their loads: lengths,
// table, rows, partials (300 tokens 8.1 us).  Many very short sequences cost 25 to 28 us
// for every 1000 of 8 key/value heads.
//
// Shares.  The tiles of all sequences and heads, in order, are cut into one
// contiguous share of equal size per warp, whatever the lengths (a sequence's
// start counts as kHead tiles more: its queries, its result).  A warp works alone
// until its share is done: what lies in its share as a whole it writes out; the
// end of a (sequence, head) that began before and the start of one that goes on
// are partial.  One block per SM then joins the partials of its warps, once, and
// what lies in several blocks is joined by a block that finishes last: partial
// m, sum and O^T go to the workspace, a flag of each block says that they are
// there, and who sees all flags adds them in their order.  (A share per block,
// whose warps meet at every sequence: 64 ragged sequences 144 us; arrivals counted
// with an atomic instead of flags: 131000 tokens 10 us more.)
//
// Copies.  Every warp has a ring of tiles in shared memory that it fills with
// 16-byte asynchronous copies, through sequences without a stop.  128-byte lines are
// permuted so that neither product's loads meet in a bank.  What does not count
// never reaches the result: rows of bf16 are filled with zeros, codes are whatever
// they are and get the weight 0.
//
// Codes.  8- and 4-bit codes become exact 16-bit floating-point integers with one
// to two operations a value: of K in fp16 (1024 + code as a pattern, less the bias),
// with queries scaled by a power of two per head (the largest to 2^13..2^14: what is
// lost lies 2^-38 below it) and, if fp32, as the sum of two fp16 (22 bits); of V in
// bf16 (128 + low bits, less 128, 256 or 136), because weights have no least size:
// the sum of two bf16 for bf16 results (16 bits), of three for fp32 ones (24
// bits).  With bf16 rows all is bf16, fp32 queries the sum of three.  A row's scale
// multiplies its score, and its weight before P V.  fp32 results add every 16
// positions to the sum in fp32, because the tensor cores cut off instead of
// rounding (131000 tokens: 2.7e-6 off without, 3.9e-7 with); sums of bf16 results stay
// there over a warp's part of a sequence (2500 positions of one sign: 8e-6 off by the
// arithmetic's restatement, their rounding 4e-3).
#pragma once

#include <atomic>
#include <type_traits>

#include "uq_attn.h"
#include "uq_kv.cuh"
#include "uq_launch.h"

namespace uq {
namespace attn {

constexpr int most_warps(int head_dim) { return head_dim <= 128 ? 16 : 8; }              // warps of a block, at most
constexpr int kSmem = 226 * 1024;      // shared memory of a block
constexpr int kMinWarps = 8;           // warps of a block that have a share, where there are few tiles
// Where warps have few places, blocks begin with whole (sequence, head)s of up to so many tiles a warp: 300 tokens 8.0
// us (9.3 without), 48 ragged sequences of 16 heads 14.6 (16.4), 32 x 500 tokens 14.5 (16.0), 16 of up to 1000 tokens
// 14.5 (13.7); with 8 tiles 2000 tokens take 18.8 instead of 12.1.
constexpr int kSnapPlaces = 8, kSnapTiles = 4;

template <int FMT, int HD, int WD, int NT>
struct Plan {
    static constexpr bool F16 = FMT != UQ_KV_BF16;                // K and Q in fp16, else in bf16
    static constexpr int RB = KvRow<FMT, HD>::kBytes;             // bytes of a row
    static constexpr int W = KvRow<FMT, HD>::kWords;              // scale words of a row
    static constexpr int NG = FMT == UQ_KV_INT4 ? HD / kKvGroup : 1;
    static constexpr int NQ = WD == UQ_W_BF16 ? 1 : F16 ? 2 : 3;  // terms of a query
    static constexpr int NP = WD == UQ_W_F32 ? 3 : 2;             // and of a weight
    static constexpr int CO = 8 * NT;                             // query heads, columns
    static constexpr int OT = HD / 16;                            // row tiles of O^T
    // positions of a tile: 8 KB of rows, as far as the scores' registers allow (8-bit codes with 16 positions a tile:
    // 131000 tokens 71 us, with 32 63)
    static constexpr int kMostTok = NT * HD == 64 && RB == 32 ? 64 : NT * HD <= 256 ? 32 : 16;
    static constexpr int kTok = 4096 / RB < 16 ? 16 : 4096 / RB < kMostTok ? 4096 / RB : kMostTok;
    // tiles that the start of a (sequence, head) counts for; a tile of 4-bit codes lasts longer than others (2 for all:
    // 128 x 100 tokens in 8 bits 16.9 us, 3 15.3; 3 for 4 bits: 256 ragged sequences 56.6 us, 2 53.9)
    static constexpr int kHead = FMT == UQ_KV_INT4 ? 2 : 3;
    static constexpr int MT = kTok / 16;                          // blocks of 16 positions, each in one page
    static constexpr int CPR = RB / 16;                           // 16-byte chunks of a row
    static constexpr int LPB = 32 / MT;                           // lanes that copy a block of 16 positions
    static constexpr int RPI = LPB / CPR;                         // rows that they copy at a time
    static constexpr int kRows = kTok * RB;                       // bytes of K in a tile, and of V
    static constexpr int kScales = kTok * W * 4;
    // a slot of the ring: K and V of a tile, or where those are large one of them after the other, so that 8 warps have
    // room (bf16 rows of 256 channels, 16 x 4096 positions: 27.0 us, whole tiles 31.2; 131000 tokens in 8 bits: halves 72
    // us, whole 62)
    static constexpr int kHalf = (kRows + kScales + 127) / 128 * 128;
    static constexpr bool kWhole = RB <= 256;
    static constexpr int kSlot = kWhole ? 2 * kHalf : kHalf;
    static constexpr int kQStride = HD * 2 + (F16 ? 16 : 64);     // bytes of a query row: no bank twice
    static constexpr int kQ = NQ * CO * kQStride;
    static constexpr int kPart = CO * (HD + 2);                   // floats of a partial: O^T, then m and sum of each column
    static constexpr int kMisc = 3072;
    static constexpr int kQBytes = kQ + CO * 4 * (1 + NG) + 128;  // a warp's queries, their scales, their sums
    // warps: as many as shared memory with two slots each takes, and registers without spilling (4-bit codes for fp32
    // results: 256 ragged sequences 60.2 us with 12, 53.9 with 8; for bf16 ones 128 x 4096 tokens 169 with 12, 172 with 8)
    static constexpr int stages(int warps) { return ((kSmem - kMisc) / warps - kQBytes) / (kSlot + 16); }
    static constexpr int warps(int most) { return most <= 4 || stages(most) >= 2 ? most : warps(most - 4); }
    static constexpr int NW = warps(NT == 2 || HD == 256 || (FMT == UQ_KV_INT4 && WD == UQ_W_F32 && HD == 128) ? 8 : 12);
    static constexpr int kThreads = 32 * NW;
    static constexpr int kStages = stages(NW) > 6 ? 6 : stages(NW);
    static constexpr int kRing = kStages * kSlot;                 // per warp: ring, masks, queries, their scales, their sums
    static constexpr int kMasks = kRing, kQs = kMasks + 16 * kStages, kQScale = kQs + kQ, kQSum = kQScale + CO * 4;
    static constexpr int kWarpBytes = (kQSum + CO * NG * 4 + 127) / 128 * 128;
    static constexpr int kBytes = NW * kWarpBytes + kMisc;
    static_assert(kStages >= 2 && kPart * 4 <= kWarpBytes, "two slots, and room for a partial at the end");
    static_assert(kBytes <= 227 * 1024 && NW <= most_warps(HD), "shared memory, workspace");
};

__device__ __forceinline__ uint32_t smem_at(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
// 16 bytes; zeros where they are not there.
__device__ __forceinline__ void copy16(uint32_t dst, const void* src) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copy16_or_zero(uint32_t dst, const void* src, bool there) {
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
// D = A B + C of a 16 x 16 and a 16 x 8 matrix; F16: fp16 operands, else bf16.
template <bool F16>
__device__ __forceinline__ void mma(float d[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    if constexpr (F16)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                     : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// D = A B.
template <bool F16>
__device__ __forceinline__ void mma_new(float d[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    if constexpr (F16)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
                     : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
                     : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.0f));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
                     : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
                     : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.0f));
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
// Pairs of 16-bit floats, the low half first.
__device__ __forceinline__ uint32_t f16_pair(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
__device__ __forceinline__ float f16_low(uint32_t p) {
    float r;
    asm("{.reg .b16 l, h; mov.b32 {l, h}, %1; cvt.f32.f16 %0, l;}" : "=f"(r) : "r"(p));
    return r;
}
__device__ __forceinline__ float f16_high(uint32_t p) {
    float r;
    asm("{.reg .b16 l, h; mov.b32 {l, h}, %1; cvt.f32.f16 %0, h;}" : "=f"(r) : "r"(p));
    return r;
}
__device__ __forceinline__ uint32_t add_f16x2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("add.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
__device__ __forceinline__ uint32_t fma_f16x2(uint32_t a, uint32_t b, uint32_t c) {
    uint32_t r;
    asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(b), "r"(c));
    return r;
}
// Two int8 codes, already in the low bytes of halves whose high bytes are 0x64 and with their sign bits flipped (so
// that a half is 1024 + 128 + code): less 1152.
__device__ __forceinline__ uint32_t unbias_int8(uint32_t x) { return add_f16x2(x, 0xe480e480u); }
// Patterns that go into a logic operation next to a mask.  An operation takes one constant of 32 bits, so a pattern
// has to be in a register: as a kernel argument, which the compiler does not know (a constant costs a second operation).
struct Patterns {
    uint32_t f16_1024, bf16_128;
};
// Two int4 codes in bits 0-3 (HIGH: 4-7) of x's halves, less 8: 1024 + c - 1032, (1024 + 16 c) / 16 - 72.
template <bool HIGH>
__device__ __forceinline__ uint32_t f16_of_int4(uint32_t x, const Patterns& c) {
    return HIGH ? fma_f16x2(masked<0x00f000f0u>(x, c.f16_1024), 0x2c002c00u, 0xd480d480u)
                : add_f16x2(masked<0x000f000fu>(x, c.f16_1024), 0xe408e408u);
}
// The pair (x0, x1) as N pairs whose sums are x0, x1.  bf16: all but the last are cut off (so that no value
// overflows), the last is rounded; fp16: all are rounded.  FULL: no term of a number is 0, because that times an infinity
// of a bf16 row is NaN where the number times it is not: every rest has 2^-30 of the number added (2^-5 of the last bit).
template <bool F16, int N, bool FULL = false>
__device__ __forceinline__ void split_pair(float x0, float x1, uint32_t part[N]) {
    const float all0 = x0, all1 = x1;
#pragma unroll
    for (int i = 0; i < N - 1; ++i) {
        if (F16) {
            part[i] = f16_pair(x0, x1);
            x0 -= f16_low(part[i]);
            x1 -= f16_high(part[i]);
        } else {
            part[i] = __byte_perm(__float_as_uint(x0), __float_as_uint(x1), 0x7632);
            x0 -= bf16_low(part[i]);
            x1 -= bf16_high(part[i]);
            if (FULL) {
                x0 = fmaf(all0, 0x1p-30f, x0);
                x1 = fmaf(all1, 0x1p-30f, x1);
            }
        }
    }
    part[N - 1] = F16 ? f16_pair(x0, x1) : bf16_pair(x0, x1);
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

// A sequence: its tiles, and its positions first .. n - 1 that count.
struct Sequence {
    int b, n, first, tiles;
    template <int TOK>
    __device__ __forceinline__ void set(const AttnArgs& a, int seq) {
        b = seq;
        n = min(max(__ldg(a.seq_lens + seq), 0), a.max_tokens);
        first = a.window > 0 ? max(n - a.window, 0) : 0;
        tiles = max(1, (n - (first & ~15) + TOK - 1) / TOK);
    }
};

// Goes through a share: unit by unit (a key/value head and its query heads), the tiles of each that lie in it.
struct Walk {
    Sequence s;
    int u, at;                         // unit, and where in it the share enters (kHead places, then the tiles)
    int tile, end;                     // the part at hand
    int64_t rem, unit0;                // places left; place of the unit's start in the order of all
    template <int TOK, int kHead>
    __device__ __forceinline__ bool next(const AttnArgs& a, int units) {
        while (rem > 0) {
            if (at < 0) {              // on to the next unit
                unit0 += s.tiles + kHead;
                if (++u == units) {
                    u = 0;
                    s.set<TOK>(a, s.b + 1);
                }
                at = 0;
            }
            const int take = (int)min(rem, (int64_t)(s.tiles + kHead - at));
            tile = max(at - kHead, 0);
            end = max(at + take - kHead, 0);
            rem -= take;
            at = -1;
            if (end > tile) return true;
        }
        return false;
    }
};

// `total` places cut into `n` shares, the first total % n of them one place longer, `warps` to a block.
struct Split {
    int64_t per, more;
    int n, warps;
    __device__ __forceinline__ Split(int64_t total, int blocks, int most) {
        if (total <= 0x7fffffff) {
            const uint32_t t = (uint32_t)total;
            warps = (int)min((uint32_t)most, max((uint32_t)kMinWarps, (t + blocks - 1) / blocks));
            n = (int)min((uint32_t)(warps * blocks), t);
            per = t / (uint32_t)n;
        } else {
            warps = most;
            n = warps * blocks;
            per = total / n;
        }
        more = total - per * n;
    }
    // Where warps have few places, a block begins with a whole (sequence, head), unless the one that it would begin
    // in is long: a join lasts as long as several tiles.
    __device__ __forceinline__ bool snaps() const { return per <= kSnapPlaces; }
    __device__ __forceinline__ int64_t start(int i) const { return per * i + min((int64_t)i, more); }
    __device__ __forceinline__ int block_of(int64_t t) const {
        const int64_t big = more * (per + 1), x = t < big ? t : t - big;
        const int64_t d = t < big ? per + 1 : per;
        const int64_t i = x <= 0x7fffffff && d <= 0x7fffffff ? (int64_t)((uint32_t)x / (uint32_t)d) : x / d;
        return (int)((uint32_t)(t < big ? i : more + i) / (uint32_t)warps);
    }
};

// Where share i of n of `many` places begins.
__device__ __forceinline__ int64_t share_of(int64_t many, int i, int n) {
    return many <= 0xffffff ? (int64_t)((uint32_t)many * (uint32_t)i / (uint32_t)n) : many * i / n;
}

// A part of a (sequence, head) that a warp, or the warps of a block, have worked on.
struct Piece {
    int64_t unit0;
    int b, u, tiles;
    int w0, w1;                        // a block's: its warps
    int from_start;                    // it has the first tile
    int to_end;                        // and the last
};

// Floats of the flags, two of 64 bits a block, ahead of the partials.
__host__ __device__ constexpr int flag_floats(int blocks) { return 4 * blocks; }

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

// acc += a partial's O^T, which counts for f.
__device__ __forceinline__ void add_partial(float4& acc, const float4& v, float f) {
    acc.x = fmaf(v.x, f, acc.x);
    acc.y = fmaf(v.y, f, acc.y);
    acc.z = fmaf(v.z, f, acc.z);
    acc.w = fmaf(v.w, f, acc.w);
}

// Four channels of N partials that are all loaded before the first is used, and their sum.
template <int N>
struct Joined {
    float2 ms[N];                      // maximum and sum
    float4 v[N], acc;
    float top, sum;
    template <typename P>
    __device__ __forceinline__ void load(int i, const float* from, int col, int d) {
        ms[i] = *reinterpret_cast<const float2*>(from + P::kPart - 2 * P::CO + 2 * col);
        v[i] = *reinterpret_cast<const float4*>(from + col * (16 * P::OT) + d);
    }
    template <typename P>
    __device__ __forceinline__ void load_cg(int i, const float* from, int col, int d) {        // stored by another block
        ms[i] = __ldcg(reinterpret_cast<const float2*>(from + P::kPart - 2 * P::CO + 2 * col));
        v[i] = __ldcg(reinterpret_cast<const float4*>(from + col * (16 * P::OT) + d));
    }
    __device__ __forceinline__ void none(int i) {
        ms[i] = make_float2(-INFINITY, 0.0f);
        v[i] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    }
    __device__ __forceinline__ float low() const { return top == -INFINITY ? 0.0f : top; }
    __device__ __forceinline__ void join() {
        top = -INFINITY;
        sum = 0.0f;
        acc = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
        for (int i = 0; i < N; ++i) top = fmaxf(top, ms[i].x);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float f = exp2_fast(ms[i].x - low());
            sum = fmaf(ms[i].y, f, sum);
            add_partial(acc, v[i], f);
        }
    }
};

template <int FMT, int HD, int WD, int NT>
__global__ void __launch_bounds__(Plan<FMT, HD, WD, NT>::kThreads, 1) attn_kernel(const AttnArgs a, const int units, const int chunks, const Patterns pat) {
    using P = Plan<FMT, HD, WD, NT>;
    constexpr bool F16 = P::F16;
    constexpr int TOK = P::kTok, ST = P::kStages, MT = P::MT, OT = P::OT, RB = P::RB, W = P::W, NG = P::NG;
    constexpr int CO = P::CO, NQ = P::NQ, NP = P::NP, NW = P::NW, kHead = P::kHead;
    extern __shared__ __align__(128) uint8_t smem[];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, c = lane & 3;
    uint8_t* const own = smem + warp * P::kWarpBytes;
    const uint32_t ring = smem_at(own), masks = ring + P::kMasks, qs = ring + P::kQs;
    Piece* const pieces = reinterpret_cast<Piece*>(smem + NW * P::kWarpBytes);
    const int r = a.heads / a.c.kv_heads;
    inputs_ready();

    // --- this warp's share
    Walk walk;
    walk.rem = 0;
    int64_t total;
    {
        const int per = (a.batch + 31) / 32, b0 = min(a.batch, lane * per), b1 = min(a.batch, b0 + per);
        int64_t sum = 0;
        for (int b = b0; b < b1; ++b) {
            walk.s.set<TOK>(a, b);
            sum += walk.s.tiles + kHead;
        }
        sum *= units;
        total = sum;                                   // up to and with this lane's sequences
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
            const int64_t x = __shfl_up_sync(kFull, total, off);
            if (lane >= off) total += x;
        }
        const int64_t before = total - sum;
        total = __shfl_sync(kFull, total, 31);
        const Split split(total, gridDim.x, NW);
        if ((int)blockIdx.x * split.warps >= split.n) return;
        const Sequence held = walk.s;                  // with one sequence a lane: that one
        auto locate = [&](int64_t place) {             // in which sequence, unit, and where in it
            int64_t at = place - before;
            int b = b0;
            const bool here = at >= 0 && at < sum;
            if (per > 1 && here)
                for (;; ++b) {
                    walk.s.set<TOK>(a, b);
                    const int64_t all = (int64_t)(walk.s.tiles + kHead) * units;
                    if (at < all) break;
                    at -= all;
                }
            const int from = __ffs(__ballot_sync(kFull, here)) - 1;
            at = __shfl_sync(kFull, at, from);
            if (per > 1) {
                walk.s.set<TOK>(a, __shfl_sync(kFull, b, from));
            } else {
                walk.s.b = from;
                walk.s.n = __shfl_sync(kFull, held.n, from);
                walk.s.first = __shfl_sync(kFull, held.first, from);
                walk.s.tiles = __shfl_sync(kFull, held.tiles, from);
            }
            const int unit = walk.s.tiles + kHead;
            walk.u = at <= 0x7fffffff ? (int)((uint32_t)at / (uint32_t)unit) : (int)(at / unit);
            walk.at = (int)(at - (int64_t)walk.u * unit);
            walk.unit0 = place - walk.at;
        };
        auto bound = [&](int block) {                  // where a block begins
            const int64_t place = split.start(min(block * split.warps, split.n));
            if (!split.snaps() || place == 0 || place >= total) return place;
            locate(place);
            const int unit = walk.s.tiles + kHead;
            return walk.s.tiles > kSnapTiles * NW ? place : walk.unit0 + (2 * walk.at < unit ? 0 : unit);
        };
        int64_t begin, end;
        if (!split.snaps()) {
            begin = bound(blockIdx.x);
            end = bound(blockIdx.x + 1);
        } else {                                       // one each by the first two warps
            volatile int64_t* const bounds = reinterpret_cast<volatile int64_t*>(pieces);
            if (warp < 2) {
                const int64_t at = bound(blockIdx.x + warp);
                if (lane == 0) bounds[warp] = at;
            }
            __syncthreads();
            begin = bounds[0];
            end = bounds[1];
            __syncthreads();
        }
        const int64_t many = end - begin;
        if (many <= 0) return;
        // a place for each warp at least, so that the warps of a piece are neighbours
        const int aw = (int)min((int64_t)(split.snaps() ? NW : split.warps), many);
        const int64_t mine = share_of(many, warp, aw);
        if (warp < aw) {
            locate(begin + mine);
            walk.rem = share_of(many, warp + 1, aw) - mine;
        }
    }
    const Split split(total, gridDim.x, NW);

    // --- the ring: `load` goes ahead of `walk`
    const int pmask = (1 << a.page_shift) - 1;
    Walk load = walk;
    bool more = load.next<TOK, kHead>(a, units);
    int load_kv = more ? load.u / chunks : 0;
    // a lane copies parts of one block of 16 positions: rows tl, tl + RPI, ..., of every row the same chunk
    constexpr int LPB = P::LPB, RPI = P::RPI;
    const int lb = lane / LPB, ll = lane % LPB, tl = ll / P::CPR;
    const uint32_t lane_dst = 16 * lb * RB + chunk_at<RB>(tl, ll % P::CPR, line_swizzle<RB>(tl));
    int page = -1;                                     // of this lane's block of the next tile; -1: none
    auto find_page = [&] {
        page = -1;
        if (more) {
            const int t = (load.s.first & ~15) + load.tile * TOK + 16 * lb;
            if (t < load.s.n) {
                page = __ldg(a.table + load.s.b * a.table_stride + (t >> a.page_shift));
                if ((uint32_t)page >= (uint64_t)a.c.pages) page = -1;
            }
        }
    };
    int64_t row = 0;                                   // of this lane's block of the tile, in the pool
    uint32_t mask[2] = {0, 0};                         // positions of the tile that count
    bool whole = false, v_next = false;
    auto copy_half = [&](const void* base, const void* scales, uint32_t at) {
        const uint8_t* const from = static_cast<const uint8_t*>(base) + row * RB + ll * 16;
        const uint32_t dst = at + lane_dst;
        if (W > 0 ? page >= 0 : whole) {
#pragma unroll
            for (int i = 0; i < 16 / RPI; ++i)
                copy16((dst ^ (line_swizzle<RB>(i * RPI) << 4)) + i * RPI * RB, from + i * LPB * 16);
        } else if (W == 0) {                           // what does not count must be zero: codes get the weight 0 instead
#pragma unroll
            for (int i = 0; i < 16 / RPI; ++i) {
                const int x = 16 * lb + tl + i * RPI;
                copy16_or_zero((dst ^ (line_swizzle<RB>(i * RPI) << 4)) + i * RPI * RB, from + i * LPB * 16,
                               ((x < 32 ? mask[0] : mask[1]) >> (x & 31)) & 1);
            }
        }
        if constexpr (W > 0) {
#pragma unroll
            for (int i = 0; i < (4 * W + LPB - 1) / LPB; ++i) {
                const int id = i * LPB + ll;
                if (page >= 0 && id < 4 * W)
                    copy16(at + P::kRows + 64 * W * lb + id * 16, static_cast<const uint8_t*>(scales) + row * (4 * W) + id * 16);
            }
        }
    };
    auto issue = [&](int slot) {
        const uint32_t at = ring + slot * P::kSlot;
        auto next = [&] {
            if (++load.tile == load.end) {
                more = load.next<TOK, kHead>(a, units);
                if (more) load_kv = load.u / chunks;
            }
            find_page();
        };
        if (!P::kWhole && v_next) {
            copy_half(a.c.v, a.c.v_scale, at);
            v_next = false;
            next();
        } else if (more) {
            const int t0 = (load.s.first & ~15) + load.tile * TOK;
            row = (((int64_t)max(page, 0) * a.c.kv_heads + load_kv) << a.page_shift) + ((t0 + 16 * lb) & pmask);
            whole = __all_sync(kFull, page >= 0) && t0 >= load.s.first && t0 + TOK <= load.s.n;
            mask[0] = mask[1] = ~0u;
            if (!whole) {
#pragma unroll
                for (int h = 0; h < (TOK + 31) / 32; ++h) {
                    const int x = 32 * h + lane, p = __shfl_sync(kFull, page, x / 16 % MT * LPB);
                    mask[h] = __ballot_sync(kFull, x < TOK && t0 + x >= load.s.first && t0 + x < load.s.n && p >= 0);
                }
            }
            if (lane == 0)
                asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(masks + slot * 16), "r"(mask[0]), "r"(mask[1]), "r"((uint32_t)whole), "r"(0u));
            copy_half(a.c.k, a.c.k_scale, at);
            if (P::kWhole) {
                copy_half(a.c.v, a.c.v_scale, at + P::kHalf);
                next();
            } else {
                v_next = true;
            }
        }
        copies_commit();
    };
    // queries of a part, 8 channels a lane as they are; rows beyond the heads are zero
    constexpr int kQLoads = CO * (HD / 8) / 32;
    uint32_t q_raw[kQLoads][WD == UQ_W_F32 ? 8 : 4];
    auto load_queries = [&] {
        const int kvh = walk.u / chunks, col0 = (walk.u - kvh * chunks) * CO;
#pragma unroll
        for (int k = 0; k < kQLoads; ++k) {
            const int i = 32 * k + lane, n = i / (HD / 8), d = (i % (HD / 8)) * 8;
            uint4 w0 = make_uint4(0, 0, 0, 0), w1 = w0;
            if (n < r - col0) {
                const int64_t e = walk.s.b * a.q_batch + (kvh * r + col0 + n) * a.q_head + d;
                const uint4* const src = reinterpret_cast<const uint4*>(static_cast<const uint8_t*>(a.q) + e * (WD == UQ_W_F32 ? 4 : 2));
                w0 = __ldg(src);
                if (WD == UQ_W_F32) w1 = __ldg(src + 1);
            }
            q_raw[k][0] = w0.x; q_raw[k][1] = w0.y; q_raw[k][2] = w0.z; q_raw[k][3] = w0.w;
            if constexpr (WD == UQ_W_F32) { q_raw[k][4] = w1.x; q_raw[k][5] = w1.y; q_raw[k][6] = w1.z; q_raw[k][7] = w1.w; }
        }
    };
    // first of the 8 channels of a lane's part of Q for steps 2 s and 2 s + 1
    auto q_channel = [&](int s) {
        return FMT == UQ_KV_BF16 ? 32 * s + 8 * c : 64 * (s >> 1) + 16 * c + 8 * (s & 1);
    };
    bool part = walk.next<TOK, kHead>(a, units);
    find_page();
    if (part) load_queries();
#pragma unroll
    for (int s = 0; s < ST; ++s) issue(s);
    int slot = 0;                                      // that comes next
    auto release = [&] {                               // the slot that was read is filled again
        __syncwarp();
        issue(slot);
        slot = slot + 1 == ST ? 0 : slot + 1;
    };

    const float to_log2 = a.scale * 1.4426950408889634f;
    const uint32_t k_swz = line_swizzle<RB>(g), v_swz0 = line_swizzle<RB>(2 * c), v_swz1 = line_swizzle<RB>(2 * c + 1);
    // pieces of this warp that are not whole: 0 the share's first, begun before, 1 its last, begun here.  Their partials
    // are in this warp's shared memory (the ring is free once nothing is left to load), or in the workspace if it goes on
    enum { kNone, kShared, kWorkspace };
    int* const places = reinterpret_cast<int*>(pieces + 3 * NW + 1);
    float* const block_parts = a.work + flag_floats(gridDim.x);
    float* const early = block_parts + ((int64_t)2 * gridDim.x + blockIdx.x * NW + warp) * P::kPart;
    if (lane < 2) places[2 * warp + lane] = kNone;

    while (part) {
        const int kvh = walk.u / chunks, col0 = (walk.u - kvh * chunks) * CO;
        const int head0 = kvh * r + col0, cols = min(CO, r - col0);
        const int t_begin = walk.tile, t_end = walk.end;

        // queries to this warp's shared memory, 8 channels a lane
        __syncwarp();
#pragma unroll
        for (int k = 0; k < kQLoads; ++k) {
            const int i = 32 * k + lane, n = i / (HD / 8), d = (i % (HD / 8)) * 8;
            float x[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if (WD == UQ_W_F32) x[j] = __uint_as_float(q_raw[k][j]);
                else x[j] = (j & 1) ? bf16_high(q_raw[k][j >> 1]) : bf16_low(q_raw[k][j >> 1]);
            }
            if constexpr (F16) {                       // the largest of the head to 2^13..2^14
                uint32_t top = 0;
#pragma unroll
                for (int j = 0; j < 8; ++j) top = max(top, __float_as_uint(x[j]) & 0x7fffffffu);
#pragma unroll
                for (int off = HD / 16; off >= 1; off >>= 1) top = max(top, __shfl_xor_sync(kFull, top, off));
                const uint32_t e = max(top >> 23, 14u);
                const float up = __uint_as_float(e == 255 ? 127u << 23 : (267u - e) << 23);
                const float down = __uint_as_float(e == 255 ? 127u << 23 : (e - 13u) << 23);
#pragma unroll
                for (int j = 0; j < 8; ++j) x[j] *= up;
                // What a score is multiplied by besides its row's scale.  It comes before that scale (4 bits), or together
                // with it (8 bits): a sum (2^29 at most) times the scale alone overflows for keys from 1e33 on.
                const float factor = down * to_log2;
                if (d == 0) reinterpret_cast<float*>(own + P::kQScale)[n] = factor;
                if constexpr (FMT == UQ_KV_INT4) {     // a group's sum of the query meets its rows' minima
                    float s = ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
#pragma unroll
                    for (int off = 4; off >= 1; off >>= 1) s += __shfl_xor_sync(kFull, s, off);
                    if ((lane & 7) == 0) reinterpret_cast<float*>(own + P::kQSum)[n * NG + d / kKvGroup] = s * factor;
                }
            }
            uint32_t terms[4][NQ];
#pragma unroll
            for (int j = 0; j < 4; ++j)                // codes of 4 bits come as pairs (i, i + 4)
                split_pair<F16, NQ, !F16>(FMT == UQ_KV_INT4 ? x[j] : x[2 * j], FMT == UQ_KV_INT4 ? x[j + 4] : x[2 * j + 1], terms[j]);
#pragma unroll
            for (int q = 0; q < NQ; ++q)
                *reinterpret_cast<uint4*>(own + P::kQs + (q * CO + n) * P::kQStride + d * 2) =
                    make_uint4(terms[0][q], terms[1][q], terms[2][q], terms[3][q]);
        }
        __syncwarp();

        float m[NT][2], l[NT][2], o[OT][NT][4], bias[NG][NT][2], q_scale[NT][2], q_sum[NG][NT][2];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                m[nt][j] = -INFINITY;
                l[nt][j] = 0.0f;
                if (F16) q_scale[nt][j] = reinterpret_cast<const float*>(own + P::kQScale)[8 * nt + 2 * c + j];
#pragma unroll
                for (int k = 0; k < NG; ++k) {
                    bias[k][nt][j] = 0.0f;
                    if (FMT == UQ_KV_INT4) q_sum[k][nt][j] = reinterpret_cast<const float*>(own + P::kQSum)[(8 * nt + 2 * c + j) * NG + k];
                }
            }
#pragma unroll
        for (int i = 0; i < OT; ++i)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int j = 0; j < 4; ++j) o[i][nt][j] = 0.0f;

        for (int tile = t_begin; tile < t_end; ++tile) {
            copies_wait<ST - 1>();
            __syncwarp();
            const uint32_t at = ring + slot * P::kSlot, sk = at + P::kRows;
            const uint4 mk = lds128(masks + slot * 16);
            const bool full = mk.z;

            // scores, to base 2: rows of a tile are positions 16 mt + g and + 8
            float x[MT][NT][4];
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                // two sums: fp32 queries' first terms and the others; else, where the steps are many, even and odd ones
                constexpr int kSums = NQ > 1 || (NG == 1 && HD > 64) ? 2 : 1;
                float acc[kSums][NT][4];
                // steps 2 s and 2 s + 1 of 16 channels
                auto two = [&](int s, bool first, const uint32_t av[2][4]) {
#pragma unroll
                    for (int q = 0; q < NQ; ++q)
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) {
                            const uint4 b = lds128(qs + (q * CO + 8 * nt + g) * P::kQStride + q_channel(s) * 2);
                            float (&even)[4] = acc[q ? kSums - 1 : 0][nt], (&odd)[4] = acc[q || NQ == 1 ? kSums - 1 : 0][nt];
                            if (first && q < 2) mma_new<F16>(even, av[0][0], av[0][1], av[0][2], av[0][3], b.x, b.y);
                            else mma<F16>(even, av[0][0], av[0][1], av[0][2], av[0][3], b.x, b.y);
                            if (first && NQ == 1 && kSums == 2) mma_new<F16>(odd, av[1][0], av[1][1], av[1][2], av[1][3], b.z, b.w);
                            else mma<F16>(odd, av[1][0], av[1][1], av[1][2], av[1][3], b.z, b.w);
                        }
                };
                auto sum = [&](int nt, int e) { return kSums == 2 ? acc[0][nt][e] + acc[kSums - 1][nt][e] : acc[0][nt][e]; };
                const int t0 = 16 * mt + g, t1 = t0 + 8;
                if constexpr (FMT == UQ_KV_BF16) {
#pragma unroll
                    for (int kk = 0; kk < HD / 32; ++kk) {
                        const uint4 lo = lds128(at + chunk_at<RB>(t0, 4 * kk + c, k_swz));
                        const uint4 hi = lds128(at + chunk_at<RB>(t1, 4 * kk + c, k_swz));
                        const uint32_t av[2][4] = {{lo.x, hi.x, lo.y, hi.y}, {lo.z, hi.z, lo.w, hi.w}};
                        two(kk, kk == 0, av);
                    }
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int e = 0; e < 4; ++e) x[mt][nt][e] = sum(nt, e) * to_log2;
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
                                const uint32_t f0 = lo[s + k] ^ 0x80808080u, f1 = hi[s + k] ^ 0x80808080u;
                                av[k][0] = unbias_int8(__byte_perm(f0, 0x64646464u, 0x4140));
                                av[k][1] = unbias_int8(__byte_perm(f1, 0x64646464u, 0x4140));
                                av[k][2] = unbias_int8(__byte_perm(f0, 0x64646464u, 0x4342));
                                av[k][3] = unbias_int8(__byte_perm(f1, 0x64646464u, 0x4342));
                            }
                            two(2 * kk + s / 2, kk + s == 0, av);
                        }
                    }
                    const float s0 = __uint_as_float(lds32(sk + 4 * t0)), s1 = __uint_as_float(lds32(sk + 4 * t1));
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int e = 0; e < 4; ++e) x[mt][nt][e] = sum(nt, e) * ((e < 2 ? s0 : s1) * q_scale[nt][e & 1]);
                } else {
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                        for (int e = 0; e < 4; ++e) x[mt][nt][e] = 0.0f;
#pragma unroll
                    for (int kk = 0; kk < NG; ++kk) {
                        const uint2 lo2 = lds64(at + chunk_at<RB>(t0, 2 * kk + (c >> 1), k_swz) + (c & 1) * 8);
                        const uint2 hi2 = lds64(at + chunk_at<RB>(t1, 2 * kk + (c >> 1), k_swz) + (c & 1) * 8);
#pragma unroll
                        for (int w = 0; w < 2; ++w) {
                            const uint32_t lo = w ? lo2.y : lo2.x, hi = w ? hi2.y : hi2.x;
                            uint32_t av[2][4];
#pragma unroll
                            for (int k = 0; k < 2; ++k) {
                                av[k][0] = f16_of_int4<false>(k ? lo >> 8 : lo, pat);
                                av[k][1] = f16_of_int4<false>(k ? hi >> 8 : hi, pat);
                                av[k][2] = f16_of_int4<true>(k ? lo >> 8 : lo, pat);
                                av[k][3] = f16_of_int4<true>(k ? hi >> 8 : hi, pat);
                            }
                            two(2 * kk + w, w == 0, av);
                        }
                        // value = scale (c - 8) + (minimum + 8 scale): the second part meets the sum of the query's group
                        const uint32_t p0 = lds32(sk + 4 * (t0 * W + kk)), p1 = lds32(sk + 4 * (t1 * W + kk));
                        const float s0 = bf16_low(p0), s1 = bf16_low(p1);
                        const float z0 = fmaf(8.0f, s0, bf16_high(p0)), z1 = fmaf(8.0f, s1, bf16_high(p1));
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                x[mt][nt][e] = fmaf(sum(nt, e) * q_scale[nt][e & 1], e < 2 ? s0 : s1,
                                                    fmaf(e < 2 ? z0 : z1, q_sum[kk][nt][e & 1], x[mt][nt][e]));
                    }
                }
            }
            if (!P::kWhole) release();
            if (!full) {
#pragma unroll
                for (int mt = 0; mt < MT; ++mt)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const bool in = ((mt < 2 ? mk.x : mk.y) >> (16 * (mt & 1) + g + (e < 2 ? 0 : 8))) & 1;
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
            if (!P::kWhole) {
                copies_wait<ST - 1>();
                __syncwarp();
            }
            const uint32_t av = ring + slot * P::kSlot + (P::kWhole ? P::kHalf : 0), sv = av + P::kRows;
            if (W > 0 && !full) {                      // values that do not count get the scale (and minimum) 0
                for (int x = lane; x < TOK; x += 32)
                    if (!(((x < 32 ? mk.x : mk.y) >> (x & 31)) & 1))
#pragma unroll
                        for (int w = 0; w < W; ++w) asm volatile("st.shared.b32 [%0], %1;" ::"r"(sv + 4 * (x * W + w)), "r"(0) : "memory");
                __syncwarp();
            }
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) {
                const int ta[4] = {16 * mt + 2 * c, 16 * mt + 2 * c + 1, 16 * mt + 2 * c + 8, 16 * mt + 2 * c + 9};
#pragma unroll
                for (int kk = 0; kk < NG; ++kk) {
                    float vs[2] = {1.0f, 1.0f}, vz[2] = {0.0f, 0.0f};      // scales; int4: values of code 8
                    if constexpr (W > 0) {
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const int t = 16 * mt + g + 8 * h;
                            const uint32_t p = lds32(sv + 4 * (t * W + kk));
                            vs[h] = FMT == UQ_KV_INT8 ? __uint_as_float(p) : bf16_low(p);
                            if (FMT == UQ_KV_INT4) vz[h] = fmaf(8.0f, vs[h], bf16_high(p));
                        }
                    }
                    uint32_t b[NT][NP][2];
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) {
                        if constexpr (FMT == UQ_KV_INT4) {
#pragma unroll
                            for (int j = 0; j < 2; ++j)
                                bias[kk][nt][j] = fmaf(x[mt][nt][j], vz[0], fmaf(x[mt][nt][j + 2], vz[1], bias[kk][nt][j]));
                        }
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            uint32_t part_of[NP];
                            split_pair<false, NP, !F16>(W > 0 ? x[mt][nt][2 * h] * vs[h] : x[mt][nt][2 * h],
                                                  W > 0 ? x[mt][nt][2 * h + 1] * vs[h] : x[mt][nt][2 * h + 1], part_of);
#pragma unroll
                            for (int p = 0; p < NP; ++p) b[nt][p][h] = transposed(part_of[p]);
                        }
                    }
                    auto add = [&](int i, uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3) {
#pragma unroll
                        for (int nt = 0; nt < NT; ++nt) {
                            if constexpr (WD == UQ_W_F32) {
                                float d[4];
                                mma_new<false>(d, a0, a1, a2, a3, b[nt][NP - 1][0], b[nt][NP - 1][1]);
#pragma unroll
                                for (int p = NP - 2; p >= 0; --p) mma<false>(d, a0, a1, a2, a3, b[nt][p][0], b[nt][p][1]);
#pragma unroll
                                for (int e = 0; e < 4; ++e) o[i][nt][e] += d[e];
                            } else {
#pragma unroll
                                for (int p = 0; p < NP; ++p) mma<false>(o[i][nt], a0, a1, a2, a3, b[nt][p][0], b[nt][p][1]);
                            }
                        }
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
                        constexpr int NWD = HD >= 128 ? 4 : 2;    // words of a lane's part of a row
                        auto pair = [&](uint32_t x0, uint32_t x1, int sel) { return bf16_of_int8(__byte_perm(x0, x1, sel), pat.bf16_128); };
#pragma unroll
                        for (int jj = 0; jj < HD / (32 * NWD); ++jj) {
                            uint32_t v[4][4];
#pragma unroll
                            for (int k = 0; k < 4; ++k) {
                                const uint32_t swz = (k & 1) ? v_swz1 : v_swz0;
                                if constexpr (NWD == 4) {
                                    const uint4 w = lds128(av + chunk_at<RB>(ta[k], 8 * jj + g, swz));
                                    v[k][0] = w.x; v[k][1] = w.y; v[k][2] = w.z; v[k][3] = w.w;
                                } else {
                                    const uint2 w = lds64(av + chunk_at<RB>(ta[k], g >> 1, swz) + (g & 1) * 8);
                                    v[k][0] = w.x; v[k][1] = w.y;
                                }
                            }
#pragma unroll
                            for (int w = 0; w < NWD; ++w)
#pragma unroll
                                for (int h = 0; h < 2; ++h)
                                    add(2 * NWD * jj + 2 * w + h, pair(v[0][w], v[1][w], h ? 0x6662 : 0x4440),
                                        pair(v[0][w], v[1][w], h ? 0x7773 : 0x5551), pair(v[2][w], v[3][w], h ? 0x6662 : 0x4440),
                                        pair(v[2][w], v[3][w], h ? 0x7773 : 0x5551));
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
                                add(4 * kk + 2 * h + i, bf16_of_int4(w0 >> (8 * i), pat.bf16_128, 0x43084308u), bf16_of_int4(w0 >> (8 * i + 4), pat.bf16_128, 0x43084308u),
                                    bf16_of_int4(w1 >> (8 * i), pat.bf16_128, 0x43084308u), bf16_of_int4(w1 >> (8 * i + 4), pat.bf16_128, 0x43084308u));
                        }
                    }
                }
            }
            release();
        }

        // --- sums over the positions of all lanes
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
        const bool from_start = t_begin == 0, to_end = t_end == walk.s.tiles;
        const Piece piece{walk.unit0, walk.s.b, walk.u, walk.s.tiles, warp, warp, from_start, to_end};
        part = walk.next<TOK, kHead>(a, units);
        if (part) load_queries();
        float* to = nullptr;
        if (!(from_start && to_end)) {
            to = part ? early : reinterpret_cast<float*>(own);
            if (!part) {
                copies_wait<0>();
                __syncwarp();
            }
            if (lane == 0) {
                pieces[2 * warp + from_start] = piece;
                places[2 * warp + from_start] = part ? kWorkspace : kShared;
            }
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int col = 8 * nt + 2 * c + j;
                const float low = m[nt][j] == -INFINITY ? 0.0f : m[nt][j];
                if (to != nullptr && g == 0) *reinterpret_cast<float2*>(to + CO * HD + 2 * col) = make_float2(m[nt][j], l[nt][j]);
#pragma unroll
                for (int i = 0; i < OT; i += 2) {      // four channels from d on
                    const int d = channel_of<FMT, HD>(i, g);
                    const float z = FMT == UQ_KV_INT4 ? bias[(16 * i) / kKvGroup % NG][nt][j] : 0.0f;
                    const float4 acc = make_float4(o[i][nt][j] + z, o[i][nt][j + 2] + z, o[i + 1][nt][j] + z, o[i + 1][nt][j + 2] + z);
                    if (to != nullptr) *reinterpret_cast<float4*>(to + col * HD + d) = acc;
                    else if (col < cols) put_out<WD>(a, piece.b, head0 + col, d, acc, low, l[nt][j]);
                }
            }
    }
    copies_wait<0>();
    __syncthreads();

    // --- join the warps: runs of pieces of one (sequence, head), the first perhaps begun in an earlier block
    Piece* const runs = pieces + 2 * NW;
    int* const info = reinterpret_cast<int*>(places + 2 * NW);    // number of runs; which two go beyond the block; more on them
    if (warp == 0) {
        const bool has0 = lane < NW && places[2 * lane] != kNone, has1 = lane < NW && places[2 * lane + 1] != kNone;
        const uint32_t kept = __ballot_sync(kFull, has0 && places[2 * lane] == kWorkspace);
        const uint32_t on = __ballot_sync(kFull, has0), begin = __ballot_sync(kFull, has1);
        const uint32_t done = __ballot_sync(kFull, has0 && pieces[2 * lane].to_end);
        const int first = on ? __ffs(on) - 1 : 32;
        const bool earlier = on && (begin & ((1u << first) - 1)) == 0;
        const uint32_t behind = ~((2u << lane) - 1);               // warps after this one
        auto run = [&](int i, const Piece& p, uint32_t rest, uint32_t ends) {
            runs[i] = p;
            runs[i].w1 = ends ? __ffs(ends) - 1 : rest ? 31 - __clz(rest) : lane;
            runs[i].to_end = ends != 0;
        };
        if (lane == first && earlier) run(0, pieces[2 * lane], on, done);
        if (has1) run(earlier + __popc(begin & ~behind) - 1, pieces[2 * lane + 1], on & behind, done & behind);
        const uint32_t open = __ballot_sync(kFull, has1 && (done & behind) == 0);
        if (lane == 0) {
            info[0] = earlier + __popc(begin);
            info[9] = (int)kept;
            info[1] = earlier ? 0 : -1;
            info[2] = open ? info[0] - 1 : -1;
        }
    }
    __syncthreads();
    const int n_runs = info[0];
    const uint32_t in_work = info[9];
    auto stored = [&](int w, bool begins) -> const float* {        // warp w's partial
        return !begins && (in_work >> w & 1) ? block_parts + ((int64_t)2 * gridDim.x + blockIdx.x * NW + w) * P::kPart
                                             : reinterpret_cast<const float*>(smem + w * P::kWarpBytes);
    };
    constexpr int kOut = CO * (HD / 4);                            // a result's groups of four channels
    auto finish = [&](int i, const auto& all) {                    // the result of a run, or the block's partial
        const Piece& p = runs[i / kOut];
        const int col = i / (HD / 4) % CO, d = (i % (HD / 4)) * 4;
        if (p.from_start && p.to_end) {
            const int kvh = p.u / chunks, col0 = (p.u - kvh * chunks) * CO;
            if (col0 + col < r) put_out<WD>(a, p.b, kvh * r + col0 + col, d, all.acc, all.low(), all.sum);
        } else {
            float* const to = block_parts + (int64_t)(2 * blockIdx.x + p.from_start) * P::kPart;
            *reinterpret_cast<float4*>(to + col * HD + d) = all.acc;
            if (d == 0) *reinterpret_cast<float2*>(to + CO * HD + 2 * col) = make_float2(all.top, all.sum);
        }
    };
    // runs of few warps two at a time: their partials may be in the workspace, and loads do not pass stores
    constexpr int kFewWarps = 4;
    for (int i0 = tid; i0 < n_runs * kOut; i0 += 2 * P::kThreads) {
        Joined<kFewWarps> two[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int i = i0 + e * P::kThreads;
            if (i >= n_runs * kOut) continue;
            const Piece& p = runs[i / kOut];
            const int col = i / (HD / 4) % CO, d = (i % (HD / 4)) * 4, w0 = p.w0, many = p.w1 - w0 + 1;
            const bool begins = p.from_start;
#pragma unroll
            for (int k = 0; k < kFewWarps; ++k)
                if (many <= kFewWarps && k < many) two[e].template load<P>(k, stored(w0 + k, begins && k == 0), col, d);
                else two[e].none(k);
        }
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const int i = i0 + e * P::kThreads;
            if (i >= n_runs * kOut) continue;
            const Piece& p = runs[i / kOut];
            const int w0 = p.w0, w1 = p.w1;
            if (w1 - w0 < kFewWarps) {
                two[e].join();
                finish(i, two[e]);
            } else {
                const int col = i / (HD / 4) % CO, d = (i % (HD / 4)) * 4;
                const bool begins = p.from_start;
                Joined<NW> all;
#pragma unroll
                for (int w = 0; w < NW; ++w)
                    if (w >= w0 && w <= w1) all.template load<P>(w, stored(w, begins && w == w0), col, d);
                    else all.none(w);
                all.join();
                finish(i, all);
            }
        }
    }
    if (info[1] < 0 && info[2] < 0) return;

    // --- join the blocks.  A block that has stored its partial raises its flag and looks at the others' flags: whoever
    // sees all of them raised adds the partials, in order.  If two see that, both write the same.  The flags go down
    // again, so that a replay of this launch finds them down.
    // Somebody sees all of them.  A lane's look misses a flag only if its fence comes before the fences of all lanes of
    // that flag's block, which are all behind the raising (__threadfence is sequentially consistent, and __syncwarp
    // passes the raising on).  If every block missed one, each of these would come before the next, in a circle.
    __syncthreads();
    if (warp < 2 && info[1 + warp] >= 0) {
        const Piece& p = runs[info[1 + warp]];
        const int own0 = split.block_of(p.unit0 + kHead), own1 = split.block_of(p.unit0 + kHead + p.tiles - 1);
        volatile uint64_t* const flags = reinterpret_cast<volatile uint64_t*>(a.work);
        auto flag = [&](int o) { return flags + 2 * o + (o == own0 ? 1 : 0); };
        if (lane == 0) {
            __threadfence();                           // this block's partial before its flag
            *flag(blockIdx.x) = a.nonce;
        }
        __syncwarp();
        __threadfence();                               // its flag before the look at the others
        bool all = true;
        for (int o = own0 + lane; o <= own1; o += 32) all &= *flag(o) == a.nonce;
        all = __all_sync(kFull, all);
        __threadfence();                               // their flags before their partials
        if (all)
            for (int o = own0 + lane; o <= own1; o += 32) *flag(o) = 0;
        if (lane == 0) {
            info[3 + 3 * warp] = all;
            info[4 + 3 * warp] = own0;
            info[5 + 3 * warp] = own1;
        }
    }
    __syncthreads();
    // groups of four channels a thread has, or threads that share one; loads that are in flight at a time
    constexpr int kEach = (kOut + P::kThreads - 1) / P::kThreads, kSplits = kOut < P::kThreads ? P::kThreads / kOut : 1;
    constexpr int kFlight = kEach >= 8 ? 2 : 16 / kEach;
    float* const weights = reinterpret_cast<float*>(smem);                                   // [partial][column]
    for (int k = 0; k < 2; ++k) {
        if (info[1 + k] < 0 || !info[3 + 3 * k]) continue;
        const Piece& p = runs[info[1 + k]];
        const int own0 = info[4 + 3 * k], n = info[5 + 3 * k] - own0 + 1;
        const int kvh = p.u / chunks, col0 = (p.u - kvh * chunks) * CO, cols = min(CO, r - col0);
        float* const stats = weights + n * CO;                                               // sums, columns' maxima and sums
        float4* const sums = reinterpret_cast<float4*>(stats + n * CO + 2 * CO);
        const float* const second = block_parts + (int64_t)2 * own0 * P::kPart;              // the first block's is its second
        auto partial = [&](int i) { return second + (2 * i + (i == 0)) * P::kPart; };
        constexpr int kFew = 12;
        if (n <= kFew) {
            for (int i = tid; i < cols * (HD / 4); i += P::kThreads) {
                const int col = i / (HD / 4), d = (i % (HD / 4)) * 4;
                Joined<kFew> all;
#pragma unroll
                for (int j = 0; j < kFew; ++j)
                    if (j < n) all.template load_cg<P>(j, partial(j), col, d);
                    else all.none(j);
                all.join();
                put_out<WD>(a, p.b, kvh * r + col0 + col, d, all.acc, all.low(), all.sum);
            }
            continue;
        }
        for (int i = tid; i < n * CO; i += P::kThreads) {
            const float2 ms = __ldcg(reinterpret_cast<const float2*>(partial(i / CO) + CO * HD) + i % CO);
            weights[i] = ms.x;
            stats[i] = ms.y;
        }
        __syncthreads();
        for (int col = warp; col < CO; col += NW) {
            float top = -INFINITY, sum = 0.0f;
            for (int i = lane; i < n; i += 32) top = fmaxf(top, weights[i * CO + col]);
#pragma unroll
            for (int off = 16; off >= 1; off >>= 1) top = fmaxf(top, __shfl_xor_sync(kFull, top, off));
            const float low = top == -INFINITY ? 0.0f : top;
            for (int i = lane; i < n; i += 32) {
                const float f = exp2_fast(weights[i * CO + col] - low);
                weights[i * CO + col] = f;
                sum = fmaf(stats[i * CO + col], f, sum);
            }
            sum = warp_sum(sum);
            if (lane == 0) {
                stats[n * CO + 2 * col] = low;
                stats[n * CO + 2 * col + 1] = sum;
            }
        }
        __syncthreads();
        float4 acc[kEach];
#pragma unroll
        for (int e = 0; e < kEach; ++e) acc[e] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        if (tid < kOut * kSplits)
            for (int w0 = tid / kOut; w0 < n; w0 += kFlight * kSplits) {
                float4 v[kFlight][kEach];
#pragma unroll
                for (int j = 0; j < kFlight; ++j)
#pragma unroll
                    for (int e = 0; e < kEach; ++e) {
                        const int w = w0 + j * kSplits, o = (tid + e * P::kThreads) % kOut;
                        if (w < n) v[j][e] = __ldcg(reinterpret_cast<const float4*>(partial(w)) + o);
                    }
#pragma unroll
                for (int j = 0; j < kFlight; ++j)
#pragma unroll
                    for (int e = 0; e < kEach; ++e) {
                        const int w = w0 + j * kSplits, o = (tid + e * P::kThreads) % kOut;
                        if (w < n) add_partial(acc[e], v[j][e], weights[w * CO + o / (HD / 4)]);
                    }
            }
        if (kSplits > 1 && tid < kOut * kSplits) sums[tid] = acc[0];
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
            const int o = tid + e * P::kThreads, col = o / (HD / 4), d = (o % (HD / 4)) * 4;
            if (kSplits == 1 && o < kOut && col < cols)
                put_out<WD>(a, p.b, kvh * r + col0 + col, d, acc[e], stats[n * CO + 2 * col], stats[n * CO + 2 * col + 1]);
        }
        __syncthreads();
        if (kSplits > 1 && tid < kOut) {
            const int col = tid / (HD / 4), d = (tid % (HD / 4)) * 4;
            float4 acc = sums[tid];
#pragma unroll
            for (int s = 1; s < kSplits; ++s) {
                const float4 v = sums[s * kOut + tid];
                acc.x += v.x; acc.y += v.y; acc.z += v.z; acc.w += v.w;
            }
            if (col < cols) put_out<WD>(a, p.b, kvh * r + col0 + col, d, acc, stats[n * CO + 2 * col], stats[n * CO + 2 * col + 1]);
        }
        __syncthreads();
    }
}

// A kernel's shared memory allowed, once per device.
template <int FMT, int HD, int WD, int NT>
cudaError_t allow_smem() {
    constexpr int kDevices = 64;
    static std::atomic<bool> done[kDevices];
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess || (dev < kDevices && done[dev].load(std::memory_order_acquire))) return e;
    e = cudaFuncSetAttribute(attn_kernel<FMT, HD, WD, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                             Plan<FMT, HD, WD, NT>::kBytes);
    if (e == cudaSuccess && dev < kDevices) done[dev].store(true, std::memory_order_release);
    return e;
}

template <int FMT, int HD, int WD, int NT>
cudaError_t go(const AttnArgs& a, cudaStream_t st) {
    using P = Plan<FMT, HD, WD, NT>;
    const cudaError_t e = allow_smem<FMT, HD, WD, NT>();
    if (e != cudaSuccess) return e;
    const int r = a.heads / a.c.kv_heads, chunks = (r + P::CO - 1) / P::CO, units = a.c.kv_heads * chunks;
    // no more blocks than the table has room for tiles
    const int64_t places = ((int64_t)(a.max_tokens + P::kTok - 1) / P::kTok + P::kHead) * units;
    const int64_t most = (places + kMinWarps - 1) / kMinWarps, full = sm_count();
    const int grid = (int)(most > full / a.batch ? full : most * a.batch);
    return launch_dependent(attn_kernel<FMT, HD, WD, NT>, dim3(grid), dim3(P::kThreads), P::kBytes, st, a, units, chunks,
                            Patterns{0x64006400u, kKvBf16_128});
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
        case 128:
            if (a.dtype == UQ_W_F32) return go<FMT, 128, UQ_W_F32, 1>(a, st);
            return two ? go<FMT, 128, UQ_W_BF16, 2>(a, st) : go<FMT, 128, UQ_W_BF16, 1>(a, st);
        default: return by_type<FMT, 256, 1>(a, st);
    }
}

}  // namespace attn
}  // namespace uq
