// Attention of several new tokens of each sequence over the paged key-value
// cache on the tensor cores (see uq_api.h): chunks of prompts, trees of drafts.
//
// The new tokens of a sequence and the r query heads that share a key/value head
// are the rows of two products, with t the cached positions, kTok at a time:
//     S [128, t] = Q [128, hd] K^T      O [128, hd] += P [128, t] V,  P = exp2(S - m)
// Row = token * r + head, so that what is read of K and V serves all of them.  A block
// has one or two tiles of 128 rows (a unit).  Its warps: one copies K and plans the
// units, one copies V, one issues the products, one keeps what goes with a tile of
// positions; four turn codes into numbers; and eight for each tile of rows make the
// weights, two threads to a row that share its positions and its channels.  With two
// tiles of rows one's products run while the other's weights are made.  Plans for one
// (fp32, 4 bits in groups, 256 channels) have two buffers of scores: those of the next
// positions are made meanwhile.  A unit of up to 128 rows under a plan for two has
// neither: its scores, weights and products come one after the other.
//
// Types.  Rows of bf16: Q, K, P, V in bf16, fp32 queries as three bf16 that add up to
// them.  Codes of 8 and 4 bits become 16-bit numbers on their way into shared memory
// without a rounding: K in fp16, for 4 bits (c - 8) s with s the group's scale over a
// power of two of the row (4 x 8 bits: 11 bits), queries scaled by a power of two per
// row and head (what lies 2^-38 below the largest is lost), fp32 ones as two fp16; V in
// bf16 as c or 2 c - 15 (c - 8 is -0.5 on average: sums that meet the minima's with the
// other sign, 1.1e-5 off instead of 6e-7 after 16400 positions).  A row's scale
// multiplies its score, and its weight before the second product, for 4 bits one
// weight per group; minima meet the sums of the query's groups, and of the weights.
// Weights for bf16 results are one bf16 over bf16 rows (2^-9 of each, as much as the
// result's own rounding: 0.0021 off in all, 0.0016 with exact ones) and the sum of two
// over codes, whose scales take from the largest weight that it is 1 and exact (0.0025
// with one, 0.0017; 4 bits of 256 channels have room for one only); for fp32 results
// three (24 bits), and these add every kTok positions to an fp32 sum in registers,
// because the tensor cores' sums are cut off instead of rounded.
//
// The maximum that weights are taken relative to follows a row's largest score only
// when that is 2^8 above it: sums in tensor memory are seldom rescaled.
//
// Shares.  Tiles of all units, in order, are cut into one contiguous share per
// block; what begins or goes on in another block leaves its maxima, sums and O in
// the workspace, and a second kernel adds them in their order.
//
// Positions that some rows of a tile see and others do not have the weight 0.  Rows
// of V behind the last position become zeros, and what is not copied is an older
// number.  A number of V that is not finite still gives NaN to all rows of its tile:
// rows whose result is not finite are done again by the second kernel, one by one
// (uq_rows_plain.cuh), with what they see and nothing else.
//
// What bounds it: the chain of a tile of rows, S to weights to O and the next S, with
// two of them in a block.  128 positions take 4100 clocks, of which the weights of a
// row's 64 positions and what they wait for are 2000, the waits for each other's
// barriers 1200, the two products 1000 (both tiles': 2050, half of the time; copies
// 2200, beside them).  A prompt of 8192 tokens, 32 heads of 128, window 4096, bf16: 415 us,
// 0.99 PFLOP/s.  What cost most on the way (that prompt, in the kernel's earlier forms):
// registers that are spilled, because the shared memory leaves next to nothing of L1 and
// they come back from L2 (576 us with 200 bytes of them, 465 without); one warp for both
// copies (507 to 475).  Small calls are the chain of their loads: 10 us to the first
// results of 16 drafts, 8 more with their join.
#pragma once

#include <cuda.h>   // CUtensorMap

#include "uq_attn.cuh"
#include "uq_pipe.cuh"
#include "uq_rows_plain.cuh"
#include "uq_tc.cuh"

namespace uq {

// Tensor map of a cache's bf16 rows, boxes of `block` rows and 64 channels, or all of them, 64 after 64 (uq_gemv.cu); false
// if the driver cannot encode it.
bool kv_rows_map(const uq_kv_cache& c, void* rows, int block, bool whole, CUtensorMap* map);

namespace rows {

using attn::f16_of_int4;
using attn::f16_pair;
using attn::Patterns;
using attn::split_pair;
using attn::unbias_int8;

static __device__ unsigned int g_err = 0;

// Tiles that the start of a unit counts for.  2 / 3 / 4 / 6, us, replayed from a graph: a prompt of 8192 tokens in bf16 487 /
// 423 / 417 / 424; 8 ragged prompts over 8 bits 54.5 / 53.6 / 52.2 / 53.6, 32 ragged trees 81 / 76 / 74 / 79; 3 prompts of fp32
// 32.1 / 30.8 / 32.8 / 34.8; a tree of 16 on bf16 21.1 / 21.4 / 21.6 / 22.5, 16 trees of fp32 over 4 bits 592 / 590 / 592 / 586.
constexpr int kHead = 4;
constexpr long long kWaitClocks = 1ll << 31;   // a wait gives up after about a second
constexpr long long kTileClocks = 1 << 15;     // what a tile may take who waits for a whole unit of them (measured: 5000 at most)
constexpr float kLazy = 8.0f;          // how far (log2) a score may lie above the maximum that is used

template <int FMT, int HD, int WD>
struct Plan {
    static constexpr bool F32 = WD == UQ_W_F32, CODES = FMT != UQ_KV_BF16;
    static constexpr int RB = KvRow<FMT, HD>::kBytes, W = KvRow<FMT, HD>::kWords;
    static constexpr int QT = !F32 ? 1 : CODES ? 2 : 3;           // terms of a query
    static constexpr int PG = FMT == UQ_KV_INT4 ? HD / kKvGroup : 1;   // weights of a position
    static constexpr int PT = F32 ? 3 : CODES && PG <= 2 ? 2 : 1;      // terms of a weight
    static constexpr int MT = !F32 && HD <= 128 && PG == 1 ? 2 : 1;    // tiles of 128 rows
    static constexpr int kTok = MT == 2 && !CODES ? 128 : 64;
    static constexpr int NB = kTok / 16;                          // blocks of 16 positions, each in one page
    static constexpr bool ALIAS = MT == 2 && PG == 1;             // P where S was
    static constexpr int SB = MT == 1 ? 2 : 1;                    // buffers of S
    // columns of tensor memory
    static constexpr int kPCols = PT * PG * kTok / 2;
    static constexpr int kO = MT * SB * kTok, kP = ALIAS ? 0 : kO + MT * HD;
    static constexpr int kCols = kP + (ALIAS ? kO + MT * HD : MT * kPCols);
    static_assert(kCols <= 512 && (!ALIAS || kPCols <= kTok), "tensor memory");
    static __host__ __device__ constexpr int p_col(int m) { return ALIAS ? m * kTok : kP + m * kPCols; }
    // what rows' threads tell each other, a query's factors, maxima and sums, and what they look up seldom: what a row sees
    static constexpr int kFactors = CODES ? 128 * MT * (1 + PG) : 0, kShared = MT * 128 * (4 + 2 * (1 + PG) + 12);
    static constexpr int kX = 4 * (kFactors + kShared);
    // shared memory: Q, the ring of K and V, what goes with a tile of positions
    static constexpr int kQTerm = 128 * HD * 2, kQ = MT * QT * kQTerm;
    static constexpr int kSlot = kTok * HD * 2;
    static constexpr int KF = FMT == UQ_KV_BF16 ? 0 : FMT == UQ_KV_INT8 ? 1 : 1 + PG;      // factors of a row of K
    static constexpr int VF = FMT == UQ_KV_BF16 ? 0 : FMT == UQ_KV_INT8 ? 1 : 2 * PG;      // and of V
    static constexpr int kInfo = 4 * (KF + VF) * kTok + 128;      // bytes: factors; pages that are there
    // codes as they are kept: rows and scales of K or V of a tile, and which of its pages are there
    static constexpr int kRaw = CODES ? kTok * (RB + 4 * W) + 128 : 0;
    static constexpr int kInfos = CODES ? 4 : 8;                  // (a tile's are free again when kSlots / 2 + 2 more begin)
    static constexpr int kRoom = 227 * 1024 - 1536 - 1024 - kQ - kInfos * kInfo - kX;
    static constexpr int kSlots = CODES ? (kRoom >= 4 * kSlot + 6 * kRaw ? 4 : 3) : kRoom >= 8 * kSlot ? 8 : kRoom >= 6 * kSlot ? 6 : 4;
    static constexpr int raws(int most) { return most > 16 ? 16 : most; }
    static constexpr int kRaws = CODES ? raws((kRoom - kSlots * kSlot) / kRaw) : 0;
    static_assert(kRoom >= kSlots * kSlot && (!CODES || kRaws >= 3), "shared memory");
    static constexpr int kBytes = 1024 + kQ + kSlots * kSlot + kInfos * kInfo + kRaws * kRaw + kX;
    static_assert(kBytes + 1536 <= 227 * 1024, "shared memory, with what is not dynamic");
    // warpgroups: two for every tile of rows that make weights, codes: one that turns them into numbers, and one whose warps
    // issue, copy and look for what is not finite.  Their registers a thread (setmaxnreg; in all what the block is
    // launched with)
    static constexpr int kGroups = 2 * MT + CODES + 1, kThreads = 128 * kGroups, kAtLaunch = 65536 / kThreads / 8 * 8;
    static constexpr int kWeightRegs = MT == 2 ? (CODES ? 88 : 104) : CODES ? 184 : 216, kLoadRegs = MT == 2 ? 64 : 72, kIssueRegs = MT == 2 ? 64 : 72;
    static_assert(2 * MT * kWeightRegs + CODES * kLoadRegs + kIssueRegs <= kGroups * kAtLaunch, "registers");
    static constexpr int kPart = MT * 128 * (HD + 2);             // floats of a partial
};

// --- the order of the work

// A unit: up to MT * 128 rows of a sequence and key/value head, and the positions that any of them sees.
struct Unit {
    int b, j, kvh, groups;
    int n, c, ctx, start;              // tokens, new ones, those before them; prompts: first row of q
    int row0, rows;
    int hi_min, lo_max;                // every row sees lo_max .. hi_min
    int lo, end, lead, base, tiles;    // some row sees lo .. end - 1 (and sinks); tiles as attn::Sequence has them
};

struct Geometry {
    int r, group;                      // heads of a key/value head, rows of a unit (a power of two)
    int tok, block;                    // positions of a tile; of what is copied at once, all in one page
};

__device__ __forceinline__ void load_sequence(const RowsArgs& a, const Geometry& g, int b, Unit& u) {
    u.b = b;
    u.n = min(max(__ldg(a.seq_lens + b), 0), a.max_tokens);
    if (a.starts != nullptr) {
        const int64_t s0 = min(max((int64_t)__ldg(a.starts + b), (int64_t)0), a.tokens);
        u.start = (int)s0;
        u.c = (int)min(max((int64_t)__ldg(a.starts + b + 1) - s0, (int64_t)0), a.tokens - s0);
    } else {
        u.start = 0;
        u.c = a.counts != nullptr ? min(max(__ldg(a.counts + b), 0), a.most) : a.most;
    }
    u.ctx = u.n - u.c;
    u.groups = (int)(((int64_t)u.c * g.r + g.group - 1) >> (31 - __clz(g.group)));
}

__device__ __forceinline__ void load_group(const RowsArgs& a, const Geometry& g, int j, Unit& u) {
    u.j = j;
    u.row0 = j * g.group;
    u.rows = min(g.group, u.c * g.r - u.row0);
    int p_min, p_max;
    if (a.starts != nullptr) {
        p_min = u.ctx + u.row0 / g.r;
        p_max = u.ctx + (u.row0 + u.rows - 1) / g.r;
        u.hi_min = p_min;
        u.end = p_max + 1;
    } else {                           // depths from -1 (a draft that does not see itself) to c - 1
        p_min = u.ctx - 1;
        p_max = u.ctx + u.c - 1;
        u.hi_min = u.ctx - 1;
        u.end = u.n;
    }
    u.lo = a.window > 0 ? max(p_min - a.window + 1, 0) : 0;
    u.lo_max = a.window > 0 ? max(p_max - a.window + 1, 0) : 0;
    const int sinks = min(a.sinks, u.lo), shift = 31 - __clz(g.tok);
    u.lead = (sinks + g.tok - 1) >> shift;
    const int from = u.lo & ~(g.block - 1);
    if (u.lead * g.tok >= from) u.lead = 0;
    u.base = u.lead == 0 && sinks > 0 ? 0 : from;
    u.tiles = u.lead + max(1, (u.end - u.base + g.tok - 1) >> shift);
}

__device__ __forceinline__ int tile_start(const Unit& u, int tok, int tile) {
    return tile < u.lead ? tile * tok : u.base + (tile - u.lead) * tok;
}
// Whether every row sees all of the tile's positions (if their pages are there).
__device__ __forceinline__ bool all_seen(const RowsArgs& a, const Unit& u, int t0, int tok) {
    return t0 + tok <= u.hi_min + 1 && (t0 >= u.lo_max || t0 + tok <= a.sinks);
}

// Goes through a share, unit by unit: key/value heads of a group of rows, then the next group.
struct Walk {
    Unit u;
    int at, tile, end;                 // place in the unit where the share enters it; its tiles that lie in the share
    int64_t rem, unit0;
    __device__ __forceinline__ bool next(const RowsArgs& a, const Geometry& g) {
        while (rem > 0) {
            if (at < 0) {
                unit0 += u.tiles + kHead;
                if (++u.kvh == a.c.kv_heads) {
                    u.kvh = 0;
                    int j = u.j + 1;
                    while (j >= u.groups) {
                        if (u.b + 1 >= a.batch) {
                            rem = 0;
                            return false;
                        }
                        load_sequence(a, g, u.b + 1, u);
                        j = 0;
                    }
                    load_group(a, g, j, u);
                }
                at = 0;
            }
            const int take = (int)min(rem, (int64_t)(u.tiles + kHead - at));
            tile = max(at - kHead, 0);
            end = max(at + take - kHead, 0);
            rem -= take;
            at = -1;
            if (end > tile) return true;
        }
        return false;
    }
};

// A unit's part in the share, as the warps of a block hand it on.
struct Item {
    Unit u;
    int tile, end;
    int64_t unit0;
};
constexpr int kItems = 4;

// `total` places cut into n shares, the first total % n of them one place longer.
struct Split {
    int64_t per, more;
    int n;
    __device__ __forceinline__ void cut(int64_t total, int blocks) {
        n = (int)min((int64_t)blocks, total);
        per = n == 0 ? 0 : total <= 0x7fffffff ? (int64_t)((uint32_t)total / (uint32_t)n) : total / n;
        more = total - per * n;
    }
    __device__ __forceinline__ int64_t start(int i) const { return per * i + min((int64_t)i, more); }
    __device__ __forceinline__ int block_of(int64_t t) const {
        const int64_t big = more * (per + 1);
        return (int)(t < big ? t / (per + 1) : more + (t - big) / per);
    }
};

// Sequence and group of slot s: prompts have a slot more for every sequence than their rows fill, trees as many as the
// largest has; false: the slot has none.
__device__ __forceinline__ bool slot_of(const RowsArgs& a, const Geometry& g, int s, Unit& u) {
    int b = 0, j;
    if (a.starts != nullptr) {
        const int shift = 31 - __clz(g.group);
        auto first = [&](int i) { return ((int64_t)__ldg(a.starts + i) * g.r >> shift) + i; };
        int hi = a.batch;
        while (hi - b > 1) {
            const int mid = (b + hi) / 2;
            if ((int)first(mid) <= s) b = mid;
            else hi = mid;
        }
        j = b == 0 && a.batch == 1 ? s : s - (int)first(b);
    } else {
        const uint32_t each = (uint32_t)(((int64_t)a.most * g.r + g.group - 1) / g.group);
        b = (int)((uint32_t)s / each);
        j = s - b * (int)each;
    }
    if (b >= a.batch || j < 0) return false;
    load_sequence(a, g, b, u);
    if (j >= u.groups) return false;
    load_group(a, g, j, u);
    return true;
}

// What the second kernel has to know of a block's share: the unit that begins in it and goes on behind it, and what is to
// be done again.
struct Open {
    int last, b, row0, rows, kvh, start;                          // last: the block that ends the unit; < 0: there is none
    int odd;                                                      // whether a result of the share is not finite
    int first_b, first_j, first_kvh, first_tile, units;           // then, the units of the share
};
static_assert(sizeof(Open) <= 64, "workspace");

// --- arithmetic

__device__ __forceinline__ float2 mul2(float2 x, float2 y) {
    unsigned long long r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(reinterpret_cast<unsigned long long&>(x)), "l"(reinterpret_cast<unsigned long long&>(y)));
    return reinterpret_cast<float2&>(r);
}
__device__ __forceinline__ float2 add2(float2 x, float2 y) {
    unsigned long long r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(reinterpret_cast<unsigned long long&>(x)), "l"(reinterpret_cast<unsigned long long&>(y)));
    return reinterpret_cast<float2&>(r);
}
__device__ __forceinline__ float2 fma2(float2 x, float2 y, float2 z) {
    unsigned long long r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(reinterpret_cast<unsigned long long&>(x)),
        "l"(reinterpret_cast<unsigned long long&>(y)), "l"(reinterpret_cast<unsigned long long&>(z)));
    return reinterpret_cast<float2&>(r);
}
__device__ __forceinline__ uint32_t mul_f16x2(uint32_t x, uint32_t y) {
    uint32_t r;
    asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(x), "r"(y));
    return r;
}
// Two int4 codes c in bits 1-4 of x's halves as bf16: 2 c - 15.
__device__ __forceinline__ uint32_t odd_of_int4(uint32_t x, uint32_t bf16_128) {
    return sub_bf16x2(masked<0x001e001eu>(x, bf16_128), 0x430f430fu);
}
// Bits of the positions lo .. hi among base .. base + 31.
__device__ __forceinline__ uint32_t range_bits(int lo, int hi, int base) {
    const int l = max(lo - base, 0), h = min(hi - base, 31);
    return h < l ? 0u : (0xffffffffu >> (31 - (h - l))) << l;
}

// All of an SM's; by one warp.
__device__ __forceinline__ void take_tensor_memory(uint32_t* address) { tc::alloc(tma::smem_addr(address), 512); }

// What a row sees: positions low .. hi, sinks up to hi, and drafts (bit j: position ctx + j).
struct Sees {
    int low, hi, sinks, ctx;
    uint64_t drafts;
    __device__ __forceinline__ uint32_t word(int base) const {
        uint32_t w = range_bits(low, hi, base) | range_bits(0, min(hi, sinks - 1), base);
        const int off = ctx - base;
        if (off > -64 && off < 32) w |= (uint32_t)(off >= 0 ? drafts << off : drafts >> -off);
        return w;
    }
};

template <int FMT, int HD, int WD>
__global__ void __launch_bounds__(Plan<FMT, HD, WD>::kThreads, 1)
rows_kernel(const RowsArgs a, const int slots, const Patterns pat, const __grid_constant__ CUtensorMap k_map,
            const __grid_constant__ CUtensorMap v_map) {
    using P = Plan<FMT, HD, WD>;
    constexpr int KT = P::kTok, MT = P::MT, NB = P::NB, QT = P::QT, PT = P::PT, PG = P::PG, RB = P::RB, W = P::W;
    constexpr bool F32 = P::F32, CODES = P::CODES;
    constexpr int kLoad = 8 * MT, kIssue = kLoad + 4 * CODES;     // first warps that turn codes into numbers, and that issue
    extern __shared__ uint8_t smem_raw[];
    __shared__ unsigned long long full[P::kSlots], empty[P::kSlots], q_ready[MT], s_ready[2], p_ready[MT], pv_done[MT], info_full[P::kInfos], drain;
    __shared__ unsigned long long raw_full[P::kRaws > 0 ? P::kRaws : 1], raw_empty[P::kRaws > 0 ? P::kRaws : 1];
    __shared__ uint32_t tm_addr;
    __shared__ unsigned long long x_ready[MT];
    __shared__ int64_t sums[P::kThreads / 32];
    __shared__ Walk first;                                        // where the share begins
    __shared__ Item items[kItems];                                // its units, one after the other; an empty one ends them
    __shared__ unsigned long long item_full[kItems], item_empty[kItems];
    __shared__ Split split;
    const int tid = threadIdx.x, warp = __shfl_sync(kFull, tid >> 5, 0), lane = tid & 31;
    uint8_t* const smem = smem_raw + ((1024u - (tma::smem_addr(smem_raw) & 1023u)) & 1023u);
    const uint32_t q_at = tma::smem_addr(smem), ring = q_at + P::kQ;
    uint8_t* const infos = smem + P::kQ + P::kSlots * P::kSlot;
    uint8_t* const raws = infos + P::kInfos * P::kInfo;
    float* const x_all = reinterpret_cast<float*>(raws + P::kRaws * P::kRaw);
    const Geometry g{a.heads / a.c.kv_heads, MT * 128, KT, min(1 << a.page_shift, KT)};

    {                                  // barriers, a thread each or a few (by one thread: 1000 clocks)
        const int i = lane;
        if (warp == 0 && i < P::kSlots) {
            tma::bar_init(tma::smem_addr(&full[i]), CODES ? 4 : 1);
            tma::bar_init(tma::smem_addr(&empty[i]), 1);
        } else if (warp == 1 && i < MT) {
            tma::bar_init(tma::smem_addr(&q_ready[i]), 8);
            tma::bar_init(tma::smem_addr(&p_ready[i]), 8);
            tma::bar_init(tma::smem_addr(&x_ready[i]), 8);
            tma::bar_init(tma::smem_addr(&pv_done[i]), 1);
        } else if (warp == 2 && i < P::kInfos) {
            tma::bar_init(tma::smem_addr(&info_full[i]), CODES ? 4 : 1);
        } else if (warp == 3 && i < P::kRaws) {
            tma::bar_init(tma::smem_addr(&raw_full[i]), 1);
            tma::bar_init(tma::smem_addr(&raw_empty[i]), 4);
        } else if (warp == 4 && i < kItems) {                     // read by the warps that weigh, load, issue and copy
            tma::bar_init(tma::smem_addr(&item_full[i]), 1);
            tma::bar_init(tma::smem_addr(&item_empty[i]), 8 * MT + 2 + (CODES ? 4 : 1));
        } else if (warp == 5 && i < 3) {
            tma::bar_init(tma::smem_addr(i < 2 ? &s_ready[i] : &drain), 1);
        }
        tma::bar_init_fence();
    }
    if (!CODES)                        // what is not copied of V has the weight 0, so it must be a number
        for (int i = tid; i < P::kSlots * P::kSlot / 16; i += P::kThreads) reinterpret_cast<uint4*>(smem + P::kQ)[i] = make_uint4(0, 0, 0, 0);
    tma::fence_async_smem();
    // nothing global is touched and no tensor memory taken before the work ahead has completed (uq_bcq_tc.cu)
    inputs_ready();
    if (warp == 0) take_tensor_memory(&tm_addr);

    Open* const open = reinterpret_cast<Open*>(a.work) + blockIdx.x;
    if (tid == 0) open->odd = 0;
    // --- this block's share: places of every slot, their sums, and the slot that the share begins in
    {
        const int per = (slots + P::kThreads - 1) / P::kThreads, s0 = min(slots, per * tid), s1 = min(slots, s0 + per);
        int64_t sum = 0;
        Unit u;
        for (int s = s0; s < s1; ++s)
            if (slot_of(a, g, s, u)) sum += (int64_t)(u.tiles + kHead) * a.c.kv_heads;
        int64_t upto = sum;
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
            const int64_t x = __shfl_up_sync(kFull, upto, off);
            if (lane >= off) upto += x;
        }
        if (lane == 31) sums[warp] = upto;
        if (tid == 0) first.rem = 0;
        __syncthreads();
        int64_t total = 0;
#pragma unroll
        for (int w = 0; w < P::kThreads / 32; ++w) {
            const int64_t x = sums[w];
            if (w < warp) upto += x;
            total += x;
        }
        const int64_t before = upto - sum;
        Split cut;
        cut.cut(total, gridDim.x);
        if (tid == 0) split = cut;
        const int64_t begin = cut.start(min((int)blockIdx.x, cut.n));
        if ((int)blockIdx.x < cut.n && begin >= before && begin < upto) {
            int64_t at = begin - before;
            for (int s = s0; s < s1; ++s)
                if (per == 1 || slot_of(a, g, s, u)) {            // (one slot a thread: u is that one)
                    const int unit = u.tiles + kHead;
                    if (at < (int64_t)unit * a.c.kv_heads) {
                        u.kvh = at <= 0x7fffffff ? (int)((uint32_t)at / (uint32_t)unit) : (int)(at / unit);
                        first.u = u;
                        first.at = (int)(at - (int64_t)u.kvh * unit);
                        first.rem = cut.start(blockIdx.x + 1) - begin;
                        first.unit0 = begin - first.at;
                        break;
                    }
                    at -= (int64_t)unit * a.c.kv_heads;
                }
        }
    }
    tc::fence_before();
    __syncthreads();
    tc::fence_after();
    dependents_may_start();            // every block has its tensor memory (uq_bcq_tc.cu)
    float* const parts = a.work + (sizeof(Open) / 4) * gridDim.x + (int64_t)2 * blockIdx.x * P::kPart;
    bool alive = true;
    // every wait is bounded; who runs out leaves, and then nobody waits for long
    auto wait = [&](unsigned long long& bar, uint32_t parity, long long limit = kWaitClocks) {
        if (!__all_sync(kFull, tma::bar_wait(tma::smem_addr(&bar), parity, limit))) {
            if (lane == 0) atomicOr(&g_err, 1u);
            alive = false;
        }
        return alive;
    };
    auto arrive = [&](unsigned long long& bar) {
        __syncwarp();
        if (lane == 0) tma::bar_arrive(tma::smem_addr(&bar));
    };
    // the next unit of the share (nullptr: there is none), and the one before it is not needed any more
    uint32_t item_no = 0;
    auto next_item = [&](long long limit = kWaitClocks) -> const Item* {
        const Item& it = items[item_no % kItems];
        if (!wait(item_full[item_no % kItems], (item_no / kItems) & 1, limit) || it.end == 0) return nullptr;
        ++item_no;
        return &it;
    };
    auto item_done = [&](uint32_t i) { arrive(item_empty[i % kItems]); };
    const uint32_t tm = tm_addr;
    const int pmask = (1 << a.page_shift) - 1;
    // Lanes that have a block of the tile: its page; -1: none, or nobody sees the block.  (As it is loaded: whether the pool
    // has such a page is looked at when it is needed, a tile later, in `there`.)
    const int n_blocks = KT / g.block, block_shift = 31 - __clz(g.block) - 4;
    auto page_of = [&](const Unit& u, int t0) {
        const int t = t0 + g.block * lane;
        int page = -1;
        if (lane < n_blocks && t >= 0 && t < u.end && (t + g.block - 1 >= u.lo || t < a.sinks)) {
            page = __ldg(a.table + u.b * a.table_stride + (t >> a.page_shift));
        }
        return page;
    };
    auto there_of = [&](int page) { return __ballot_sync(kFull, (uint32_t)page < (uint64_t)a.c.pages); };
    // Which of the tile's sixteens of positions have one.
    auto sixteens = [&](uint32_t there) {
        return __ballot_sync(kFull, lane < NB && (there >> (lane >> block_shift) & 1));
    };
    const int v_block = CODES ? KT : g.block;                     // rows of V that lie in lines of 128 bytes one after the other
    auto slot_at = [&](uint32_t h) { return ring + (h % P::kSlots) * P::kSlot; };
    auto slot_free = [&](uint32_t h) { return h < (uint32_t)P::kSlots || wait(empty[h % P::kSlots], ((h / P::kSlots) & 1) ^ 1); };

    if (CODES && warp >= kLoad && warp < kIssue) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(P::kLoadRegs));
        // --- codes into numbers, and the factors that go with a tile of positions
        const int lt = tid - 32 * kLoad;
        uint32_t half = 0, tile_no = 0;                           // halves and tiles so far
        if constexpr (CODES) {
            constexpr int CPR = RB / 16, RPI = 128 / CPR, IT = KT / RPI;     // 16 bytes a thread, rows RPI apart
            static_assert(IT >= 1, "a tile has a row for every thread's chunk");
            const int r0 = lt / CPR, ch = lt % CPR;
            auto put = [&](uint32_t at, int r, int chunk, uint32_t x0, uint32_t x1, uint32_t x2, uint32_t x3) {   // 8 channels
                asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(at + (chunk >> 3) * (KT * 128) + r * 128 + (((chunk & 7) ^ (r & 7)) << 4)),
                             "r"(x0), "r"(x1), "r"(x2), "r"(x3) : "memory");
            };
            // scales of a row of K in 4 bits over a power of two: 2^8 .. 2^9 the largest
            auto up_of = [&](const uint32_t* w, float& down) {
                uint32_t e = 9;
#pragma unroll
                for (int k = 0; k < W; ++k) e = max(e, (w[k] >> 7) & 255);
                down = e == 255 ? 1.0f : __uint_as_float((e - 8) << 23);
                return e == 255 ? 1.0f : __uint_as_float((262 - e) << 23);
            };
            while (const Item* const it = alive ? next_item() : nullptr) {
                const int tiles = it->end - it->tile;
                item_done(item_no - 1);
                for (int tile = 0; tile < tiles && alive; ++tile, ++tile_no) {
                    uint8_t* const info = infos + (tile_no % P::kInfos) * P::kInfo;
                    float* const kf = reinterpret_cast<float*>(info + 128);
                    float* const vf = kf + P::KF * KT;
#pragma unroll
                    for (int v = 0; v < 2; ++v, ++half) {
                        const uint8_t* const raw = raws + (half % P::kRaws) * P::kRaw;
                        const uint32_t* const words = reinterpret_cast<const uint32_t*>(raw + KT * RB);
                        if (!wait(raw_full[half % P::kRaws], (half / P::kRaws) & 1) || !slot_free(half)) break;
                        if (v == 0 && lt == 0) *reinterpret_cast<volatile uint32_t*>(info) = *reinterpret_cast<const volatile uint32_t*>(raw + P::kRaw - 128);
                        const uint32_t at = slot_at(half);
                        if (lt < KT) {                            // factors of row lt
                            const uint32_t* const w = words + lt * W;
                            if constexpr (FMT == UQ_KV_INT8) {
                                (v ? vf : kf)[lt] = __uint_as_float(w[0]);
                            } else if (v == 0) {
                                float down;
                                up_of(w, down);
                                kf[lt] = down;
#pragma unroll
                                for (int k = 0; k < W; ++k) kf[(1 + k) * KT + lt] = fmaf(8.0f, bf16_low(w[k]), bf16_high(w[k]));
                            } else {
#pragma unroll
                                for (int k = 0; k < W; ++k) {
                                    const float s = bf16_low(w[k]);
                                    vf[k * KT + lt] = 0.5f * s;
                                    vf[(PG + k) * KT + lt] = fmaf(7.5f, s, bf16_high(w[k]));
                                }
                            }
                        }
#pragma unroll 2
                        for (int i = 0; i < IT; ++i) {
                            const int r = r0 + i * RPI;
                            const uint4 code = *reinterpret_cast<const uint4*>(raw + r * RB + ch * 16);
                            const uint32_t u[4] = {code.x, code.y, code.z, code.w};
                            if constexpr (FMT == UQ_KV_INT8) {
                                uint32_t x[8];
#pragma unroll
                                for (int k = 0; k < 4; ++k) {
                                    if (v == 0) {
                                        const uint32_t f = u[k] ^ 0x80808080u;
                                        x[2 * k] = unbias_int8(__byte_perm(f, 0x64646464u, 0x4140));
                                        x[2 * k + 1] = unbias_int8(__byte_perm(f, 0x64646464u, 0x4342));
                                    } else {
                                        x[2 * k] = bf16_of_int8(__byte_perm(u[k], 0, 0x4140), pat.bf16_128);
                                        x[2 * k + 1] = bf16_of_int8(__byte_perm(u[k], 0, 0x4342), pat.bf16_128);
                                    }
                                }
                                put(at, r, 2 * ch, x[0], x[1], x[2], x[3]);
                                put(at, r, 2 * ch + 1, x[4], x[5], x[6], x[7]);
                            } else if (v == 0) {
                                float down;
                                const float up = up_of(words + r * W, down), s = bf16_low(words[r * W + ch * 32 / kKvGroup]) * up;
                                const uint32_t ss = f16_pair(s, s);
#pragma unroll
                                for (int k = 0; k < 4; ++k)
                                    put(at, r, 4 * ch + k, mul_f16x2(f16_of_int4<false>(u[k], pat), ss), mul_f16x2(f16_of_int4<true>(u[k], pat), ss),
                                        mul_f16x2(f16_of_int4<false>(u[k] >> 8, pat), ss), mul_f16x2(f16_of_int4<true>(u[k] >> 8, pat), ss));
                            } else {
#pragma unroll
                                for (int k = 0; k < 4; ++k)
                                    put(at, r, 4 * ch + k, odd_of_int4(u[k] << 1, pat.bf16_128), odd_of_int4(u[k] >> 3, pat.bf16_128),
                                        odd_of_int4(u[k] >> 7, pat.bf16_128), odd_of_int4(u[k] >> 11, pat.bf16_128));
                            }
                        }
                        arrive(raw_empty[half % P::kRaws]);
                        if (v) arrive(info_full[tile_no % P::kInfos]);
                        tma::fence_async_smem();
                        arrive(full[half % P::kSlots]);
                    }
                }
            }
        }
    } else if (warp >= kIssue) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(P::kIssueRegs));
        if (warp == kIssue + 1 || warp == kIssue + 2) {
            // --- copies of K, and of V, tile by tile, by blocks that lie next to each other.  Rows of bf16 go where the products
            // read them, codes and scales as they are to the warps that turn them into numbers.  What has no page, or is
            // seen by nobody, is not copied.  Operands are uniform and one lane issues, as for the products: each copy
            // takes 60 to 75 clocks, and both by one warp were the longest part of a tile
            const int v = warp - (kIssue + 1);
            constexpr int kRing = CODES ? P::kRaws : P::kSlots;
            const uint32_t e = tc::elect(), raws_u = __shfl_sync(kFull, tma::smem_addr(raws), 0), ring_u = __shfl_sync(kFull, ring, 0);
            // The first of them plans too, one lane of it, with what it has to know in shared memory: with L1 all taken for
            // that, a register that is spilled comes back from L2
            uint32_t planned = 0, half = v;
            auto plan = [&]() -> const Item* {                    // the next unit of the share, for all others too
                const uint32_t i = planned++ % kItems;
                if (planned > kItems && !wait(item_empty[i], (((planned - 1) / kItems) & 1) ^ 1)) return nullptr;
                Item& it = items[i];
                if (lane == 0) {
                    const bool more = first.next(a, g);
                    if (more) {
                        it.u = first.u;
                        it.tile = first.tile;
                        it.unit0 = first.unit0;
                    }
                    it.end = more ? first.end : 0;
                }
                arrive(item_full[i]);
                return it.end > 0 ? &it : nullptr;
            };
            const Item* it = v ? next_item() : plan();
            int tile = it ? it->tile : 0, page = it ? page_of(it->u, tile_start(it->u, KT, tile)) : -1;
            for (; it && alive; half += 2) {
                const int t0 = __shfl_sync(kFull, tile_start(it->u, KT, tile), 0), mine = page, kvh = __shfl_sync(kFull, it->u.kvh, 0);
                const uint32_t there = there_of(mine);
                if (++tile == it->end) {
                    if (v) item_done(item_no - 1);
                    it = v ? next_item() : plan();
                    if (it) tile = it->tile;
                }
                if (it) page = page_of(it->u, tile_start(it->u, KT, tile));
                const int s = half % kRing;
                if (half >= (uint32_t)kRing && !wait(CODES ? raw_empty[s] : empty[s], ((half / kRing) & 1) ^ 1)) break;
                const uint32_t bar = tma::smem_addr(CODES ? &raw_full[s] : &full[s]);
                const uint32_t to = CODES ? raws_u + s * P::kRaw : ring_u + s * P::kSlot;
                if (CODES) {
                    const uint32_t all = sixteens(there);
                    if (lane == 0) *reinterpret_cast<volatile uint32_t*>(raws + s * P::kRaw + P::kRaw - 128) = all;
                }
                if (lane == 0) {
                    tma::fence_async_smem();                      // the reads of this stage come first
                    tma::bar_arrive_tx(bar, __popc(there) * g.block * (RB + 4 * W));
                }
                __syncwarp();
                for (int i = 0; i < n_blocks; ++i) {
                    const int from = __shfl_sync(kFull, mine, i), row = (t0 + g.block * i) & pmask;
                    if (!(there >> i & 1)) continue;
                    if constexpr (CODES) {
                        const int64_t at = (((int64_t)from * a.c.kv_heads + kvh) << a.page_shift) + row;
                        tc::copy(to + i * g.block * RB, static_cast<const uint8_t*>(v ? a.c.v : a.c.k) + at * RB, g.block * RB, bar, e);
                        tc::copy(to + KT * RB + i * g.block * 4 * W, static_cast<const uint8_t*>(v ? a.c.v_scale : a.c.k_scale) + at * (4 * W), g.block * 4 * W, bar, e);
                    } else if (v) {
                        tc::load_box(to + i * g.block * (HD * 2), &v_map, 0, (kvh << a.page_shift) + row, 0, from, bar, e);
                    } else {
#pragma unroll
                        for (int c = 0; c < HD / 64; ++c)
                            tc::load_box(to + c * (KT * 128) + i * g.block * 128, &k_map, 64 * c, (kvh << a.page_shift) + row, from, bar, e);
                    }
                }
                __syncwarp();
            }
            if (!alive)                                           // copies may still be on their way: they land before the block leaves
                for (uint32_t h = half > (uint32_t)kRing + v ? half - kRing - (kRing & 1) : v; h < half; h += 2) {
                    const uint32_t bar = tma::smem_addr(CODES ? &raw_full[h % kRing] : &full[h % kRing]);
                    if (!__all_sync(kFull, tma::bar_wait(bar, (h / kRing) & 1)) && lane == 0) atomicOr(&g_err, kDrainTimeoutBit);
                }
        }
        else if (!CODES && warp == kIssue + 3) {
            // --- what goes with a tile of positions; rows of V behind the last position become zeros
            uint32_t half = 0, tile_no = 0;
            const Item* it = next_item();
            if (it && lane == 0) {
                open->first_b = it->u.b;
                open->first_j = it->u.j;
                open->first_kvh = it->u.kvh;
                open->first_tile = it->tile;
            }
            int tile = it ? it->tile : 0, page = it ? page_of(it->u, tile_start(it->u, KT, tile)) : -1;
            for (; it && alive; ++tile_no, half += 2) {
                uint8_t* const info = infos + (tile_no % P::kInfos) * P::kInfo;
                const uint32_t there = sixteens(there_of(page));
                const int rows = it->u.end - tile_start(it->u, KT, tile);
                if (++tile == it->end) {
                    item_done(item_no - 1);
                    it = next_item();
                    if (it) tile = it->tile;
                }
                if (it) page = page_of(it->u, tile_start(it->u, KT, tile));
                // V's place, not K's: that one may be free, taken and free again before this tile has its info, and a phase
                // that is two behind looks like the one to come.  Its last V gone says too that nobody reads this info's place
                if (!slot_free(half + 1)) break;
                if (lane == 0) *reinterpret_cast<volatile uint32_t*>(info) = there;
                if (rows < KT) {
                    if (!wait(full[(half + 1) % P::kSlots], ((half + 1) / P::kSlots) & 1)) break;
                    constexpr int CPR = RB / 16;
                    for (int i = max(rows, 0) * CPR + lane; i < KT * CPR; i += 32) {
                        const int r = i / CPR, c = i % CPR;
                        asm volatile("st.shared.v4.b32 [%0], {%1,%1,%1,%1};" ::"r"(slot_at(half + 1) + (r & ~(v_block - 1)) * (HD * 2) + (c >> 3) * v_block * 128 +
                                                                                  (r & (v_block - 1)) * 128 + (((c & 7) ^ (r & 7)) << 4)), "r"(0) : "memory");
                    }
                    tma::fence_async_smem();
                }
                arrive(info_full[tile_no % P::kInfos]);
            }
            if (lane == 0) open->units = (int)item_no;
        }
      else if (warp == kIssue) {
        // --- the products: the whole warp, uniformly; one lane issues
        const uint32_t e = tc::elect();
        uint32_t half = 0;                                        // of the tile at hand: 2 * its number
        uint32_t units[MT] = {}, done[MT] = {}, scored = 0;       // q_ready, p_ready waits; tiles scored (one tile of rows)
        // Uniform operands, known to be (an issue takes 25 clocks then, else around 100: uq_bcq_tc.cu), so addresses and
        // counts come from one lane, and a descriptor's lower word is all that changes from one product to the next.
        const uint32_t tm_u = __shfl_sync(kFull, tm, 0), q_u = __shfl_sync(kFull, q_at, 0) >> 4, ring_u = __shfl_sync(kFull, ring, 0) >> 4;
        const int v_block_u = __shfl_sync(kFull, v_block, 0);
        const uint64_t k_desc = tc::desc128(0, 16), v_desc = tc::desc128(0, v_block_u * 128);
        auto scores = [&](int m, uint32_t h, int buf) {           // S of the tile whose K is half h
            const uint64_t q_at0 = k_desc | (q_u + m * (QT * P::kQTerm >> 4)), k_at0 = k_desc | (ring_u + (h % P::kSlots) * (P::kSlot >> 4));
            const uint32_t d = tm_u + (m * P::SB + buf) * KT;
#pragma unroll
            for (int t = QT - 1; t >= 0; --t)                     // the smallest terms first
#pragma unroll
                for (int kk = 0; kk < HD / 16; ++kk)
                    tc::mma_ss(d, q_at0 + ((t * P::kQTerm + (kk >> 2) * (128 * 128) + (kk & 3) * 32) >> 4), k_at0 + (((kk >> 2) * (KT * 128) + (kk & 3) * 32) >> 4),
                               tc::idesc128(KT, !CODES, false), t < QT - 1 || kk > 0, e);
            if (e) tc::commit(tma::smem_addr(&s_ready[MT == 2 ? m : buf]));
            __syncwarp();
        };
        auto values = [&](int m, uint32_t h, uint32_t add) {      // O += P V, V half h
            const uint64_t v_at0 = v_desc | (ring_u + (h % P::kSlots) * (P::kSlot >> 4));
            constexpr int N = PG > 1 ? kKvGroup : HD;
#pragma unroll
            for (int gi = 0; gi < PG; ++gi)
#pragma unroll
                for (int t = PT - 1; t >= 0; --t)
#pragma unroll
                    for (int kk = 0; kk < KT / 16; ++kk)
                        tc::mma(tm_u + P::kO + m * HD + gi * kKvGroup, tm_u + P::p_col(m) + (gi * PT + t) * (KT / 2) + kk * 8,
                                v_at0 + ((gi * v_block_u * 128 + ((16 * kk) & ~(v_block_u - 1)) * (HD * 2) + ((16 * kk) & (v_block_u - 1)) * 128) >> 4), tc::idesc128(N, true, true),
                                t < PT - 1 || kk > 0 ? 1u : F32 ? 0u : add, e);
            if (e) tc::commit(tma::smem_addr(&pv_done[m]));
            __syncwarp();
        };
        auto have = [&](uint32_t h) { return wait(full[h % P::kSlots], (h / P::kSlots) & 1); };
        auto release = [&](uint32_t h) {
            if (e) tc::commit(tma::smem_addr(&empty[h % P::kSlots]));
            __syncwarp();
        };
        while (const Item* const it = alive ? next_item() : nullptr) {
            const int nm = MT == 2 && __shfl_sync(kFull, it->u.rows, 0) > 128 ? 2 : 1, tiles = __shfl_sync(kFull, it->end - it->tile, 0);
            item_done(item_no - 1);
            if (!have(half)) break;
            for (int m = 0; m < nm && alive; ++m) {
                if (!wait(q_ready[m], units[m]++ & 1)) break;
                tc::fence_after();
                scores(m, half, scored & 1 & (P::SB - 1));
            }
            if (!alive) break;
            release(half);
            ++scored;
            for (int tile = 0; tile < tiles && alive; ++tile, half += 2) {
                const bool more = tile + 1 < tiles;
                if (MT == 1 && more) {                            // S of the next tile while this one's weights are made
                    if (!have(half + 2)) break;
                    tc::fence_after();
                    scores(0, half + 2, scored & 1);
                    release(half + 2);
                    ++scored;
                }
                // (what was copied has mostly been there for long: not to be waited for one by one behind the weights)
                if (!have(half + 1) || (MT == 2 && more && !have(half + 2))) break;
                for (int m = 0; m < nm && alive; ++m) {
                    if (!wait(p_ready[m], done[m]++ & 1)) break;
                    tc::fence_after();
                    values(m, half + 1, tile > 0);
                    if (m == nm - 1) release(half + 1);
                    if (MT == 2 && more) {
                        // Where P was S goes only when the product that reads it is done: one product may begin to write before
                        // another ahead of it has read its left operand in tensor memory
                        if (P::ALIAS && !wait(pv_done[m], (done[m] & 1) ^ 1)) break;
                        tc::fence_after();
                        scores(m, half + 2, 0);
                        if (m == nm - 1) release(half + 2);
                    }
                }
            }
        }
        if (!alive) {                                             // products may still run: they end before tensor memory is given back
            if (e) tc::commit(tma::smem_addr(&drain));
            __syncwarp();
            if (!__all_sync(kFull, tma::bar_wait(tma::smem_addr(&drain), 0)) && lane == 0) atomicOr(&g_err, kDrainTimeoutBit);
        }
      }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(P::kWeightRegs));
        // --- weights: two threads for a row, in two warpgroups, that share its positions (and the channels of its result)
        constexpr int KC = KT / 2, NW = KC / 32, HC = HD / 2;     // a thread's positions, by 32; its channels
        const int m_tile = warp >> 3, part = (warp >> 2) & 1, row_in = (warp & 3) * 32 + lane;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t t_o = tm + lanes + P::kO + m_tile * HD + part * HC, t_p = tm + lanes + P::p_col(m_tile) + part * (KC / 2);
        const float to_log2 = a.scale * 1.4426950408889634f;
        const float factor = CODES || to_log2 == 0.0f ? 1.0f : fabsf(to_log2);     // (scale 0: queries are 0, factor 1)
        float* const q_factors = x_all + (m_tile * 128 + row_in) * (1 + PG);
        float* const x_tops = x_all + P::kFactors + m_tile * (P::kShared / MT);      // [2][2][128], then [2][1 + PG][128]
        float* const x_sums = x_tops + 4 * 128;
        int* const x_sees = reinterpret_cast<int*>(x_sums + 2 * (1 + PG) * 128) + part * 128 + row_in;             // [6][2][128]
        uint32_t exchanged = 0;
        auto exchange = [&] {                                     // what the other warpgroup has written is there
            arrive(x_ready[m_tile]);
            return wait(x_ready[m_tile], exchanged++ & 1);
        };
        uint32_t tiles_done = 0, tile_no = 0;                     // of this tile of rows; of the block
        bool opened = false;

        // --- queries: 8 channels a lane, so that a warp reads whole lines; all loads of a unit before the first is used
        constexpr int LPR = HD / 8, RPS = 32 / LPR, NR = 16, STEPS = NR / RPS;
        uint4 raw[STEPS][F32 ? 2 : 1];
        // of this thread in the unit (again at its end: a division is less than registers that are spilled)
        struct Place {
            int token, head;
            bool real;
        };
        auto place_of = [&](const Unit& u) {
            const int in = m_tile * 128 + row_in, row = u.row0 + in, token = row / g.r;
            return Place{token, u.kvh * g.r + row - token * g.r, in < u.rows};
        };
        bool apart = false;                                       // units were passed over
        auto next_unit = [&]() -> const Item* {
            // (the unit after one that is passed over is planned when the others are through with that one)
            for (long long limit = kWaitClocks;;) {
                const Item* const it = next_item(limit);
                if (!it || m_tile * 128 < it->u.rows) return it;
                limit = kWaitClocks + (it->end - it->tile) * kTileClocks;
                tile_no += it->end - it->tile;
                apart = true;
                item_done(item_no - 1);
            }
        };
        auto load_queries = [&](const Unit& u) {
            const Place p = place_of(u);
            const int64_t at = p.real ? (a.starts != nullptr ? (int64_t)(u.start + p.token) * a.q_row : u.b * a.q_batch + p.token * a.q_row) + (int64_t)p.head * a.q_head : -1;
#pragma unroll
            for (int i = 0; i < STEPS; ++i) {
                const int64_t from = __shfl_sync(kFull, at, part * NR + i * RPS + lane / LPR);
                const uint4* const src = reinterpret_cast<const uint4*>(static_cast<const uint8_t*>(a.q) + (from + (lane % LPR) * 8) * (F32 ? 4 : 2));
                raw[i][0] = from >= 0 ? __ldg(src) : make_uint4(0, 0, 0, 0);
                if (F32) raw[i][F32 ? 1 : 0] = from >= 0 ? __ldg(src + 1) : make_uint4(0, 0, 0, 0);
            }
        };
        auto store_queries = [&] {
#pragma unroll
            for (int i = 0; i < STEPS; ++i) {
                const int r_at = (warp & 3) * 32 + part * NR + i * RPS + lane / LPR, c8 = lane % LPR;
                const uint32_t w[8] = {raw[i][0].x, raw[i][0].y, raw[i][0].z, raw[i][0].w,
                                       raw[i][F32 ? 1 : 0].x, raw[i][F32 ? 1 : 0].y, raw[i][F32 ? 1 : 0].z, raw[i][F32 ? 1 : 0].w};
                float x[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) x[k] = F32 ? __uint_as_float(w[k]) : (k & 1) ? bf16_high(w[k >> 1]) : bf16_low(w[k >> 1]);
                float up = to_log2 < 0.0f ? -1.0f : to_log2 == 0.0f ? 0.0f : 1.0f;
                if constexpr (CODES) {                            // the largest of the row to 2^13 .. 2^14
                    uint32_t most = 0;
#pragma unroll
                    for (int k = 0; k < 8; ++k) most = max(most, __float_as_uint(x[k]) & 0x7fffffffu);
#pragma unroll
                    for (int off = LPR / 2; off >= 1; off >>= 1) most = max(most, __shfl_xor_sync(kFull, most, off));
                    const uint32_t ex = max(most >> 23, 14u);
                    up = __uint_as_float(ex == 255 ? 127u << 23 : (267u - ex) << 23);
                    const float qf = __uint_as_float(ex == 255 ? 127u << 23 : (ex - 13u) << 23) * to_log2;
                    float* const f = x_all + (m_tile * 128 + r_at) * (1 + PG);
                    if (c8 == 0) f[0] = qf;
                    if constexpr (FMT == UQ_KV_INT4) {            // a group's sum of the query meets its rows' minima
                        float sum = (((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]))) * up;
#pragma unroll
                        for (int off = 4; off >= 1; off >>= 1) sum += __shfl_xor_sync(kFull, sum, off);
                        if (c8 % 8 == 0) f[1 + c8 / 8] = sum * qf;
                    }
                }
#pragma unroll
                for (int k = 0; k < 8; ++k) x[k] *= up;
                uint32_t terms[4][QT];
#pragma unroll
                for (int k = 0; k < 4; ++k) {                     // codes of 4 bits come as pairs (i, i + 4)
                    const float x0 = FMT == UQ_KV_INT4 ? x[k] : x[2 * k], x1 = FMT == UQ_KV_INT4 ? x[k + 4] : x[2 * k + 1];
                    if constexpr (QT == 1) terms[k][0] = CODES ? f16_pair(x0, x1) : bf16_pair(x0, x1);
                    else split_pair<CODES, QT, !CODES>(x0, x1, terms[k]);
                }
#pragma unroll
                for (int t = 0; t < QT; ++t)
                    asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(q_at + (m_tile * QT + t) * P::kQTerm + (r_at >> 3) * 1024 + (r_at & 7) * 128 +
                                                                              (c8 >> 3) * (128 * 128) + (((c8 & 7) ^ (r_at & 7)) << 4)),
                                 "r"(terms[0][t]), "r"(terms[1][t]), "r"(terms[2][t]), "r"(terms[3][t]) : "memory");
            }
        };

        const Item* it = next_unit();
        while (alive && it) {
            const uint32_t this_no = item_no - 1;
            const int first_tile = it->tile, end_tile = it->end;
            Unit seen_by;                                         // (what the loop over tiles needs of the unit, in registers)
            seen_by.lead = it->u.lead;
            seen_by.base = it->u.base;
            seen_by.hi_min = it->u.hi_min;
            seen_by.lo_max = it->u.lo_max;
            load_queries(it->u);
            store_queries();
            tma::fence_async_smem();
            arrive(q_ready[m_tile]);
            if (CODES && !exchange()) break;                      // the row's factors, from who loaded it
            float qf = 1.0f, qs[PG];
            if constexpr (CODES) {
                qf = q_factors[0];
#pragma unroll
                for (int k = 0; k < PG; ++k) qs[k] = FMT == UQ_KV_INT4 ? q_factors[1 + k] : 0.0f;
            }
            {
                const int ctx = it->u.ctx;
                const auto [token, head, real] = place_of(it->u);
                Sees sees{0, -1, 0, ctx, 0};
                if (real) {
                    if (a.starts != nullptr) {
                        sees.hi = ctx + token;
                        sees.low = a.window > 0 ? sees.hi - a.window + 1 : 0;
                    } else {
                        const unsigned long long* const masks = reinterpret_cast<const unsigned long long*>(a.tree) + it->u.b * a.tree_stride;
                        const uint64_t drafts = it->u.c >= 64 ? ~0ull : (1ull << it->u.c) - 1;
                        const uint64_t mine = __ldg(masks + token) & drafts;
                        const int p = ctx + __popcll(mine) - 1;
                        sees.hi = ctx - 1;
                        sees.low = a.window > 0 ? p - a.window + 1 : 0;
                        sees.drafts = mine;
                        if (a.window > 0)
                            for (uint64_t left = mine; left; left &= left - 1) {
                                const int j = __ffsll((long long)left) - 1, at = ctx + __popcll(__ldg(masks + j) & drafts) - 1;
                                if (!(at >= sees.low || at < a.sinks)) sees.drafts &= ~(1ull << j);
                            }
                        if (ctx < 0) sees.drafts = ctx <= -64 ? 0 : sees.drafts >> -ctx << -ctx;
                    }
                    sees.sinks = a.window > 0 ? a.sinks : 0;
                }
                x_sees[0] = sees.low;
                x_sees[256] = sees.hi;
                x_sees[512] = sees.sinks;
                x_sees[768] = ctx;
                x_sees[1024] = (int)(uint32_t)sees.drafts;
                x_sees[1280] = (int)(uint32_t)(sees.drafts >> 32);
            }
            __syncwarp();

            // the maximum that weights are relative to; the same, or 0
            float top = -INFINITY, base = 0.0f, sum = 0.0f;
            float acc[F32 ? HC : 1], bias[PG];
#pragma unroll
            for (int k = 0; k < (F32 ? HC : 1); ++k) acc[k] = 0.0f;
#pragma unroll
            for (int k = 0; k < PG; ++k) bias[k] = 0.0f;
            auto drained = [&] {                                  // the products of the tile before, into registers
                if constexpr (F32) {
#pragma unroll
                    for (int d = 0; d < HC; d += 16) {
                        float v[16];
                        tc::load(t_o + d, v);
#pragma unroll
                        for (int k = 0; k < 16; ++k) acc[d + k] += v[k];
                    }
                }
            };

            for (int tile = first_tile; tile < end_tile && alive; ++tile, ++tile_no, ++tiles_done) {
                const uint8_t* const info = infos + (tile_no % P::kInfos) * P::kInfo;
                const float* const kf = reinterpret_cast<const float*>(info + 128) + part * KC;
                const float* const vf = kf + P::KF * KT;
                const int t0 = tile_start(seen_by, KT, tile);
                const int buf = MT == 1 ? tile_no & 1 : 0;
                // A tile of rows that had no part in the units before knows by its scores alone how far the others are, and the
                // infos' phases repeat after two rounds: there they are looked at behind the scores.  (32 ragged trees over 8 bits
                // and the prompt of 8192, us: so 74.0 and 417, always behind 76.5 and 417, the second tile of rows always behind and the
                // first ahead 75.3 and 424.)
                if (!apart && !wait(info_full[tile_no % P::kInfos], (tile_no / P::kInfos) & 1)) break;
                if (MT == 2 ? !wait(s_ready[m_tile], tiles_done & 1) : !wait(s_ready[buf], (tile_no >> 1) & 1)) break;
                if (apart && !wait(info_full[tile_no % P::kInfos], (tile_no / P::kInfos) & 1)) break;
                apart = false;
                const uint32_t there = *reinterpret_cast<const volatile uint32_t*>(info);
                const bool mixed = !all_seen(a, seen_by, t0, KT) || there != (1u << NB) - 1;
                tc::fence_after();
                const uint32_t t_s = tm + lanes + (m_tile * P::SB + buf) * KT + part * KC;
                auto pages_of = [&](int w) { return ((there >> (2 * w)) & 1 ? 0xffffu : 0u) | ((there >> (2 * w + 1)) & 1 ? 0xffff0000u : 0u); };
                const bool before = tile > first_tile;             // there is a product of this unit's
                // scores of 32 positions, times `factor` to base 2
                auto score = [&](int w, float (&x)[32]) {
                    if constexpr (CODES) {
#pragma unroll
                        for (int k = 0; k < 32; k += 4) {
                            const float4 f = *reinterpret_cast<const float4*>(kf + 32 * w + k);
                            const float2 q2 = make_float2(qf, qf);
                            float2 s0 = mul2(make_float2(x[k], x[k + 1]), mul2(make_float2(f.x, f.y), q2));
                            float2 s1 = mul2(make_float2(x[k + 2], x[k + 3]), mul2(make_float2(f.z, f.w), q2));
                            if constexpr (FMT == UQ_KV_INT4) {
#pragma unroll
                                for (int gi = 0; gi < PG; ++gi) {
                                    const float4 z = *reinterpret_cast<const float4*>(kf + (1 + gi) * KT + 32 * w + k);
                                    const float2 x2 = make_float2(qs[gi], qs[gi]);
                                    s0 = fma2(make_float2(z.x, z.y), x2, s0);
                                    s1 = fma2(make_float2(z.z, z.w), x2, s1);
                                }
                            }
                            x[k] = s0.x; x[k + 1] = s0.y; x[k + 2] = s1.x; x[k + 3] = s1.y;
                        }
                    }
                };
                float s[NW][32], tops[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
                float2 sums2[2];
                float biases[PG];
                auto raise = [&](const float (&x)[32]) {
#pragma unroll
                    for (int k = 0; k < 32; k += 8)
#pragma unroll
                        for (int c = 0; c < 4; ++c) tops[c] = fmaxf(fmaxf(tops[c], x[k + 2 * c]), x[k + 2 * c + 1]);
                };
                auto highest = [&] { return fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3])) * factor; };
                // weights of 32 positions, relative to `base`, into tensor memory; MIXED: some rows do not see some of them
                auto weigh = [&](auto MIXED, int w, uint32_t vis) {
                    [[maybe_unused]] constexpr bool M = decltype(MIXED)::value;
                    const float2 f2 = make_float2(factor, factor), b2 = make_float2(-base, -base);
                    float (&p)[32] = s[w], extra[CODES ? PG : 1];
#pragma unroll
                    for (int k = 0; k < 32; k += 2) {
                        const float2 x = make_float2(p[k], p[k + 1]), y = CODES ? add2(x, b2) : fma2(x, f2, b2);
                        p[k] = y.x;
                        p[k + 1] = y.y;
                    }
#pragma unroll
                    for (int k = 0; k < 32; ++k) p[k] = attn::exp2_fast(p[k]);
#pragma unroll
                    for (int k = 0; k < 32; k += 2) sums2[(k >> 1) & 1] = add2(sums2[(k >> 1) & 1], make_float2(p[k], p[k + 1]));
#pragma unroll
                    for (int gi = 0; gi < PG; ++gi) {
                        uint32_t words[PT][16];
                        if (FMT == UQ_KV_INT4) extra[gi % (CODES ? PG : 1)] = 0.0f;
#pragma unroll
                        for (int k = 0; k < 32; k += 4) {
                            float2 x0 = make_float2(p[k], p[k + 1]), x1 = make_float2(p[k + 2], p[k + 3]);
                            if constexpr (CODES) {
                                if constexpr (FMT == UQ_KV_INT4) {
                                    float4 z = *reinterpret_cast<const float4*>(vf + (PG + gi) * KT + 32 * w + k);
                                    if constexpr (M) {
                                        z.x = vis >> k & 1 ? z.x : 0.0f;
                                        z.y = vis >> (k + 1) & 1 ? z.y : 0.0f;
                                        z.z = vis >> (k + 2) & 1 ? z.z : 0.0f;
                                        z.w = vis >> (k + 3) & 1 ? z.w : 0.0f;
                                    }
                                    extra[gi] = fmaf(x0.x, z.x, fmaf(x0.y, z.y, fmaf(x1.x, z.z, fmaf(x1.y, z.w, extra[gi]))));
                                }
                                const float4 f = *reinterpret_cast<const float4*>(vf + gi * KT + 32 * w + k);
                                x0 = mul2(x0, make_float2(f.x, f.y));
                                x1 = mul2(x1, make_float2(f.z, f.w));
                                if constexpr (M) {
                                    x0.x = vis >> k & 1 ? x0.x : 0.0f;
                                    x0.y = vis >> (k + 1) & 1 ? x0.y : 0.0f;
                                    x1.x = vis >> (k + 2) & 1 ? x1.x : 0.0f;
                                    x1.y = vis >> (k + 3) & 1 ? x1.y : 0.0f;
                                }
                            }
                            if constexpr (PT == 1) {
                                words[0][k / 2] = bf16_pair(x0.x, x0.y);
                                words[0][k / 2 + 1] = bf16_pair(x1.x, x1.y);
                            } else {
                                uint32_t t3[PT];
                                split_pair<false, PT, !CODES>(x0.x, x0.y, t3);
#pragma unroll
                                for (int t = 0; t < PT; ++t) words[t][k / 2] = t3[t];
                                split_pair<false, PT, !CODES>(x1.x, x1.y, t3);
#pragma unroll
                                for (int t = 0; t < PT; ++t) words[t][k / 2 + 1] = t3[t];
                            }
                        }
                        if constexpr (FMT == UQ_KV_INT4) biases[gi] += extra[gi];
#pragma unroll
                        for (int t = 0; t < PT; ++t) tc::store(t_p + (gi * PT + t) * (KT / 2) + 16 * w, words[t]);
                    }
                };
                // the maximum moves on to `most` where that is far above it; sums so far follow
                auto lift_to = [&](float most) {
                    const bool lift = most > top + kLazy || (top == -INFINITY && most > top);
                    const bool rescale = lift && top != -INFINITY;
                    const float down = rescale ? attn::exp2_fast(top - most) : 1.0f;
                    if (lift) {
                        top = most;
                        base = most;
                    }
                    const bool any = __any_sync(kFull, rescale);
                    if (before && (MT == 1 || any)) {
                        if (!wait(pv_done[m_tile], (tiles_done - 1) & 1)) return;
                        tc::fence_after();
                        drained();
                    }
                    if (any) {
                        sum *= down;
#pragma unroll
                        for (int k = 0; k < PG; ++k) bias[k] *= down;
                        if constexpr (F32) {
#pragma unroll
                            for (int k = 0; k < HC; ++k) acc[k] *= down;
                        } else if (before) {
#pragma unroll 1
                            for (int d = 0; d < HC; d += 16) {
                                float v[16];
                                tc::load(t_o + d, v);
                                uint32_t x[16];
#pragma unroll
                                for (int k = 0; k < 16; ++k) x[k] = __float_as_uint(v[k] * down);
                                tc::store(t_o + d, x);
                            }
                            tc::wait_store();
                        }
                    }
                };
                // the maximum first, then weights
                auto in_order = [&](auto MIXED) {
                    constexpr bool M = decltype(MIXED)::value;
                    uint32_t vis[NW];
                    if constexpr (M) {
                        const Sees sees{x_sees[0], x_sees[256], x_sees[512], x_sees[768], (uint32_t)x_sees[1024] | (uint64_t)(uint32_t)x_sees[1280] << 32};
#pragma unroll
                        for (int w = 0; w < NW; ++w) vis[w] = sees.word(t0 + part * KC + 32 * w) & pages_of(part * NW + w);
                    } else {
#pragma unroll
                        for (int w = 0; w < NW; ++w) vis[w] = ~0u;
                    }
#pragma unroll
                    for (int w = 0; w < NW; ++w) tc::load32(t_s + 32 * w, s[w]);
#pragma unroll
                    for (int w = 0; w < NW; ++w) {
                        if (w == 0) tc::wait_load(s[w]);
                        else tc::after_wait(s[w]);
                        score(w, s[w]);
                        if constexpr (M) {
#pragma unroll
                            for (int k = 0; k < 32; ++k) s[w][k] = vis[w] >> k & 1 ? s[w][k] : -INFINITY;
                        }
                        raise(s[w]);
                    }
                    float* const mine = x_tops + (tiles_done & 1) * 256;
                    const float most = highest();
                    mine[part * 128 + row_in] = most;
                    // the other half's scores lie where this one's weights go: read there, told here, then written
                    tc::fence_before();
                    if (!exchange()) return;
                    tc::fence_after();
                    lift_to(fmaxf(most, mine[(part ^ 1) * 128 + row_in]));
                    if (!alive) return;
                    sums2[0] = sums2[1] = make_float2(0.0f, 0.0f);
#pragma unroll
                    for (int k = 0; k < PG; ++k) biases[k] = 0.0f;
#pragma unroll
                    for (int w = 0; w < NW; ++w) weigh(MIXED, w, vis[w]);
                };
                if (mixed) in_order(std::true_type{});
                else in_order(std::false_type{});
                sum += (sums2[0].x + sums2[0].y) + (sums2[1].x + sums2[1].y);
#pragma unroll
                for (int k = 0; k < PG; ++k) bias[k] += biases[k];
                if (!alive) break;
                tc::wait_store();
                tc::fence_before();
                arrive(p_ready[m_tile]);
            }
            if (!alive) break;
            // --- the unit's results, or its part of them
            const bool from_start = first_tile == 0, to_end = end_tile == it->u.tiles, whole = from_start && to_end;
            const Unit& u = it->u;
            const auto [token, head, mine] = place_of(u);
            const int64_t out_row = a.starts != nullptr ? (int64_t)(u.start + token) : (int64_t)u.b * a.most + token;
            const int64_t lse_at = out_row * a.heads + head;
            const int64_t out_at = mine ? (a.starts != nullptr ? (int64_t)(u.start + token) * a.out_row : u.b * a.out_batch + token * a.out_row) + (int64_t)head * a.out_head : -1;
            if (from_start && !to_end) {
                opened = true;
                if (tid == 0) {
                    Open& o = *open;
                    o.last = split.block_of(it->unit0 + kHead + u.tiles - 1);
                    o.b = u.b;
                    o.row0 = u.row0;
                    o.rows = u.rows;
                    o.kvh = u.kvh;
                    o.start = u.start;
                }
            }
            item_done(this_no);                                   // (a few words of it are in registers)
            it = alive ? next_unit() : nullptr;
            x_sums[part * (1 + PG) * 128 + row_in] = sum;
#pragma unroll
            for (int k = 0; k < PG; ++k) x_sums[(part * (1 + PG) + 1 + k) * 128 + row_in] = bias[k];
            if (!exchange()) break;
            sum += x_sums[(part ^ 1) * (1 + PG) * 128 + row_in];
#pragma unroll
            for (int k = 0; k < PG; ++k) bias[k] += x_sums[((part ^ 1) * (1 + PG) + 1 + k) * 128 + row_in];
            if (!wait(pv_done[m_tile], (tiles_done - 1) & 1)) break;
            tc::fence_after();
            drained();
            if (!CODES && !(fabsf(base) < INFINITY)) sum = kKvNan;    // the product with the scale is no number
            bool odd = false;                                     // (of bf16 rows)
            const float inv = whole ? (sum == 0.0f ? 0.0f : __fdiv_rn(1.0f, sum)) : 1.0f;
            float* const to = parts + (from_start ? P::kPart : 0);
            const int in_unit = m_tile * 128 + row_in;
            // a row's results lie next to each other: through shared memory, where the queries were, a warp writes whole lines
            constexpr int RW = HC * (F32 ? 4 : 2), CPO = RW / 16, RPO = 32 / CPO;
            // (where this row's own query was: other warps may have put their next ones beside it)
            const uint32_t stage = q_at + m_tile * QT * P::kQTerm + (F32 ? part * P::kQTerm : 0);
            auto staged = [&](int r, int c) {
                const int chunk = c + (F32 ? 0 : part * (HC / 8));
                return stage + (chunk >> 3) * (128 * 128) + (r >> 3) * 1024 + (r & 7) * 128 + (((chunk & 7) ^ (r & 7)) << 4);
            };
            auto keep = [&](int chunk, uint32_t x0, uint32_t x1, uint32_t x2, uint32_t x3) {
                asm volatile("st.shared.v4.b32 [%0], {%1,%2,%3,%4};" ::"r"(staged(row_in, chunk)), "r"(x0), "r"(x1), "r"(x2), "r"(x3) : "memory");
            };
#pragma unroll
            for (int d = 0; d < HC; d += 32) {
                float v[32];
                if constexpr (F32) {
#pragma unroll
                    for (int k = 0; k < 32; ++k) v[k] = acc[d + k];
                } else {
                    tc::load32(t_o + d, v);
                    tc::wait_load(v);
                }
                if constexpr (FMT == UQ_KV_INT4) {                // pairs (i, i + 4) of every 8 channels, and the minima
                    float x[32], z = bias[0];
#pragma unroll
                    for (int k = 1; k < PG; ++k) z = (part * HC + d) / kKvGroup == k ? bias[k] : z;
#pragma unroll
                    for (int k = 0; k < 32; ++k) x[(k & ~7) + ((k & 7) >> 1) + 4 * (k & 1)] = v[k] + z;
#pragma unroll
                    for (int k = 0; k < 32; ++k) v[k] = x[k];
                }
                if (!CODES) {
#pragma unroll
                    for (int k = 0; k < 32; ++k) odd |= !(fabsf(v[k] * inv) < INFINITY);
                }
                if (!whole) {
                    if (mine) {
#pragma unroll
                        for (int k = 0; k < 32; ++k) to[(part * HC + d + k) * (MT * 128) + in_unit] = v[k];
                    }
                } else if constexpr (F32) {
#pragma unroll
                    for (int k = 0; k < 8; ++k)
                        keep(d / 4 + k, __float_as_uint(v[4 * k] * inv), __float_as_uint(v[4 * k + 1] * inv), __float_as_uint(v[4 * k + 2] * inv), __float_as_uint(v[4 * k + 3] * inv));
                } else {
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        keep(d / 8 + k, bf16_pair(v[8 * k] * inv, v[8 * k + 1] * inv), bf16_pair(v[8 * k + 2] * inv, v[8 * k + 3] * inv),
                             bf16_pair(v[8 * k + 4] * inv, v[8 * k + 5] * inv), bf16_pair(v[8 * k + 6] * inv, v[8 * k + 7] * inv));
                }
            }
            if (whole) {
                __syncwarp();
#pragma unroll 4
                for (int i = 0; i < 32 / RPO; ++i) {
                    const int r_at = i * RPO + lane / CPO, chunk = lane % CPO;
                    const int64_t at = __shfl_sync(kFull, out_at, r_at);
                    const uint4 v = attn::lds128(staged((warp & 3) * 32 + r_at, chunk));
                    if (at >= 0) *reinterpret_cast<uint4*>(static_cast<uint8_t*>(a.out) + (at + part * HC) * (F32 ? 4 : 2) + chunk * 16) = v;
                }
            }
            if (whole && mine && odd) open->odd = 1;
            if (mine && part == 0) {
                if (!whole) {
                    to[HD * (MT * 128) + in_unit] = top;
                    to[(HD + 1) * (MT * 128) + in_unit] = sum;
                } else if (a.lse != nullptr) {
                    a.lse[lse_at] = sum == 0.0f ? -INFINITY : (base + log2f(sum)) * 0.6931471805599453f;
                }
            }
            __syncwarp();
            if (it && !exchange()) break;            // nobody reads what the next queries overwrite
        }
        if (tid == 0 && !opened) open->last = -1;
    }
    tc::fence_before();
    __syncthreads();
    if (warp == 0) tc::dealloc(tm, 512);
}

// Adds up the parts of the units that lie in several blocks: block (i, d) those of the unit that begins in share i and
// goes on, channels 32 d .. 32 d + 31; a thread has 8 channels of a row, and loads several parts at a time.
constexpr int kJoinThreads = 256;
// A number of a bf16 row of V that is not finite gives NaN to all rows of a tile, those too whose weight is 0 because
// they do not see it.  So rows whose result is not finite are done again one by one, with what they see and nothing else,
// and what is not finite takes its value from that.  A unit belongs to the share that it begins in; `own`: all of them,
// `open`: the last, which goes on behind it.  Block (i, d) has channels 32 d .. 32 d + 31, behind its sums of parts.
template <int FMT, int HD, int WD>
__device__ __noinline__ void again(const RowsArgs& a, const Open& o, bool own, bool open) {
    using P = Plan<FMT, HD, WD>;
    __shared__ float qs[kJoinThreads / 32][HD];
    const Geometry g{a.heads / a.c.kv_heads, P::MT * 128, P::kTok, min(1 << a.page_shift, P::kTok)};
    Unit u;
    load_sequence(a, g, o.first_b, u);
    load_group(a, g, o.first_j, u);
    u.kvh = o.first_kvh;
    for (int i = 0; i < o.units; ++i) {
        const bool begins = i > 0 || o.first_tile == 0, last = i == o.units - 1 && o.last >= 0;
        if (begins && (last ? open : own))
            for (int at = threadIdx.x >> 5; at < u.rows; at += kJoinThreads / 32) {
                const int row = u.row0 + at, token = row / g.r, head = u.kvh * g.r + row - token * g.r;
                const bool prompt = a.starts != nullptr;
                const int64_t out = (prompt ? (int64_t)(u.start + token) * a.out_row : u.b * a.out_batch + token * a.out_row) + (int64_t)head * a.out_head +
                                    32 * blockIdx.y + (threadIdx.x & 31);
                const float x = WD == UQ_W_F32 ? static_cast<const float*>(a.out)[out] : __uint_as_float((uint32_t)static_cast<const uint16_t*>(a.out)[out] << 16);
                if (__all_sync(kFull, finite(x))) continue;
                plain::attend<FMT, HD, WD>(a, u.b, token, u.c, head,
                                           prompt ? (int64_t)(u.start + token) * a.q_row : u.b * a.q_batch + token * a.q_row,
                                           prompt ? (int64_t)(u.start + token) * a.out_row : u.b * a.out_batch + token * a.out_row, 0,
                                           qs[threadIdx.x >> 5], 32 * blockIdx.y);
                __syncwarp();
            }
        if (++u.kvh < a.c.kv_heads) continue;
        u.kvh = 0;
        int j = u.j + 1;
        while (j >= u.groups) {
            if (u.b + 1 >= a.batch) return;
            load_sequence(a, g, u.b + 1, u);
            j = 0;
        }
        load_group(a, g, j, u);
    }
}

template <int FMT, int HD, int WD>
__global__ void __launch_bounds__(kJoinThreads) join_kernel(const RowsArgs a, const int shares) {
    using P = Plan<FMT, HD, WD>;
    constexpr int R = P::MT * 128, kAtOnce = 8;
    inputs_ready();
    const Open* const opens = reinterpret_cast<const Open*>(a.work);
    const Open& o = opens[blockIdx.x];                            // (rows and last of no meaning where last < 0)
    const bool own = FMT == UQ_KV_BF16 && o.odd;
    if (o.last < 0 && !own) return;
    bool odd = false;
    const float* const parts = a.work + (sizeof(Open) / 4) * shares;
    const int first = blockIdx.x, r = a.heads / a.c.kv_heads;
    for (int item = threadIdx.x; o.last >= 0 && item < 4 * ((o.rows + 31) & ~31); item += kJoinThreads) {
        // 32 rows next to each other, then the next 8 channels of them
        const int row = (item >> 7) * 32 + (item & 31), d0 = 32 * blockIdx.y + 8 * ((item >> 5) & 3);
        if (row >= o.rows) continue;
        auto part = [&](int i) { return parts + (int64_t)(2 * i + (i == first)) * P::kPart + row; };
        float top = -INFINITY, sum = 0.0f, acc[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) acc[k] = 0.0f;
        for (int i0 = first; i0 <= o.last; i0 += kAtOnce) {
            float m[kAtOnce], l[kAtOnce], v[kAtOnce][8];
#pragma unroll
            for (int j = 0; j < kAtOnce; ++j) {
                const bool in = i0 + j <= o.last;
                const float* const p = part(in ? i0 + j : i0);
                m[j] = in ? p[HD * R] : -INFINITY;
                l[j] = in ? p[(HD + 1) * R] : 0.0f;
#pragma unroll
                for (int k = 0; k < 8; ++k) v[j][k] = in ? p[(d0 + k) * R] : 0.0f;
            }
            float most = top;
#pragma unroll
            for (int j = 0; j < kAtOnce; ++j) most = fmaxf(most, m[j]);
            const float base = most == -INFINITY ? 0.0f : most, f0 = attn::exp2_fast(top - base);
            if (i0 > first) {
                sum *= f0;
#pragma unroll
                for (int k = 0; k < 8; ++k) acc[k] *= f0;
            }
            top = most;
#pragma unroll
            for (int j = 0; j < kAtOnce; ++j) {
                if (i0 + j > o.last) continue;
                const float f = attn::exp2_fast(m[j] - base);
                sum = fmaf(l[j], f, sum);
#pragma unroll
                for (int k = 0; k < 8; ++k) acc[k] = fmaf(v[j][k], f, acc[k]);
            }
        }
        const float base = top == -INFINITY ? 0.0f : top;
        const int at = o.row0 + row, token = at / r, head = o.kvh * r + at - token * r;
        const float inv = sum == 0.0f ? 0.0f : __fdiv_rn(1.0f, sum);
        if (FMT == UQ_KV_BF16) {
#pragma unroll
            for (int k = 0; k < 8; ++k) odd |= !finite(acc[k] * inv);
        }
        const int64_t to = (a.starts != nullptr ? (int64_t)(o.start + token) * a.out_row : o.b * a.out_batch + token * a.out_row) + (int64_t)head * a.out_head + d0;
        if constexpr (P::F32) {
            float4* const dst = reinterpret_cast<float4*>(static_cast<float*>(a.out) + to);
            dst[0] = make_float4(acc[0] * inv, acc[1] * inv, acc[2] * inv, acc[3] * inv);
            dst[1] = make_float4(acc[4] * inv, acc[5] * inv, acc[6] * inv, acc[7] * inv);
        } else {
            *reinterpret_cast<uint4*>(static_cast<uint16_t*>(a.out) + to) =
                make_uint4(bf16_pair(acc[0] * inv, acc[1] * inv), bf16_pair(acc[2] * inv, acc[3] * inv), bf16_pair(acc[4] * inv, acc[5] * inv),
                           bf16_pair(acc[6] * inv, acc[7] * inv));
        }
        if (a.lse != nullptr && d0 == 0) {
            const int64_t out_row = a.starts != nullptr ? (int64_t)(o.start + token) : (int64_t)o.b * a.most + token;
            a.lse[out_row * a.heads + head] = sum == 0.0f ? -INFINITY : (base + log2f(sum)) * 0.6931471805599453f;
        }
    }
    odd = __syncthreads_or(odd);
    if (own || odd) again<FMT, HD, WD>(a, o, own, odd);
}

static cudaError_t error(bool clear, unsigned int* flag) {
    unsigned int v = 0;
    cudaError_t e = cudaMemcpyFromSymbol(&v, g_err, sizeof(v));
    if (e != cudaSuccess) return e;
    *flag = v;
    if (clear && v) {
        const unsigned int z = 0;
        e = cudaMemcpyToSymbol(g_err, &z, sizeof(z));
    }
    return e;
}

// A kernel's shared memory allowed, once per device.
template <int FMT, int HD, int WD>
cudaError_t allow_smem() {
    static std::atomic<bool> done[kMaxDevices];
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess || (dev < kMaxDevices && done[dev].load(std::memory_order_acquire))) return e;
    e = cudaFuncSetAttribute(rows_kernel<FMT, HD, WD>, cudaFuncAttributeMaxDynamicSharedMemorySize, Plan<FMT, HD, WD>::kBytes);
    if (e == cudaSuccess && dev < kMaxDevices) done[dev].store(true, std::memory_order_release);
    return e;
}

template <int FMT, int HD, int WD>
cudaError_t go(const RowsArgs& a, cudaStream_t st) {
    using P = Plan<FMT, HD, WD>;
    cudaError_t e = allow_smem<FMT, HD, WD>();
    if (e != cudaSuccess) return e;
    const int r = a.heads / a.c.kv_heads, group = P::MT * 128;
    const int slots = (int)(a.starts != nullptr ? a.tokens * r / group + a.batch
                                              : (int64_t)a.batch * (((int64_t)a.most * r + group - 1) / group));
    const int grid = sm_count();
    CUtensorMap k_map = {}, v_map = {};
    const int block = a.c.page_size < P::kTok ? a.c.page_size : P::kTok;
    if (FMT == UQ_KV_BF16 && !(kv_rows_map(a.c, a.c.k, block, false, &k_map) && kv_rows_map(a.c, a.c.v, block, true, &v_map))) return cudaErrorNotSupported;
    e = launch_dependent(rows_kernel<FMT, HD, WD>, dim3(grid), dim3(P::kThreads), P::kBytes, st, a, slots, Patterns{0x64006400u, kKvBf16_128}, k_map, v_map);
    if (e != cudaSuccess) return e;
    return launch_dependent(join_kernel<FMT, HD, WD>, dim3(grid, HD / 32), dim3(kJoinThreads), 0, st, a, grid);
}

// (fp32 results of 256 channels have no room for their sums in a thread's registers: uq_attn_rows.cu.)
template <int FMT>
cudaError_t by_head(const RowsArgs& a, cudaStream_t st) {
    const bool f32 = a.dtype == UQ_W_F32;
    switch (a.c.head_dim) {
        case 64: return f32 ? go<FMT, 64, UQ_W_F32>(a, st) : go<FMT, 64, UQ_W_BF16>(a, st);
        case 128: return f32 ? go<FMT, 128, UQ_W_F32>(a, st) : go<FMT, 128, UQ_W_BF16>(a, st);
        default: return go<FMT, 256, UQ_W_BF16>(a, st);
    }
}

}  // namespace rows
}  // namespace uq
