// C-ABI front end: argument validation, error reporting, dispatch to the
// kernel launchers.  Nothing here allocates device memory or keeps a
// pointer beyond the call.
#include <algorithm>
#include <cstdarg>
#include <cstdio>
#include <cstring>
#include <cstdint>
#include <utility>
#include <cmath>

#include "uq_attn.h"
#include "uq_launch.h"

namespace {

thread_local char g_err[512] = "";

uq_status fail(uq_status st, const char* fmt, ...) {
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(g_err, sizeof(g_err), fmt, ap);
    va_end(ap);
    return st;
}

uq_status ok() {
    g_err[0] = '\0';
    return UQ_OK;
}

constexpr int64_t kMaxIn = int64_t(1) << 24;   // row lengths whose 32-bit per-row offsets stay exact

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// Checks shape, q, g, W dtype.  Returns UQ_OK or an error status.
uq_status check_shape(int64_t out, int64_t in, int q, int g, int wdtype) {
    if (q < 1 || q > 4) return fail(UQ_ERR_UNSUPPORTED, "q=%d: bit-widths 1..4 are supported", q);
    if (out < 1 || in < 1) return fail(UQ_ERR_ARG, "empty matrix: out=%lld in=%lld", (long long)out, (long long)in);
    if (out > 0x7fffffffLL) return fail(UQ_ERR_ARG, "out=%lld exceeds 2^31-1 rows", (long long)out);
    if (g < 32 || g % 32 != 0) return fail(UQ_ERR_ARG, "g=%d must be a positive multiple of 32", g);
    if (in % g != 0) return fail(UQ_ERR_ARG, "in=%lld is not a multiple of g=%d", (long long)in, g);
    if (!(g == 32 || g == 64 || g % 128 == 0))
        return fail(UQ_ERR_UNSUPPORTED, "g=%d: supported group sizes are 32, 64 and multiples of 128", g);
    if (in > kMaxIn) return fail(UQ_ERR_UNSUPPORTED, "in=%lld exceeds %lld", (long long)in, (long long)kMaxIn);
    if (wdtype != UQ_W_F32 && wdtype != UQ_W_BF16) return fail(UQ_ERR_ARG, "unknown weight dtype %d", wdtype);
    return UQ_OK;
}

uq_status check_ptr(const void* p, const char* name) {
    if (p == nullptr) return fail(UQ_ERR_ARG, "%s is NULL", name);
    if (!aligned16(p)) return fail(UQ_ERR_ALIGN, "%s=%p is not 16-byte aligned", name, p);
    return UQ_OK;
}

#define UQ_TRY(expr)                      \
    do {                                  \
        uq_status _s = (expr);            \
        if (_s != UQ_OK) return _s;       \
    } while (0)

uq_status cuda_status(cudaError_t e, const char* what) {
    if (e != cudaSuccess) return fail(UQ_ERR_CUDA, "%s: %s", what, cudaGetErrorString(e));
    return ok();
}

// The product cuts the columns into tiles of 512; a row's groups must either
// tile a column tile exactly (g divides 512) or be made of whole tiles (512
// divides g), so that every group boundary falls on a lane boundary the
// kernels know at compile time.
uq_status check_gemv_group(int g) {
    if (512 % g != 0 && g % 512 != 0)
        return fail(UQ_ERR_UNSUPPORTED,
                    "g=%d: the BCQ product needs g to divide 512 or to be a multiple of 512 (32, 64, 128, 256, "
                    "512, 1024, ...)",
                    g);
    return UQ_OK;
}

// The key-value cache's description.
uq_status check_kv(const uq_kv_cache& c) {
    if (c.format != UQ_KV_BF16 && c.format != UQ_KV_INT8 && c.format != UQ_KV_INT4)
        return fail(UQ_ERR_ARG, "unknown cache format %d", (int)c.format);
    if (c.pages < 1 || c.pages > 0x7fffffffLL)
        return fail(UQ_ERR_ARG, "cache.pages=%lld must be in 1..2^31-1", (long long)c.pages);
    if (c.kv_heads < 1 || c.kv_heads > 4096) return fail(UQ_ERR_ARG, "cache.kv_heads=%d must be in 1..4096", c.kv_heads);
    if (c.page_size < 16 || c.page_size > 256 || (c.page_size & (c.page_size - 1)) != 0)
        return fail(UQ_ERR_UNSUPPORTED, "cache.page_size=%d: powers of two from 16 to 256 are supported", c.page_size);
    if (c.head_dim != 64 && c.head_dim != 128 && c.head_dim != 256)
        return fail(UQ_ERR_UNSUPPORTED, "cache.head_dim=%d: 64, 128 and 256 are supported", c.head_dim);
    UQ_TRY(check_ptr(c.k, "cache.k"));
    UQ_TRY(check_ptr(c.v, "cache.v"));
    if (c.format != UQ_KV_BF16) {
        UQ_TRY(check_ptr(c.k_scale, "cache.k_scale"));
        UQ_TRY(check_ptr(c.v_scale, "cache.v_scale"));
    }
    return UQ_OK;
}

// Rows of `width` contiguous elements at i * s0 + j * s1 (i < n0, j < n1):
// 16-byte aligned, and apart from each other where they are written.
uq_status check_rows(const char* name, int64_t s0, int64_t n0, int64_t s1, int64_t n1, int width, int dtype, bool written) {
    constexpr int64_t kMost = int64_t(1) << 56;                  // elements: byte offsets stay far from overflow
    const int64_t per = dtype == UQ_W_F32 ? 4 : 8;
    if (s0 < 0 || s1 < 0 || s0 > kMost / n0 || s1 > kMost / n1)
        return fail(UQ_ERR_ARG, "%s: strides %lld, %lld must be >= 0 and within 2^56 elements", name, (long long)s0,
                    (long long)s1);
    if ((n0 > 1 && s0 % per != 0) || (n1 > 1 && s1 % per != 0))
        return fail(UQ_ERR_ALIGN, "%s: strides %lld, %lld give rows that are not 16-byte aligned", name, (long long)s0,
                    (long long)s1);
    if (!written) return UQ_OK;
    const bool first = n1 == 1 || (n0 > 1 && s0 <= s1);          // the dimension of the smaller step
    const int64_t sa = first ? s0 : s1, na = first ? n0 : n1, sb = first ? s1 : s0, nb = first ? n1 : n0;
    if ((na > 1 && sa < width) || (nb > 1 && sb < (na - 1) * sa + width))
        return fail(UQ_ERR_ARG, "%s: strides %lld, %lld make rows of %d overlap", name, (long long)s0, (long long)s1, width);
    return UQ_OK;
}

uq_status check_float(int dtype) {
    if (dtype != UQ_W_F32 && dtype != UQ_W_BF16) return fail(UQ_ERR_ARG, "unknown dtype %d", dtype);
    return UQ_OK;
}

// Rows at i * s0 + j * s1 + k * s2: as check_rows, the rows of one i and then the blocks of all i.
uq_status check_rows3(const char* name, int64_t s0, int64_t n0, int64_t s1, int64_t n1, int64_t s2, int64_t n2, int width,
                      int dtype, bool written) {
    UQ_TRY(check_rows(name, s1, n1, s2, n2, width, dtype, false));
    UQ_TRY(check_rows(name, s0, n0, s2, n2, width, dtype, false));
    if (!written) return UQ_OK;
    std::pair<int64_t, int64_t> d[3] = {{s0, n0}, {s1, n1}, {s2, n2}};     // smallest step first; a single one has none
    for (auto& x : d)
        if (x.second == 1) x.first = 0;
    std::sort(d, d + 3);
    int64_t extent = width;
    for (const auto& x : d) {
        if (x.second == 1) continue;
        if (x.first < extent)
            return fail(UQ_ERR_ARG, "%s: strides %lld, %lld, %lld make rows of %d overlap", name, (long long)s0,
                        (long long)s1, (long long)s2, width);
        extent += (x.second - 1) * x.first;
    }
    return UQ_OK;
}

uq_status check_ints(const void* p, const char* name, unsigned bytes) {
    if (p == nullptr) return fail(UQ_ERR_ARG, "%s is NULL", name);
    if (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) return fail(UQ_ERR_ALIGN, "%s=%p is not %u-byte aligned", name, p, bytes);
    return UQ_OK;
}

uq_status kv_copy(bool write, const char* what, const uq_kv_cache& c, const int64_t* slots, int64_t tokens, void* k,
                  void* v, int dtype, const int64_t strides[4], void* stream) {
    UQ_TRY(check_kv(c));
    UQ_TRY(check_float(dtype));
    if (tokens < 0 || tokens > 0x7fffffffLL / c.kv_heads)
        return fail(UQ_ERR_ARG, "tokens=%lld: tokens * kv_heads must be in 0..2^31-1", (long long)tokens);
    if (tokens == 0) return ok();
    UQ_TRY(check_rows("k", strides[0], tokens, strides[1], c.kv_heads, c.head_dim, dtype, !write));
    UQ_TRY(check_rows("v", strides[2], tokens, strides[3], c.kv_heads, c.head_dim, dtype, !write));
    UQ_TRY(check_ptr(k, "k"));
    UQ_TRY(check_ptr(v, "v"));
    if (slots == nullptr) return fail(UQ_ERR_ARG, "slots is NULL");
    if (reinterpret_cast<uintptr_t>(slots) & 7u) return fail(UQ_ERR_ALIGN, "slots=%p is not 8-byte aligned", (const void*)slots);
    return cuda_status(uq::launch_kv_copy(write, c, slots, tokens, k, v, dtype, strides, (cudaStream_t)stream), what);
}

// What the attentions over the cache have in common: numbers, buffers, workspace.
uq_status check_attn(const uq_kv_cache& cache, int64_t batch, int heads, int64_t table_stride, int64_t max_pages,
                     float scale, int64_t window, int64_t sinks) {
    if (batch < 0 || batch > 65535) return fail(UQ_ERR_ARG, "batch=%lld must be in 0..65535", (long long)batch);
    if (heads < 1 || heads > 65536 || heads % cache.kv_heads != 0)
        return fail(UQ_ERR_ARG, "heads=%d must be a multiple of kv_heads=%d, 65536 at most", heads, cache.kv_heads);
    if (max_pages < 1 || max_pages > (int64_t(1) << 30) / cache.page_size)
        return fail(UQ_ERR_ARG, "max_pages=%lld: max_pages * page_size must be in %d..2^30", (long long)max_pages,
                    cache.page_size);
    if (table_stride < (batch > 1 ? max_pages : 0) || table_stride > (int64_t(1) << 40))
        return fail(UQ_ERR_ARG, "table_stride=%lld must be at least max_pages=%lld", (long long)table_stride,
                    (long long)max_pages);
    if (window < 0) return fail(UQ_ERR_ARG, "window=%lld must be >= 0 (0: every position)", (long long)window);
    if (sinks < 0) return fail(UQ_ERR_ARG, "sinks=%lld must be >= 0", (long long)sinks);
    if (!(std::fabs(scale) <= 0x1p127f)) return fail(UQ_ERR_ARG, "scale must be finite, 2^127 at most");   // to base 2 too
    return UQ_OK;
}

uq_status check_attn_buffers(const void* q, const void* out, const int32_t* block_table, const int32_t* seq_lens,
                             const float* lse, const void* workspace) {
    UQ_TRY(check_ptr(q, "q"));
    UQ_TRY(check_ptr(out, "out"));
    UQ_TRY(check_ints(block_table, "block_table", 4));
    UQ_TRY(check_ints(seq_lens, "seq_lens", 4));
    if (reinterpret_cast<uintptr_t>(lse) & 3u) return fail(UQ_ERR_ALIGN, "lse=%p is not 4-byte aligned", (const void*)lse);
    return check_ptr(workspace, "workspace");
}

uq_status check_workspace(int64_t bytes, int64_t need, const char* says) {
    if (bytes < need)
        return fail(UQ_ERR_ARG, "workspace of %lld bytes; this attention needs %lld (%s)", (long long)bytes, (long long)need, says);
    return UQ_OK;
}

// Attention of one new token; sinks = 0: none.
uq_status one_token(const char* what, const uq_kv_cache& cache, const void* q, int dtype, int64_t batch, int heads,
                    int64_t q_batch_stride, int64_t q_head_stride, const int32_t* block_table, int64_t table_stride,
                    int64_t max_pages, const int32_t* seq_lens, float scale, int64_t window, int64_t sinks, void* out,
                    int64_t out_batch_stride, int64_t out_head_stride, float* lse, void* workspace,
                    int64_t workspace_bytes, void* stream) {
    UQ_TRY(check_kv(cache));
    UQ_TRY(check_float(dtype));
    UQ_TRY(check_attn(cache, batch, heads, table_stride, max_pages, scale, window, sinks));
    if (batch == 0) return ok();
    UQ_TRY(check_rows("q", q_batch_stride, batch, q_head_stride, heads, cache.head_dim, dtype, false));
    UQ_TRY(check_rows("out", out_batch_stride, batch, out_head_stride, heads, cache.head_dim, dtype, true));
    UQ_TRY(check_attn_buffers(q, out, block_table, seq_lens, lse, workspace));
    UQ_TRY(check_workspace(workspace_bytes, uq::attn_workspace_bytes(heads, cache.kv_heads, cache.head_dim),
                           "uq_paged_attn_workspace_bytes"));
    uq::AttnArgs a{};
    a.c = cache;
    a.q = q;
    a.out = out;
    a.lse = lse;
    a.table = block_table;
    a.seq_lens = seq_lens;
    a.work = static_cast<float*>(workspace);
    a.q_batch = q_batch_stride;
    a.q_head = q_head_stride;
    a.out_batch = out_batch_stride;
    a.out_head = out_head_stride;
    a.table_stride = table_stride;
    a.max_tokens = (int)(max_pages * cache.page_size);
    a.window = window >= a.max_tokens ? 0 : (int)window;
    a.sinks = a.window == 0 ? 0 : (int)std::min<int64_t>(sinks, a.max_tokens);
    a.batch = (int)batch;
    a.heads = heads;
    a.dtype = dtype;
    a.page_shift = __builtin_ctz((unsigned)cache.page_size);
    a.scale = scale;
    return cuda_status(uq::launch_attn(a, (cudaStream_t)stream), what);
}

// The arguments that prompts and trees share.
uq::RowsArgs rows_args(const uq_kv_cache& cache, const void* q, int dtype, int64_t batch, int heads,
                       const int32_t* block_table, int64_t table_stride, int64_t max_pages, const int32_t* seq_lens,
                       float scale, int64_t window, int64_t sinks, void* out, float* lse, void* workspace) {
    uq::RowsArgs a{};
    a.c = cache;
    a.q = q;
    a.out = out;
    a.lse = lse;
    a.table = block_table;
    a.seq_lens = seq_lens;
    a.table_stride = table_stride;
    a.batch = (int)batch;
    a.heads = heads;
    a.dtype = dtype;
    a.page_shift = __builtin_ctz((unsigned)cache.page_size);
    a.max_tokens = (int)(max_pages * cache.page_size);
    a.window = window >= a.max_tokens ? 0 : (int)window;
    a.sinks = a.window == 0 ? 0 : (int)std::min<int64_t>(sinks, a.max_tokens);
    a.scale = scale;
    a.work = static_cast<float*>(workspace);
    return a;
}

}  // namespace

extern "C" {

int uq_abi_version(void) { return 1; }

const char* uq_last_error(void) { return g_err; }

uq_status uq_init_params(const void* W, uq_wdtype wdtype, int64_t out, int64_t in, int q, int g, int G, int T,
                         uq_clip clip, uq_params p, uint8_t* codes, void* stream) {
    UQ_TRY(check_shape(out, in, q, g, wdtype));
    if (g > 32768) return fail(UQ_ERR_UNSUPPORTED, "initialization supports g <= 32768 (g=%d)", g);
    if (G < 1) return fail(UQ_ERR_ARG, "G=%d must be >= 1", G);
    if (T < 0) return fail(UQ_ERR_ARG, "T=%d must be >= 0", T);
    if (clip != UQ_CLIP_FIXED_MIN && clip != UQ_CLIP_FIXED_MAX && clip != UQ_CLIP_BALANCED)
        return fail(UQ_ERR_ARG, "unknown clipping strategy %d", (int)clip);
    UQ_TRY(check_ptr(W, "W"));
    UQ_TRY(check_ptr(p.delta, "params.delta"));
    UQ_TRY(check_ptr(p.zu, "params.zu"));
    UQ_TRY(check_ptr(p.s, "params.s"));
    UQ_TRY(check_ptr(p.sr, "params.sr"));
    UQ_TRY(check_ptr(p.alpha, "params.alpha"));
    UQ_TRY(check_ptr(p.zb, "params.zb"));
    UQ_TRY(check_ptr(codes, "codes"));
    const uq::Shape sh{out, (int)in, q, g, (int)wdtype};
    return cuda_status(uq::launch_init(sh, W, G, T, (int)clip, p, codes, (cudaStream_t)stream), "uq_init_params");
}

uq_status uq_quantize_fwd(const void* W, uq_wdtype wdtype, int64_t out, int64_t in, int q, int g, uq_params p,
                          uint8_t* codes, uq_map map, int64_t step, int p_period, float* W_hat, void* stream) {
    UQ_TRY(check_shape(out, in, q, g, wdtype));
    if (map != UQ_MAP_FULL && map != UQ_MAP_LOCAL_PERIODIC) return fail(UQ_ERR_ARG, "unknown mapping %d", (int)map);
    if (p_period < 1) return fail(UQ_ERR_ARG, "p_period=%d must be >= 1", p_period);
    if (step < 0) return fail(UQ_ERR_ARG, "step=%lld must be >= 0", (long long)step);
    const int mode = map == UQ_MAP_FULL ? uq::FWD_FULL : (step % p_period == 0 ? uq::FWD_REMAP : uq::FWD_KEEP);
    if (mode != uq::FWD_KEEP) {
        UQ_TRY(check_ptr(W, "W"));
        UQ_TRY(check_ptr(p.s, "params.s"));
        UQ_TRY(check_ptr(p.sr, "params.sr"));
    }
    UQ_TRY(check_ptr(p.delta, "params.delta"));
    UQ_TRY(check_ptr(p.zu, "params.zu"));
    UQ_TRY(check_ptr(p.alpha, "params.alpha"));
    UQ_TRY(check_ptr(p.zb, "params.zb"));
    UQ_TRY(check_ptr(codes, "codes"));
    UQ_TRY(check_ptr(W_hat, "W_hat"));
    const uq::Shape sh{out, (int)in, q, g, (int)wdtype};
    return cuda_status(uq::launch_fwd(sh, W, p, codes, mode, W_hat, (cudaStream_t)stream), "uq_quantize_fwd");
}

uq_status uq_quantize_bwd(const void* W, uq_wdtype wdtype, int64_t out, int64_t in, int q, int g, uq_params p,
                          const uint8_t* codes, const float* dL_dWhat, uq_grads gr, void* stream) {
    UQ_TRY(check_shape(out, in, q, g, wdtype));
    UQ_TRY(check_ptr(W, "W"));
    UQ_TRY(check_ptr(p.delta, "params.delta"));
    UQ_TRY(check_ptr(p.zu, "params.zu"));
    UQ_TRY(check_ptr(p.s, "params.s"));
    UQ_TRY(check_ptr(p.sr, "params.sr"));
    UQ_TRY(check_ptr(p.alpha, "params.alpha"));
    UQ_TRY(check_ptr(p.zb, "params.zb"));
    UQ_TRY(check_ptr(codes, "codes"));
    UQ_TRY(check_ptr(dL_dWhat, "dL_dWhat"));
    UQ_TRY(check_ptr(gr.ddelta, "grads.ddelta"));
    UQ_TRY(check_ptr(gr.dzu, "grads.dzu"));
    UQ_TRY(check_ptr(gr.ds, "grads.ds"));
    UQ_TRY(check_ptr(gr.dsr, "grads.dsr"));
    UQ_TRY(check_ptr(gr.dalpha, "grads.dalpha"));
    UQ_TRY(check_ptr(gr.dzb, "grads.dzb"));
    const uq::Shape sh{out, (int)in, q, g, (int)wdtype};
    return cuda_status(uq::launch_bwd(sh, W, p, codes, dL_dWhat, gr, (cudaStream_t)stream), "uq_quantize_bwd");
}

uq_status uq_quantize_bwd_ex(const void* W, uq_wdtype wdtype, int64_t out, int64_t in, int q, int g, uq_params p,
                             const uint8_t* codes, const float* dL_dWhat, uq_grads gr, uq_filter filter,
                             void* stream) {
    if (filter != UQ_FILTER_STE && filter != UQ_FILTER_ELEMENT)
        return fail(UQ_ERR_ARG, "unknown gradient filter %d", (int)filter);
    UQ_TRY(check_shape(out, in, q, g, wdtype));
    UQ_TRY(check_ptr(W, "W"));
    UQ_TRY(check_ptr(p.delta, "params.delta"));
    UQ_TRY(check_ptr(p.zu, "params.zu"));
    UQ_TRY(check_ptr(p.s, "params.s"));
    UQ_TRY(check_ptr(p.sr, "params.sr"));
    UQ_TRY(check_ptr(p.alpha, "params.alpha"));
    UQ_TRY(check_ptr(p.zb, "params.zb"));
    UQ_TRY(check_ptr(codes, "codes"));
    UQ_TRY(check_ptr(dL_dWhat, "dL_dWhat"));
    UQ_TRY(check_ptr(gr.ddelta, "grads.ddelta"));
    UQ_TRY(check_ptr(gr.dzu, "grads.dzu"));
    UQ_TRY(check_ptr(gr.ds, "grads.ds"));
    UQ_TRY(check_ptr(gr.dsr, "grads.dsr"));
    UQ_TRY(check_ptr(gr.dalpha, "grads.dalpha"));
    UQ_TRY(check_ptr(gr.dzb, "grads.dzb"));
    const uq::Shape sh{out, (int)in, q, g, (int)wdtype};
    return cuda_status(uq::launch_bwd(sh, W, p, codes, dL_dWhat, gr, (cudaStream_t)stream, (int)filter),
                       "uq_quantize_bwd_ex");
}

uq_status uq_export_bcq_half(const void* W, uq_wdtype wdtype, int64_t out, int64_t in, int q, int g, uq_params p,
                             const uint8_t* codes, uq_export_mode mode, uint32_t* bitplanes, uint16_t* alpha_star,
                             uint16_t* zb_star, void* stream) {
    UQ_TRY(check_shape(out, in, q, g, wdtype));
    if (mode != UQ_EXPORT_REUSE_CODES && mode != UQ_EXPORT_REMAP_EQ4)
        return fail(UQ_ERR_ARG, "unknown export mode %d", (int)mode);
    if (mode == UQ_EXPORT_REMAP_EQ4) UQ_TRY(check_ptr(W, "W"));
    else UQ_TRY(check_ptr(codes, "codes"));
    UQ_TRY(check_ptr(p.delta, "params.delta"));
    UQ_TRY(check_ptr(p.zu, "params.zu"));
    UQ_TRY(check_ptr(p.alpha, "params.alpha"));
    UQ_TRY(check_ptr(p.zb, "params.zb"));
    UQ_TRY(check_ptr(bitplanes, "bitplanes"));
    UQ_TRY(check_ptr(alpha_star, "alpha_star"));
    UQ_TRY(check_ptr(zb_star, "zb_star"));
    const uq::Shape sh{out, (int)in, q, g, (int)wdtype};
    return cuda_status(uq::launch_export_half(sh, W, p, codes, (int)mode, bitplanes, alpha_star, zb_star,
                                              (cudaStream_t)stream),
                       "uq_export_bcq_half");
}

uq_status uq_train_step(const void* W, uq_wdtype wdtype, int64_t out, int64_t in, int q, int g, uq_params p,
                        uint8_t* codes, const float* dL_dWhat, float lr_F, float lr_B, uq_map map, int64_t step,
                        int p_period, float* W_hat, void* stream) {
    UQ_TRY(check_shape(out, in, q, g, wdtype));
    if (map != UQ_MAP_FULL && map != UQ_MAP_LOCAL_PERIODIC) return fail(UQ_ERR_ARG, "unknown mapping %d", (int)map);
    if (p_period < 1) return fail(UQ_ERR_ARG, "p_period=%d must be >= 1", p_period);
    if (step < 0 || step == INT64_MAX) return fail(UQ_ERR_ARG, "step=%lld must be in [0, 2^63 - 1)", (long long)step);
    const uq::Shape sh{out, (int)in, q, g, (int)wdtype};
    if (!uq::step_path_ok(sh))
        return fail(UQ_ERR_UNSUPPORTED,
                    "the fused step handles g in {32, 64, 128} with in a multiple of %d and at most %d (g=%d in=%lld); "
                    "use uq_quantize_bwd and uq_quantize_fwd",
                    g == 32 ? 256 : 512, g == 32 ? 16384 : 32768, g, (long long)in);
    UQ_TRY(check_ptr(W, "W"));
    UQ_TRY(check_ptr(p.delta, "params.delta"));
    UQ_TRY(check_ptr(p.zu, "params.zu"));
    UQ_TRY(check_ptr(p.s, "params.s"));
    UQ_TRY(check_ptr(p.sr, "params.sr"));
    UQ_TRY(check_ptr(p.alpha, "params.alpha"));
    UQ_TRY(check_ptr(p.zb, "params.zb"));
    UQ_TRY(check_ptr(codes, "codes"));
    UQ_TRY(check_ptr(dL_dWhat, "dL_dWhat"));
    UQ_TRY(check_ptr(W_hat, "W_hat"));
    const int64_t next = step + 1;
    const int mode = map == UQ_MAP_FULL ? uq::FWD_FULL : (next % p_period == 0 ? uq::FWD_REMAP : uq::FWD_KEEP);
    return cuda_status(uq::launch_step(sh, W, p, codes, dL_dWhat, lr_F, lr_B, mode, W_hat, (cudaStream_t)stream),
                       "uq_train_step");
}

uq_status uq_train_step_bf16(const void* W, uq_wdtype wdtype, int64_t out, int64_t in, int q, int g, uq_params p,
                             uint8_t* codes, const uint16_t* dL_dWhat, float lr_F, float lr_B, uq_map map,
                             int64_t step, int p_period, uint16_t* W_hat, void* stream) {
    UQ_TRY(check_shape(out, in, q, g, wdtype));
    if (map != UQ_MAP_FULL && map != UQ_MAP_LOCAL_PERIODIC) return fail(UQ_ERR_ARG, "unknown mapping %d", (int)map);
    if (p_period < 1) return fail(UQ_ERR_ARG, "p_period=%d must be >= 1", p_period);
    if (step < 0 || step == INT64_MAX) return fail(UQ_ERR_ARG, "step=%lld must be in [0, 2^63 - 1)", (long long)step);
    const uq::Shape sh{out, (int)in, q, g, (int)wdtype};
    if (!uq::step_path_ok(sh))
        return fail(UQ_ERR_UNSUPPORTED,
                    "the fused step handles g in {32, 64, 128} with in a multiple of %d and at most %d (g=%d in=%lld)",
                    g == 32 ? 256 : 512, g == 32 ? 16384 : 32768, g, (long long)in);
    UQ_TRY(check_ptr(W, "W"));
    UQ_TRY(check_ptr(p.delta, "params.delta"));
    UQ_TRY(check_ptr(p.zu, "params.zu"));
    UQ_TRY(check_ptr(p.s, "params.s"));
    UQ_TRY(check_ptr(p.sr, "params.sr"));
    UQ_TRY(check_ptr(p.alpha, "params.alpha"));
    UQ_TRY(check_ptr(p.zb, "params.zb"));
    UQ_TRY(check_ptr(codes, "codes"));
    UQ_TRY(check_ptr(dL_dWhat, "dL_dWhat"));
    UQ_TRY(check_ptr(W_hat, "W_hat"));
    const int64_t next = step + 1;
    const int mode = map == UQ_MAP_FULL ? uq::FWD_FULL : (next % p_period == 0 ? uq::FWD_REMAP : uq::FWD_KEEP);
    return cuda_status(
        uq::launch_step_bf16(sh, W, p, codes, dL_dWhat, lr_F, lr_B, mode, W_hat, (cudaStream_t)stream),
        "uq_train_step_bf16");
}

uq_status uq_quantize_fwd_omni(const void* W, uq_wdtype wdtype, int64_t out, int64_t in, int q, int g,
                               uq_params_omni p, uint8_t* codes, uq_map map, int64_t step, int p_period,
                               float* W_hat, void* stream) {
    UQ_TRY(check_shape(out, in, q, g, wdtype));
    const uq::Shape sh{out, (int)in, q, g, (int)wdtype};
    if (!uq::omni_ok(sh)) return fail(UQ_ERR_UNSUPPORTED, "g=%d: the OmniQuant maps take g in {32, 64, 128, 256, 512}", g);
    if (map != UQ_MAP_FULL && map != UQ_MAP_LOCAL_PERIODIC) return fail(UQ_ERR_ARG, "unknown mapping %d", (int)map);
    if (p_period < 1) return fail(UQ_ERR_ARG, "p_period=%d must be >= 1", p_period);
    if (step < 0) return fail(UQ_ERR_ARG, "step=%lld must be >= 0", (long long)step);
    UQ_TRY(check_ptr(W, "W"));
    UQ_TRY(check_ptr(p.beta, "params.beta"));
    UQ_TRY(check_ptr(p.gamma, "params.gamma"));
    UQ_TRY(check_ptr(p.alpha, "params.alpha"));
    UQ_TRY(check_ptr(p.zb, "params.zb"));
    UQ_TRY(check_ptr(codes, "codes"));
    UQ_TRY(check_ptr(W_hat, "W_hat"));
    const int mode = map == UQ_MAP_FULL ? uq::FWD_FULL : (step % p_period == 0 ? uq::FWD_REMAP : uq::FWD_KEEP);
    return cuda_status(uq::launch_omni_fwd(sh, W, p, codes, mode, W_hat, (cudaStream_t)stream), "uq_quantize_fwd_omni");
}

uq_status uq_quantize_bwd_omni(const void* W, uq_wdtype wdtype, int64_t out, int64_t in, int q, int g,
                               uq_params_omni p, const uint8_t* codes, const float* dL_dWhat, uq_grads_omni gr,
                               void* stream) {
    UQ_TRY(check_shape(out, in, q, g, wdtype));
    const uq::Shape sh{out, (int)in, q, g, (int)wdtype};
    if (!uq::omni_ok(sh)) return fail(UQ_ERR_UNSUPPORTED, "g=%d: the OmniQuant maps take g in {32, 64, 128, 256, 512}", g);
    UQ_TRY(check_ptr(W, "W"));
    UQ_TRY(check_ptr(p.beta, "params.beta"));
    UQ_TRY(check_ptr(p.gamma, "params.gamma"));
    UQ_TRY(check_ptr(p.alpha, "params.alpha"));
    UQ_TRY(check_ptr(p.zb, "params.zb"));
    UQ_TRY(check_ptr(codes, "codes"));
    UQ_TRY(check_ptr(dL_dWhat, "dL_dWhat"));
    UQ_TRY(check_ptr(gr.dbeta, "grads.dbeta"));
    UQ_TRY(check_ptr(gr.dgamma, "grads.dgamma"));
    UQ_TRY(check_ptr(gr.dalpha, "grads.dalpha"));
    UQ_TRY(check_ptr(gr.dzb, "grads.dzb"));
    return cuda_status(uq::launch_omni_bwd(sh, W, p, codes, dL_dWhat, gr, (cudaStream_t)stream), "uq_quantize_bwd_omni");
}

uq_status uq_omni_scales(const void* W, uq_wdtype wdtype, int64_t out, int64_t in, int q, int g, const float* beta,
                         const float* gamma, float* delta, float* zo, void* stream) {
    UQ_TRY(check_shape(out, in, q, g, wdtype));
    const uq::Shape sh{out, (int)in, q, g, (int)wdtype};
    if (!uq::omni_ok(sh)) return fail(UQ_ERR_UNSUPPORTED, "g=%d: the OmniQuant maps take g in {32, 64, 128, 256, 512}", g);
    UQ_TRY(check_ptr(W, "W"));
    UQ_TRY(check_ptr(beta, "beta"));
    UQ_TRY(check_ptr(gamma, "gamma"));
    UQ_TRY(check_ptr(delta, "delta"));
    UQ_TRY(check_ptr(zo, "zo"));
    return cuda_status(uq::launch_omni_scales(sh, W, beta, gamma, delta, zo, (cudaStream_t)stream), "uq_omni_scales");
}

uq_status uq_quantize_fwd_awq(const void* W, uq_wdtype wdtype, int64_t out, int64_t in, int q, int g,
                              uq_params_awq p, uint8_t* codes, uq_map map, int64_t step, int p_period, float* W_hat,
                              void* stream) {
    UQ_TRY(check_shape(out, in, q, g, wdtype));
    const uq::Shape sh{out, (int)in, q, g, (int)wdtype};
    if (!uq::awq_ok(sh)) return fail(UQ_ERR_UNSUPPORTED, "g=%d: the AWQ maps take g in {32, 64, 128, 256, 512}", g);
    if (map != UQ_MAP_FULL && map != UQ_MAP_LOCAL_PERIODIC) return fail(UQ_ERR_ARG, "unknown mapping %d", (int)map);
    if (p_period < 1) return fail(UQ_ERR_ARG, "p_period=%d must be >= 1", p_period);
    if (step < 0) return fail(UQ_ERR_ARG, "step=%lld must be >= 0", (long long)step);
    const int mode = map == UQ_MAP_FULL ? uq::FWD_FULL : (step % p_period == 0 ? uq::FWD_REMAP : uq::FWD_KEEP);
    if (mode != uq::FWD_KEEP) UQ_TRY(check_ptr(W, "W"));
    UQ_TRY(check_ptr(p.sa, "params.sa"));
    UQ_TRY(check_ptr(p.delta, "params.delta"));
    UQ_TRY(check_ptr(p.za, "params.za"));
    UQ_TRY(check_ptr(p.alpha, "params.alpha"));
    UQ_TRY(check_ptr(p.zb, "params.zb"));
    UQ_TRY(check_ptr(codes, "codes"));
    UQ_TRY(check_ptr(W_hat, "W_hat"));
    return cuda_status(uq::launch_awq_fwd(sh, W, p, codes, mode, W_hat, (cudaStream_t)stream), "uq_quantize_fwd_awq");
}

int64_t uq_awq_bwd_workspace_bytes(int64_t out, int64_t in, int q, int g) {
    if (q < 1 || q > 4 || out < 1 || in < 1 || g < 32 || in % g != 0 || in > kMaxIn || out > 0x7fffffffLL) return -1;
    const uq::Shape sh{out, (int)in, q, g, UQ_W_BF16};
    if (!uq::awq_ok(sh)) return -1;
    return uq::awq_workspace_floats(sh) * (int64_t)sizeof(float);
}

uq_status uq_quantize_bwd_awq(const void* W, uq_wdtype wdtype, int64_t out, int64_t in, int q, int g,
                              uq_params_awq p, const uint8_t* codes, const float* dL_dWhat, uq_grads_awq gr,
                              float* workspace, int64_t workspace_bytes, void* stream) {
    UQ_TRY(check_shape(out, in, q, g, wdtype));
    const uq::Shape sh{out, (int)in, q, g, (int)wdtype};
    if (!uq::awq_ok(sh)) return fail(UQ_ERR_UNSUPPORTED, "g=%d: the AWQ maps take g in {32, 64, 128, 256, 512}", g);
    UQ_TRY(check_ptr(W, "W"));
    UQ_TRY(check_ptr(p.sa, "params.sa"));
    UQ_TRY(check_ptr(p.delta, "params.delta"));
    UQ_TRY(check_ptr(p.za, "params.za"));
    UQ_TRY(check_ptr(p.alpha, "params.alpha"));
    UQ_TRY(check_ptr(p.zb, "params.zb"));
    UQ_TRY(check_ptr(codes, "codes"));
    UQ_TRY(check_ptr(dL_dWhat, "dL_dWhat"));
    UQ_TRY(check_ptr(gr.dsa, "grads.dsa"));
    UQ_TRY(check_ptr(gr.ddelta, "grads.ddelta"));
    UQ_TRY(check_ptr(gr.dza, "grads.dza"));
    UQ_TRY(check_ptr(gr.dalpha, "grads.dalpha"));
    UQ_TRY(check_ptr(gr.dzb, "grads.dzb"));
    UQ_TRY(check_ptr(workspace, "workspace"));
    const int64_t need = uq::awq_workspace_floats(sh) * (int64_t)sizeof(float);
    if (workspace_bytes < need)
        return fail(UQ_ERR_ARG, "workspace of %lld bytes; the backward needs %lld (uq_awq_bwd_workspace_bytes)",
                    (long long)workspace_bytes, (long long)need);
    return cuda_status(uq::launch_awq_bwd(sh, W, p, codes, dL_dWhat, gr, workspace, (cudaStream_t)stream),
                       "uq_quantize_bwd_awq");
}

uq_status uq_export_bcq(const void* W, uq_wdtype wdtype, int64_t out, int64_t in, int q, int g, uq_params p,
                        const uint8_t* codes, uq_export_mode mode, uint32_t* bitplanes, float* alpha_star,
                        float* zb_star, void* stream) {
    UQ_TRY(check_shape(out, in, q, g, wdtype));
    if (mode != UQ_EXPORT_REUSE_CODES && mode != UQ_EXPORT_REMAP_EQ4)
        return fail(UQ_ERR_ARG, "unknown export mode %d", (int)mode);
    if (mode == UQ_EXPORT_REMAP_EQ4) UQ_TRY(check_ptr(W, "W"));
    else UQ_TRY(check_ptr(codes, "codes"));
    UQ_TRY(check_ptr(p.delta, "params.delta"));
    UQ_TRY(check_ptr(p.zu, "params.zu"));
    UQ_TRY(check_ptr(p.alpha, "params.alpha"));
    UQ_TRY(check_ptr(p.zb, "params.zb"));
    UQ_TRY(check_ptr(bitplanes, "bitplanes"));
    UQ_TRY(check_ptr(alpha_star, "alpha_star"));
    UQ_TRY(check_ptr(zb_star, "zb_star"));
    const uq::Shape sh{out, (int)in, q, g, (int)wdtype};
    return cuda_status(uq::launch_export(sh, W, p, codes, (int)mode, bitplanes, alpha_star, zb_star,
                                         (cudaStream_t)stream),
                       "uq_export_bcq");
}

int64_t uq_bcq_gemv_workspace_bytes(int64_t out, int64_t in, int batch) {
    if (out < 1 || in < 32 || in % 32 != 0 || in > kMaxIn || batch < 1 || batch > 64) return -1;
    return uq::gemv_workspace_floats(out, in, batch) * (int64_t)sizeof(float);
}

uq_status uq_bcq_gemv(const uint32_t* bitplanes, const float* alpha_star, const float* zb_star, int64_t out,
                      int64_t in, int q, int g, const void* x, uq_wdtype xdtype, int batch, float* y, float* workspace,
                      int64_t workspace_bytes, void* stream) {
    UQ_TRY(check_shape(out, in, q, g, xdtype));
    UQ_TRY(check_gemv_group(g));
    if (batch < 1 || batch > 64) return fail(UQ_ERR_ARG, "batch=%d must be in 1..64", batch);
    UQ_TRY(check_ptr(bitplanes, "bitplanes"));
    UQ_TRY(check_ptr(alpha_star, "alpha_star"));
    UQ_TRY(check_ptr(zb_star, "zb_star"));
    UQ_TRY(check_ptr(x, "x"));
    UQ_TRY(check_ptr(y, "y"));
    UQ_TRY(check_ptr(workspace, "workspace"));
    const int64_t need = uq_bcq_gemv_workspace_bytes(out, in, batch);
    if (workspace_bytes < need)
        return fail(UQ_ERR_ARG, "workspace of %lld bytes; this product needs %lld (uq_bcq_gemv_workspace_bytes)",
                    (long long)workspace_bytes, (long long)need);
    return cuda_status(uq::launch_gemv(bitplanes, alpha_star, zb_star, out, (int)in, q, g, x, (int)xdtype, batch, y,
                                       workspace, (cudaStream_t)stream),
                       "uq_bcq_gemv");
}

uq_status uq_bcq_gemv_noalloc(const uint32_t* bitplanes, const float* alpha_star, const float* zb_star,
                              int64_t out, int64_t in, int q, int g, const void* x, uq_wdtype xdtype, int batch,
                              float* y, void* stream) {
    UQ_TRY(check_shape(out, in, q, g, xdtype));
    UQ_TRY(check_gemv_group(g));
    if (batch < 1 || batch > 64) return fail(UQ_ERR_ARG, "batch=%d must be in 1..64", batch);
    UQ_TRY(check_ptr(bitplanes, "bitplanes"));
    UQ_TRY(check_ptr(alpha_star, "alpha_star"));
    UQ_TRY(check_ptr(zb_star, "zb_star"));
    UQ_TRY(check_ptr(x, "x"));
    UQ_TRY(check_ptr(y, "y"));
    const int64_t need = uq::gemv_workspace_floats(out, in, batch);
    const int64_t have = uq::gemv_static_workspace_floats();
    if (need > have)
        return fail(UQ_ERR_UNSUPPORTED,
                    "this product needs %lld floats of scratch (ceil(in/512) * batch * out); the built-in scratch "
                    "holds %lld: pass a workspace to uq_bcq_gemv instead",
                    (long long)need, (long long)have);
    float* work = nullptr;
    const cudaError_t e = uq::gemv_static_workspace(&work);
    if (e != cudaSuccess) return cuda_status(e, "uq_bcq_gemv_noalloc: looking up the built-in scratch");
    return cuda_status(uq::launch_gemv(bitplanes, alpha_star, zb_star, out, (int)in, q, g, x, (int)xdtype, batch, y,
                                       work, (cudaStream_t)stream),
                       "uq_bcq_gemv_noalloc");
}

uq_status uq_kv_write(uq_kv_cache cache, const void* k, const void* v, uq_wdtype dtype, int64_t tokens,
                      int64_t k_token_stride, int64_t k_head_stride, int64_t v_token_stride, int64_t v_head_stride,
                      const int64_t* slots, void* stream) {
    const int64_t strides[4] = {k_token_stride, k_head_stride, v_token_stride, v_head_stride};
    return kv_copy(true, "uq_kv_write", cache, slots, tokens, const_cast<void*>(k), const_cast<void*>(v), (int)dtype,
                   strides, stream);
}

uq_status uq_kv_read(uq_kv_cache cache, const int64_t* slots, int64_t tokens, void* k_out, void* v_out,
                     uq_wdtype dtype, int64_t k_token_stride, int64_t k_head_stride, int64_t v_token_stride,
                     int64_t v_head_stride, void* stream) {
    const int64_t strides[4] = {k_token_stride, k_head_stride, v_token_stride, v_head_stride};
    return kv_copy(false, "uq_kv_read", cache, slots, tokens, k_out, v_out, (int)dtype, strides, stream);
}

uq_status uq_kv_append(uq_kv_cache cache, const void* k, const void* v, uq_wdtype dtype, int64_t tokens,
                       int64_t k_token_stride, int64_t k_head_stride, int64_t v_token_stride, int64_t v_head_stride,
                       const int64_t* slots, const int64_t* positions, const float* rope, int64_t rope_rows,
                       int rotated, const void* q, int heads, int64_t q_token_stride, int64_t q_head_stride,
                       void* q_out, int64_t out_token_stride, int64_t out_head_stride, void* stream) {
    UQ_TRY(check_kv(cache));
    UQ_TRY(check_float((int)dtype));
    if (tokens < 0 || tokens > 0x7fffffffLL / cache.kv_heads)
        return fail(UQ_ERR_ARG, "tokens=%lld: tokens * kv_heads must be in 0..2^31-1", (long long)tokens);
    if (rotated < 16 || rotated > cache.head_dim || rotated % 16 != 0)
        return fail(UQ_ERR_UNSUPPORTED, "rotated=%d: multiples of 16 up to head_dim=%d are supported", rotated, cache.head_dim);
    if (rope_rows < 1 || rope_rows > (int64_t(1) << 40))
        return fail(UQ_ERR_ARG, "rope_rows=%lld must be in 1..2^40", (long long)rope_rows);
    if ((q == nullptr) != (q_out == nullptr)) return fail(UQ_ERR_ARG, "q and q_out are given together");
    if (q != nullptr && (heads < 1 || heads > 65536 || (tokens > 0 && tokens > 0x7fffffffLL / heads)))
        return fail(UQ_ERR_ARG, "heads=%d must be in 1..65536, and tokens * heads in 0..2^31-1", heads);
    if (tokens == 0) return ok();
    UQ_TRY(check_rows("k", k_token_stride, tokens, k_head_stride, cache.kv_heads, cache.head_dim, (int)dtype, false));
    UQ_TRY(check_rows("v", v_token_stride, tokens, v_head_stride, cache.kv_heads, cache.head_dim, (int)dtype, false));
    UQ_TRY(check_ptr(k, "k"));
    UQ_TRY(check_ptr(v, "v"));
    if (q != nullptr) {
        UQ_TRY(check_rows("q", q_token_stride, tokens, q_head_stride, heads, cache.head_dim, (int)dtype, false));
        UQ_TRY(check_rows("q_out", out_token_stride, tokens, out_head_stride, heads, cache.head_dim, (int)dtype, true));
        UQ_TRY(check_ptr(q, "q"));
        UQ_TRY(check_ptr(q_out, "q_out"));
    }
    UQ_TRY(check_ints(slots, "slots", 8));
    UQ_TRY(check_ints(positions, "positions", 8));
    UQ_TRY(check_ptr(rope, "rope"));
    uq::AppendArgs a{};
    a.c = cache;
    a.k = k;
    a.v = v;
    a.q = q;
    a.q_out = q_out;
    a.slots = slots;
    a.positions = positions;
    a.rope = rope;
    a.tokens = tokens;
    a.rope_rows = rope_rows;
    a.k_token = k_token_stride;
    a.k_head = k_head_stride;
    a.v_token = v_token_stride;
    a.v_head = v_head_stride;
    a.q_token = q_token_stride;
    a.q_head = q_head_stride;
    a.out_token = out_token_stride;
    a.out_head = out_head_stride;
    a.heads = heads;
    a.rot = rotated;
    a.dtype = (int)dtype;
    a.page_shift = __builtin_ctz((unsigned)cache.page_size);
    return cuda_status(uq::launch_kv_append(a, (cudaStream_t)stream), "uq_kv_append");
}

int64_t uq_paged_attn_workspace_bytes(int heads, int kv_heads, int head_dim) {
    if (kv_heads < 1 || kv_heads > 4096 || heads < 1 || heads > 65536 || heads % kv_heads != 0) return -1;
    if (head_dim != 64 && head_dim != 128 && head_dim != 256) return -1;
    return uq::attn_workspace_bytes(heads, kv_heads, head_dim);
}

uq_status uq_paged_attn(uq_kv_cache cache, const void* q, uq_wdtype dtype, int64_t batch, int heads,
                        int64_t q_batch_stride, int64_t q_head_stride, const int32_t* block_table,
                        int64_t table_stride, int64_t max_pages, const int32_t* seq_lens, float scale,
                        int64_t window, void* out, int64_t out_batch_stride, int64_t out_head_stride, float* lse,
                        void* workspace, int64_t workspace_bytes, void* stream) {
    return one_token("uq_paged_attn", cache, q, (int)dtype, batch, heads, q_batch_stride, q_head_stride, block_table,
                     table_stride, max_pages, seq_lens, scale, window, 0, out, out_batch_stride, out_head_stride, lse,
                     workspace, workspace_bytes, stream);
}

uq_status uq_paged_attn_sinks(uq_kv_cache cache, const void* q, uq_wdtype dtype, int64_t batch, int heads,
                              int64_t q_batch_stride, int64_t q_head_stride, const int32_t* block_table,
                              int64_t table_stride, int64_t max_pages, const int32_t* seq_lens, float scale,
                              int64_t window, int64_t sinks, void* out, int64_t out_batch_stride,
                              int64_t out_head_stride, float* lse, void* workspace, int64_t workspace_bytes,
                              void* stream) {
    return one_token("uq_paged_attn_sinks", cache, q, (int)dtype, batch, heads, q_batch_stride, q_head_stride,
                     block_table, table_stride, max_pages, seq_lens, scale, window, sinks, out, out_batch_stride,
                     out_head_stride, lse, workspace, workspace_bytes, stream);
}

int64_t uq_paged_rows_workspace_bytes(int heads, int kv_heads, int head_dim) {
    if (kv_heads < 1 || kv_heads > 4096 || heads < 1 || heads > 65536 || heads % kv_heads != 0) return -1;
    if (head_dim != 64 && head_dim != 128 && head_dim != 256) return -1;
    return uq::attn_rows_workspace_bytes(heads, kv_heads, head_dim);
}

uq_status uq_paged_prompt_attn(uq_kv_cache cache, const void* q, uq_wdtype dtype, int64_t tokens, int heads,
                               int64_t q_token_stride, int64_t q_head_stride, const int32_t* starts, int64_t batch,
                               const int32_t* block_table, int64_t table_stride, int64_t max_pages,
                               const int32_t* seq_lens, float scale, int64_t window, int64_t sinks, void* out,
                               int64_t out_token_stride, int64_t out_head_stride, float* lse, void* workspace,
                               int64_t workspace_bytes, void* stream) {
    UQ_TRY(check_kv(cache));
    UQ_TRY(check_float((int)dtype));
    UQ_TRY(check_attn(cache, batch, heads, table_stride, max_pages, scale, window, sinks));
    if (tokens < 0 || tokens > 0x7fffffffLL / heads)
        return fail(UQ_ERR_ARG, "tokens=%lld: tokens * heads must be in 0..2^31-1", (long long)tokens);
    if (batch == 0 || tokens == 0) return ok();
    UQ_TRY(check_rows("q", q_token_stride, tokens, q_head_stride, heads, cache.head_dim, (int)dtype, false));
    UQ_TRY(check_rows("out", out_token_stride, tokens, out_head_stride, heads, cache.head_dim, (int)dtype, true));
    UQ_TRY(check_attn_buffers(q, out, block_table, seq_lens, lse, workspace));
    UQ_TRY(check_ints(starts, "starts", 4));
    UQ_TRY(check_workspace(workspace_bytes, uq_paged_rows_workspace_bytes(heads, cache.kv_heads, cache.head_dim),
                           "uq_paged_rows_workspace_bytes"));
    uq::RowsArgs a = rows_args(cache, q, (int)dtype, batch, heads, block_table, table_stride, max_pages, seq_lens, scale,
                               window, sinks, out, lse, workspace);
    a.starts = starts;
    a.tokens = tokens;
    a.q_row = q_token_stride;
    a.q_head = q_head_stride;
    a.out_row = out_token_stride;
    a.out_head = out_head_stride;
    return cuda_status(uq::launch_attn_rows(a, (cudaStream_t)stream), "uq_paged_prompt_attn");
}

uq_status uq_paged_tree_attn(uq_kv_cache cache, const void* q, uq_wdtype dtype, int64_t batch, int64_t drafts,
                             int heads, int64_t q_batch_stride, int64_t q_draft_stride, int64_t q_head_stride,
                             const uint64_t* tree, int64_t tree_stride, const int32_t* counts,
                             const int32_t* block_table, int64_t table_stride, int64_t max_pages,
                             const int32_t* seq_lens, float scale, int64_t window, int64_t sinks, void* out,
                             int64_t out_batch_stride, int64_t out_draft_stride, int64_t out_head_stride, float* lse,
                             void* workspace, int64_t workspace_bytes, void* stream) {
    UQ_TRY(check_kv(cache));
    UQ_TRY(check_float((int)dtype));
    UQ_TRY(check_attn(cache, batch, heads, table_stride, max_pages, scale, window, sinks));
    if (drafts < 0 || drafts > 64) return fail(UQ_ERR_ARG, "drafts=%lld must be in 0..64", (long long)drafts);
    if (batch == 0 || drafts == 0) return ok();
    if (batch * drafts > 0x7fffffffLL / heads)
        return fail(UQ_ERR_ARG, "batch * drafts * heads must be in 0..2^31-1 (%lld * %lld * %d)", (long long)batch,
                    (long long)drafts, heads);
    if (tree_stride < (batch > 1 ? drafts : 0) || tree_stride > (int64_t(1) << 40))
        return fail(UQ_ERR_ARG, "tree_stride=%lld must be at least drafts=%lld", (long long)tree_stride, (long long)drafts);
    UQ_TRY(check_rows3("q", q_batch_stride, batch, q_draft_stride, drafts, q_head_stride, heads, cache.head_dim, (int)dtype, false));
    UQ_TRY(check_rows3("out", out_batch_stride, batch, out_draft_stride, drafts, out_head_stride, heads, cache.head_dim, (int)dtype, true));
    UQ_TRY(check_attn_buffers(q, out, block_table, seq_lens, lse, workspace));
    UQ_TRY(check_ints(tree, "tree", 8));
    if (reinterpret_cast<uintptr_t>(counts) & 3u) return fail(UQ_ERR_ALIGN, "counts=%p is not 4-byte aligned", (const void*)counts);
    UQ_TRY(check_workspace(workspace_bytes, uq_paged_rows_workspace_bytes(heads, cache.kv_heads, cache.head_dim),
                           "uq_paged_rows_workspace_bytes"));
    uq::RowsArgs a = rows_args(cache, q, (int)dtype, batch, heads, block_table, table_stride, max_pages, seq_lens, scale,
                               window, sinks, out, lse, workspace);
    a.tree = tree;
    a.tree_stride = tree_stride;
    a.counts = counts;
    a.most = (int)drafts;
    a.q_batch = q_batch_stride;
    a.q_row = q_draft_stride;
    a.q_head = q_head_stride;
    a.out_batch = out_batch_stride;
    a.out_row = out_draft_stride;
    a.out_head = out_head_stride;
    return cuda_status(uq::launch_attn_rows(a, (cudaStream_t)stream), "uq_paged_tree_attn");
}

uq_status uq_check_device(void* stream) {
    cudaError_t e = cudaStreamSynchronize((cudaStream_t)stream);
    if (e != cudaSuccess) return fail(UQ_ERR_CUDA, "uq_check_device: %s", cudaGetErrorString(e));
    unsigned int flag = 0, flag_step = 0, flag_omni = 0, flag_awq = 0, flag_gemv = 0;
    e = uq::stream_error(true, &flag);
    for (auto more : {uq::ragged_fwd_error, uq::ragged_bwd_error}) {
        unsigned int flag_ragged = 0;
        if (e == cudaSuccess) e = more(true, &flag_ragged);
        flag |= flag_ragged;
    }
    if (e == cudaSuccess) e = uq::step_error(true, &flag_step);
    if (e == cudaSuccess) {
        unsigned int flag_step_bf16 = 0;
        e = uq::step_bf16_error(true, &flag_step_bf16);
        flag_step |= flag_step_bf16;
    }
    if (e == cudaSuccess) e = uq::omni_error(true, &flag_omni);
    if (e == cudaSuccess) e = uq::awq_error(true, &flag_awq);
    if (e == cudaSuccess) e = uq::gemv_error(true, &flag_gemv);
    if (e == cudaSuccess) {
        unsigned int flag_tc = 0;
        e = uq::bcq_tc_error(true, &flag_tc);
        flag_gemv |= flag_tc;
    }
    unsigned int flag_rows = 0;
    for (auto more : {uq::rows_bf16_error, uq::rows_int8_error, uq::rows_int4_error}) {
        unsigned int one = 0;
        if (e == cudaSuccess) e = more(true, &one);
        flag_rows |= one;
    }
    if (e != cudaSuccess) return fail(UQ_ERR_CUDA, "uq_check_device: %s", cudaGetErrorString(e));
    flag |= (flag_rows << 20) | (flag_step << 4) | (flag_omni << 8) | (flag_awq << 12) | (flag_gemv << 16);
    const unsigned int drain_bits = 0x888888u;   // kDrainTimeoutBit of each kernel family
    if (flag & drain_bits)
        return fail(UQ_ERR_CUDA, "a bounded wait ran out on the device (flag %u): a kernel gave up waiting "
                                 "for its own data copies, and its wait for the copies still in flight ran out "
                                 "too, so a block may have exited with copies landing in its shared memory",
                    flag);
    if (flag) return fail(UQ_ERR_CUDA, "a bounded wait ran out on the device (flag %u): a kernel gave up waiting "
                                       "for its own data copies", flag);
    return ok();
}

uq_status uq_selftest_wait_timeout(void* stream) {
    return cuda_status(uq::launch_wait_selftest((cudaStream_t)stream), "uq_selftest_wait_timeout");
}

}  // extern "C"
