// The operators on a paged KV cache of 8-bit rows, in windows and for drafted tokens: the host side of their part of the C ABI, the kernels that append and read,
// and attention over plain rows.
#include "quant_launch.hpp"

using namespace ctkvr;

namespace {

int check_format(int format, bool plain)
{
    if (format == CTKVR_KV_INT8 || format == CTKVR_KV_FP8 || (plain && format == CTKVR_KV_PLAIN)) return CTKVR_OK;
    return fail(CTKVR_EINVAL, "unknown format %d of rows", format);
}
int check_codes(int format, const void *codes, const float *scales, const char *name)
{
    if (!codes || !aligned16(codes)) return fail(CTKVR_EINVAL, "%s: must begin on a 16-byte boundary", name);
    if ((format == CTKVR_KV_PLAIN) != !scales)
        return fail(CTKVR_EINVAL, format == CTKVR_KV_PLAIN ? "%s: plain rows have no scales" : "%s: 8-bit rows need scales", name);
    if ((uintptr_t)scales & 3) return fail(CTKVR_EINVAL, "%s: scales must begin on a 4-byte boundary", name);
    return CTKVR_OK;
}

struct AttnCall {
    const void *q;
    int64_t q_stride;
    int format;
    const void *k;
    const float *k_scales;
    const void *v;
    const float *v_scales;
    const int32_t *cu, *cur, *table;
    int total;
    void *out;
    float *lse;
};
int check_attn(const ctkvr_cache *c, const AttnCall &x)
{
    if (!x.q || !x.cu || !x.cur || !x.table || !x.out) return fail(CTKVR_EINVAL, "a required pointer is NULL");
    TRY(check_rows(c, "q", x.q, x.q_stride, c->p.n_q_heads));
    TRY(check_codes(x.format, x.k, x.k_scales, "k"));
    TRY(check_codes(x.format, x.v, x.v_scales, "v"));
    if (!aligned16(x.out)) return fail(CTKVR_EINVAL, "out must begin on a 16-byte boundary");
    return CTKVR_OK;
}

template <typename T, int SIGHT> int plain_launch(const ctkvr_cache *c, QuantAttnArgs &qa, int log, int opt, hipStream_t st)
{
    AttnArgs &a = qa.a;
    const unsigned grid = (unsigned)((int64_t)a.tiles * c->p.n_kv_heads * a.nsplit);
    TRY(with_opts(opt, [&](auto o) {
        constexpr int kOpt = decltype(o)::value & (SIGHT == kTree ? kCap : ~0);   // (drafted tokens have no distance)
        if constexpr (sizeof(T) == 2) {
            constexpr bool kWide = SIGHT == kTree;   // (tiles of 256 plain rows are slower in windows)
            if (log == 4) tokens_kernel<kPlain, T, kOpt, SIGHT, 1><<<dim3(grid), 256, 0, st>>>(qa);
            else if (log == 5) tokens_kernel<kPlain, T, kOpt, SIGHT, 2><<<dim3(grid), 256, 0, st>>>(qa);
            else if (log == 7) rows_kernel<kPlain, T, kOpt, SIGHT, 4><<<dim3(grid), 256, 0, st>>>(qa);
            else if (!kWide || log != 8) return no_kernel(log);
            if constexpr (kWide) {
                if (log == 8) rows_kernel<kPlain, T, kOpt, SIGHT, 8><<<dim3(grid), 512, 0, st>>>(qa);
            }
        } else {
            if (log == 5) attn_few_kernel<T, kOpt, 2, SIGHT><<<dim3(grid), 128, 0, st>>>(a);
            else if (log == 7) attn_kernel<T, kOpt, 4, SIGHT><<<dim3(grid), 256, 0, st>>>(a);
            else return no_kernel(log);
        }
        return (int)CTKVR_OK;
    }));
    join_launch<T>(c, a, st);
    return launched(SIGHT == kWindow ? "ctkvr_cache_window_attn" : "ctkvr_cache_tree_attn");
}

template <int SIGHT> int attend(const ctkvr_cache *c, const AttnCall &x, const ScoreOpts &o, hipStream_t st)
{
    DeviceScope on(c->dev);
    HIP_TRY(on.err);
    QuantAttnArgs qa{};
    AttnArgs &a = qa.a;
    a.v = view(c, x.table, x.cu, x.cur, x.total);
    a.o = o;
    a.q = x.q;
    a.q_stride = x.q_stride;
    a.k_pages = x.k;
    a.v_pages = x.v;
    a.out = x.out;
    a.lse = x.lse;
    a.part_o = c->part_o;
    a.part_lse = c->part_lse;
    qa.k_scales = x.k_scales;
    qa.v_scales = x.v_scales;
    const int64_t slots = (int64_t)c->p.max_pages * c->p.page_size;
    SightPlan plan = sight_plan(c, x.total, SIGHT == kWindow ? std::min<int64_t>(slots, (int64_t)o.window + o.sinks + x.total) : slots,
                                x.format != CTKVR_KV_PLAIN, SIGHT == kWindow);
    fit_plan(c, x.total, Room{c->part_rows, c->counts}, plan);
    a.tiles = plan.tiles;
    a.nsplit = plan.nsplit;
    a.done = plan.join_inside ? c->done : nullptr;
    const int opt = (c->p.softcap > 0.0f ? kCap : 0) | (o.slopes ? kBias : 0);
    const bool bf16 = c->p.dtype == CTKVR_BF16;
    if (x.format != CTKVR_KV_PLAIN)
        return bf16 ? quant_attn_launch<bf16_t>(c, qa, plan, x.format, SIGHT, opt, st) : quant_attn_launch<float>(c, qa, plan, x.format, SIGHT, opt, st);
    if constexpr (SIGHT != kRange)
        return bf16 ? plain_launch<bf16_t, SIGHT>(c, qa, plan.log, opt, st) : plain_launch<float, SIGHT>(c, qa, plan.log, opt, st);
    return fail(CTKVR_EINVAL, "plain rows are ctkvr_cache_attn's");   // (refused before)
}

}  // namespace

#pragma GCC visibility push(default)
extern "C" {

int ctkvr_cache_quant_append(ctkvr_cache *c, const void *q, int64_t q_stride, const void *k, int64_t k_stride, const void *v, int64_t v_stride,
                             const int32_t *positions, const int32_t *cu_new, const int32_t *cur_lens, const int32_t *block_table, int32_t total,
                             void *q_out, int32_t format, void *k_codes, float *k_scales, void *v_codes, float *v_scales, void *hip_stream)
{
    if (!c) return fail(CTKVR_EINVAL, "cache is NULL");
    TRY(check_tokens(c, total));
    TRY(check_format(format, false));
    if (total == 0) return CTKVR_OK;
    if (!cu_new || !cur_lens || !block_table || !k || !v) return fail(CTKVR_EINVAL, "a required pointer is NULL");
    if (!q != !q_out) return fail(CTKVR_EINVAL, "q and q_out go together");
    if (q) TRY(check_rows(c, "q", q, q_stride, c->p.n_q_heads));
    TRY(check_rows(c, "k", k, k_stride, c->p.n_kv_heads));
    TRY(check_rows(c, "v", v, v_stride, c->p.n_kv_heads));
    TRY(check_codes(format, k_codes, k_scales, "k_codes"));
    TRY(check_codes(format, v_codes, v_scales, "v_codes"));
    if (!aligned16(q_out)) return fail(CTKVR_EINVAL, "q_out must begin on a 16-byte boundary");
    DeviceScope on(c->dev);
    HIP_TRY(on.err);
    QuantAppendArgs a{};
    a.a.v = view(c, block_table, cu_new, cur_lens, total);
    a.a.rope = c->rope;
    a.a.q = q;
    a.a.k = k;
    a.a.val = v;
    a.a.q_stride = q_stride;
    a.a.k_stride = k_stride;
    a.a.v_stride = v_stride;
    a.a.positions = positions;
    a.a.q_out = q_out;
    a.k = QuantRows{(uint8_t *)k_codes, k_scales};
    a.v = QuantRows{(uint8_t *)v_codes, v_scales};
    const int share = total <= 2 * c->num_cu ? 4 : 2;   // (waves a token; of 1024, 2048, 4096, 8192 tokens one, two, four 15.5, 13.7, 13.6; 19.4, 18.0, 20.0; 28.4, 29.2, 30.8; 52, 49, 52 us)
    const dim3 grid((unsigned)(((int64_t)total * share + 3) / 4));
    hipStream_t st = (hipStream_t)hip_stream;
    if (c->p.dtype == CTKVR_BF16) {
        if (format == CTKVR_KV_INT8) quant_append_kernel<bf16_t, kInt8><<<grid, 256, 0, st>>>(a, share);
        else quant_append_kernel<bf16_t, kFp8><<<grid, 256, 0, st>>>(a, share);
    } else {
        if (format == CTKVR_KV_INT8) quant_append_kernel<float, kInt8><<<grid, 256, 0, st>>>(a, share);
        else quant_append_kernel<float, kFp8><<<grid, 256, 0, st>>>(a, share);
    }
    return launched("ctkvr_cache_quant_append");
}

int ctkvr_cache_quant_read(ctkvr_cache *c, int32_t format, const void *k_codes, const float *k_scales, const void *v_codes, const float *v_scales,
                           const int32_t *first_tokens, const int32_t *cur_lens, const int32_t *block_table, const int32_t *out_table, int32_t out_max_pages,
                           int32_t out_num_pages, void *k_pages, void *v_pages, void *hip_stream)
{
    if (!c) return fail(CTKVR_EINVAL, "cache is NULL");
    TRY(check_format(format, false));
    if (!cur_lens || !block_table || !out_table) return fail(CTKVR_EINVAL, "a required pointer is NULL");
    if (!k_pages && !v_pages) return fail(CTKVR_EINVAL, "neither k_pages nor v_pages");
    if (k_pages) TRY(check_codes(format, k_codes, k_scales, "k_codes"));
    if (v_pages) TRY(check_codes(format, v_codes, v_scales, "v_codes"));
    if (!aligned16(k_pages) || !aligned16(v_pages)) return fail(CTKVR_EINVAL, "pages must begin on 16-byte boundaries");
    if (out_num_pages < 1 || out_max_pages < 1 || (int64_t)out_max_pages * c->p.page_size > (1 << 20))
        return fail(CTKVR_EINVAL, "out_num_pages %d, out_max_pages %d: at least 1, sequences of 2^20 tokens at most", out_num_pages, out_max_pages);
    DeviceScope on(c->dev);
    HIP_TRY(on.err);
    QuantReadArgs a{};
    a.v = view(c, block_table, nullptr, cur_lens, 0);
    a.first = first_tokens;
    if (k_pages) {
        a.codes[0] = (const uint8_t *)k_codes;
        a.scales[0] = k_scales;
        a.out[0] = k_pages;
    }
    if (v_pages) {
        a.codes[1] = (const uint8_t *)v_codes;
        a.scales[1] = v_scales;
        a.out[1] = v_pages;
    }
    a.out_table = out_table;
    a.out_cols = out_max_pages;
    a.out_pages = (uint32_t)out_num_pages;
    // (a run of 64 tokens a block, up to 16 blocks a CU; the rest of a wide table goes round)
    const int64_t units = (int64_t)c->p.batch * c->p.n_kv_heads, most = (int64_t)std::min(c->p.max_pages, out_max_pages) * c->p.page_size;
    const dim3 grid((unsigned)units, (unsigned)std::max<int64_t>(1, std::min<int64_t>((most + 63) / 64, 16ll * c->num_cu / units)));
    hipStream_t st = (hipStream_t)hip_stream;
    if (c->p.dtype == CTKVR_BF16) {
        if (format == CTKVR_KV_INT8) quant_read_kernel<bf16_t, kInt8><<<grid, 256, 0, st>>>(a);
        else quant_read_kernel<bf16_t, kFp8><<<grid, 256, 0, st>>>(a);
    } else {
        if (format == CTKVR_KV_INT8) quant_read_kernel<float, kInt8><<<grid, 256, 0, st>>>(a);
        else quant_read_kernel<float, kFp8><<<grid, 256, 0, st>>>(a);
    }
    return launched("ctkvr_cache_quant_read");
}

int ctkvr_cache_quant_attn(ctkvr_cache *c, const void *q, int64_t q_stride, int32_t format, const void *k_codes, const float *k_scales, const void *v_codes,
                           const float *v_scales, const int32_t *cu_new, const int32_t *cur_lens, const int32_t *block_table, int32_t total,
                           const float *slopes, const int32_t *prefix_lens, const int32_t *first_key, void *out, float *out_lse, void *hip_stream)
{
    if (!c) return fail(CTKVR_EINVAL, "cache is NULL");
    TRY(check_tokens(c, total));
    TRY(check_format(format, false));
    if (total == 0) return CTKVR_OK;
    const AttnCall x{q, q_stride, format, k_codes, k_scales, v_codes, v_scales, cu_new, cur_lens, block_table, total, out, out_lse};
    TRY(check_attn(c, x));
    return attend<kRange>(c, x, score_opts(c, slopes, prefix_lens, first_key), (hipStream_t)hip_stream);
}

int ctkvr_cache_window_attn(ctkvr_cache *c, const void *q, int64_t q_stride, int32_t format, const void *k_pages, const float *k_scales, const void *v_pages,
                            const float *v_scales, const int32_t *cu_new, const int32_t *cur_lens, const int32_t *block_table, int32_t total, int32_t window,
                            int32_t n_sink, const float *slopes, void *out, float *out_lse, void *hip_stream)
{
    if (!c) return fail(CTKVR_EINVAL, "cache is NULL");
    TRY(check_tokens(c, total));
    TRY(check_format(format, true));
    if (window < 1 || n_sink < 0) return fail(CTKVR_EINVAL, "window %d, n_sink %d: at least 1 and 0", window, n_sink);
    if (total == 0) return CTKVR_OK;
    const AttnCall x{q, q_stride, format, k_pages, k_scales, v_pages, v_scales, cu_new, cur_lens, block_table, total, out, out_lse};
    TRY(check_attn(c, x));
    ScoreOpts o = score_opts(c, slopes, nullptr, nullptr);
    o.window = std::min(window, 1 << 30);   // (slots are below that, also those beyond the table)
    o.sinks = std::min(n_sink, 1 << 20);
    return attend<kWindow>(c, x, o, (hipStream_t)hip_stream);
}

int ctkvr_cache_tree_attn(ctkvr_cache *c, const void *q, int64_t q_stride, int32_t format, const void *k_pages, const float *k_scales, const void *v_pages,
                          const float *v_scales, const int32_t *cu_new, const int32_t *cur_lens, const int32_t *block_table, int32_t total,
                          const uint32_t *tree_mask, int32_t mask_words, const int32_t *first_key, void *out, float *out_lse, void *hip_stream)
{
    if (!c) return fail(CTKVR_EINVAL, "cache is NULL");
    TRY(check_tokens(c, total));
    TRY(check_format(format, true));
    if (mask_words < 1 || mask_words > (1 << 15)) return fail(CTKVR_EINVAL, "mask_words %d outside 1..2^15", mask_words);
    if (total == 0) return CTKVR_OK;
    const AttnCall x{q, q_stride, format, k_pages, k_scales, v_pages, v_scales, cu_new, cur_lens, block_table, total, out, out_lse};
    TRY(check_attn(c, x));
    if (!tree_mask || ((uintptr_t)tree_mask & 3)) return fail(CTKVR_EINVAL, "tree_mask: NULL, or not on a 4-byte boundary");
    ScoreOpts o = score_opts(c, nullptr, nullptr, first_key);
    o.drafts = tree_mask;
    o.words = mask_words;
    return attend<kTree>(c, x, o, (hipStream_t)hip_stream);
}

}  // extern "C"
#pragma GCC visibility pop
