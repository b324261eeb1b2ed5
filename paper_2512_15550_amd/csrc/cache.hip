// The operators on the paged KV cache: the host side of their part of the C ABI, and their kernels.
#include <new>

#include "cache_host.hpp"
#include "sight_plan.hpp"

using namespace ctkvr;

namespace {

int check_cache_params(const ctkvr_cache_params *p)
{
    if (!p) return fail(CTKVR_EINVAL, "params is NULL");
    if (p->batch < 1 || p->n_q_heads < 1 || p->n_kv_heads < 1) return fail(CTKVR_EINVAL, "batch/heads must be >= 1");
    if (p->n_q_heads % p->n_kv_heads) return fail(CTKVR_EINVAL, "n_q_heads %% n_kv_heads != 0");
    if (p->head_dim != 128) return fail(CTKVR_EUNSUPPORTED, "head_dim %d: only 128 is supported", p->head_dim);
    const int G = p->n_q_heads / p->n_kv_heads;
    if (G != 1 && G != 2 && G != 4 && G != 8) return fail(CTKVR_EUNSUPPORTED, "group size %d: only 1, 2, 4, 8", G);
    if (p->dtype != CTKVR_F32 && p->dtype != CTKVR_BF16) return fail(CTKVR_EINVAL, "unknown dtype %d", p->dtype);
    if (p->page_size < 1 || p->page_size > 256 || (p->page_size & (p->page_size - 1)))
        return fail(CTKVR_EUNSUPPORTED, "page_size %d: powers of two up to 256", p->page_size);
    if (p->num_pages < 1 || p->max_pages < 1 || p->max_new < 1) return fail(CTKVR_EINVAL, "num_pages, max_pages and max_new must be >= 1");
    if ((int64_t)p->max_pages * p->page_size > (1 << 20))
        return fail(CTKVR_EUNSUPPORTED, "max_pages %d of %d tokens: sequences of 2^20 tokens at most", p->max_pages, p->page_size);
    if (p->max_new > (1 << 20) || p->batch > (1 << 16) || p->n_q_heads > (1 << 10))
        return fail(CTKVR_EUNSUPPORTED, "max_new %d, batch %d, n_q_heads %d: at most 2^20, 2^16, 2^10", p->max_new, p->batch, p->n_q_heads);
    // A launch has fewer than 2^32 threads a dimension.  Units (a sequence's KV head) are one of weights and eviction, of up to 1024 threads; attention's blocks
    // of 256 are max_new * n_q_heads / 128 + units at most, or three a unit, and those of split keys a few a CU.
    if ((int64_t)p->batch * p->n_kv_heads >= 1 << 22)
        return fail(CTKVR_EUNSUPPORTED, "%d sequences of %d KV heads: fewer than 2^22 together", p->batch, p->n_kv_heads);
    if ((int64_t)p->num_pages * p->page_size * p->n_kv_heads >= 0xffffffffll)
        return fail(CTKVR_EUNSUPPORTED, "%d pages: a cache of 2^32 - 2 rows at most", p->num_pages);
    if ((((int64_t)p->max_pages * p->page_size + 127) / 128) * p->batch * p->n_kv_heads >= (1ll << 31))
        return fail(CTKVR_EUNSUPPORTED, "%d sequences of %d pages: too large a batch", p->batch, p->max_pages);
    if (!(p->sm_scale >= 0.0f && p->sm_scale <= 1e15f)) return fail(CTKVR_EINVAL, "sm_scale must be 0 to 1e15");
    // (so that its products with the scale and with the convergent's constants are finite)
    if (!(p->softcap == 0.0f || (p->softcap >= 1e-6f && p->softcap <= 1e15f))) return fail(CTKVR_EINVAL, "softcap must be 0, or 1e-6 to 1e15");
    if (!p->rope_freq && !(p->rope_base > 0.0 && !std::isinf(p->rope_base))) return fail(CTKVR_EINVAL, "rope_base must be finite and > 0");
    for (int i = 0; i < 64; ++i) {
        if (p->rope_freq && !std::isfinite(p->rope_freq[i])) return fail(CTKVR_EINVAL, "rope_freq[%d] is not finite", i);
        if (p->rope_axis && p->rope_axis[i] > 2) return fail(CTKVR_EINVAL, "rope_axis[%d] = %d: axes are 0, 1 and 2", i, p->rope_axis[i]);
    }
    return CTKVR_OK;
}

template <typename T> int attn_launch(const ctkvr_cache *c, AttnArgs &a, bool few, int opt, hipStream_t st)
{
    const unsigned grid = (unsigned)((int64_t)a.tiles * c->p.n_kv_heads * a.nsplit);
    with_opts(opt, [&](auto o) {
        constexpr int kOpt = decltype(o)::value, kFew = sizeof(T) == 2 ? 4 : 2;
        if (few) attn_few_kernel<T, kOpt, kFew><<<dim3(grid), 64 * kFew, 0, st>>>(a);
        else attn_kernel<T, kOpt, 4><<<dim3(grid), 256, 0, st>>>(a);
        return 0;
    });
    join_launch<T>(c, a, st);
    return launched("ctkvr_cache_attn");
}
template <typename T> int weights_launch(const ctkvr_cache *c, WeightArgs &a, int opt, hipStream_t st)
{
    const int64_t keys = (int64_t)c->p.max_pages * c->p.page_size, units = (int64_t)c->p.batch * c->p.n_kv_heads;
    // Rows that fit a block's shared memory once or twice: keys go past them.  More rows: they go past the keys.
    const int held = 65536 / (128 * (int)sizeof(T)), used = std::max(1, std::min(a.v.total, c->p.batch));
    if (((int64_t)a.v.total << c->lg) <= 2ll * held * used) {
        a.nsplit = (int)std::max<int64_t>(1, std::min<int64_t>((c->p.batch > 1 ? 8 : 2) * c->num_cu / units, (keys + 127) / 128));
        with_opts(opt, [&](auto o) {
            weights_few_kernel<T, decltype(o)::value><<<dim3((unsigned)units, (unsigned)a.nsplit), 256, 0, st>>>(a);
            return 0;
        });
    } else {
        // (rows go past 256 keys of a block, 128 in fp32, unless that leaves CUs without one)
        constexpr int kWide = sizeof(T) == 2 ? 256 : 128;
        const unsigned wide = (unsigned)((keys + kWide - 1) / kWide), narrow = (unsigned)((keys + kWide / 4 - 1) / (kWide / 4));
        with_opts(opt, [&](auto o) {
            if (wide * units >= c->num_cu) weights_kernel<T, decltype(o)::value><<<dim3((unsigned)units, wide), 512, 0, st>>>(a);
            else weights_rows_kernel<T, decltype(o)::value><<<dim3((unsigned)units, narrow), 512, 0, st>>>(a);
            return 0;
        });
    }
    return launched("ctkvr_cache_weights");
}

}  // namespace

#pragma GCC visibility push(default)
extern "C" {

int ctkvr_cache_create(const ctkvr_cache_params *p, void *hip_stream, ctkvr_cache **out_cache)
{
    if (!out_cache) return fail(CTKVR_EINVAL, "out_cache is NULL");
    *out_cache = nullptr;
    TRY(check_cache_params(p));
    ctkvr_cache *c = new (std::nothrow) ctkvr_cache();
    if (!c) return fail(CTKVR_ENOMEM, "host allocation failed");
    if (hipGetDevice(&c->dev) != hipSuccess) {
        delete c;
        return fail(CTKVR_EHIP, "no current device");
    }
    c->p = *p;
    c->p.rope_freq = nullptr;
    c->p.rope_axis = nullptr;
    c->G = p->n_q_heads / p->n_kv_heads;
    c->lg = __builtin_ctz(c->G);
    c->page_shift = __builtin_ctz(p->page_size);
    c->scale = p->sm_scale > 0.0f ? p->sm_scale : (float)(1.0 / sqrt(128.0));
    int cus = 0;
    if (hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, c->dev) == hipSuccess && cus > 0) c->num_cu = cus;
    for (int i = 0; i < 64; ++i) {
        c->rope.turn[i] = turn_of(p->rope_freq ? (long double)p->rope_freq[i] : rope_freq(p->rope_base, i));
        c->rope.axis[i] = p->rope_axis ? p->rope_axis[i] : 0;
        c->axes = std::max(c->axes, c->rope.axis[i] + 1);
    }
    // for the largest product of rows and runs that a call may take, and its tiles
    Room room = sight_room(c);
    for (int total = 1; total <= p->max_new; ++total) {
        const AttnPlan plan = attn_plan(c, total);
        if (plan.nsplit == 1 && (((int64_t)total << c->lg) >> 7) * p->n_kv_heads >= 8ll * c->num_cu) break;   // more tokens are never split again
        if (plan.nsplit == 1) continue;
        room.rows = std::max(room.rows, (size_t)plan.nsplit * total * p->n_q_heads);
        room.counts = std::max(room.counts, (size_t)plan.tiles * p->n_kv_heads);
    }
    c->part_rows = room.rows;
    c->counts = room.counts;
    if (room.rows) {
        int rc = pool_get(c->dev, (room.rows * 129 + room.counts) * 4, 4, &c->mem);
        if (rc == CTKVR_OK) {
            c->part_o = (float *)c->mem.base;
            c->part_lse = c->part_o + room.rows * 128;
            c->done = (uint32_t *)(c->part_lse + room.rows);
            hipStream_t st = (hipStream_t)hip_stream;
            cache_clear_kernel<<<dim3((unsigned)((room.counts + 255) / 256)), 256, 0, st>>>(c->done, room.counts);
            rc = launched("ctkvr_cache_create");
            const hipError_t e = hipStreamSynchronize(st);
            if (rc == CTKVR_OK && e != hipSuccess) rc = fail(CTKVR_EHIP, "ctkvr_cache_create: %s", hipGetErrorString(e));
        }
        if (rc != CTKVR_OK) {
            delete c;
            return rc;
        }
    }
    *out_cache = c;
    return CTKVR_OK;
}

void ctkvr_cache_free(ctkvr_cache *c)
{
    delete c;   // synchronises its device
}

int ctkvr_cache_append(ctkvr_cache *c, const void *q, int64_t q_stride, const void *k, int64_t k_stride, const void *v, int64_t v_stride,
                       const int32_t *positions, const int32_t *cu_new, const int32_t *cur_lens, const int32_t *block_table, int32_t total,
                       void *q_out, void *k_pages, void *v_pages, void *hip_stream)
{
    if (!c) return fail(CTKVR_EINVAL, "cache is NULL");
    TRY(check_tokens(c, total));
    if (total == 0) return CTKVR_OK;
    if (!cu_new || !cur_lens || !block_table) return fail(CTKVR_EINVAL, "a required pointer is NULL");
    if (!q != !q_out) return fail(CTKVR_EINVAL, "q and q_out go together");
    if (!k != !v || (k && (!k_pages || !v_pages))) return fail(CTKVR_EINVAL, "k, v, k_pages and v_pages go together");
    if (!q && !k) return fail(CTKVR_EINVAL, "neither q nor k and v");
    if (q) TRY(check_rows(c, "q", q, q_stride, c->p.n_q_heads));
    if (k) TRY(check_rows(c, "k", k, k_stride, c->p.n_kv_heads));
    if (k) TRY(check_rows(c, "v", v, v_stride, c->p.n_kv_heads));
    if (!aligned16(q_out) || !aligned16(k_pages) || !aligned16(v_pages)) return fail(CTKVR_EINVAL, "outputs must begin on 16-byte boundaries");
    DeviceScope on(c->dev);
    HIP_TRY(on.err);
    AppendArgs a{};
    a.v = view(c, block_table, cu_new, cur_lens, total);
    a.rope = c->rope;
    a.q = q;
    a.k = k;
    a.val = v;
    a.q_stride = q_stride;
    a.k_stride = k_stride;
    a.v_stride = v_stride;
    a.positions = positions;
    a.q_out = q_out;
    a.k_pages = k_pages;
    a.v_pages = v_pages;
    const unsigned grid = (unsigned)((total + 3) / 4);
    if (c->p.dtype == CTKVR_BF16) append_kernel<bf16_t><<<dim3(grid), 256, 0, (hipStream_t)hip_stream>>>(a);
    else append_kernel<float><<<dim3(grid), 256, 0, (hipStream_t)hip_stream>>>(a);
    return launched("ctkvr_cache_append");
}

int ctkvr_cache_attn(ctkvr_cache *c, const void *q, int64_t q_stride, const void *k_pages, const void *v_pages, const int32_t *cu_new,
                     const int32_t *cur_lens, const int32_t *block_table, int32_t total, const float *slopes, const int32_t *prefix_lens,
                     const int32_t *first_key, void *out, float *out_lse, void *hip_stream)
{
    if (!c) return fail(CTKVR_EINVAL, "cache is NULL");
    TRY(check_tokens(c, total));
    if (total == 0) return CTKVR_OK;
    if (!q || !k_pages || !v_pages || !cu_new || !cur_lens || !block_table || !out) return fail(CTKVR_EINVAL, "a required pointer is NULL");
    TRY(check_rows(c, "q", q, q_stride, c->p.n_q_heads));
    if (!aligned16(k_pages) || !aligned16(v_pages) || !aligned16(out)) return fail(CTKVR_EINVAL, "pages and outputs must begin on 16-byte boundaries");
    DeviceScope on(c->dev);
    HIP_TRY(on.err);
    AttnArgs a{};
    a.v = view(c, block_table, cu_new, cur_lens, total);
    a.o = score_opts(c, slopes, prefix_lens, first_key);
    a.q = q;
    a.q_stride = q_stride;
    a.k_pages = k_pages;
    a.v_pages = v_pages;
    a.out = out;
    a.lse = out_lse;
    a.part_o = c->part_o;
    a.part_lse = c->part_lse;
    const AttnPlan plan = attn_plan(c, total);
    a.tiles = plan.tiles;
    a.nsplit = plan.nsplit;
    a.done = plan.join_inside ? c->done : nullptr;
    const int opt = (c->p.softcap > 0.0f ? kCap : 0) | (slopes ? kBias : 0);
    return c->p.dtype == CTKVR_BF16 ? attn_launch<bf16_t>(c, a, plan.few, opt, (hipStream_t)hip_stream)
                                    : attn_launch<float>(c, a, plan.few, opt, (hipStream_t)hip_stream);
}

int ctkvr_cache_weights(ctkvr_cache *c, const void *q, int64_t q_stride, const float *lse, const void *k_pages, const int32_t *cu_new,
                        const int32_t *cur_lens, const int32_t *block_table, int32_t total, const float *slopes, const int32_t *prefix_lens,
                        const int32_t *first_key, float decay, const float *weights_in, float *weights_out, int32_t weights_stride,
                        void *hip_stream)
{
    if (!c) return fail(CTKVR_EINVAL, "cache is NULL");
    TRY(check_tokens(c, total));
    if ((total && (!q || !lse)) || !k_pages || !cu_new || !cur_lens || !block_table || !weights_out) return fail(CTKVR_EINVAL, "a required pointer is NULL");
    if (total) TRY(check_rows(c, "q", q, q_stride, c->p.n_q_heads));
    if (!aligned16(k_pages)) return fail(CTKVR_EINVAL, "pages must begin on 16-byte boundaries");
    if (weights_stride < c->p.max_pages * c->p.page_size)
        return fail(CTKVR_EINVAL, "weights_stride %d < %d tokens of a table's row", weights_stride, c->p.max_pages * c->p.page_size);
    if (!std::isfinite(decay)) return fail(CTKVR_EINVAL, "decay is not finite");
    DeviceScope on(c->dev);
    HIP_TRY(on.err);
    WeightArgs a{};
    a.v = view(c, block_table, cu_new, cur_lens, total);
    a.o = score_opts(c, slopes, prefix_lens, first_key);
    a.q = q;
    a.q_stride = q_stride;
    a.lse = lse;
    a.k_pages = k_pages;
    a.w_in = weights_in;
    a.w_out = weights_out;
    a.w_stride = weights_stride;
    a.decay = decay;
    const int opt = (c->p.softcap > 0.0f ? kCap : 0) | (slopes ? kBias : 0);
    return c->p.dtype == CTKVR_BF16 ? weights_launch<bf16_t>(c, a, opt, (hipStream_t)hip_stream)
                                    : weights_launch<float>(c, a, opt, (hipStream_t)hip_stream);
}

int ctkvr_cache_evict(ctkvr_cache *c, const float *weights_in, int32_t weights_stride, const int32_t *cur_lens, const int32_t *block_table,
                      int32_t budget, int32_t n_init, int32_t n_local, void *k_pages, void *v_pages, float *weights_out, int32_t *out_ids,
                      int32_t *out_lens, void *hip_stream)
{
    if (!c) return fail(CTKVR_EINVAL, "cache is NULL");
    if (!weights_in || !cur_lens || !block_table || !k_pages || !v_pages || !out_ids) return fail(CTKVR_EINVAL, "a required pointer is NULL");
    if (weights_stride < c->p.max_pages * c->p.page_size)
        return fail(CTKVR_EINVAL, "weights_stride %d < %d tokens of a table's row", weights_stride, c->p.max_pages * c->p.page_size);
    if (budget < 1 || budget > (1 << 20)) return fail(CTKVR_EINVAL, "budget %d outside 1..2^20", budget);
    if (n_init < 0 || n_local < 0 || (int64_t)n_init + n_local > budget)
        return fail(CTKVR_EINVAL, "n_init %d and n_local %d: not negative, and budget %d at most together", n_init, n_local, budget);
    if (!aligned16(k_pages) || !aligned16(v_pages)) return fail(CTKVR_EINVAL, "pages must begin on 16-byte boundaries");
    const bool lens_in_place = out_lens == cur_lens;
    const uintptr_t cur0 = (uintptr_t)cur_lens, lens0 = (uintptr_t)out_lens, lens_bytes = (uintptr_t)c->p.batch * 4;
    if (out_lens && !lens_in_place && cur0 < lens0 + lens_bytes && lens0 < cur0 + lens_bytes)
        return fail(CTKVR_EINVAL, "out_lens overlaps cur_lens: it may be cur_lens, or none of it");
    DeviceScope on(c->dev);
    HIP_TRY(on.err);
    EvictArgs a{};
    a.v = view(c, block_table, nullptr, cur_lens, 0);
    a.w_in = weights_in;
    a.w_out = weights_out;
    a.w_stride = weights_stride;
    a.budget = budget;
    a.n_init = n_init;
    a.n_local = n_local;
    a.ids = out_ids;
    a.lens = lens_in_place ? nullptr : out_lens;
    a.k_pages = k_pages;
    a.v_pages = v_pages;
    const int units = c->p.batch * c->p.n_kv_heads, keys = c->p.max_pages * c->p.page_size;
    hipStream_t st = (hipStream_t)hip_stream;
    // (a thread holds the ranks of so many keys of the longest sequence that the table has room for)
    if (keys <= 8192) evict_select_kernel<8><<<dim3((unsigned)units), 1024, 0, st>>>(a);
    else if (keys <= 32768) evict_select_kernel<32><<<dim3((unsigned)units), 1024, 0, st>>>(a);
    else if (keys <= 65536) evict_select_kernel<64><<<dim3((unsigned)units), 1024, 0, st>>>(a);
    else evict_select_kernel<0><<<dim3((unsigned)units), 1024, 0, st>>>(a);
    // Slices of 128 bytes, a line, and down to 32 while every block still has a CU.  8 / 32 / 128 units of 4096 or 5000 kept rows, us, with
    // slices of 128, 64, 32 and 16 bytes: 19.0, 12.5, 11.6, 14.1 / 29.1, 26.2, 33.6, 55.0 / 44.4, 45.3, 86.5, 191.
    const int pieces = c->p.dtype == CTKVR_BF16 ? 32 : 64;
    a.slices = pieces / 8;
    while (a.slices < pieces / 2 && 2 * units * a.slices <= c->num_cu) a.slices *= 2;
    if (c->p.dtype == CTKVR_BF16) evict_move_kernel<bf16_t><<<dim3((unsigned)units, (unsigned)a.slices), 1024, 0, st>>>(a);
    else evict_move_kernel<float><<<dim3((unsigned)units, (unsigned)a.slices), 1024, 0, st>>>(a);
    if (lens_in_place) {   // (every block above reads the lengths as they were)
        a.lens = out_lens;
        evict_lens_kernel<<<dim3((unsigned)((c->p.batch + 255) / 256)), 256, 0, st>>>(a);
    }
    return launched("ctkvr_cache_evict");
}

}  // extern "C"
#pragma GCC visibility pop
