// What the host sides of the cache operators share: the handle, checks of arguments, how attention falls into blocks.
#pragma once
#include "../../include/ctkvr.h"

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "cache.hpp"
#include "host.hpp"

struct ctkvr_cache {
    ctkvr_cache_params p{};
    int G = 0, lg = 0, page_shift = 0, dev = 0, num_cu = 256;
    float scale = 0.f;
    ctkvr::RopeTable rope{};
    int axes = 1;
    ctkvr::PoolBlock mem{nullptr, 0};   // the workspace: a split attention's partial outputs, their log-sum-exps, and a count for each tile
    float *part_o = nullptr, *part_lse = nullptr;
    uint32_t *done = nullptr;
    size_t part_rows = 0, counts = 0;   // what there is room for

    ~ctkvr_cache()
    {
        ctkvr::DeviceScope on(dev);
        ctkvr::pool_put(dev, mem, on.err == hipSuccess && ctkvr::device_idle());
    }
};

namespace ctkvr {

constexpr int kMaxSplit = 128;

inline bool aligned16(const void *p) { return ((uintptr_t)p & 15) == 0; }

inline CacheView view(const ctkvr_cache *c, const int32_t *table, const int32_t *cu, const int32_t *cur, int total)
{
    CacheView v{};
    v.table = table;
    v.cu = cu;
    v.cur = cur;
    v.batch = c->p.batch;
    v.h = c->p.n_q_heads;
    v.g = c->p.n_kv_heads;
    v.lg = c->lg;
    v.page_shift = c->page_shift;
    v.max_pages = c->p.max_pages;
    v.total = total;
    v.num_pages = (uint32_t)c->p.num_pages;
    return v;
}

inline ScoreOpts score_opts(const ctkvr_cache *c, const float *slopes, const int32_t *prefix, const int32_t *first)
{
    ScoreOpts o{};
    o.slopes = slopes;
    o.prefix = prefix;
    o.first = first;
    o.c2 = c->scale * kLog2e;
    if (c->p.softcap > 0.0f) {
        o.cap_in = c->scale / c->p.softcap;
        o.cap_out = c->p.softcap * kLog2e;
        o.cap_105 = o.cap_out * 105.0f;
        o.cap_945 = o.cap_out * 945.0f;
    }
    return o;
}

inline int check_tokens(const ctkvr_cache *c, int total)
{
    if (total < 0 || total > c->p.max_new) return fail(CTKVR_EINVAL, "total %d outside 0..max_new = %d", total, c->p.max_new);
    return CTKVR_OK;
}
inline int check_rows(const ctkvr_cache *c, const char *name, const void *p, int64_t stride, int heads)
{
    const int64_t unit = c->p.dtype == CTKVR_BF16 ? 8 : 4;
    if (!aligned16(p) || stride % unit) return fail(CTKVR_EINVAL, "%s: rows must begin on 16-byte boundaries", name);
    if (stride < (int64_t)heads * 128 || stride > (1 << 30)) return fail(CTKVR_EINVAL, "%s: stride %lld outside %d..2^30", name, (long long)stride, heads * 128);
    return CTKVR_OK;
}

// How a call's rows and keys fall into blocks.
//   Tiles of 128 rows read a key once for all of them; tiles of 32, whose keys a block's waves share out, where 128 would be mostly empty (64 rows a unit), and
// where those would leave CUs without a block, unless the keys are many and the rows are too: 574 tokens of 8 heads a KV head on 13K keys 67 us with 128 rows a block
// and the keys split, 101 with 32; but up to 122 tokens of 4 heads 45 and 30, and in fp32, where a row more is a row's products more, 42 tokens 64 and 31.
//   Keys are split into runs where blocks would be too few: to a block a CU for one sequence in bf16, two in fp32 (500 tokens on 2 KV heads 36 -> 27 us), eight for
// several, whose lengths differ.  A run has 256 keys at least, 64 in fp32, but 2048 where a unit has several tiles and they fill half the chip by
// themselves: 93 tokens on 520 keys, two sequences, 23 us in three runs and 17 in one.
//   The runs' outputs are joined by the block that ends last where it has little to read, by a launch of its own otherwise.  One token of 32 heads on 32K keys 31.6
// and 32.6 us, and 6.6 and 10.4 where a document leaves one run; but 29 tokens on 856 keys 19.2 and 14.3, 2 tokens of 8 heads a KV head on 3769 keys in fp32 40 and 22,
// one token of 13 sequences 33.0 and 31.1.
struct AttnPlan {
    bool few, join_inside;
    int tiles, nsplit;
};
inline AttnPlan attn_plan(const ctkvr_cache *c, int total)
{
    const int64_t rows = (int64_t)total << c->lg, keys = (int64_t)c->p.max_pages * c->p.page_size, g = c->p.n_kv_heads, cus = c->num_cu;
    const int used = std::min(total, c->p.batch);   // sequences with new tokens, at most
    const bool bf16 = c->p.dtype == CTKVR_BF16;
    AttnPlan p{};
    const int64_t wide = (rows >> 7) + used, narrow = (rows >> 5) + used;
    p.few = rows <= 64ll * used || (wide * g < cus && (!bf16 || keys < 4096 || rows < 512ll * used));
    p.tiles = (int)(p.few ? narrow : wide);
    const bool enough = narrow >= 2 * used && narrow * g >= cus / 2;
    const int64_t want = (!p.few ? 2 : used > 1 ? 8 : bf16 ? 1 : 2) * cus, least = !p.few ? 1024 : enough ? 2048 : bf16 ? 256 : 64;
    p.nsplit = p.few || wide * g < cus ? (int)std::max<int64_t>(1, std::min({want / (p.tiles * g), (keys + least - 1) / least, (int64_t)kMaxSplit})) : 1;
    p.join_inside = p.few && used == 1 && rows <= 8 && rows * p.nsplit <= (bf16 ? 256 : 128);
    return p;
}

template <typename F> int with_opts(int opt, F f)
{
    switch (opt) {
        case 0: return f(std::integral_constant<int, 0>());
        case kCap: return f(std::integral_constant<int, kCap>());
        case kBias: return f(std::integral_constant<int, kBias>());
        default: return f(std::integral_constant<int, kCap | kBias>());
    }
}
inline int launched(const char *what)
{
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? CTKVR_OK : fail(CTKVR_EHIP, "%s: %s", what, hipGetErrorString(e));
}

// the runs of a split attention, where they are not joined by its own blocks
template <typename T> void join_launch(const ctkvr_cache *c, AttnArgs &a, hipStream_t st)
{
    if (a.nsplit == 1 || a.done) return;
    const unsigned rows = (unsigned)((int64_t)a.v.total * c->p.n_q_heads);
    if (a.nsplit >= 8) attn_join_kernel<T, 8><<<dim3(rows), 256, 0, st>>>(a);
    else attn_join_kernel<T, 1><<<dim3((rows + 7) / 8), 256, 0, st>>>(a);
}

}  // namespace ctkvr
