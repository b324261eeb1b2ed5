// How attention over 8-bit rows, in windows and of drafted tokens falls into blocks.
#pragma once
#include <stdlib.h>

#include "cache_host.hpp"

namespace ctkvr {

// How a call's rows and keys fall into blocks: tiles of 16, 32 or 128 rows
struct SightPlan {
    int log;   // of a tile's rows
    int tiles, nsplit;
    bool join_inside;
};
// keys: those that a row may see, at most
inline SightPlan sight_plan(const ctkvr_cache *c, int total, int64_t keys, bool codes)
{
    const int64_t rows = (int64_t)total << c->lg, g = c->p.n_kv_heads, cus = c->num_cu;
    const int used = std::min(total, c->p.batch);   // sequences with new tokens, at most
    const bool bf16 = c->p.dtype == CTKVR_BF16;
    // a sequence's rows are a multiple of the group's size, so that rounding each up to tiles adds no more than that
    auto tiles = [&](int log) { return (rows + used * (int64_t)((1 << log) - c->G)) >> log; };
    SightPlan p{};
    p.log = rows <= 16ll * used && (bf16 || codes) ? 4 : rows <= 64ll * used || (tiles(7) * g < cus && (!bf16 || keys < 4096 || rows < 512ll * used)) ? 5 : 7;
    if (const char *e = getenv("SP_LOG")) p.log = atoi(e);
    p.tiles = (int)tiles(p.log);
    const bool few = p.log < 7, enough = tiles(5) >= 2 * used && tiles(5) * g >= cus / 2;
    int64_t want = (!few ? 2 : used > 1 ? 8 : bf16 ? 1 : 2) * cus, least = !few ? 1024 : enough ? 2048 : bf16 ? 256 : 64;
    if (const char *e = getenv("SP_WANT")) want = atoi(e) * cus;
    if (const char *e = getenv("SP_LEAST")) least = atoi(e);
    p.nsplit = few || tiles(7) * g < cus ? (int)std::max<int64_t>(1, std::min({want / (p.tiles * g), (keys + least - 1) / least, (int64_t)kMaxSplit})) : 1;
    p.join_inside = few && used == 1 && rows <= 8 && rows * p.nsplit <= (bf16 ? 256 : 128);
    if (const char *e = getenv("SP_JOIN")) p.join_inside = atoi(e) && few;
    return p;
}

}  // namespace ctkvr
