// How attention over 8-bit rows, in windows and of drafted tokens falls into blocks.
#pragma once
#include "cache_host.hpp"

namespace ctkvr {

// How a call's rows and keys fall into blocks: tiles of 16, 32, 128 or 256 rows.  us, in that order, 32 heads on 8 KV heads in bf16:
//   Up to 16 rows a unit take tiles of 16.  More take tiles of 128 where these fill the chip (2048 tokens on as many keys 129, 87, 69; four sequences of 300 in a
// window of 1024 106, 65, 48) and where the keys are long enough to be split and the rows enough (one sequence's 16 / 32 tokens on 32K codes 40, 35, 44 / 68, 52, 48;
// 64 rows a unit of eight sequences, codes 120 and 149, plain 180 and 161); else those of 32 (500 tokens on as many keys 20, 15, 23), or of 16 where that leaves half the
// CUs idle (on 2 KV heads 11, 15, 23).
//   Over codes, and for several drafts over plain rows, long keys or twice as many tiles as CUs make it 256 rows in place of 128 where a sequence has more than that: a block
// of 8 waves has a CU for itself and converts and reads a key for twice as many rows (codes: 2048 tokens on 32K keys 1243 -> 1146, 1024 849 -> 596, which are split then,
// 512 353 -> 319, 33 62 -> 54, 4096 on themselves 199 -> 176, four sequences of 300 on 8K to 64K 1555 -> 652, split, eight drafts of 64 on 32K 443 -> 366, plain ones 398 -> 361;
// but one plain draft of 64 61 -> 63, 2048 and 1024 on themselves 73 -> 80 and 41 -> 46, 8192 plain rows in windows of 1024 and 128 185 -> 199 and 82 -> 94, and 20 tokens of
// eight sequences, 80 rows, 142 -> 198).  Runs are as many as use all CUs to the end (five drafts of 27 on 8K, 450 blocks and 250: 94 -> 79).
//   With fp32 queries a tile of 32 rows has more registers than two waves a SIMD: 16 or 128 rows (100 / 512 tokens on 8192 keys 70, 83, 62 / 220, 266, 203; 8 on 32K 32,
// 34, 57; 500 on as many, 2 KV heads, 13, 16, 35).  Over plain fp32 rows it is 32 or 128, as in ctkvr_cache_attn.
//   Keys are split into runs where blocks would be too few, to so many blocks a CU: single tokens of one sequence, and in windows, whose runs are alike, one; of
// several sequences, whose lengths differ, half as many as these, 2 to 8 (up to 64K keys, two sequences 25, 31, 36 with 2, 4, 8; four 63, 65, 69; sixteen 267, 248, 240); tiles
// of 32 as many as the sequences, up to 6 (eight of 32 rows 96, 93, 94, 109 with 4, 6, 8, 16, of 32 to 100 rows 97, 90, 98, 98); one sequence's larger tiles, and with fp32
// queries, two; several sequences' tiles of 128 four, and of 256, which are alone on a CU, half of what tiles of 128 have (drafts of 40 in eight sequences 213, 225, 234 with 2,
// 3, 4, of 64 366, 382, 413; four of 300 652, 643, 636).
//   A run has 256 keys at least, 512 with tiles of 256 and one sequence's of 128 (64 tokens on 8K keys 51 -> 38, 28 43 -> 31), 1024 with several sequences' of 128 (four of 28 on
// 16K 70, with 512 92), 2048 where the tiles fill half the chip by themselves: the join of the runs costs 4 us and more.  It is done by the block that ends last, without a launch
// of its own, where that reads little and all blocks run at once (16 sequences in windows of 4096 55.4 -> 54.1, but causal in eight blocks a CU 239 -> 241).
struct SightPlan {
    int log;   // of a tile's rows
    int tiles, nsplit;
    bool join_inside;   // by the block that ends last, not by a launch of its own
};
// keys: those that a row may see, at most
inline SightPlan sight_plan(const ctkvr_cache *c, int total, int64_t keys, bool codes, bool window)
{
    const int64_t rows = (int64_t)total << c->lg, g = c->p.n_kv_heads, cus = c->num_cu;
    const int used = std::min(total, c->p.batch);   // sequences with new tokens, at most
    const bool bf16 = c->p.dtype == CTKVR_BF16, is_long = keys >= 4096;
    // (a sequence's rows are a multiple of the group's size, so that rounding each up to tiles adds no more than that)
    auto tiles = [&](int log) { return (rows + used * (int64_t)((1 << log) - c->G)) >> log; };
    const bool wide = tiles(7) * g >= cus;
    SightPlan p{};
    if (!bf16) p.log = codes ? (rows <= 64ll * used || (tiles(7) * g < cus / 2 && !is_long) ? 4 : 7) : rows <= 64ll * used || (!wide && (!is_long || rows < 512ll * used)) ? 5 : 7;
    else if (rows <= 16ll * used) p.log = 4;
    else if (wide || (is_long && rows > (codes ? 64ll : 48ll) * used)) p.log = 7;
    else p.log = is_long || tiles(5) * g >= cus / 2 ? 5 : 4;
    if (p.log == 7 && bf16 && rows > 128ll * used && (codes || (!window && used > 1)) && (is_long || tiles(8) * g >= 2 * cus)) p.log = 8;
    p.tiles = (int)tiles(p.log);
    // (what larger tiles come to where sequences have as many tokens; the bound would be up to twice that)
    const int64_t alike = p.log >= 7 ? used * ((rows / used + (1 << p.log) - 1) >> p.log) : p.tiles;
    const int per_cu = !bf16 ? 2 : p.log == 4 ? (window || used == 1 ? 1 : std::min(8, std::max(2, used / 2))) : p.log == 8 ? (used == 1 || window ? 1 : 2) : used == 1 || window ? 2 : p.log == 5 ? std::min(6, used) : 4;
    const int64_t want = (int64_t)per_cu * cus, least = p.tiles * g >= cus / 2 ? 2048 : p.log < 7 ? 256 : bf16 && (p.log == 8 || used == 1) ? 512 : 1024;
    p.nsplit = p.log >= 7 && p.tiles * g >= cus ? 1 : (int)std::max<int64_t>(1, std::min({want / (alike * g), (keys + least - 1) / least, (int64_t)kMaxSplit}));
    if (p.log == 8) {   // (all CUs at once, a run each)
        auto turns = [&](int n) { return (alike * g * n + cus - 1) / cus; };
        for (int n = p.nsplit - 1; n > 0; --n)
            if (turns(n) * p.nsplit < turns(p.nsplit) * n) p.nsplit = n;
    }
    p.join_inside = p.log < 7 && rows <= 8 * used && rows * p.nsplit <= (bf16 ? 256 : 128) * used && p.tiles * g * p.nsplit <= 2 * cus;
    return p;
}

// A plan's tiles that a launch has no kernel for
inline int no_kernel(int log) { return fail(CTKVR_EHIP, "no kernel for tiles of 2^%d rows", log); }

// What a workspace has room for: rows of partial outputs, and counts of the tiles whose runs are joined by the block that ends last
struct Room {
    size_t rows, counts;
};
// ... that every call of up to max_new tokens finds room in.  Plans are looked up at a number of tokens and a sixteenth more, and what lies between is taken to have as many
// runs as either, so that a handle's creation does not go through all numbers (one KV head, two sequences, 32768 tokens: 7.8 ms -> 0.3); it makes the workspace larger by a
// sixteenth at most.  A call with more runs all the same gets as many as there is room for (fit_plan).
inline Room sight_room(const ctkvr_cache *c)
{
    const int64_t slots = (int64_t)c->p.max_pages * c->p.page_size, spans[2] = {slots, std::min<int64_t>(slots, 4095)};   // (fewer keys are split less, in the form that they get)
    Room room{0, 0};
    for (int total = 1, upto; total <= c->p.max_new; total = upto + 1) {
        upto = std::min(c->p.max_new, total + total / 16);
        int most = 1;
        for (int at = total; at <= upto; at += std::max(1, upto - total))
            for (int span = 0; span < (slots > 4095 ? 2 : 1); ++span)
                for (const int form : {0, 1, 2, 3}) most = std::max(most, sight_plan(c, at, spans[span], form & 1, form & 2).nsplit);
        if (most > 1) room = Room{std::max(room.rows, (size_t)most * upto * c->p.n_q_heads), (size_t)c->num_cu};   // (runs are joined inside in up to two blocks a CU: a tile has two at least)
        else if ((((int64_t)total << c->lg) >> 7) * c->p.n_kv_heads >= 8ll * c->num_cu) break;   // more tokens are never split again
    }
    return room;
}
inline void fit_plan(const ctkvr_cache *c, int total, const Room &room, SightPlan &p)
{
    p.nsplit = (int)std::max<size_t>(1, std::min<size_t>(p.nsplit, room.rows / ((size_t)total * c->p.n_q_heads)));
    if ((size_t)p.tiles * c->p.n_kv_heads > room.counts) p.join_inside = false;
}

}  // namespace ctkvr
