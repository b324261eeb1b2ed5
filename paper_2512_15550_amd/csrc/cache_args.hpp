// Where the operators on the paged KV cache find a sequence's tokens, its rows and what a token sees; plain functions, for the kernels and for the host.
#pragma once
#include <hip/hip_runtime.h>
#include <math.h>
#include <stddef.h>
#include <stdint.h>

namespace ctkvr {

// What every operator needs of the cache and of the call's tokens
struct CacheView {
    const int32_t *table;   // [batch][max_pages]
    const int32_t *cu;      // [batch + 1]: new tokens cu[b] .. cu[b + 1] - 1 belong to sequence b
    const int32_t *cur;     // [batch]: tokens in the cache, the new ones among them
    int batch, h, g, lg;    // lg: log2 of the group size
    int page_shift, max_pages, total;
    uint32_t num_pages;
};

struct SeqSpan {
    int c0, n, len, old;   // first new token, new tokens, tokens in the cache (as far as the table goes), those before the new ones
};
// (values that make no sense are brought into range: nothing is read or written outside the caller's arrays)
__host__ __device__ __forceinline__ SeqSpan seq_span(const CacheView &v, int b)
{
    SeqSpan s;
    s.c0 = min(max(v.cu[b], 0), v.total);
    s.n = min(max(v.cu[b + 1], s.c0), v.total) - s.c0;
    const int cur = min(max(v.cur[b], 0), 1 << 30);
    s.len = min(cur, v.max_pages << v.page_shift);
    s.old = cur - s.n;
    return s;
}

// KV row (in units of 128 elements) of token t < max_pages << page_shift, or -1 where its page is none of the cache's
__host__ __device__ __forceinline__ int64_t cache_row(const CacheView &v, int b, int kv, int t)
{
    const uint32_t page = (uint32_t)v.table[(size_t)b * v.max_pages + (t >> v.page_shift)];
    if (page >= v.num_pages) return -1;
    return (((int64_t)page * v.g + kv) << v.page_shift) + (t & ((1 << v.page_shift) - 1));
}

struct ScoreOpts {
    const float *slopes;      // [h] or null
    const int32_t *prefix;    // [batch] or null
    const int32_t *first;     // [total] or null
    float c2;                 // scale * log2 e
    float cap_in, cap_out, cap_105, cap_945;   // scale / cap, cap * log2 e, the latter times 105 and 945 (cap != 0)
};
// What a row sees: keys from lo on, before hi
struct RowSight {
    int pos, lo, hi;
};
__host__ __device__ __forceinline__ RowSight row_sight(const CacheView &v, const ScoreOpts &o, const SeqSpan &s, int prefix, int token)
{
    RowSight r;
    r.pos = s.old + token;
    r.hi = r.pos < 0 ? 0 : min(max(r.pos + 1, prefix), s.len);
    r.lo = o.first ? max(o.first[s.c0 + token], 0) : 0;
    return r;
}

// A frequency (radians per position) as a fraction of a turn, in 2^-64: freq / (2 pi) modulo 1, off by one of them at most for frequencies up to 2^32.
// 1 / (2 pi) is held as two long doubles, and what the product is off by is added back, so that a frequency of many turns keeps its fraction.
inline uint64_t turn_of(long double freq)
{
    const long double hi = 0xa2f9836e4e44152ap-66L, lo = -0xf62a0b82b2c88fc9p-136L;
    const long double p = freq * hi, off = fmal(freq, hi, -p) + freq * lo;
    long double t = p - floorl(p) + off;
    t -= floorl(t);
    const long double u = roundl(ldexpl(t, 64));
    return u >= ldexpl(1.0L, 64) ? 0 : (uint64_t)u;
}
// the frequency of pair i; for bases from 1 on its turn is off by 1.25 of 2^-64 at most
inline long double rope_freq(double base, int i) { return powl((long double)base, -i / 64.0L); }

}  // namespace ctkvr
