// Attention of single tokens and few rows: tiles of 16 and 32 rows, over plain bf16 rows and rows of 8 bits.
#pragma once
#include "quant.hpp"

namespace ctkvr {

typedef float f32x8_t __attribute__((ext_vector_type(8)));

// Waits until shared memory has answered
__device__ __forceinline__ void lds_answered()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0xc07f);
    asm volatile("" ::: "memory");
}
// One exchange of the four groups of 16 lanes
__device__ __forceinline__ float groups_max(float x)
{
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return half_max(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}
__device__ __forceinline__ float groups_sum(float x)
{
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return half_sum(__uint_as_float(r[0]) + __uint_as_float(r[1]));
}

// A tile of 32 keys in shared memory: their rows of codes, those of their values, and their scales (K's, then V's); of bf16 the values alone, since there is not the
// room for twice as many blocks otherwise (16 sequences of 4100 keys 62 us with both, 57 so).  The 16-byte chunk c of row r stands at
// chunk c ^ r / 2 % 8 (keys) or c ^ swz(r) (values), so that the 16 rows of keys that lanes take at one chunk, and those that 32 lanes of the transposing loads take, fall
// on all 64 banks once: 16 of a chunk of codes (8 g .. 8 g + 7 and 16 more), eight of two chunks of bf16 (8 g .. 8 g + 7).
template <int STORE> struct TokenTile {
    static constexpr int kRowBytes = STORE == kPlain ? 256 : 128, kHalf = 32 * kRowBytes, kChunks = kRowBytes / 16;
    static constexpr int kBytes = STORE == kPlain ? kHalf : 2 * kHalf + 256;
    static constexpr int kPer = 64 / kChunks, kRowLoads = 32 / kPer;   // rows of one load of a wave, and loads of K or V
    static constexpr int kLoads = 2 * kRowLoads + 1;   // of a tile of codes
    static __device__ __forceinline__ int swz(int r) { return STORE == kPlain ? (r & 7) << 1 : ((r >> 1) & 3) | ((r >> 2) & 4); }
};
// 4 bytes a lane from `from` into shared memory at byte `to` + 4 * lane
__device__ __forceinline__ void word_to_lds(uint32_t to, const void *from)
{
    asm volatile("s_nop 0\n\tglobal_load_lds_dword %1, off" :: "{m0}"(__builtin_amdgcn_readfirstlane(to)), "v"(from) : "memory");
}

// Values of a plain tile that are not finite, to the rows that see them (cf. OddValues)
template <int RB, typename F> __device__ __forceinline__ void add_odd(f32x4_t (&o)[RB][8], const char *vt, int part, F sees_key)
{
    for (int n = 0; n < 32; ++n) {
        int k = n;
        asm volatile("" : "+s"(k));
        bool sees[RB];
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) sees[rb] = sees_key(rb, k);
#pragma unroll
        for (int db = 0; db < 8; ++db)
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const int d = 16 * db + 4 * part + c;
                const float x = __uint_as_float((uint32_t)*reinterpret_cast<const bf16_t *>(vt + k * 256 + (((d >> 3) ^ TokenTile<kPlain>::swz(k)) << 4) + 2 * (d & 7)) << 16);
                if (!(fabsf(x) < INFINITY)) {
#pragma unroll
                    for (int rb = 0; rb < RB; ++rb)
                        if (sees[rb]) o[rb][db][c] += x;
                }
            }
    }
}

// One block a tile of 16 RB rows and a run of their keys, which its waves share out, 32 at a time; no wave waits for another before the end.  Keys and values go straight
// to shared memory, BUFS - 1 tiles ahead of the one that is worked on.  Scores come as S^T = K Q^T on 16 x 16 x 32 products: a lane has one row (lane % 16) of each 16 and, of
// each 16 keys, those from 4 (lane / 16) on, and its probabilities of 32 keys are, where they stand, an operand of O^T = V^T P^T.  What it reads bounds tiles of 16 rows: 5.4 TB/s for
// 16 sequences of 8K to 64K keys (238 us), one token on 32K 21 us, 9 of them launch, dependent loads and the runs' join; tiles of 32 the conversion of codes and the softmax
// (vector instructions half of the cycles, matrix cores 11 %; drafts of 8 to 25 tokens of 8 sequences 90 us).
template <int STORE, typename T, int OPT, int SIGHT, int RB>
__global__ __launch_bounds__(256, sizeof(T) == 2 || RB == 1 ? 2 : 1) void tokens_kernel(QuantAttnArgs qa)
{
    using Tile = TokenTile<STORE>;
    constexpr bool kCodes = STORE != kPlain;
    constexpr int NW = 4, BUFS = 2, kRows = 16 * RB, kParts = sizeof(T) == 2 ? 1 : 3, kWeights = sizeof(T) == 2 ? 1 : 2;
    static_assert((RB == 1 || RB == 2) && (kCodes || sizeof(T) == 2) && BUFS * Tile::kBytes >= kRows * 512, "");
    __shared__ __align__(16) char smem[NW][BUFS * Tile::kBytes];
    __shared__ float join[NW][2][kRows];
    __shared__ bool last;
    const AttnArgs &a = qa.a;
    const CacheView &v = a.v;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), part = lane >> 4, r16 = lane & 15;
    const int kv = blockIdx.x % v.g, rest = blockIdx.x / v.g, split = rest % a.nsplit, tile = a.tiles - 1 - rest / a.nsplit;
    int b, at;
    SeqSpan s;
    if (!locate_span<3 + RB>(v, tile, &b, &at, &s)) return;
    const int rows = s.n << v.lg, r0 = at * kRows, have = min(kRows, rows - r0);
    const int prefix = a.o.prefix ? min(max(a.o.prefix[b], 0), s.len) : 0;
    int token[RB], head[RB];
    RowSight sight[RB];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        const int row = min(r0 + 16 * rb + r16, rows - 1);
        token[rb] = row >> v.lg;
        head[rb] = (kv << v.lg) + (row & ((1 << v.lg) - 1));
        sight[rb] = sight_of<SIGHT>(v, a.o, s, prefix, token[rb]);
    }

    // step i of the product over 128 dimensions has, of codes, those from 64 (i / 2) + 16 part + 8 (i % 2) on, 16 of a lane at a time; of bf16 those from 32 i + 8 part on
    bf16x8_t q[RB][4][kParts];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            query_parts<T, kParts>((const T *)a.q + (int64_t)(s.c0 + token[rb]) * a.q_stride + head[rb] * 128,
                                   kCodes ? 64 * (i >> 1) + 16 * part + 8 * (i & 1) : 32 * i + 8 * part, q[rb][i]);

    const int tok0 = r0 >> v.lg, tok1 = (min(r0 + kRows, rows) - 1) >> v.lg;
    const KeyRange range = key_range_of<SIGHT>(s, prefix, tok0, tok1);
    int k_lo = 0, all_lo = 0;
    if (SIGHT == kWindow) {
        k_lo = max(s.old + tok0 + 1 - a.o.window, 0);
        all_lo = max(s.old + tok1 + 1 - a.o.window, 0);
    } else if (a.o.first) {
        k_lo = all_lo = sight[0].lo;
        if constexpr (RB == 2) {
            k_lo = min(k_lo, sight[RB - 1].lo);
            all_lo = max(all_lo, sight[RB - 1].lo);
        }
#pragma unroll
        for (int d = 1; d < 16; d <<= 1) {
            k_lo = min(k_lo, __shfl_xor(k_lo, d));
            all_lo = max(all_lo, __shfl_xor(all_lo, d));
        }
        k_lo = __builtin_amdgcn_readfirstlane(k_lo);
        all_lo = __builtin_amdgcn_readfirstlane(all_lo);
    }
    int first_tile = k_lo / 32, tiles = range.hi > k_lo ? (range.hi + 31) / 32 - first_tile : 0;
    KeyTiles kt{};
    if constexpr (SIGHT == kWindow) {
        kt = window_tiles(a.o, k_lo, range.hi, 32);
        first_tile = kt.from;
        tiles = kt.to;
    }
    auto tile_of = [&](int i) { return SIGHT == kWindow ? kt.at(i) : i; };
    // (as many runs as there are two tiles for each wave)
    const int used = max(1, min(a.nsplit, (tiles + 2 * NW - 1) / (2 * NW)));
    if (split >= used) {
        auto row_out = [&](int r) { return (size_t)(s.c0 + ((r0 + r) >> v.lg)) * v.h + (kv << v.lg) + ((r0 + r) & ((1 << v.lg) - 1)); };
        if (!a.done && (int)threadIdx.x < have) a.part_lse[(size_t)split * v.total * v.h + row_out(threadIdx.x)] = -INFINITY;
        return;
    }
    const bool whole = a.nsplit == 1 || (a.done && used == 1);   // this block's outputs are the rows'
    const int64_t runs = (int64_t)used * NW, run = split * NW + wave;
    const int t0 = __builtin_amdgcn_readfirstlane(first_tile + (int)(tiles * run / runs));
    const int t1 = __builtin_amdgcn_readfirstlane(first_tile + (int)(tiles * (run + 1) / runs));

    // the row of key lane % 32; 64 of the table's entries at a time
    const int max_key = max(range.hi - 1, 0);
    const int32_t *table = v.table + (size_t)b * v.max_pages;
    int e0 = -64;
    uint32_t page = 0, bad = 0;
    auto rows_of = [&](int t) -> uint32_t {
        const int key = min(t * 32 + (lane & 31), max_key), e = key >> v.page_shift;
        const int last_e = min(t * 32 + 31, max_key) >> v.page_shift;
        if (last_e >= e0 + 64) {
            e0 = (t * 32) >> v.page_shift;
            page = (uint32_t)table[min(e0 + lane, v.max_pages - 1)];
            loads_landed<0>();
        }
        const uint32_t p = (uint32_t)__shfl((int)page, e - e0);
        const uint32_t r = p < v.num_pages ? (uint32_t)((p * (uint64_t)v.g + kv) << v.page_shift) + (key & ((1 << v.page_shift) - 1)) : kNoRow;
        const uint64_t ok = __ballot(r != kNoRow);
        bad = (uint32_t)~ok;
        if (ok == ~0ull) return r;
        if (!ok) return 0;
        const uint32_t other = __builtin_amdgcn_readlane(r, __builtin_ctzll(ok));
        return r != kNoRow ? r : other;
    };
    const uint32_t lds0 = __builtin_amdgcn_readfirstlane(lds_at(smem[wave]));
    auto fetch = [&](int buf, uint32_t r) {
        const uint32_t to = lds0 + buf * Tile::kBytes, values_to = kCodes ? to + Tile::kHalf : to;
#pragma unroll
        for (int j = 0; j < Tile::kRowLoads; ++j) {
            const int key = j * Tile::kPer + lane / Tile::kChunks, c = lane % Tile::kChunks;
            const int64_t from = (int64_t)(uint32_t)__shfl((int)r, key) * Tile::kRowBytes;
            if constexpr (kCodes) row_to_lds(to + j * 1024, (const char *)a.k_pages + from + 16 * (c ^ ((key >> 1) & 7)));
            row_to_lds(values_to + j * 1024, (const char *)a.v_pages + from + 16 * (c ^ Tile::swz(key)));
        }
        if constexpr (kCodes) word_to_lds(to + 2 * Tile::kHalf, (lane < 32 ? qa.k_scales : qa.v_scales) + r);
    };

    bf16x8_t k[2][4];   // keys of bf16
    auto fetch_keys = [&](uint32_t r) {
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            const char *from = (const char *)a.k_pages + (int64_t)(uint32_t)__shfl((int)r, 16 * kb + r16) * 256 + 16 * part;
#pragma unroll
            for (int i = 0; i < 4; ++i) k[kb][i] = *reinterpret_cast<const bf16x8_t *>(from + 64 * i);
        }
    };

    f32x4_t o[RB][8] = {};
    float m[RB], l[RB], slope2[RB];
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        m[rb] = -INFINITY;
        l[rb] = 0.0f;
        slope2[rb] = (OPT & kBias) ? a.o.slopes[head[rb]] * kLog2e : 0.0f;
    }
    int exponent[RB], least = kLeastExponent;   // of the rows' weights; a bound of all from below
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) exponent[rb] = kLeastExponent;
    auto raise = [&](int rb, int to) {
        const float f = ldexpf(1.0f, exponent[rb] - to);
        exponent[rb] = to;
#pragma unroll
        for (int db = 0; db < 8; ++db) o[rb][db] *= f;
    };
    uint32_t bads[BUFS] = {};   // (of the tiles on their way, the next one first)
    uint32_t r = t0 < t1 ? rows_of(tile_of(t0)) : 0;
    loads_landed<0>();   // (of all that the compiler knows of: it would wait for these, and for all that it does not know of, in every turn)
#pragma unroll
    for (int i = 0; i < BUFS - 1; ++i) {
        if (i && t0 + i < t1) r = rows_of(tile_of(t0 + i));
        bads[i] = bad;
        if (t0 + i < t1) fetch(i, r);
    }
    if (!kCodes && t0 < t1) fetch_keys(r);
    int buf = 0;
    for (int t = t0; t < t1; ++t) {
        const int key0 = tile_of(t) * 32;
        const uint32_t bad_now = bads[0];
        // this tile is there, and what its buffer's successor held has been read
        const int ahead = t + BUFS - 1;
        if (ahead < t1) r = rows_of(tile_of(ahead));
        if constexpr (!kCodes) settled();   // (the compiler's own waits for the keys in registers count no loads to shared memory)
        lds_answered();
        if (!kCodes) {
            if (ahead < t1) fetch(buf ^ 1, r);
        } else if (ahead < t1) {
            fetch(buf == 0 ? BUFS - 1 : buf - 1, r);
            loads_landed<(BUFS - 1) * Tile::kLoads>();
        } else {
            loads_landed<0>();
        }
#pragma unroll
        for (int i = 0; i < BUFS - 2; ++i) bads[i] = bads[i + 1];
        bads[BUFS - 2] = bad;
        char *kt_ = smem[wave] + buf * Tile::kBytes, *vt = kCodes ? kt_ + Tile::kHalf : kt_;
        float *scales = reinterpret_cast<float *>(kt_ + 2 * Tile::kHalf);
        const bool masked = key0 + 32 > range.all_hi || (key0 < all_lo && !(SIGHT == kWindow && key0 + 32 <= a.o.sinks)) || bad_now != 0;
        if constexpr (kCodes) {
            const float scale = fabsf(scales[lane]);
            if (!masked && __any(lane >= 32 && scale > ldexpf(1.0f, least))) {
                least = max(least, exponent_of_all(lane >= 32 ? scale : 0.0f));
#pragma unroll
                for (int rb = 0; rb < RB; ++rb) raise(rb, max(exponent[rb], least));
            }
        }
        // (Operands are requested of shared memory ahead of what comes before their use, and stay there: a load that the compiler puts right before it has the wave wait.)
        uint4 key_codes[2][2];
        if constexpr (kCodes) {
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    key_codes[kb][i] = *reinterpret_cast<const uint4 *>(kt_ + (16 * kb + r16) * Tile::kRowBytes + (((part + 4 * i) ^ (r16 >> 1)) << 4));
            asm volatile("" ::: "memory");
        }
        f32x8_t sc[RB];
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            f32x4_t z[RB] = {};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                bf16x8_t x;
                if constexpr (kCodes) {
                    const uint4 &w = key_codes[kb][i >> 1];
                    x = (i & 1) ? codes8<STORE>(w.z, w.w) : codes8<STORE>(w.x, w.y);
                } else {
                    x = k[kb][i];
                }
#pragma unroll
                for (int p = kParts - 1; p >= 0; --p)
#pragma unroll
                    for (int rb = 0; rb < RB; ++rb) z[rb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, q[rb][i][p], z[rb], 0, 0, 0);
            }
#pragma unroll
            for (int rb = 0; rb < RB; ++rb)
#pragma unroll
                for (int c = 0; c < 4; ++c) sc[rb][4 * kb + c] = z[rb][c];
        }
        if (!kCodes && ahead < t1) fetch_keys(r);
        if constexpr (kCodes) {
#pragma unroll
            for (int kb = 0; kb < 2; ++kb) {
                const f32x4_t x = *reinterpret_cast<const f32x4_t *>(scales + 16 * kb + 4 * part);
#pragma unroll
                for (int rb = 0; rb < RB; ++rb)
#pragma unroll
                    for (int c = 0; c < 4; ++c) sc[rb][4 * kb + c] *= x[c];
            }
        }
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) score_regs<OPT, 8, 16>(sc[rb], a.o, slope2[rb], sight[rb].pos - key0, part);
        uint32_t seen[RB];   // by the lane's rows, a bit for each key
        if (masked) {
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) {
                seen[rb] = sight_bits<SIGHT>(a.o, s, sight[rb], token[rb], key0) & ~bad_now;
#pragma unroll
                for (int i = 0; i < 8; ++i) sc[rb][i] = (seen[rb] >> (4 * part + 16 * (i >> 2) + (i & 3))) & 1 ? sc[rb][i] : -INFINITY;
            }
            if constexpr (kCodes) {   // (the scales of keys that no row sees are whatever stands there)
                float top[RB] = {};
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int n = 4 * part + 16 * (i >> 2) + (i & 3);
                    const float x = fabsf(scales[32 + n]);
#pragma unroll
                    for (int rb = 0; rb < RB; ++rb) top[rb] = fmaxf(top[rb], (seen[rb] >> n) & 1 ? x : 0.0f);
                }
#pragma unroll
                for (int rb = 0; rb < RB; ++rb) {
                    const int to = max(exponent[rb], exponent_above(groups_max(top[rb])));
                    if (__any(to != exponent[rb])) raise(rb, to);
                }
            } else {
                if (__any(OddValues<bf16_t, 32, 64>::any(vt, lane))) {
                    add_odd(o, vt, part, [&](int rb, int n) { return (bool)((seen[rb] >> n) & 1); });
                    __builtin_amdgcn_wave_barrier();
                    OddValues<bf16_t, 32, 64>::clean(vt, lane);
                    __builtin_amdgcn_wave_barrier();
                }
            }
        }
        // the values' operands of d block db: eight codes, or eight bf16 values in two parts
        union ValueOperand { i32x2_t codes; s16x4_t h[2]; bf16x8_t w; } value[8];
        if constexpr (kCodes) {
            const int key = 4 * part + ((lane >> 1) & 3) + 16 * ((lane >> 3) & 1);
#pragma unroll
            for (int db = 0; db < 8; ++db)
                value[db].codes = __builtin_amdgcn_ds_read_tr8_b64_v2i32((CTKVR_LDS i32x2_t *)(vt + key * 128 + ((db ^ Tile::swz(key)) << 4) + 8 * (lane & 1)));
        } else {
            const int key = 4 * part + (r16 >> 2);
#pragma unroll
            for (int db = 0; db < 8; ++db)
#pragma unroll
                for (int aa = 0; aa < 2; ++aa)
                    value[db].h[aa] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((CTKVR_LDS s16x4_t *)(
                        vt + (key + 16 * aa) * 256 + (((2 * db + ((lane & 3) >> 1)) ^ Tile::swz(key + 16 * aa)) << 4) + 8 * (lane & 1)));
        }
        asm volatile("" ::: "memory");
        // probabilities under the running maximum, their sum, the outputs so far to the new maximum
        float w[RB][8];
#pragma unroll
        for (int rb = 0; rb < RB; ++rb) {
            float top = sc[rb][0];
#pragma unroll
            for (int i = 1; i < 8; ++i) top = fmaxf(top, sc[rb][i]);
            top = groups_max(top);
            if constexpr (OPT == 0) top *= a.o.c2;
            if (__any(kCodes ? top > m[rb] + (float)kLag : top > m[rb])) {
                const float m_new = fmaxf(m[rb], top), f = m[rb] == -INFINITY ? 1.0f : exp2_fast(m[rb] - m_new);
                m[rb] = m_new;
                l[rb] *= f;
#pragma unroll
                for (int db = 0; db < 8; ++db) o[rb][db] *= f;
            }
            const float ref = m[rb] == -INFINITY ? 0.0f : m[rb];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                w[rb][i] = exp2_fast(OPT == 0 ? fmaf(sc[rb][i], a.o.c2, -ref) : sc[rb][i] - ref);
                l[rb] += w[rb][i];
            }
        }
        if constexpr (kCodes) {
#pragma unroll
            for (int kb = 0; kb < 2; ++kb) {
                const f32x4_t x = *reinterpret_cast<const f32x4_t *>(scales + 32 + 16 * kb + 4 * part);
#pragma unroll
                for (int rb = 0; rb < RB; ++rb) {
                    const float by = ldexpf(1.0f, kWeightPower - exponent[rb]);
#pragma unroll
                    for (int c = 0; c < 4; ++c) w[rb][4 * kb + c] *= x[c] * by;
                }
            }
            f16x8_t p[RB][kWeights];
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) {
                if (masked) {   // (a hidden row's scale may be anything)
#pragma unroll
                    for (int i = 0; i < 8; ++i) w[rb][i] = (seen[rb] >> (4 * part + 16 * (i >> 2) + (i & 3))) & 1 ? w[rb][i] : 0.0f;
                }
                split_parts(w[rb], p[rb]);
            }
#pragma unroll
            for (int db = 0; db < 8; ++db) {
                uint32_t lo = (uint32_t)value[db].codes[0], hi = (uint32_t)value[db].codes[1];
                if (masked) lo = no_nan<STORE>(lo), hi = no_nan<STORE>(hi);
                const f16x8_t y = codes8h<STORE>(lo, hi);
#pragma unroll
                for (int i = kWeights - 1; i >= 0; --i)
#pragma unroll
                    for (int rb = 0; rb < RB; ++rb) o[rb][db] = __builtin_amdgcn_mfma_f32_16x16x32_f16(y, p[rb][i], o[rb][db], 0, 0, 0);
            }
        } else {
            bf16x8_t p[RB][1];
#pragma unroll
            for (int rb = 0; rb < RB; ++rb) split_parts(w[rb], p[rb]);   // (rounded to the values' type, as in attn_kernel)
#pragma unroll
            for (int db = 0; db < 8; ++db)
#pragma unroll
                for (int rb = 0; rb < RB; ++rb) o[rb][db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(value[db].w, p[rb][0], o[rb][db], 0, 0, 0);
        }
        buf = buf + 1 == BUFS ? 0 : buf + 1;
        __builtin_amdgcn_wave_barrier();
    }

    // the waves' outputs to one maximum, through shared memory (16-byte chunks at chunk ^ row)
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        l[rb] = groups_sum(l[rb]);
        if (part == 0) {
            join[wave][0][16 * rb + lane] = m[rb];
            join[wave][1][16 * rb + lane] = l[rb];
        }
    }
    loads_landed<0>();
    __syncthreads();   // (and nobody needs its values any more)
#pragma unroll
    for (int rb = 0; rb < RB; ++rb) {
        const int r = 16 * rb + r16;
        float top = join[0][0][r];
#pragma unroll
        for (int w = 1; w < NW; ++w) top = fmaxf(top, join[w][0][r]);
        const float f = (m[rb] == -INFINITY ? 1.0f : exp2_fast(m[rb] - top)) * (kCodes ? ldexpf(1.0f, exponent[rb] - kWeightPower) : 1.0f);
#pragma unroll
        for (int db = 0; db < 8; ++db) *reinterpret_cast<f32x4_t *>(smem[0] + (wave * kRows + r) * 512 + (((4 * db + part) ^ r) << 4)) = o[rb][db] * f;
    }
    __syncthreads();
    few_join<T, NW, kRows>(a, s, kv, r0, have, tile, split, used, whole, smem[0], join, &last);
}

}  // namespace ctkvr
