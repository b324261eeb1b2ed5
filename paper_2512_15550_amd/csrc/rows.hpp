// Attention of many rows: tiles of 128 and 256 rows, over plain bf16 rows and rows of 8 bits.
#pragma once
#include "quant.hpp"

namespace ctkvr {

// A tile of 64 keys and their values in shared memory, as bf16 (keys) and bf16 or, from codes, fp16 (values), and where a lane finds its operands.  Shared memory
// answers 16 lanes of 16 bytes or 32 of 8 at a time, from 64 banks: the 16 rows that lanes take at one chunk of keys, and the four rows that 16 lanes of the transposing
// load take at two chunks of values, with the 16 lanes beside them at two more, have to fall on all banks once.
//   Rows of codes are turned into 16 bits on their way.  The 16 codes of a lane become the chunks c and c + 8 of a row, c the lane of its eight, so that eight lanes write
// a line; the queries and outputs follow this order (column()).  Rows of 272 and 320 bytes then put an operand at a constant distance from a lane's first.
//   Plain rows come straight from memory, 16 bytes a lane, one row of 256 bytes behind the other: there the chunk c of row r stands at c ^ r % 16 (keys) or
// c ^ 4 (r % 4) (values).
template <bool CODES> struct RowsTile {
    static constexpr int kKeyRow = CODES ? 272 : 256, kValueRow = CODES ? 320 : 256;
    static constexpr int kKeyBytes = 64 * kKeyRow, kBytes = kKeyBytes + 64 * kValueRow;
    // the first of the 8 dimensions that chunk c of a row holds
    static __host__ __device__ __forceinline__ constexpr int column(int c) { return CODES ? 16 * (c & 7) + 8 * (c >> 3) : 8 * c; }
    static __device__ __forceinline__ int key_at(int lane, int kb, int i)
    {
        const int r = lane & 31, half = lane >> 5;
        if constexpr (CODES) return r * kKeyRow + 16 * half + 32 * kb * kKeyRow + 32 * i;
        else return r * 256 + (((2 * i + half) ^ (r & 15)) << 4) + 32 * kb * 256;
    }
    // rows 8 aa + 4 (lane / 32) + 0 .. 3 of 16 from 32 kb + 16 k2 on, chunks 4 db on
    static __device__ __forceinline__ int value_at(int lane, int kb, int k2, int aa, int db)
    {
        const int half = lane >> 5, in = (lane & 15) >> 2, r = 4 * half + in, rows = 32 * kb + 16 * k2 + 8 * aa;
        if constexpr (CODES) return kKeyBytes + r * kValueRow + 32 * ((lane >> 4) & 1) + 8 * (lane & 3) + rows * kValueRow + 64 * db;
        else return kKeyBytes + r * 256 + ((db ^ in) << 6) + 32 * ((lane >> 4) & 1) + 8 * (lane & 3) + rows * 256;
    }
};

// One block a tile of 32 NW rows of a unit and, where the keys are split, one of nsplit runs of them; a wave has 32 rows.  While a tile of 64 keys is worked on the
// next one is put into shared memory (codes: turned into bf16 and fp16 by the block, each once for all its waves) and the one behind it requested.  Two waves a SIMD: two blocks of four
// a CU, or one of eight, which does half of that work for a row (2048 tokens on 32K codes 1243 -> 1146 us, 903 to 952 TFLOP/s; 8192 plain rows in a window of 1024 take 185 us in blocks of four, 199 in blocks of eight).  Products and the vector instructions of softmax, scales and
// conversion bound it, which two waves of a SIMD hardly overlap.
template <int STORE, typename T, int OPT, int SIGHT, int NW> __global__ __launch_bounds__(64 * NW, sizeof(T) == 2 ? 2 : 1) void rows_kernel(QuantAttnArgs qa)
{
    constexpr bool kCodes = STORE != kPlain;
    using Tile = RowsTile<kCodes>;
    constexpr int kRowsLog = NW == 8 ? 8 : 7, kKeys = 64, kShare = kKeys / NW, kParts = sizeof(T) == 2 ? 1 : 3, kWeights = sizeof(T) == 2 ? 1 : 2;
    static_assert((kCodes || sizeof(T) == 2) && (NW == 4 || (NW == 8 && sizeof(T) == 2)), "");
    __shared__ __align__(16) char smem[2][Tile::kBytes];
    __shared__ __align__(16) float scales[2][2][kKeys];   // [buffer][K, V]
    __shared__ int exponents[2];   // of the values' scales in a buffer
    __shared__ __align__(8) uint8_t far_rows[2][NW];   // [step % 2][wave]
    const AttnArgs &a = qa.a;
    const CacheView &v = a.v;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
    // (a KV head's tiles stay on an XCD where the heads are a multiple of 8; the tiles with most keys go first)
    const int kv = blockIdx.x % v.g, rest = blockIdx.x / v.g, split = rest % a.nsplit;
    int b, at;
    SeqSpan s;
    if (!locate_span<kRowsLog>(v, a.tiles - 1 - rest / a.nsplit, &b, &at, &s)) return;
    const int rows = s.n << v.lg, r0 = at << kRowsLog, row = r0 + 32 * wave + (lane & 31);
    const int prefix = a.o.prefix ? min(max(a.o.prefix[b], 0), s.len) : 0;
    const int token = min(row, rows - 1) >> v.lg, head = (kv << v.lg) + (min(row, rows - 1) & ((1 << v.lg) - 1));
    const RowSight sight = sight_of<SIGHT>(v, a.o, s, prefix, token);
    bf16x8_t q[8][kParts];
#pragma unroll
    for (int i = 0; i < 8; ++i) query_parts<T, kParts>((const T *)a.q + (int64_t)(s.c0 + token) * a.q_stride + head * 128, Tile::column(2 * i + half), q[i]);

    const int tok0 = r0 >> v.lg, tok1 = (min(r0 + 32 * NW, rows) - 1) >> v.lg;
    const KeyRange range = key_range_of<SIGHT>(s, prefix, tok0, tok1);
    int k_lo = 0, all_lo = 0;
    if (SIGHT == kWindow) {
        k_lo = max(s.old + tok0 + 1 - a.o.window, 0);
        all_lo = max(s.old + tok1 + 1 - a.o.window, 0);
    } else if (a.o.first) {
        int lo = sight.lo, hi = sight.lo;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            lo = min(lo, __shfl_xor(lo, d));
            hi = max(hi, __shfl_xor(hi, d));
        }
        int *ex = reinterpret_cast<int *>(scales);
        if (lane == 0) {
            ex[2 * wave] = lo;
            ex[2 * wave + 1] = hi;
        }
        __syncthreads();
        k_lo = ex[0];
        all_lo = ex[1];
#pragma unroll
        for (int w = 1; w < NW; ++w) {
            k_lo = min(k_lo, ex[2 * w]);
            all_lo = max(all_lo, ex[2 * w + 1]);
        }
        k_lo = __builtin_amdgcn_readfirstlane(k_lo);
        all_lo = __builtin_amdgcn_readfirstlane(all_lo);
        __syncthreads();
    }
    int t0 = k_lo / kKeys, t1 = range.hi > k_lo ? (range.hi + kKeys - 1) / kKeys : t0;
    KeyTiles kt{};
    if constexpr (SIGHT == kWindow) {
        kt = window_tiles(a.o, k_lo, range.hi, kKeys);
        t0 = kt.from;
        t1 = kt.to;
    }
    auto tile_of = [&](int i) { return SIGHT == kWindow ? kt.at(i) : i; };
    if (a.nsplit > 1) {   // this block's run of them: as many runs as there are eight tiles for
        const int n = t1 - t0, used = max(1, min(a.nsplit, n / 8)), at_run = min(split, used);
        const int from = (int)((int64_t)n * at_run / used), to = (int)((int64_t)n * min(at_run + 1, used) / used);
        t1 = t0 + to;
        t0 += from;
    }
    t0 = __builtin_amdgcn_readfirstlane(t0);
    t1 = __builtin_amdgcn_readfirstlane(t1);

    // Key `lane` of a tile: its entry of the table, requested a step before it is needed, and its row.  Keys that have none, and what lies behind the last key, take a row
    // that is there: whatever the memory behind them holds reaches no product.
    const int max_key = max(range.hi - 1, 0);
    const int32_t *table = v.table + (size_t)b * v.max_pages;
    auto key_of = [&](int i) { return min(tile_of(i) * kKeys + lane, max_key); };
    auto page_of = [&](int i) { return (uint32_t)table[key_of(i) >> v.page_shift]; };
    uint64_t bad = 0;
    auto row_of = [&](int i, uint32_t page) -> uint32_t {
        const uint32_t r = page < v.num_pages ? (uint32_t)((page * (uint64_t)v.g + kv) << v.page_shift) + (key_of(i) & ((1 << v.page_shift) - 1)) : kNoRow;
        const uint64_t ok = __ballot(r != kNoRow);
        bad = ~ok;
        if (ok == ~0ull) return r;
        if (!ok) return 0;
        const uint32_t other = __builtin_amdgcn_readlane(r, __builtin_ctzll(ok));
        return r != kNoRow ? r : other;
    };
    auto seen_by_all = [&](int i, uint64_t none) {
        const int t = tile_of(i);
        return (t + 1) * kKeys <= range.all_hi && (t * kKeys >= all_lo || (SIGHT == kWindow && (t + 1) * kKeys <= a.o.sinks)) && none == 0;
    };

    // A wave's share of a tile is kShare rows.  Codes: 8 lanes a row, 16 codes a lane, to registers and from there to shared memory.
    uint4 codes[2][kShare / 8];
    float scale = 0.0f;
    // A tile that all rows see has its values' scales times 2^(11 - tile_exponent), which wave 1 holds and leaves with the tile; of another they are as they are, since
    // there every row has an exponent of its own.
    //   A row that has seen values more than 2^kFar times as large as such a tile's keeps its exponent there, since its outputs, below 2^44 at that with 2^20 keys, have no
    // room at the tile's; the tile's weights are next to nothing to it.  While a block has such rows, or may have, it takes its tiles one at a time.
    constexpr int kRowsOwn = INT_MIN, kFar = 80;
    int tile_exponent = kLeastExponent;
    auto request = [&](uint32_t r) {
        if (wave < 2) scale = (wave ? qa.v_scales : qa.k_scales)[r];
#pragma unroll
        for (int j = 0; j < kShare / 8; ++j) {
            const int64_t from = (int64_t)(uint32_t)__shfl((int)r, wave * kShare + 8 * j + (lane >> 3)) * 128 + 16 * (lane & 7);
            codes[0][j] = *reinterpret_cast<const uint4 *>((const char *)a.k_pages + from);
            codes[1][j] = *reinterpret_cast<const uint4 *>((const char *)a.v_pages + from);
        }
    };
    auto put = [&](auto buf, int i, uint64_t none) {
        if (wave == 0) scales[buf][0][lane] = OPT == 0 ? scale * a.o.c2 : scale;
        if (wave == 1) {
            const bool all = seen_by_all(i, none);
            if (all && __any(fabsf(scale) > ldexpf(1.0f, tile_exponent))) tile_exponent = max(tile_exponent, exponent_of_all(scale));
            scales[buf][1][lane] = all ? scale * ldexpf(1.0f, kWeightPower - tile_exponent) : scale;
            if (lane == 0) exponents[buf] = all ? tile_exponent : kRowsOwn;
        }
        if (STORE == kFp8 && !seen_by_all(i, none)) {
#pragma unroll
            for (int j = 0; j < kShare / 8; ++j) {
                uint4 &w = codes[1][j];
                w = make_uint4(no_nan<STORE>(w.x), no_nan<STORE>(w.y), no_nan<STORE>(w.z), no_nan<STORE>(w.w));
            }
        }
#pragma unroll
        for (int j = 0; j < kShare / 8; ++j) {
            const int key = wave * kShare + 8 * j + (lane >> 3);
            char *k_to = smem[buf] + key * Tile::kKeyRow + 16 * (lane & 7), *v_to = smem[buf] + Tile::kKeyBytes + key * Tile::kValueRow + 16 * (lane & 7);
            *reinterpret_cast<bf16x8_t *>(k_to) = codes8<STORE>(codes[0][j].x, codes[0][j].y);
            *reinterpret_cast<bf16x8_t *>(k_to + 128) = codes8<STORE>(codes[0][j].z, codes[0][j].w);
            *reinterpret_cast<f16x8_t *>(v_to) = codes8h<STORE>(codes[1][j].x, codes[1][j].y);
            *reinterpret_cast<f16x8_t *>(v_to + 128) = codes8h<STORE>(codes[1][j].z, codes[1][j].w);
        }
    };
    // Plain rows: four a load, straight to shared memory.  Where a wave's are in one page the address of the first is the wave's, not a lane's.
    const uint32_t lds0 = __builtin_amdgcn_readfirstlane(lds_at(smem));
    const bool one_page = (1 << v.page_shift) >= kShare;
    const int in4 = lane >> 4, c16 = lane & 15;
    auto load = [&](auto buf, uint32_t r, bool whole) {
        const uint32_t to = lds0 + buf * Tile::kBytes + wave * kShare * 256;
        if (one_page && whole) {
            const int64_t from = (int64_t)(uint32_t)__builtin_amdgcn_readlane(r, wave * kShare) * 256;
#pragma unroll
            for (int j = 0; j < kShare / 4; ++j) {
                load_to_lds(to + j * 1024, (const char *)a.k_pages + from, (4 * j + in4) * 256 + 16 * (c16 ^ ((wave * kShare + 4 * j + in4) & 15)));
                load_to_lds(to + Tile::kKeyBytes + j * 1024, (const char *)a.v_pages + from, (4 * j + in4) * 256 + 16 * (c16 ^ (in4 << 2)));
            }
            return;
        }
#pragma unroll
        for (int j = 0; j < kShare / 4; ++j) {
            const int64_t from = (int64_t)(uint32_t)__shfl((int)r, wave * kShare + 4 * j + in4) * 256;
            row_to_lds(to + j * 1024, (const char *)a.k_pages + from + 16 * (c16 ^ ((wave * kShare + 4 * j + in4) & 15)));
            row_to_lds(to + Tile::kKeyBytes + j * 1024, (const char *)a.v_pages + from + 16 * (c16 ^ (in4 << 2)));
        }
    };
    auto whole = [&](int i, uint64_t none) { return none == 0 && (tile_of(i) + 1) * kKeys <= range.hi; };

    f32x16_t o[4] = {};
    float m = -INFINITY, l = 0.0f;
    int exponent = kLeastExponent;   // of the row's outputs
    const float slope2 = (OPT & kBias) ? a.o.slopes[head] * kLog2e : 0.0f;
    uint64_t bad_now = 0, bad_next = 0;   // of the tile that is worked on, and of the next
    uint32_t page = 0, r = 0;             // codes: entries of the tile behind the next; plain: the next tile's rows, and those entries
    auto step = [&](auto buf, auto masked, int i) {
        const auto other = [&] {
            if constexpr (std::is_same_v<decltype(buf), int>) return buf ^ 1;
            else return std::integral_constant<int, decltype(buf)::value ^ 1>();
        }();
        const uint64_t bad_1 = bad_next;
        if constexpr (kCodes) {
            if (i + 1 < t1) put(other, i + 1, bad_1);
            if (i + 2 < t1) {
                request(row_of(i + 2, page));
                bad_next = bad;
            }
        } else {
            if (i + 1 < t1) load(other, r, whole(i + 1, bad_1));
            if (i + 2 < t1) {
                r = row_of(i + 2, page);
                bad_next = bad;
            }
        }
        if (i + 3 < t1) page = page_of(i + 3);
        char *tile = smem[buf];
        const int key0 = tile_of(i) * kKeys;
        uint32_t seen[2];
        if constexpr (decltype(masked)::value) {
#pragma unroll
            for (int kb = 0; kb < 2; ++kb) seen[kb] = sight_bits<SIGHT>(a.o, s, sight, token, key0 + 32 * kb) & ~(uint32_t)(bad_now >> (32 * kb));
            if constexpr (!kCodes) {
                // values that are not finite, to the rows that see them, and out of the tile (cf. OddValues)
                const u32x4_t *w = reinterpret_cast<const u32x4_t *>(tile + Tile::kKeyBytes) + threadIdx.x;
                uint32_t odd = 0;
#pragma unroll
                for (int j = 0; j < 16 / NW; ++j) {
                    const u32x4_t x = w[j * 64 * NW];
#pragma unroll
                    for (int e = 0; e < 4; ++e) odd |= ((x[e] & 0x7f807f80u) + 0x00800080u) & 0x80008000u;
                }
                if (__syncthreads_or(odd)) {
                    for (int n = 0; n < kKeys; ++n) {
                        int k = n;
                        asm volatile("" : "+s"(k));
                        const bool sees = ((k < 32 ? seen[0] : seen[1]) >> (k & 31)) & 1;
                        const char *from = tile + Tile::kKeyBytes + k * 256;
#pragma unroll
                        for (int db = 0; db < 4; ++db)
#pragma unroll
                            for (int e = 0; e < 16; ++e) {
                                const int d = 32 * db + 8 * (e >> 2) + 4 * half + (e & 3);
                                const float x = __uint_as_float((uint32_t)*reinterpret_cast<const bf16_t *>(from + (((d >> 3) ^ ((k & 3) << 2)) << 4) + 2 * (d & 7)) << 16);
                                if (sees && !(fabsf(x) < INFINITY)) o[db][e] += x;
                            }
                    }
                    __syncthreads();
                    OddValues<bf16_t, kKeys, 64 * NW>::clean(tile + Tile::kKeyBytes, threadIdx.x);
                    __syncthreads();
                }
            }
        }
        f32x16_t sc[2] = {};
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const bf16x8_t x = *reinterpret_cast<const bf16x8_t *>(tile + Tile::key_at(lane, kb, j));
#pragma unroll
                for (int p = kParts - 1; p >= 0; --p) sc[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, q[j][p], sc[kb], 0, 0, 0);
            }
        int e = 0;
        if constexpr (kCodes) {
            e = __builtin_amdgcn_readfirstlane(exponents[buf]);
            if constexpr (decltype(masked)::value) {
                int to = e;
                if (e == kRowsOwn) {
                    float top = 0.0f;
#pragma unroll
                    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                        for (int n = 0; n < 16; ++n) {
                            const int k = 8 * (n >> 2) + 4 * half + (n & 3);
                            top = fmaxf(top, (seen[kb] >> k) & 1 ? fabsf(scales[buf][1][32 * kb + k]) : 0.0f);
                        }
                    to = max(exponent, exponent_above(half_max(top)));
                } else if (exponent - e > kFar) {
                    to = exponent;
                }
                if (__any(to != exponent)) {
                    scale_outputs(o, exponent - to);
                    exponent = to;
                }
                const bool is_far = __any(exponent - max(e, kLeastExponent) > kFar);
                if (lane == 0) far_rows[i & 1][wave] = is_far;
            } else {
                if (__any(exponent != e)) {
                    scale_outputs(o, exponent - e);
                    exponent = e;
                }
            }
        }
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            if constexpr (kCodes) scale_regs(sc[kb], scales[buf][0] + 32 * kb, half);
            score_regs<OPT>(sc[kb], a.o, slope2, sight.pos - key0 - 32 * kb, half);
            if constexpr (decltype(masked)::value) mask_bits(sc[kb], seen[kb], half, -INFINITY);
        }
        // (codes: the factor of the exponent is in their keys' scales)
        softmax_regs<(kCodes && OPT == 0 ? kBias : OPT), 2, (kCodes ? kLag : 0)>(sc, o, m, l, a.o.c2);
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            if constexpr (kCodes) {
                if (decltype(masked)::value && __any(exponent != e)) {   // (some rows' weights take a power of their own)
                    scale_regs_by(sc[kb], scales[buf][1] + 32 * kb, ldexpf(1.0f, (e == kRowsOwn ? kWeightPower : e) - exponent), half);
                } else {
                    scale_regs(sc[kb], scales[buf][1] + 32 * kb, half);
                }
                if constexpr (decltype(masked)::value) mask_bits(sc[kb], seen[kb], half, 0.0f);   // (a hidden row's scale may be anything)
            }
#pragma unroll
            for (int k2 = 0; k2 < 2; ++k2) {
                float y[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) y[j] = sc[kb][8 * k2 + j];
                std::conditional_t<kCodes, f16x8_t, bf16x8_t> p[kCodes ? kWeights : 1];   // (plain: rounded to the values' type, as in attn_kernel)
                split_parts(y, p);
#pragma unroll
                for (int db = 0; db < 4; ++db) {
                    union { s16x4_t h[2]; std::remove_reference_t<decltype(p[0])> w; } x;
#pragma unroll
                    for (int aa = 0; aa < 2; ++aa)
                        x.h[aa] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((CTKVR_LDS s16x4_t *)(tile + Tile::value_at(lane, kb, k2, aa, db)));
                    if constexpr (kCodes) {
#pragma unroll
                        for (int j = kWeights - 1; j >= 0; --j) o[db] = __builtin_amdgcn_mfma_f32_32x32x16_f16(x.w, p[j], o[db], 0, 0, 0);
                    } else {
                        o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x.w, p[0], o[db], 0, 0, 0);
                    }
                }
            }
        }
        bad_now = bad_1;
        if constexpr (!kCodes) loads_landed<0>();
        __syncthreads();
    };
    using Zero = std::integral_constant<int, 0>;
    if (t0 < t1) {
        r = row_of(t0, page_of(t0));
        bad_now = bad;
        if constexpr (kCodes) {
            request(r);
            put(Zero(), t0, bad_now);
        } else {
            load(Zero(), r, whole(t0, bad_now));
        }
        if (t0 + 1 < t1) {
            r = row_of(t0 + 1, page_of(t0 + 1));
            bad_next = bad;
            if constexpr (kCodes) request(r);
        }
        if (t0 + 2 < t1) page = page_of(t0 + 2);
        if constexpr (!kCodes) loads_landed<0>();
        __syncthreads();
    }
    int i = t0;
    while (i < t1) {
        // (two at a time: where a tile is in shared memory is then part of the instructions)
        bool pairs = ((i - t0) & 1) == 0;
        if (kCodes && pairs && i > t0 && i + 1 < t1 && seen_by_all(i, bad_now) && seen_by_all(i + 1, bad_next)) {
            using Waves = std::conditional_t<NW == 8, uint64_t, uint32_t>;
            pairs = !__any(*reinterpret_cast<const Waves *>(far_rows[(i - 1) & 1]) != 0);
        }
        if (pairs)
            while (i + 1 < t1 && seen_by_all(i, bad_now) && seen_by_all(i + 1, bad_next)) {
                step(Zero(), std::false_type(), i);
                step(std::integral_constant<int, 1>(), std::false_type(), i + 1);
                i += 2;
            }
        if (i >= t1) break;
        step((i - t0) & 1, std::true_type(), i);
        ++i;
    }
    if constexpr (kCodes) scale_outputs(o, exponent - kWeightPower);
    many_finish<T, RowsTile<kCodes>>(a, s, split, t0 == t1, row < rows, token, head, m, half_sum(l), o, half);
}

}  // namespace ctkvr
