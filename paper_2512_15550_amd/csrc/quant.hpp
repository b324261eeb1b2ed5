// Kernels of a paged KV cache whose rows are held in 8 bits: append with rotary positions, reading back, attention.  gfx950, wave64, matrix cores.
//
// A row is 128 codes of one byte, int8 or e4m3, and an fp32 scale: its largest magnitude over the largest code.  Both kinds of code are exact in bf16 and fp16, so that
// the products take them as they are, two bytes each from the conversion on; a key's scale multiplies its score, a value's its probability.  Such a weight enters the
// product in fp16, which has three bits more than bf16 (with weights in bf16 the outputs of a single token on 32K keys were 2.5e-3 off, of which their own rounding is
// 1.6e-3), under a power of two that goes with the largest scale that its row has seen (kWeightPower).  With fp32 queries a query is three bf16 parts and a weight two of
// fp16: as exact as fp32 products (outputs 4e-7 to 9e-7 off, elementary operations in fp32 8e-7 to 2.6e-6), at a sixth of their cost.
#pragma once
#include "cache.hpp"

namespace ctkvr {

constexpr int kPlain = 0, kInt8 = 1, kFp8 = 2;   // (ctkvr_kv_format)
template <int STORE> constexpr float kTop = STORE == kInt8 ? 127.0f : 448.0f;

typedef int i32x2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2_t __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8_t __attribute__((ext_vector_type(8)));

// ---- append -------------------------------------------------------------------------------------------------
struct QuantRows {
    uint8_t *codes;    // [num_pages][g][page][128]
    float *scales;     // [num_pages][g][page]
};
struct QuantAppendArgs {
    AppendArgs a;      // (k_pages, v_pages: null)
    QuantRows k, v;
};

// A row's largest magnitude, as bits, over its 8 lanes (NaN above infinity above all numbers)
__device__ __forceinline__ uint32_t largest_bits(const float (&p)[8], const float (&q)[8])
{
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = max(m, max(__float_as_uint(p[i]) & 0x7fffffffu, __float_as_uint(q[i]) & 0x7fffffffu));
#pragma unroll
    for (int d = 1; d < 8; d <<= 1) m = max(m, (uint32_t)__shfl_xor((int)m, d));
    return m;
}
// x * top / amax, correctly rounded, so that what lies half way between two codes goes to the even one: a quotient from the reciprocal and one step of its
// remainder (Markstein's division), four instructions a value where a division takes ten.  `inv`: 1 / amax.
template <int STORE> __device__ __forceinline__ float in_codes(float x, float amax, float inv)
{
    const float n = x * kTop<STORE>, y = n * inv;
    return fmaf(fmaf(-y, amax, n), inv, y);
}
template <int STORE> __device__ __forceinline__ uint2 encode(const float (&y)[8])
{
    uint2 c;
    if constexpr (STORE == kInt8) {
        uint32_t w[2] = {0, 0};
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i >> 2] |= ((uint32_t)(int)rintf(y[i]) & 0xffu) << (8 * (i & 3));
        c = make_uint2(w[0], w[1]);
    } else {
        int lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false), hi = __builtin_amdgcn_cvt_pk_fp8_f32(y[4], y[5], 0, false);
        lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], lo, true);
        hi = __builtin_amdgcn_cvt_pk_fp8_f32(y[6], y[7], hi, true);
        c = make_uint2((uint32_t)lo, (uint32_t)hi);
    }
    return c;
}
// A row's chunks i8 and i8 + 8 of 8 elements, as codes.  A row that holds an infinity or NaN gets the scale NaN and codes of 0.
template <int STORE> __device__ __forceinline__ void store_codes(const QuantRows &to, int64_t row, int i8, float (&p)[8], float (&q)[8])
{
    const uint32_t bits = largest_bits(p, q);
    const float amax = __uint_as_float(bits);
    const bool odd = bits >= 0x7f800000u, none = odd || bits == 0;
    // (far from 1 the row is taken by a power of two, so that neither the products nor the reciprocal leave the range)
    const float by = amax > 0x1p100f ? 0x1p-64f : amax < 0x1p-62f ? 0x1p64f : 1.0f, scaled = none ? 1.0f : amax * by, inv = 1.0f / scaled;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        p[i] = none ? 0.0f : in_codes<STORE>(p[i] * by, scaled, inv);
        q[i] = none ? 0.0f : in_codes<STORE>(q[i] * by, scaled, inv);
    }
    uint8_t *at = to.codes + row * 128;
    *reinterpret_cast<uint2 *>(at + 8 * i8) = encode<STORE>(p);
    *reinterpret_cast<uint2 *>(at + 64 + 8 * i8) = encode<STORE>(q);
    if (i8 == 0) to.scales[row] = odd ? __uint_as_float(0x7fc00000u) : amax / kTop<STORE>;
}

// `share` waves have a token, 8 lanes a row of it, the chunks i and i + 8 of 8 elements each.  A wave's first rows are requested before it looks its token up.  Many
// tokens: reading and writing, two waves each.  Few: loads that wait for each other, so that four waves a token have two rounds of them in place of six
// (16 tokens 7.3 -> 5.6 us).  Memory bounds it: 8192 tokens in 38 us, 4.8 TB/s, as a copy.
template <typename T, int STORE> __global__ __launch_bounds__(256) void quant_append_kernel(QuantAppendArgs qa, int share)
{
    __shared__ float2 turn[4][64];
    const AppendArgs &a = qa.a;
    const CacheView &v = a.v;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, at = blockIdx.x * 4 + wave, token = at / share;
    if (token >= v.total) return;
    const int i8 = lane & 7, nq = a.q ? v.h : 0, rows = nq + 2 * v.g, step = 8 * share;
    auto row = [&](int r) {
        return r < nq ? (const T *)a.q + (int64_t)token * a.q_stride + r * 128
               : r < nq + v.g ? (const T *)a.k + (int64_t)token * a.k_stride + (r - nq) * 128
                              : (const T *)a.val + (int64_t)token * a.v_stride + (r - nq - v.g) * 128;
    };
    int r = (at % share) * 8 + (lane >> 3);
    Chunk<T> lo, hi;
    if (r < rows) {
        lo = load_chunk_nt(row(r), i8);
        hi = load_chunk_nt(row(r), i8 + 8);
    }
    AppendToken t;
    if (!append_token(a, token, lane, turn[wave], &t)) return;
    while (r < rows) {
        const int kv = r - nq, next = r + step;
        float x[8], y[8], p[8], q[8];
        unpack(lo, x);
        unpack(hi, y);
        if (next < rows) {
            lo = load_chunk_nt(row(next), i8);
            hi = load_chunk_nt(row(next), i8 + 8);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            p[i] = kv >= v.g ? x[i] : fmaf(x[i], t.cs[i], -(y[i] * t.sn[i]));
            q[i] = kv >= v.g ? y[i] : fmaf(y[i], t.cs[i], x[i] * t.sn[i]);
        }
        if (r < nq) {
            T *to = (T *)a.q_out + ((size_t)token * v.h + r) * 128;
            store_chunk(to + 8 * i8, p);
            store_chunk(to + 64 + 8 * i8, q);
        } else if (t.page < v.num_pages) {
            const int64_t to = (((int64_t)t.page * v.g + (kv < v.g ? kv : kv - v.g)) << v.page_shift) + (t.slot & ((1 << v.page_shift) - 1));
            store_codes<STORE>(kv < v.g ? qa.k : qa.v, to, i8, p, q);
        }
        r = next;
    }
}

// ---- reading back -------------------------------------------------------------------------------------------
struct QuantReadArgs {
    CacheView v;              // (cu: null)
    const int32_t *first;     // [batch] or null: the first token that is read
    const uint8_t *codes[2];  // K, V; null: not read
    const float *scales[2];
    void *out[2];             // [out_pages][g][page][128]
    const int32_t *out_table; // [batch][out_cols]
    int out_cols;
    uint32_t out_pages;
};
// four codes times their row's scale
template <int STORE> __device__ __forceinline__ f32x4_t decode(uint32_t w, float scale)
{
    if constexpr (STORE == kInt8) {
        return f32x4_t{(float)(int8_t)w, (float)(int8_t)(w >> 8), (float)(int8_t)(w >> 16), (float)(int8_t)(w >> 24)} * scale;
    } else {
        const auto a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
        return f32x4_t{a[0], a[1], b[0], b[1]} * scale;
    }
}
// A block takes runs of 64 tokens of a unit: 16 lanes a row, 8 codes a lane, so that a row's values are written in a line, and four rows a lane on their way at once.
// Memory bounds it: 32K tokens in 44 us, 4.6 TB/s, where a copy reaches 4.8.
template <typename T, int STORE> __global__ __launch_bounds__(256) void quant_read_kernel(QuantReadArgs a)
{
    constexpr int kRun = 64, kEach = 4;
    const CacheView &v = a.v;
    const int b = blockIdx.x / v.g, kv = blockIdx.x % v.g, i16 = threadIdx.x & 15;
    const int len = min(max(v.cur[b], 0), v.max_pages << v.page_shift), from = a.first ? max(a.first[b], 0) : 0;
    const int n = min(len - from, a.out_cols << v.page_shift), mask = (1 << v.page_shift) - 1;
    for (int run = blockIdx.y * kRun; run < n; run += gridDim.y * kRun) {
        int64_t src[kEach], dst[kEach];
        bool ok[kEach];
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
            const int j = run + 16 * e + (threadIdx.x >> 4), at = min(j, n - 1);
            const uint32_t page = (uint32_t)a.out_table[(size_t)b * a.out_cols + (at >> v.page_shift)];
            src[e] = cache_row(v, b, kv, from + at);
            dst[e] = (((int64_t)page * v.g + kv) << v.page_shift) + (at & mask);
            ok[e] = j < n && src[e] >= 0 && page < a.out_pages;
            if (!ok[e]) src[e] = 0;
        }
        uint2 w[2][kEach];
        float scale[2][kEach];
#pragma unroll
        for (int x = 0; x < 2; ++x)
            if (a.codes[x]) {
#pragma unroll
                for (int e = 0; e < kEach; ++e) {
                    w[x][e] = *reinterpret_cast<const uint2 *>(a.codes[x] + src[e] * 128 + 8 * i16);
                    scale[x][e] = a.scales[x][src[e]];
                }
            }
#pragma unroll
        for (int x = 0; x < 2; ++x)
            if (a.codes[x]) {
#pragma unroll
                for (int e = 0; e < kEach; ++e) {
                    if (!ok[e]) continue;
                    const f32x4_t lo = decode<STORE>(w[x][e].x, scale[x][e]), hi = decode<STORE>(w[x][e].y, scale[x][e]);
                    const float y[8] = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
                    store_chunk((T *)a.out[x] + dst[e] * 128 + 8 * i16, y);
                }
            }
    }
}

// ---- attention ----------------------------------------------------------------------------------------------
// locate_tile with the sequence's span, from the lane that has looked it up: no second trip to memory
template <int LOG> __device__ __forceinline__ bool locate_span(const CacheView &v, int tile, int *b, int *at, SeqSpan *s)
{
    const int lane = threadIdx.x & 63;
    int base = 0;
    for (int b0 = 0; b0 < v.batch; b0 += 64) {
        SeqSpan mine{};
        if (b0 + lane < v.batch) mine = seq_span(v, b0 + lane);
        const int tiles = ((mine.n << v.lg) + (1 << LOG) - 1) >> LOG;
        int upto = tiles;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int o = __shfl_up(upto, d);
            if (lane >= d) upto += o;
        }
        const int all = __builtin_amdgcn_readlane(upto, 63);
        if (tile < base + all) {
            const int l = __builtin_ctzll(__ballot(base + upto > tile));
            *b = b0 + l;
            *at = tile - base - (__builtin_amdgcn_readlane(upto, l) - __builtin_amdgcn_readlane(tiles, l));
            *s = SeqSpan{__builtin_amdgcn_readlane(mine.c0, l), __builtin_amdgcn_readlane(mine.n, l), __builtin_amdgcn_readlane(mine.len, l),
                         __builtin_amdgcn_readlane(mine.old, l)};
            return true;
        }
        base += all;
    }
    return false;
}

struct QuantAttnArgs {
    AttnArgs a;                         // (k_pages and v_pages are codes)
    const float *k_scales, *v_scales;   // [num_pages][g][page]: a row's number is its scale's
};

// eight codes as bf16, exactly
template <int STORE> __device__ __forceinline__ bf16x8_t codes8(uint32_t lo, uint32_t hi)
{
    bf16x8_t x;
    if constexpr (STORE == kInt8) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[i] = (__bf16)(float)(int8_t)(lo >> (8 * i));
            x[4 + i] = (__bf16)(float)(int8_t)(hi >> (8 * i));
        }
    } else {
        union { bf16x2_t h[4]; bf16x8_t w; } u;
        u.h[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)lo, 1.0f, false);
        u.h[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)lo, 1.0f, true);
        u.h[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)hi, 1.0f, false);
        u.h[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)hi, 1.0f, true);
        x = u.w;
    }
    return x;
}
// ... as fp16
template <int STORE> __device__ __forceinline__ f16x8_t codes8h(uint32_t lo, uint32_t hi)
{
    union { f16x2_t h[4]; f16x8_t w; } u;
    if constexpr (STORE == kInt8) {
        // the byte 128 + code as the last of the mantissa of 1024 + it, less 1152
        lo ^= 0x80808080u;
        hi ^= 0x80808080u;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t pair = __builtin_amdgcn_perm(0x64646464u, i < 2 ? lo : hi, (i & 1) ? 0x04030402u : 0x04010400u);
            u.h[i] = __builtin_bit_cast(f16x2_t, pair) - f16x2_t{(_Float16)1152.0f, (_Float16)1152.0f};
        }
    } else {
        u.h[0] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)lo, 1.0f, false);
        u.h[1] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)lo, 1.0f, true);
        u.h[2] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)hi, 1.0f, false);
        u.h[3] = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8((int)hi, 1.0f, true);
    }
    return u.w;
}
// e4m3's two NaN codes become 0: memory behind a sequence or before its window may hold them, and 0 times NaN is no 0
template <int STORE> __device__ __forceinline__ uint32_t no_nan(uint32_t w)
{
    if constexpr (STORE == kInt8) return w;
    const uint32_t nan = ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
    return w & ~(nan | (nan - (nan >> 7)));
}

// x as the sum of PARTS values, the first the nearest: three of bf16 have all bits of an fp32 value, two of fp16 all but two.  What is left of x is less the part as it was
// rounded: where x is a product the compiler would otherwise round it to fp16 in one step for the part and in two for the difference, and where these do not agree, one
// time in ten thousand, the sum is off by 2^-10 (outputs of 128 tokens on 32K keys by 9.7e-6 where 9e-7 is what the sums leave; the time is the same).
template <typename V, int PARTS> __device__ __forceinline__ void split_parts(const float (&x)[8], V (&part)[PARTS])
{
    using E = std::remove_reference_t<decltype(part[0][0] + part[0][0])>;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        float rest = x[j];
#pragma unroll
        for (int p = 0; p < PARTS; ++p) {
            E h = (E)rest;
            if (p + 1 < PARTS) {
                asm("" : "+v"(h));
                rest -= (float)h;
            }
            part[p][j] = h;
        }
    }
}
// The query's 8 elements from d on as parts
template <typename T, int PARTS> __device__ __forceinline__ void query_parts(const T *row, int d, bf16x8_t (&part)[PARTS])
{
    if constexpr (sizeof(T) == 2) {
        part[0] = *reinterpret_cast<const bf16x8_t *>(row + d);
    } else {
        const f32x4_t a = *reinterpret_cast<const f32x4_t *>(row + d), b = *reinterpret_cast<const f32x4_t *>(row + d + 4);
        const float x[8] = {a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
        split_parts(x, part);
    }
}

// 32 keys' scores or probabilities times their scales, which stand in shared memory in the keys' order
__device__ __forceinline__ void scale_regs(f32x16_t &s, const float *scales, int half)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const f32x4_t x = *reinterpret_cast<const f32x4_t *>(scales + 8 * i + 4 * half);
#pragma unroll
        for (int c = 0; c < 4; ++c) s[4 * i + c] *= x[c];
    }
}
// ... times their scales times `by`, which brings scales that probabilities above 1 would take beyond fp32 into range first
__device__ __forceinline__ void scale_regs_by(f32x16_t &s, const float *scales, float by, int half)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const f32x4_t x = *reinterpret_cast<const f32x4_t *>(scales + 8 * i + 4 * half);
#pragma unroll
        for (int c = 0; c < 4; ++c) s[4 * i + c] *= x[c] * by;
    }
}

// Values' scales as they multiply probabilities: times 2^(11 - exponent) = 2^(kWeightPower - exponent), where 2^exponent is above every scale that the row has seen so
// far, and probabilities are under a maximum that may lag by kLag = 4 powers of two, so that a weight is below 2^15, and one under its row's true maximum has all of
// fp16's bits down to 2^-25 of 2^exponent; what is left of smaller ones is off by 2^-36 of that at most.  An exponent is a row's own where rows see different keys: a value
// that one token sees and its neighbour does not may be any size.  The outputs are scaled as the exponent grows, once or twice in a run of keys as a rule, and as a maximum
// grows by more than 16 times; without the lag a row of few keys has a new one in most tiles (2048 tokens on 32K keys 1250 -> 1225 us, drafts of 2 to 24 tokens
// 101 -> 98).
constexpr int kLag = 4, kWeightPower = 15 - kLag, kLeastExponent = -80;
// (Scales may have either sign: what counts is their magnitude.)
// the least power of two above a magnitude, from kLeastExponent on.  (0 and NaN: kLeastExponent; a row that sees NaN becomes NaN anyway.)
__device__ __forceinline__ int exponent_above(float scale)
{
    return scale > 0.0f ? max((int)(__float_as_uint(scale) >> 23) - 126, kLeastExponent) : kLeastExponent;
}
// above a wave's scales together (NaN: as 0)
__device__ __forceinline__ int exponent_of_all(float scale)
{
    uint32_t bits = fabsf(scale) > 0.0f ? __float_as_uint(fabsf(scale)) : 0u;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) bits = max(bits, (uint32_t)__shfl_xor((int)bits, d));
    return max(__builtin_amdgcn_readfirstlane((int)(bits >> 23)) - 126, kLeastExponent);
}
__device__ __forceinline__ void scale_outputs(f32x16_t (&o)[4], int by)   // by 2^by, of the lane's row
{
    const float f = ldexpf(1.0f, by);
#pragma unroll
    for (int db = 0; db < 4; ++db)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[db][i] *= f;
}

}  // namespace ctkvr
