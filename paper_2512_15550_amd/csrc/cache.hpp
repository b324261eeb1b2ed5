// Kernels of the operators on the paged KV cache: append with rotary positions, attention of new tokens, accumulated attention weights,
// eviction.  gfx950, wave64, matrix cores.
//
// Rows.  The G query heads that share a KV head are rows of one problem: row r of a (sequence, KV head) unit is head r % G of the
// sequence's new token r / G, so a tile of rows reads each key once for the whole group.
//
// Scores come transposed, S^T = K Q^T: in the 32 x 32 result a lane holds one row (column lane % 32) and 16 keys, so that a row's maximum and
// sum are a chain within the lane and one exchange with the other half of the wave, and the probabilities are, where they stand, the B operand of the
// next product O^T = V^T P^T for keys in the order 8 a + 4 (lane / 32) + c, which V's operand follows.
#pragma once
#include "cache_args.hpp"
#include "common.hpp"

namespace ctkvr {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef short s16x8_t __attribute__((ext_vector_type(8)));

#define CTKVR_LDS __attribute__((address_space(3)))

constexpr uint32_t kNoRow = 0xffffffffu;
constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;

// Tile `tile` of the tiles of 2^LOG rows that the batch's units of one KV head fall into, sequence by sequence: its sequence and its
// number there (by one wave; every lane gets them)
template <int LOG> __device__ __forceinline__ bool locate_tile(const CacheView &v, int tile, int *b, int *at)
{
    const int lane = threadIdx.x & 63;
    int base = 0;
    for (int b0 = 0; b0 < v.batch; b0 += 64) {
        int mine = 0;
        if (b0 + lane < v.batch) mine = (((seq_span(v, b0 + lane).n << v.lg) + (1 << LOG) - 1) >> LOG);
        int upto = mine;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int o = __shfl_up(upto, d);
            if (lane >= d) upto += o;
        }
        const int all = __builtin_amdgcn_readlane(upto, 63);
        if (tile < base + all) {
            const int l = __builtin_ctzll(__ballot(base + upto > tile));
            *b = b0 + l;
            *at = tile - base - (__builtin_amdgcn_readlane(upto, l) - __builtin_amdgcn_readlane(mine, l));
            return true;
        }
        base += all;
    }
    return false;
}

// ---- tiles of 128-element rows in shared memory ------------------------------------------------------
// 16 KB: 64 rows of bf16 or 32 of fp32.  The 16-byte chunk c of row r stands at chunk c ^ swz(r): the 32 rows that an operand of the
// matrix instructions reads at one chunk, and the four rows at two chunks that the transposing load takes, then fall on all banks alike.
template <typename T> struct RowTile {
    static constexpr int kRows = sizeof(T) == 2 ? 64 : 32, kRowBytes = 128 * sizeof(T), kChunks = kRowBytes / 16;
    static constexpr int kRowsPerLoad = 64 / kChunks;   // rows of one load of a wave
    static constexpr int kBytes = kRows * kRowBytes;
};
template <typename T> __device__ __forceinline__ int swz(int row)
{
    if constexpr (sizeof(T) == 2) return ((row & 3) << 2) | ((row >> 2) & 3);
    else return row & 15;
}
// 16 bytes a lane from `from` straight into shared memory at byte `to` + 16 * lane (uniform `to`); waited for like a load
__device__ __forceinline__ void row_to_lds(uint32_t to, const void *from)
{
    asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %1, off" :: "{m0}"(__builtin_amdgcn_readfirstlane(to)), "v"(from) : "memory");
}
__device__ __forceinline__ uint32_t lds_at(const void *p) { return (uint32_t)(uintptr_t)(const CTKVR_LDS void *)p; }

// Waits until at most N of the wave's loads are in flight.  (The builtin, which the compiler reckons with; of loads in assembly it does not know, so
// that neither its own waits nor a barrier would be enough.)
template <int N> __device__ __forceinline__ void loads_landed()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | 0x0f70);
    asm volatile("" ::: "memory");
}

// ... and until shared memory has answered
__device__ __forceinline__ void settled()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0x0070);
    asm volatile("" ::: "memory");
}

// One exchange between the halves of a wave
__device__ __forceinline__ float half_max(float x)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float half_sum(float x)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// A row's part of a product's operand: lane (row, half) holds the chunks 2 i + half
template <typename T> struct Operand;
template <> struct Operand<bf16_t> { bf16x8_t c[8]; };
template <> struct Operand<float> { f32x4_t c[16]; };
template <typename T> __device__ __forceinline__ void load_operand(Operand<T> &o, const T *row, int half)
{
    using C = std::remove_reference_t<decltype(o.c[0])>;
#pragma unroll
    for (int i = 0; i < (int)(sizeof(o.c) / 16); ++i) o.c[i] = *reinterpret_cast<const C *>(reinterpret_cast<const char *>(row) + 32 * i + 16 * half);
}
// acc += A B^T over 128 dimensions: A's row lane % 32 of a tile in shared memory from row r0 on, B an operand in registers
template <typename T> __device__ __forceinline__ f32x16_t rows_dot(const char *tile, int r0, const Operand<T> &b, f32x16_t acc)
{
    const int lane = threadIdx.x & 63, r = r0 + (lane & 31), half = lane >> 5, s = swz<T>(r);
    const char *row = tile + r * RowTile<T>::kRowBytes;
    if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const bf16x8_t a = *reinterpret_cast<const bf16x8_t *>(row + (((2 * i + half) ^ s) << 4));
            acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b.c[i], acc, 0, 0, 0);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const f32x4_t a = *reinterpret_cast<const f32x4_t *>(row + (((2 * i + half) ^ s) << 4));
#pragma unroll
            for (int e = 0; e < 4; ++e) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(a[e], b.c[i][e], acc, 0, 0, 0);
        }
    }
    return acc;
}

// ---- scores ------------------------------------------------------------------------------------------
constexpr int kCap = 1, kBias = 2;
// scores times log2 e, from the dot products (without cap and bias the factor is left to the exponent)
// (of N registers, whose keys are STRIDE (i / 4) + i % 4 + 4 part)
template <int OPT, int N = 16, int STRIDE = 8, typename V> __device__ __forceinline__ void score_regs(V &s, const ScoreOpts &o, float slope2, int pos_minus_key0, int part)
{
    if constexpr (OPT != 0) {
        if constexpr ((OPT & kCap) != 0) {
            // cap tanh(x), x = score / cap: up to the cap, where scores are as a rule, by the fifth convergent of tanh's continued fraction, off by 1e-7 of it
            // at most; beyond by (1 - e) / (1 + e), e = exp(-2 |x|), which loses nothing there.  Which of them a score gets is its own size's matter, so that no
            // other key or row has a part in it; the wave only leaves the second out, half of the instructions, where none of its scores needs it.
            float big = 0.0f;
#pragma unroll
            for (int i = 0; i < N; ++i) big = fmaxf(big, fabsf(s[i]));
            auto capped = [&](float z, auto beyond) {
                const float x = z * o.cap_in, y = x * x;
                float n = x * fmaf(y, fmaf(y, o.cap_out, o.cap_105), o.cap_945), d = fmaf(y, fmaf(y, 15.0f, 420.0f), 945.0f);
                if constexpr (decltype(beyond)::value) {
                    const float e = exp2_fast(fabsf(x) * (-2.0f * kLog2e));
                    const bool far = fabsf(x) > 1.0f;
                    n = far ? copysignf(o.cap_out - o.cap_out * e, x) : n;
                    d = far ? 1.0f + e : d;
                }
                return n * __builtin_amdgcn_rcpf(d);
            };
            if (__any(big * o.cap_in > 1.0f)) {
#pragma unroll
                for (int i = 0; i < N; ++i) s[i] = capped(s[i], std::true_type());
            } else {
#pragma unroll
                for (int i = 0; i < N; ++i) s[i] = capped(s[i], std::false_type());
            }
        }
        const float far = (float)(pos_minus_key0 - 4 * part);   // (distances below 2^24 are exact)
#pragma unroll
        for (int i = 0; i < N; ++i) {
            float z = (OPT & kCap) ? s[i] : s[i] * o.c2;
            if constexpr ((OPT & kBias) != 0) z = fmaf(-slope2, fabsf(far - (float)(STRIDE * (i >> 2) + (i & 3))), z);
            s[i] = z;
        }
    }
}

static __global__ void cache_clear_kernel(uint32_t *p, size_t n)
{
    const size_t i = (size_t)blockIdx.x * blockDim.x + threadIdx.x;
    if (i < n) p[i] = 0;
}

// ---- attention of new tokens --------------------------------------------------------------------------
struct AttnArgs {
    CacheView v;
    ScoreOpts o;
    const void *q;
    int64_t q_stride;          // elements from a token to the next
    const void *k_pages, *v_pages;
    void *out;                 // [total][h][128]
    float *lse;                // [total][h] or null
    int tiles;
    // where keys are split into runs: [nsplit][total][h][128] and [nsplit][total][h]; how many of a tile's runs are done
    float *part_o, *part_lse;
    uint32_t *done;            // [tiles][g], zero between calls; null: attn_join_kernel joins the runs
    int nsplit;
};

// A key that a row does not see has probability 0 there, but 0 times an infinity or NaN is no 0.  So where a tile has such keys for some row, values
// that are not finite are added to the rows that see them and then taken out of the tile.
template <typename T, int KEYS, int THREADS> struct OddValues {
    static constexpr int kWords = KEYS * 128 * (int)sizeof(T) / 4 / THREADS;
    static __device__ __forceinline__ bool any(const char *vt, int tid)
    {
        const u32x4_t *w = reinterpret_cast<const u32x4_t *>(vt) + tid;
        uint32_t odd = 0;
#pragma unroll
        for (int i = 0; i < kWords / 4; ++i) {
            const u32x4_t x = w[i * THREADS];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if constexpr (sizeof(T) == 2) odd |= ((x[e] & 0x7f807f80u) + 0x00800080u) & 0x80008000u;
                else odd |= ((x[e] & 0x7f800000u) + 0x00800000u) & 0x80000000u;
            }
        }
        return odd != 0;
    }
    static __device__ __forceinline__ void clean(char *vt, int tid)
    {
        uint32_t *w = reinterpret_cast<uint32_t *>(vt) + tid;
        for (int i = 0; i < kWords; ++i) {
            uint32_t x = w[i * THREADS];
            if constexpr (sizeof(T) == 2) {
                if ((x & 0x7f80u) == 0x7f80u) x &= 0xffff0000u;
                if ((x & 0x7f800000u) == 0x7f800000u) x &= 0xffffu;
            } else if ((x & 0x7f800000u) == 0x7f800000u)
                x = 0;
            w[i * THREADS] = x;
        }
    }
    // sees(k): whether the lane's row sees key k of the tile
    template <typename F> static __device__ __forceinline__ void add(f32x16_t (&o)[4], const char *vt, int half, F sees_key)
    {
        for (int n = 0; n < KEYS; ++n) {
            int k = n;
            asm volatile("" : "+s"(k));   // (its addresses are not worth registers in the loop over the tiles)
            const bool sees = sees_key(k);
#pragma unroll
            for (int db = 0; db < 4; ++db)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int d = 32 * db + 8 * (i >> 2) + 4 * half + (i & 3), c = d * (int)sizeof(T) / 16;
                    const char *p = vt + k * RowTile<T>::kRowBytes + ((c ^ swz<T>(k)) << 4) + (d * (int)sizeof(T) & 15);
                    float x;
                    if constexpr (sizeof(T) == 2) x = __uint_as_float((uint32_t)*reinterpret_cast<const bf16_t *>(p) << 16);
                    else x = *reinterpret_cast<const float *>(p);
                    if (sees && !(fabsf(x) < INFINITY)) o[db][i] += x;
                }
        }
    }
};

// Of 32 keys from key0 on (bad: those that are not there), what a row does not see becomes `none`
__device__ __forceinline__ void mask_regs(f32x16_t &s, const RowSight &sight, int key0, uint32_t bad, int half, float none)
{
    const int lo = sight.lo - key0 - 4 * half, hi = sight.hi - key0 - 4 * half;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
        const int k = 8 * (i >> 2) + (i & 3);
        s[i] = k >= lo && k < hi ? s[i] : none;
    }
    if (bad) {
        const uint32_t mine = bad >> (4 * half);
#pragma unroll
        for (int i = 0; i < 16; ++i) s[i] = (mine >> (8 * (i >> 2) + (i & 3))) & 1 ? none : s[i];
    }
}

// ... and where that is not a range
__device__ __forceinline__ void mask_bits(f32x16_t &s, uint32_t seen, int half, float none)
{
    const uint32_t mine = seen >> (4 * half);
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = (mine >> (8 * (i >> 2) + (i & 3))) & 1 ? s[i] : none;
}

// A tile's scores to probabilities under the running maximum m (in units of log2 e, as all exponents here), their sum to l, the outputs so far to the
// new maximum.  (A maximum that may be left behind by a few powers of two, so that fewer tiles scale the outputs, was 2 % faster on 2048 tokens of 32K keys, 1130 and
// 1106 us; but the weight of a row's largest score is 1 now, which bf16 holds exactly, and the outputs there were off by 2.3e-3 in place of 2.0e-3, those of a
// single token by 2.1e-3 in place of 1.7e-3.  LAG: by so many; weights in fp16 lose nothing by it.)  While m is -infinity the outputs are 0, or infinities that stay.
template <int OPT, int NB, int LAG = 0> __device__ __forceinline__ void softmax_regs(f32x16_t (&sc)[NB], f32x16_t (&o)[4], float &m, float &l, float c2)
{
    float top = -INFINITY;
#pragma unroll
    for (int kb = 0; kb < NB; ++kb)
#pragma unroll
        for (int i = 0; i < 16; ++i) top = fmaxf(top, sc[kb][i]);
    top = half_max(top);
    if constexpr (OPT == 0) top *= c2;
    if (__any(LAG ? top > m + (float)LAG : top > m)) {
        const float m_new = fmaxf(m, top), scale = m == -INFINITY ? 1.0f : exp2_fast(m - m_new);
        m = m_new;
        l *= scale;
#pragma unroll
        for (int db = 0; db < 4; ++db)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[db][i] *= scale;
    }
    const float ref = m == -INFINITY ? 0.0f : m;
#pragma unroll
    for (int kb = 0; kb < NB; ++kb)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const float p = exp2_fast(OPT == 0 ? fmaf(sc[kb][i], c2, -ref) : sc[kb][i] - ref);
            l += p;
            sc[kb][i] = p;
        }
}

// O^T += V^T P^T.  In bf16 the probabilities are rounded to the values' type, as the matrix cores take them: off by 2^-8 of themselves at most, which
// is what rounding the output costs; the sum under them is of the unrounded ones.
template <typename T, int NB> __device__ __forceinline__ void values_dot(f32x16_t (&o)[4], const char *vt, const f32x16_t (&sc)[NB], int lane)
{
    const int half = lane >> 5;
#pragma unroll
    for (int kb = 0; kb < NB; ++kb) {
        if constexpr (sizeof(T) == 2) {
#pragma unroll
            for (int ks = 0; ks < 2; ++ks) {
                bf16x8_t p;
#pragma unroll
                for (int j = 0; j < 8; ++j) p[j] = (__bf16)sc[kb][8 * ks + j];
#pragma unroll
                for (int db = 0; db < 4; ++db) {
                    union { s16x4_t h[2]; bf16x8_t w; } x;
#pragma unroll
                    for (int aa = 0; aa < 2; ++aa) {
                        const int k = 32 * kb + 16 * ks + 8 * aa + 4 * half + ((lane & 15) >> 2);
                        const int c = (4 * db + 2 * ((lane & 31) >> 4) + ((lane & 3) >> 1)) ^ swz<T>(k);
                        x.h[aa] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((CTKVR_LDS s16x4_t *)(vt + k * 256 + (c << 4) + 8 * (lane & 1)));
                    }
                    o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x.w, p, o[db], 0, 0, 0);
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int k = 32 * kb + 8 * (i >> 2) + 4 * half + (i & 3), s = swz<T>(k);
#pragma unroll
                for (int db = 0; db < 4; ++db) {
                    const int d = 32 * db + (lane & 31);
                    const float x = *reinterpret_cast<const float *>(vt + k * 512 + (((d >> 2) ^ s) << 4) + 4 * (d & 3));
                    o[db] = __builtin_amdgcn_mfma_f32_32x32x2f32(x, sc[kb][i], o[db], 0, 0, 0);
                }
            }
        }
    }
}

// keys that some token of tok0 .. tok1 sees, and those that all of them see, as far as positions say
struct KeyRange {
    int hi, all_hi;
};
__device__ __forceinline__ KeyRange key_range(const SeqSpan &s, int prefix, int tok0, int tok1)
{
    const int pos0 = s.old + tok0, pos1 = s.old + tok1;
    KeyRange r;
    r.hi = pos1 < 0 ? 0 : min(max(pos1 + 1, prefix), s.len);
    r.all_hi = pos0 < 0 ? 0 : min(max(pos0 + 1, prefix), s.len);
    return r;
}
template <int SIGHT> __device__ __forceinline__ KeyRange key_range_of(const SeqSpan &s, int prefix, int tok0, int tok1)
{
    KeyRange r = key_range(s, SIGHT == kRange ? prefix : 0, tok0, tok1);
    if constexpr (SIGHT == kTree) {
        r.hi = s.old + tok1 < 0 ? 0 : s.len;
        r.all_hi = s.old + tok0 < 0 ? 0 : min(s.old, s.len);
    }
    return r;
}

template <typename T> __device__ __forceinline__ void store4(T *p, const f32x4_t &x)
{
    if constexpr (sizeof(T) == 2) {
        bf16x4_t y;
#pragma unroll
        for (int c = 0; c < 4; ++c) y[c] = (__bf16)x[c];
        *reinterpret_cast<bf16x4_t *>(p) = y;
    } else {
        *reinterpret_cast<f32x4_t *>(p) = x;
    }
}
// What blocks of a launch hand to each other goes past the caches that they do not share, word by word: a fence, which would write back and invalidate a whole L2
// for each of them, made a step of 16 sequences take 770 us in place of 440.
__device__ __forceinline__ void hand_over(float *p, const f32x4_t &x)
{
    union { f32x4_t f; unsigned long long w[2]; } u{x};
#pragma unroll
    for (int i = 0; i < 2; ++i)
        __hip_atomic_store(reinterpret_cast<unsigned long long *>(p) + i, u.w[i], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ void hand_over(float *p, float x) { __hip_atomic_store(p, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ f32x4_t handed4(const float *p)
{
    union { f32x4_t f; unsigned long long w[2]; } u;
#pragma unroll
    for (int i = 0; i < 2; ++i)
        u.w[i] = __hip_atomic_load(reinterpret_cast<const unsigned long long *>(p) + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    return u.f;
}
__device__ __forceinline__ float handed(const float *p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ float inv_sum(float l) { return l == 0.0f ? 0.0f : 1.0f / l; }   // (NaN stays)
__device__ __forceinline__ float lse_of(float m, float l) { return l == 0.0f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2; }

// the first dimension of a row's chunk c of 8, in order
struct ColumnsInOrder {
    static constexpr int column(int c) { return 8 * c; }
};
// A row's outputs, or its run's, from its sum l and maximum m
template <typename T, typename ORDER = ColumnsInOrder>
__device__ __forceinline__ void many_finish(const AttnArgs &a, const SeqSpan &s, int split, bool empty, bool live, int token, int head, float m, float l,
                                            const f32x16_t (&o)[4], int half)
{
    const CacheView &v = a.v;
    if (!live) return;
    const float inv = inv_sum(l), lse = lse_of(m, l);
    const size_t at_row = (size_t)(s.c0 + token) * v.h + head;
    const size_t n = (size_t)split * v.total * v.h + at_row;
    if (half == 0) {
        if (a.nsplit > 1) a.part_lse[n] = lse;
        else if (a.lse) a.lse[at_row] = lse;
    }
    if (a.nsplit > 1 && empty) return;
#pragma unroll
    for (int db = 0; db < 4; ++db)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int d = ORDER::column(4 * db + i) + 4 * half;
            f32x4_t x;
#pragma unroll
            for (int c = 0; c < 4; ++c) x[c] = o[db][4 * i + c] * inv;
            if (a.nsplit > 1) store4(a.part_o + n * 128 + d, x);
            else store4((T *)a.out + at_row * 128 + d, x);
        }
}

// Many rows: one block a tile of 32 NW rows of a unit and, where the keys are split, one of nsplit runs of them; a wave has 32 rows.  Each tile of keys goes straight to shared memory while the one before it is worked on; the maximum runs with them.
template <typename T, int OPT, int NW, int SIGHT = kRange> __global__ __launch_bounds__(64 * NW, sizeof(T) == 2 ? 2 : 1) void attn_kernel(AttnArgs a)
{
    constexpr int kRowsLog = NW == 4 ? 7 : 8, kKeys = RowTile<T>::kRows, kBlocks = kKeys / 32, kTile = RowTile<T>::kBytes;
    constexpr int kPer = RowTile<T>::kRowsPerLoad, kLoads = kKeys / (NW * kPer);   // loads a wave makes of a tile of K, and of V
    using Odd = OddValues<T, kKeys, 64 * NW>;
    static_assert(NW == 4 || NW == 8, "");
    __shared__ __align__(16) char smem[2][2][kTile];   // [buffer][K, V]
    const CacheView &v = a.v;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
    // (a KV head's tiles stay on an XCD where the heads are a multiple of 8; the tiles with most keys go first)
    const int kv = blockIdx.x % v.g, rest = blockIdx.x / v.g, split = rest % a.nsplit;
    int b, at;
    if (!locate_tile<kRowsLog>(v, a.tiles - 1 - rest / a.nsplit, &b, &at)) return;
    const SeqSpan s = seq_span(v, b);
    const int rows = s.n << v.lg, r0 = at << kRowsLog, row = r0 + 32 * wave + (lane & 31);
    const int prefix = a.o.prefix ? min(max(a.o.prefix[b], 0), s.len) : 0;
    const int token = min(row, rows - 1) >> v.lg, head = (kv << v.lg) + (min(row, rows - 1) & ((1 << v.lg) - 1));
    const RowSight sight = sight_of<SIGHT>(v, a.o, s, prefix, token);

    Operand<T> q;
    load_operand(q, (const T *)a.q + (int64_t)(s.c0 + token) * a.q_stride + head * 128, half);

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
        int *ex = reinterpret_cast<int *>(smem);
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

    // KV row of key (tile, lane), and which keys of a tile have none.  Those, and what lies behind the last key, take a row
    // that is there: whatever the memory behind them holds reaches no product.
    const int max_key = max(range.hi - 1, 0);
    uint64_t bad = 0;
    auto rows_of = [&](int t) -> uint32_t {
        const uint32_t r = (uint32_t)cache_row(v, b, kv, min(t * kKeys + (lane & (kKeys - 1)), max_key));
        const uint64_t ok = __ballot(r != kNoRow);
        bad = ~ok;
        if (ok == ~0ull) return r;
        if (!ok) return 0;
        const uint32_t other = __builtin_amdgcn_readlane(r, __builtin_ctzll(ok));
        return r != kNoRow ? r : other;
    };
    // A wave's share of a tile, 16 keys (8 in fp32) at a time.  Where they are in one page the distance to the first of them is the same in every tile and
    // the address of that one is the wave's, not a lane's.
    const uint32_t lds0 = __builtin_amdgcn_readfirstlane(lds_at(smem));
    constexpr int kShare = kKeys / NW;
    const bool one_page = (1 << v.page_shift) >= kShare;
    uint32_t lane_off[kLoads];
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
        const int in = j * kPer + lane / RowTile<T>::kChunks;
        lane_off[j] = in * RowTile<T>::kRowBytes + 16 * ((lane % RowTile<T>::kChunks) ^ swz<T>(wave * kShare + in));
    }
    auto fetch = [&](int buf, uint32_t r, bool whole) {
        const uint32_t to = lds0 + buf * 2 * kTile + wave * kShare * RowTile<T>::kRowBytes;
        if (one_page && whole) {
            const int64_t from = (int64_t)(uint32_t)__builtin_amdgcn_readlane(r, wave * kShare) * RowTile<T>::kRowBytes;
            const char *k = (const char *)a.k_pages + from, *x = (const char *)a.v_pages + from;
#pragma unroll
            for (int j = 0; j < kLoads; ++j) {
                load_to_lds(to + j * 1024, k, lane_off[j]);
                load_to_lds(to + j * 1024 + kTile, x, lane_off[j]);
            }
            return;
        }
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
            const int in = j * kPer + lane / RowTile<T>::kChunks;
            const int64_t from = (int64_t)(uint32_t)__shfl((int)r, wave * kShare + in) * RowTile<T>::kRowBytes + (lane_off[j] - in * RowTile<T>::kRowBytes);
            row_to_lds(to + j * 1024, (const char *)a.k_pages + from);
            row_to_lds(to + j * 1024 + kTile, (const char *)a.v_pages + from);
        }
    };

    f32x16_t o[4] = {};
    float m = -INFINITY, l = 0.0f;
    const float slope2 = (OPT & kBias) ? a.o.slopes[head] * kLog2e : 0.0f;
    uint64_t bad_now = 0;
    uint32_t next = 0;
    // tile t in buffer `buf`, with the tile behind it on its way; MASKED: some row may not see some key
    auto step = [&](auto buf, auto masked, int t) {
        const uint64_t bad_next = bad;
        if (t + 1 < t1) {
            fetch(buf ^ 1, next, bad == 0 && (tile_of(t + 1) + 1) * kKeys <= range.hi);
            if (t + 2 < t1) next = rows_of(tile_of(t + 2));
        }
        char *kt = smem[buf][0], *vt = smem[buf][1];
        const int key0 = tile_of(t) * kKeys;
        if constexpr (decltype(masked)::value) {
            if (__syncthreads_or(Odd::any(vt, threadIdx.x))) {
                if constexpr (SIGHT == kRange) {
                    Odd::add(o, vt, half, [&](int k) { return key0 + k >= sight.lo && key0 + k < sight.hi && !((bad_now >> k) & 1); });
                } else {
                    uint64_t seen = sight_bits<SIGHT>(a.o, s, sight, token, key0);
                    if (kBlocks > 1) seen |= (uint64_t)sight_bits<SIGHT>(a.o, s, sight, token, key0 + 32) << 32;
                    seen &= ~bad_now;
                    Odd::add(o, vt, half, [&](int k) { return (bool)((seen >> k) & 1); });
                }
                __syncthreads();
                Odd::clean(vt, threadIdx.x);
                __syncthreads();
            }
        }
        f32x16_t sc[kBlocks];
#pragma unroll
        for (int kb = 0; kb < kBlocks; ++kb) sc[kb] = rows_dot<T>(kt, 32 * kb, q, f32x16_t{});
#pragma unroll
        for (int kb = 0; kb < kBlocks; ++kb) {
            score_regs<OPT>(sc[kb], a.o, slope2, sight.pos - (key0 + 32 * kb), half);
            if constexpr (decltype(masked)::value) {
                const uint32_t none = (uint32_t)(bad_now >> (32 * kb));
                if constexpr (SIGHT == kRange) mask_regs(sc[kb], sight, key0 + 32 * kb, none, half, -INFINITY);
                else mask_bits(sc[kb], sight_bits<SIGHT>(a.o, s, sight, token, key0 + 32 * kb) & ~none, half, -INFINITY);
            }
        }
        softmax_regs<OPT, kBlocks>(sc, o, m, l, a.o.c2);
        values_dot<T, kBlocks>(o, vt, sc, lane);
        bad_now = bad_next;
        loads_landed<0>();
        __syncthreads();
    };
    if (t0 < t1) {
        const uint32_t r = rows_of(tile_of(t0));
        bad_now = bad;
        fetch(0, r, bad == 0 && (tile_of(t0) + 1) * kKeys <= range.hi);
        if (t0 + 1 < t1) next = rows_of(tile_of(t0 + 1));
        loads_landed<0>();
        __syncthreads();
    }
    auto seen_by_all = [&](int i, uint64_t none) {
        const int t = tile_of(i);
        return (t + 1) * kKeys <= range.all_hi && (t * kKeys >= all_lo || (SIGHT == kWindow && (t + 1) * kKeys <= a.o.sinks)) && none == 0;
    };
    int t = t0;
    while (t < t1) {
        // (two at a time: where a tile is in shared memory is then part of the instructions)
        if (((t - t0) & 1) == 0)
            while (t + 1 < t1 && seen_by_all(t, bad_now) && seen_by_all(t + 1, bad)) {
                step(std::integral_constant<int, 0>(), std::false_type(), t);
                step(std::integral_constant<int, 1>(), std::false_type(), t + 1);
                t += 2;
            }
        if (t >= t1) break;
        step((t - t0) & 1, std::true_type(), t);
        ++t;
    }

    many_finish<T>(a, s, split, t0 == t1, row < rows, token, head, m, half_sum(l), o, half);
}

// The end of a tile of few rows, whose waves have left their outputs, all to one maximum, in shared memory (ROWS rows of 512 bytes a wave, 16-byte chunk c of row r at
// chunk c ^ r) and their own maxima and sums in `join`: they become one, the rows' or this run's, and the run that ends last joins the runs.
template <typename T, int NW, int ROWS>
__device__ __forceinline__ void few_join(const AttnArgs &a, const SeqSpan &s, int kv, int r0, int have, int tile, int split, int used, bool whole, char *smem,
                                         float (&join)[NW][2][ROWS], bool *last)
{
    const CacheView &v = a.v;
    auto row_out = [&](int r) { return (size_t)(s.c0 + ((r0 + r) >> v.lg)) * v.h + (kv << v.lg) + ((r0 + r) & ((1 << v.lg) - 1)); };
    for (int j = threadIdx.x; j < have * 32; j += 64 * NW) {   // (row, four elements)
        const int r = j >> 5, c = j & 31;
        float t = join[0][0][r], sum = 0.0f;
#pragma unroll
        for (int w = 1; w < NW; ++w) t = fmaxf(t, join[w][0][r]);
        f32x4_t x = {};
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            const float mw = join[w][0][r];
            sum += join[w][1][r] * (mw == -INFINITY ? 1.0f : exp2_fast(mw - t));
            x += *reinterpret_cast<const f32x4_t *>(smem + w * ROWS * 512 + r * 512 + ((c ^ r) << 4));
        }
        x *= inv_sum(sum);
        const float lse = lse_of(t, sum);
        const size_t at_row = row_out(r);
        if (!whole) {
            const size_t n = (size_t)split * v.total * v.h + at_row;
            if (a.done) {
                if (c == 0) hand_over(a.part_lse + n, lse);
                hand_over(a.part_o + n * 128 + 4 * c, x);
            } else {
                if (c == 0) a.part_lse[n] = lse;
                store4(a.part_o + n * 128 + 4 * c, x);
            }
        } else {
            if (c == 0 && a.lse) a.lse[at_row] = lse;
            store4((T *)a.out + at_row * 128 + 4 * c, x);
        }
    }
    if (whole || !a.done) return;

    // The run that ends last joins the tile's runs, in their order, by their log-sum-exps: 32 lanes a row, four elements a lane, and where the
    // rows are few several such groups a row, that take the runs in turn.
    loads_landed<0>();   // (stores too)
    __syncthreads();
    if (threadIdx.x == 0) {
        uint32_t *done = a.done + (size_t)tile * v.g + kv;
        *last = atomicAdd(done, 1u) == (uint32_t)used - 1;
        if (*last) *done = 0;
    }
    __syncthreads();
    if (!*last) return;
    constexpr int kGroups = 2 * NW;
    f32x4_t(*sums)[33] = reinterpret_cast<f32x4_t(*)[33]>(smem);   // [group][lane, or the weights' sum]
    int ways = kGroups;
    while (ways > 1 && ways * have > kGroups) ways >>= 1;
    const int group = threadIdx.x >> 5, l32 = threadIdx.x & 31, way = group % ways;
    const size_t step = (size_t)v.total * v.h;
    for (int base = 0; base < have; base += kGroups / ways) {
        const int r = base + group / ways;
        f32x4_t x = {};
        float top_lse = -INFINITY, sum = 0.0f, ref = 0.0f;
        if (r < have) {
            const float *lses = a.part_lse + row_out(r), *outs = a.part_o + row_out(r) * 128 + 4 * l32;
            for (int i = l32; i < used; i += 32) top_lse = fmaxf(top_lse, handed(lses + i * step));
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) top_lse = fmaxf(top_lse, __shfl_xor(top_lse, d));
            ref = top_lse == -INFINITY ? 0.0f : top_lse;
#pragma unroll 8
            for (int i = way; i < used; i += ways) {
                const float w = exp2_fast((handed(lses + i * step) - ref) * kLog2e);
                sum += w;
                x += handed4(outs + i * step * 128) * w;
            }
        }
        if (ways > 1) {
            sums[group][l32] = x;
            if (l32 == 0) sums[group][32][0] = sum;
            __syncthreads();
            if (way == 0)
                for (int w = 1; w < ways; ++w) {
                    x += sums[group + w][l32];
                    sum += sums[group + w][32][0];
                }
            __syncthreads();
        }
        if (r < have && way == 0) {
            if (l32 == 0 && a.lse) a.lse[row_out(r)] = sum == 0.0f ? -INFINITY : ref + __builtin_amdgcn_logf(sum) * kLn2;
            store4((T *)a.out + row_out(r) * 128 + 4 * l32, x * inv_sum(sum));
        }
    }
}
// ... from a wave's outputs of 32 rows
template <typename T, int NW>
__device__ __forceinline__ void few_finish(const AttnArgs &a, const SeqSpan &s, int kv, int r0, int have, int tile, int split, int used, bool whole, float m,
                                           float l, const f32x16_t (&o)[4], char *smem, float (&join)[NW][2][32], bool *last)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
    // the waves' outputs to one maximum, through shared memory (16-byte chunks at chunk ^ row)
    l = half_sum(l);
    if (half == 0) {
        join[wave][0][lane] = m;
        join[wave][1][lane] = l;
    }
    loads_landed<0>();
    __syncthreads();   // (and nobody needs its values any more)
    const int r32 = lane & 31;
    float top = join[0][0][r32];
#pragma unroll
    for (int w = 1; w < NW; ++w) top = fmaxf(top, join[w][0][r32]);
    const float scale = m == -INFINITY ? 1.0f : exp2_fast(m - top);
    char *mine = smem + wave * 32 * 512;
#pragma unroll
    for (int db = 0; db < 4; ++db)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f32x4_t x;
#pragma unroll
            for (int c = 0; c < 4; ++c) x[c] = o[db][4 * i + c] * scale;
            *reinterpret_cast<f32x4_t *>(mine + r32 * 512 + (((8 * db + 2 * i + half) ^ r32) << 4)) = x;
        }
    __syncthreads();
    few_join<T, NW, 32>(a, s, kv, r0, have, tile, split, used, whole, smem, join, last);
}

// Few rows: one block a tile of 32 rows and a run of their keys, which its waves share out, each with a maximum and outputs of its own until
// they are joined at the end; no wave waits for another before that.  Keys go to registers as operands, values to shared memory, a tile of 32 ahead.
template <typename T, int OPT, int NW, int SIGHT = kRange> __global__ __launch_bounds__(64 * NW, sizeof(T) == 2 ? 2 : 1) void attn_few_kernel(AttnArgs a)
{
    constexpr int kTile = 32 * RowTile<T>::kRowBytes, kPer = RowTile<T>::kRowsPerLoad, kLoads = 32 / kPer;
    using Odd = OddValues<T, 32, 64>;
    __shared__ __align__(16) char smem[NW][2][kTile];
    __shared__ float join[NW][2][32];
    __shared__ bool last;
    const CacheView &v = a.v;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
    const int kv = blockIdx.x % v.g, rest = blockIdx.x / v.g, split = rest % a.nsplit, tile = a.tiles - 1 - rest / a.nsplit;
    int b, at;
    if (!locate_tile<5>(v, tile, &b, &at)) return;
    const SeqSpan s = seq_span(v, b);
    const int rows = s.n << v.lg, r0 = at << 5, row = r0 + (lane & 31);
    const int prefix = a.o.prefix ? min(max(a.o.prefix[b], 0), s.len) : 0;
    const int token = min(row, rows - 1) >> v.lg, head = (kv << v.lg) + (min(row, rows - 1) & ((1 << v.lg) - 1));
    const RowSight sight = sight_of<SIGHT>(v, a.o, s, prefix, token);

    Operand<T> q;
    load_operand(q, (const T *)a.q + (int64_t)(s.c0 + token) * a.q_stride + head * 128, half);

    const int tok0 = r0 >> v.lg, tok1 = (min(r0 + 32, rows) - 1) >> v.lg;
    const KeyRange range = key_range_of<SIGHT>(s, prefix, tok0, tok1);
    int k_lo = 0, all_lo = 0;
    if (SIGHT == kWindow) {
        k_lo = max(s.old + tok0 + 1 - a.o.window, 0);
        all_lo = max(s.old + tok1 + 1 - a.o.window, 0);
    } else if (a.o.first) {
        k_lo = all_lo = sight.lo;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            k_lo = min(k_lo, __shfl_xor(k_lo, d));
            all_lo = max(all_lo, __shfl_xor(all_lo, d));
        }
    }
    int first_tile = k_lo / 32, tiles = range.hi > k_lo ? (range.hi + 31) / 32 - first_tile : 0;
    KeyTiles kt{};
    if constexpr (SIGHT == kWindow) {
        kt = window_tiles(a.o, k_lo, range.hi, 32);
        first_tile = kt.from;
        tiles = kt.to;
    }
    auto tile_of = [&](int i) { return SIGHT == kWindow ? kt.at(i) : i; };
    const int have = min(32, rows - r0);
    // as many of the runs as the keys are worth: two tiles a wave (in fp32 one) at least; the other blocks have nothing to do
    const int per = sizeof(T) == 2 ? 2 * NW : NW, used = max(1, min(a.nsplit, (tiles + per - 1) / per));
    auto row_out = [&](int r) { return (size_t)(s.c0 + ((r0 + r) >> v.lg)) * v.h + (kv << v.lg) + ((r0 + r) & ((1 << v.lg) - 1)); };
    if (split >= used) {
        if (!a.done && (int)threadIdx.x < have) a.part_lse[(size_t)split * v.total * v.h + row_out(threadIdx.x)] = -INFINITY;
        return;
    }
    const bool whole = a.nsplit == 1 || (a.done && used == 1);   // this block's outputs are the rows'
    const int64_t runs = (int64_t)used * NW, run = split * NW + wave;
    const int t0 = __builtin_amdgcn_readfirstlane(first_tile + (int)(tiles * run / runs));
    const int t1 = __builtin_amdgcn_readfirstlane(first_tile + (int)(tiles * (run + 1) / runs));

    // 64 of the table's entries at a time, a lane each
    const int max_key = max(range.hi - 1, 0);
    const int32_t *table = v.table + (size_t)b * v.max_pages;
    int e0 = -64;
    uint32_t page = 0;
    uint64_t bad = 0;
    auto rows_of = [&](int t) -> uint32_t {
        const int key = min(t * 32 + (lane & 31), max_key), e = key >> v.page_shift;
        const int last = min(t * 32 + 31, max_key) >> v.page_shift;
        if (last >= e0 + 64) {
            e0 = (t * 32) >> v.page_shift;
            page = (uint32_t)table[min(e0 + lane, v.max_pages - 1)];
            loads_landed<0>();
        }
        const uint32_t p = (uint32_t)__shfl((int)page, e - e0);
        const uint32_t r = p < v.num_pages ? (uint32_t)((p * (uint64_t)v.g + kv) << v.page_shift) + (key & ((1 << v.page_shift) - 1)) : kNoRow;
        const uint64_t ok = __ballot(r != kNoRow);
        bad = ~ok;
        if (ok == ~0ull) return r;
        if (!ok) return 0;
        const uint32_t other = __builtin_amdgcn_readlane(r, __builtin_ctzll(ok));
        return r != kNoRow ? r : other;
    };
    const uint32_t lds0 = __builtin_amdgcn_readfirstlane(lds_at(smem[wave]));
    auto fetch_values = [&](int buf, uint32_t r) {
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
            const int key = j * kPer + lane / RowTile<T>::kChunks, c = (lane % RowTile<T>::kChunks) ^ swz<T>(key);
            row_to_lds(lds0 + buf * kTile + j * kPer * RowTile<T>::kRowBytes,
                       (const char *)a.v_pages + (int64_t)(uint32_t)__shfl((int)r, key) * RowTile<T>::kRowBytes + 16 * c);
        }
    };

    f32x16_t o[4] = {};
    float m = -INFINITY, l = 0.0f;
    const float slope2 = (OPT & kBias) ? a.o.slopes[head] * kLog2e : 0.0f;
    Operand<T> k;
    uint64_t bad_now = 0;
    if (t0 < t1) {
        const uint32_t r = rows_of(tile_of(t0));
        bad_now = bad;
        fetch_values(0, r);
        load_operand(k, (const T *)a.k_pages + (int64_t)r * 128, half);
    }
    for (int t = t0; t < t1; ++t) {
        const int buf = (t - t0) & 1, key0 = tile_of(t) * 32;
        const bool more = t + 1 < t1;
        const uint32_t r = more ? rows_of(tile_of(t + 1)) : 0;
        const uint64_t bad_next = bad;
        settled();   // this tile's keys and values are there, those of the last have been read
        f32x16_t sc[1] = {};
        Operand<T> k_next;
        if (sizeof(T) == 2 && more) {   // (fp32 operands are too wide for two)
            fetch_values(buf ^ 1, r);
            load_operand(k_next, (const T *)a.k_pages + (int64_t)r * 128, half);
        }
        if constexpr (sizeof(T) == 2) {
#pragma unroll
            for (int i = 0; i < 8; ++i) sc[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k.c[i], q.c[i], sc[0], 0, 0, 0);
        } else {
#pragma unroll
            for (int i = 0; i < 16; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) sc[0] = __builtin_amdgcn_mfma_f32_32x32x2f32(k.c[i][e], q.c[i][e], sc[0], 0, 0, 0);
        }
        if (sizeof(T) == 4 && more) {
            fetch_values(buf ^ 1, r);
            load_operand(k, (const T *)a.k_pages + (int64_t)r * 128, half);
        }
        if constexpr (sizeof(T) == 2) k = k_next;
        char *vt = smem[wave][buf];
        score_regs<OPT>(sc[0], a.o, slope2, sight.pos - key0, half);
        if (key0 + 32 > range.all_hi || (key0 < all_lo && !(SIGHT == kWindow && key0 + 32 <= a.o.sinks)) || bad_now != 0) {
            uint32_t seen = 0;
            if constexpr (SIGHT == kRange) {
                mask_regs(sc[0], sight, key0, (uint32_t)bad_now, half, -INFINITY);
            } else {
                seen = sight_bits<SIGHT>(a.o, s, sight, token, key0) & ~(uint32_t)bad_now;
                mask_bits(sc[0], seen, half, -INFINITY);
            }
            if (__any(Odd::any(vt, lane))) {
                Odd::add(o, vt, half, [&](int k) {
                    return SIGHT == kRange ? key0 + k >= sight.lo && key0 + k < sight.hi && !((bad_now >> k) & 1) : (bool)((seen >> k) & 1);
                });
                __builtin_amdgcn_wave_barrier();
                Odd::clean(vt, lane);
                __builtin_amdgcn_wave_barrier();
            }
        }
        softmax_regs<OPT, 1>(sc, o, m, l, a.o.c2);
        values_dot<T, 1>(o, vt, sc, lane);
        bad_now = bad_next;
        __builtin_amdgcn_wave_barrier();
    }

    few_finish<T, NW>(a, s, kv, r0, have, tile, split, used, whole, m, l, o, smem[0][0], join, &last);
}

// The runs of a row joined by their log-sum-exps: a row has WAYS groups of 32 lanes, four elements a lane, that take the runs in turn
template <typename T, int WAYS> __global__ __launch_bounds__(256) void attn_join_kernel(AttnArgs a)
{
    __shared__ f32x4_t part[WAYS > 1 ? 8 : 1][32];
    __shared__ float sums[WAYS > 1 ? 8 : 1];
    const int rows = min(max(a.v.cu[a.v.batch], 0), a.v.total) * a.v.h;   // (tokens behind the last sequence have no runs)
    const int group = threadIdx.x >> 5, l32 = threadIdx.x & 31, way = group % WAYS;
    const int row = blockIdx.x * (8 / WAYS) + group / WAYS;
    const bool live = row < rows && row >= a.v.cu[0] * a.v.h;
    const size_t step = (size_t)a.v.total * a.v.h;
    float top = -INFINITY;
    f32x4_t o = {};
    float sum = 0.0f, ref = 0.0f;
    if (live) {
        for (int i = l32; i < a.nsplit; i += 32) top = fmaxf(top, a.part_lse[i * step + row]);
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) top = fmaxf(top, __shfl_xor(top, d));
        ref = top == -INFINITY ? 0.0f : top;
#pragma unroll 4
        for (int i = way; i < a.nsplit; i += WAYS) {
            const float x = a.part_lse[i * step + row];
            if (x == -INFINITY) continue;   // (an empty run has no outputs)
            const float w = exp2_fast((x - ref) * kLog2e);
            sum += w;
            const f32x4_t p = *reinterpret_cast<const f32x4_t *>(a.part_o + (i * step + row) * 128 + 4 * l32);
#pragma unroll
            for (int c = 0; c < 4; ++c) o[c] = fmaf(w, p[c], o[c]);
        }
    }
    if constexpr (WAYS > 1) {
        part[group][l32] = o;
        if (l32 == 0) sums[group] = sum;
        __syncthreads();
        if (way) return;
#pragma unroll
        for (int w = 1; w < WAYS; ++w) {
            o += part[group + w][l32];
            sum += sums[group + w];
        }
    }
    if (!live) return;
    if (a.lse && l32 == 0) a.lse[row] = sum == 0.0f ? -INFINITY : ref + __builtin_amdgcn_logf(sum) * kLn2;
    store4((T *)a.out + (size_t)row * 128 + 4 * l32, o * inv_sum(sum));
}

// ---- accumulated attention weight ----------------------------------------------------------------------
struct WeightArgs {
    CacheView v;
    ScoreOpts o;
    const void *q;
    int64_t q_stride;
    const float *lse;       // [total][h]
    const void *k_pages;
    const float *w_in;      // [batch][g][w_stride] or null
    float *w_out;
    int w_stride;
    float decay;
    int nsplit;             // weights_few_kernel: blocks of a unit
};

// 16 values a lane, each added over the 32 lanes of its half: the lane gets the sum of value (lane % 32) / 2.  At every step half of what is left goes to the
// lanes of one half of the group and half to the other, so that it takes 38 instructions where 16 sums apart would take 80 and 16 exchanges.
__device__ __forceinline__ float scattered_sum(const f32x16_t &s, int lane)
{
    float r[8], t[4], u[2];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const auto x = __builtin_amdgcn_permlane16_swap(__float_as_uint(s[i]), __float_as_uint(s[i + 8]), false, false);
        r[i] = __uint_as_float(x[0]) + __uint_as_float(x[1]);
    }
    const bool b3 = lane & 8, b2 = lane & 4, b1 = lane & 2;
#pragma unroll
    for (int i = 0; i < 4; ++i) t[i] = (b3 ? r[i + 4] : r[i]) + dpp_f<0x128>(b3 ? r[i] : r[i + 4]);   // row_ror:8
#pragma unroll
    for (int i = 0; i < 2; ++i) u[i] = (b2 ? t[i + 2] : t[i]) + dpp_f<0x141>(b2 ? t[i] : t[i + 2]);
    const float v = (b1 ? u[1] : u[0]) + dpp_f<0x4E>(b1 ? u[0] : u[1]);
    return v + dpp_f<0xB1>(v);
}
__device__ __forceinline__ int scattered_key(int lane)   // the key (of 32) whose sum that is
{
    const int i = (lane & 31) >> 1;
    return 8 * (i >> 2) + 4 * (lane >> 5) + (i & 3);
}
// A row's part in the sums: what it sees and minus its log-sum-exp (in units of log2 e).  A row whose log-sum-exp is -infinity sees nothing: it may be one that
// the caller leaves out, whose scores are anything, NaN included.
struct WeightRow {
    RowSight sight;
    float nlse, slope2;
};
template <int OPT> __device__ __forceinline__ WeightRow weight_row(const WeightArgs &a, const SeqSpan &s, int prefix, int kv, int row, int rows)
{
    const int r = min(row, rows - 1), token = r >> a.v.lg, head = (kv << a.v.lg) + (r & ((1 << a.v.lg) - 1));
    WeightRow w;
    w.sight = row_sight(a.v, a.o, s, prefix, token);
    const float lse = a.lse[(size_t)(s.c0 + token) * a.v.h + head];
    w.nlse = -lse * kLog2e;
    w.slope2 = (OPT & kBias) ? a.o.slopes[head] * kLog2e : 0.0f;
    if (row >= rows || lse == -INFINITY) {
        w.sight.hi = 0;
        w.nlse = -INFINITY;
    }
    return w;
}
// sum += the probabilities of 32 NB keys from k0 on (their operands: k) under the lane's row (q)
template <typename T, int OPT, int NB> __device__ __forceinline__ void add_weights(f32x16_t (&sum)[NB], const Operand<T> (&k)[NB], const Operand<T> &q, const WeightRow &w,
                                                                                   const ScoreOpts &o, int k0, uint64_t bad, int half)
{
    const bool masked = !__all(w.sight.lo <= k0 && w.sight.hi >= k0 + 32 * NB) || bad != 0;
    if (masked && !__any(w.sight.lo < k0 + 32 * NB && w.sight.hi > k0)) return;
    f32x16_t sc[NB] = {};
    if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int kb = 0; kb < NB; ++kb) sc[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k[kb].c[i], q.c[i], sc[kb], 0, 0, 0);
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int kb = 0; kb < NB; ++kb) sc[kb] = __builtin_amdgcn_mfma_f32_32x32x2f32(k[kb].c[i][e], q.c[i][e], sc[kb], 0, 0, 0);
    }
#pragma unroll
    for (int kb = 0; kb < NB; ++kb) score_regs<OPT>(sc[kb], o, w.slope2, w.sight.pos - k0 - 32 * kb, half);
#pragma unroll
    for (int kb = 0; kb < NB; ++kb)
#pragma unroll
        for (int i = 0; i < 16; ++i) sc[kb][i] = exp2_fast(OPT == 0 ? fmaf(sc[kb][i], o.c2, w.nlse) : sc[kb][i] + w.nlse);
    if (masked) {
#pragma unroll
        for (int kb = 0; kb < NB; ++kb) mask_regs(sc[kb], w.sight, k0 + 32 * kb, (uint32_t)(bad >> (32 * kb)), half, 0.0f);
    }
#pragma unroll
    for (int kb = 0; kb < NB; ++kb)
#pragma unroll
        for (int i = 0; i < 16; ++i) sum[kb][i] += sc[kb][i];
}
// The same for bf16 rows that all see all of the 32 keys, in two parts, so that the matrix cores can have the next rows while the vector units have these
__device__ __forceinline__ f32x16_t keys_dot(const Operand<bf16_t> &k, const Operand<bf16_t> &q)
{
    f32x16_t sc = {};
#pragma unroll
    for (int i = 0; i < 8; ++i) sc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k.c[i], q.c[i], sc, 0, 0, 0);
    return sc;
}
template <int OPT> __device__ __forceinline__ void add_seen(f32x16_t &sum, f32x16_t sc, const WeightRow &w, const ScoreOpts &o, int k0, int half)
{
    score_regs<OPT>(sc, o, w.slope2, w.sight.pos - k0, half);
#pragma unroll
    for (int i = 0; i < 16; ++i) sum[i] += exp2_fast(OPT == 0 ? fmaf(sc[i], o.c2, w.nlse) : sc[i] + w.nlse);
}
// a row of a tile in shared memory as the second operand
template <typename T> __device__ __forceinline__ void tile_operand(Operand<T> &q, const char *tile, int r, int half)
{
    using C = std::remove_reference_t<decltype(q.c[0])>;
#pragma unroll
    for (int i = 0; i < (int)(sizeof(q.c) / 16); ++i)
        q.c[i] = *reinterpret_cast<const C *>(tile + r * RowTile<T>::kRowBytes + (((2 * i + half) ^ swz<T>(r)) << 4));
}

// Many rows.  One block of eight waves 4 x 32 kBlocks keys of a unit; a wave keeps its keys as operands and adds up their probabilities over half of the
// rows, which come through shared memory, 128 at a time.  A key's sum has two owners that are added at the end: the same in every call.
template <typename T, int OPT> __global__ __launch_bounds__(512, 2) void weights_kernel(WeightArgs a)
{
    constexpr int kBlocks = sizeof(T) == 2 ? 2 : 1, kKeys = 128 * kBlocks;
    constexpr int kRows = 128, kTile = kRows * RowTile<T>::kRowBytes, kPer = RowTile<T>::kRowsPerLoad, kLoads = kRows / (8 * kPer);
    __shared__ __align__(16) char smem[2][kTile];
    const CacheView &v = a.v;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5, side = wave >> 2;
    const int kv = blockIdx.x % v.g, b = blockIdx.x / v.g, key0 = blockIdx.y * kKeys, mine0 = key0 + 32 * kBlocks * (wave & 3);
    const SeqSpan s = seq_span(v, b);
    if (key0 >= s.len) return;
    const int prefix = a.o.prefix ? min(max(a.o.prefix[b], 0), s.len) : 0;
    const int rows = s.n << v.lg;

    Operand<T> k[kBlocks];
    uint64_t bad = 0;   // keys of the wave that are not there
#pragma unroll
    for (int kb = 0; kb < kBlocks; ++kb) {
        const int key = mine0 + 32 * kb + (lane & 31);
        const uint32_t r = key < s.len ? (uint32_t)cache_row(v, b, kv, key) : kNoRow;
        bad |= (__ballot(r == kNoRow) & 0xffffffffull) << (32 * kb);
        load_operand(k[kb], (const T *)a.k_pages + (int64_t)(r == kNoRow ? 0 : r) * 128, half);
    }

    // rows that may see one of the block's keys
    const int tok0 = prefix > key0 ? 0 : min(max(key0 - s.old, 0), s.n), tok_pos = min(max(0, -s.old), s.n);
    const int t0 = __builtin_amdgcn_readfirstlane((max(tok0, tok_pos) << v.lg) / kRows), t1 = __builtin_amdgcn_readfirstlane((rows + kRows - 1) / kRows);
    const uint32_t lds0 = __builtin_amdgcn_readfirstlane(lds_at(smem));
    auto fetch = [&](int buf, int t) {
#pragma unroll
        for (int j = 0; j < kLoads; ++j) {
            const int at0 = (wave * kLoads + j) * kPer, r = at0 + lane / RowTile<T>::kChunks, c = (lane % RowTile<T>::kChunks) ^ swz<T>(r);
            const int row = min(t * kRows + r, rows - 1);
            row_to_lds(lds0 + buf * kTile + at0 * RowTile<T>::kRowBytes,
                       (const char *)((const T *)a.q + (int64_t)(s.c0 + (row >> v.lg)) * a.q_stride + ((kv << v.lg) + (row & ((1 << v.lg) - 1))) * 128) + 16 * c);
        }
    };
    f32x16_t sum[kBlocks] = {};
    WeightRow w[2];
    if (t0 < t1) {
        fetch(0, t0);
#pragma unroll
        for (int rb = 0; rb < 2; ++rb) w[rb] = weight_row<OPT>(a, s, prefix, kv, t0 * kRows + 64 * side + 32 * rb + (lane & 31), rows);
    }
    for (int t = t0; t < t1; ++t) {
        loads_landed<0>();
        __syncthreads();
        WeightRow next[2];
        if (t + 1 < t1) {   // the next rows' log-sum-exps come in the shadow of this tile too
            fetch((t - t0 + 1) & 1, t + 1);
#pragma unroll
            for (int rb = 0; rb < 2; ++rb) next[rb] = weight_row<OPT>(a, s, prefix, kv, (t + 1) * kRows + 64 * side + 32 * rb + (lane & 31), rows);
        }
#pragma unroll
        for (int rb = 0; rb < 2; ++rb) {
            Operand<T> q;
            tile_operand(q, smem[(t - t0) & 1], 64 * side + 32 * rb + (lane & 31), half);
            add_weights<T, OPT, kBlocks>(sum, k, q, w[rb], a.o, mine0, bad, half);
        }
#pragma unroll
        for (int rb = 0; rb < 2; ++rb) w[rb] = next[rb];
    }
    const size_t unit = ((size_t)b * v.g + kv) * a.w_stride;
    float *other = reinterpret_cast<float *>(smem) + (wave & 3) * 32 * kBlocks;
    __syncthreads();
#pragma unroll
    for (int turn = 1; turn >= 0; --turn) {   // the second half's sums, then the first half's with them
        if (side == turn) {
#pragma unroll
            for (int kb = 0; kb < kBlocks; ++kb) {
                float x = scattered_sum(sum[kb], lane);
                const int at = 32 * kb + scattered_key(lane), key = mine0 + at;
                if (lane & 1) continue;
                if (turn) {
                    other[at] = x;
                } else if (key < s.len) {
                    x += other[at];
                    if (a.w_in && key < s.old) x = fmaf(a.decay, a.w_in[unit + key], x);
                    a.w_out[unit + key] = x;
                }
            }
        }
        if (turn) __syncthreads();
    }
}

// Many rows, few keys: one block 32 kBlocks keys, a wave an eighth of the rows, which it reads as operands where they are (the keys being few, from a
// cache); the eight sums of a key are added at the end, in order.
template <typename T, int OPT> __global__ __launch_bounds__(512, 2) void weights_rows_kernel(WeightArgs a)
{
    constexpr int kBlocks = sizeof(T) == 2 ? 2 : 1, kKeys = 32 * kBlocks;
    __shared__ float sums[8][kKeys];
    const CacheView &v = a.v;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
    const int kv = blockIdx.x % v.g, b = blockIdx.x / v.g, key0 = blockIdx.y * kKeys;
    const SeqSpan s = seq_span(v, b);
    if (key0 >= s.len) return;
    const int prefix = a.o.prefix ? min(max(a.o.prefix[b], 0), s.len) : 0, rows = s.n << v.lg;
    Operand<T> k[kBlocks];
    uint64_t bad = 0;
#pragma unroll
    for (int kb = 0; kb < kBlocks; ++kb) {
        const int key = key0 + 32 * kb + (lane & 31);
        const uint32_t r = key < s.len ? (uint32_t)cache_row(v, b, kv, key) : kNoRow;
        bad |= (__ballot(r == kNoRow) & 0xffffffffull) << (32 * kb);
        load_operand(k[kb], (const T *)a.k_pages + (int64_t)(r == kNoRow ? 0 : r) * 128, half);
    }
    const int tok0 = prefix > key0 ? 0 : min(max(key0 - s.old, 0), s.n), tok_pos = min(max(0, -s.old), s.n);
    const int t0 = (max(tok0, tok_pos) << v.lg) / 32, t1 = (rows + 31) / 32;
    f32x16_t sum[kBlocks] = {};
    auto operand = [&](Operand<T> &q, int t) {
        const int r = min(32 * t + (lane & 31), rows - 1);
        load_operand(q, (const T *)a.q + (int64_t)(s.c0 + (r >> v.lg)) * a.q_stride + ((kv << v.lg) + (r & ((1 << v.lg) - 1))) * 128, half);
    };
    int t = __builtin_amdgcn_readfirstlane(t0 + wave);
    Operand<T> q;
    WeightRow w{};
    if (t < t1) {
        operand(q, t);
        w = weight_row<OPT>(a, s, prefix, kv, 32 * t + (lane & 31), rows);
    }
    for (; t < t1; t += 8) {
        Operand<T> q_next;
        WeightRow w_next{};
        if (t + 8 < t1) {
            if constexpr (sizeof(T) == 2) operand(q_next, t + 8);
            w_next = weight_row<OPT>(a, s, prefix, kv, 32 * (t + 8) + (lane & 31), rows);
        }
        add_weights<T, OPT, kBlocks>(sum, k, q, w, a.o, key0, bad, half);
        if constexpr (sizeof(T) == 2) q = q_next;
        else if (t + 8 < t1) operand(q, t + 8);
        w = w_next;
    }
#pragma unroll
    for (int kb = 0; kb < kBlocks; ++kb) {
        const float x = scattered_sum(sum[kb], lane);
        if ((lane & 1) == 0) sums[wave][32 * kb + scattered_key(lane)] = x;
    }
    __syncthreads();
    const int key = key0 + threadIdx.x;
    if ((int)threadIdx.x < kKeys && key < s.len) {
        float x = sums[0][threadIdx.x];
#pragma unroll
        for (int i = 1; i < 8; ++i) x += sums[i][threadIdx.x];
        const size_t at = ((size_t)b * v.g + kv) * a.w_stride + key;
        if (a.w_in && key < s.old) x = fmaf(a.decay, a.w_in[at], x);
        a.w_out[at] = x;
    }
}

// Few rows, many keys: a block keeps up to 64 KB of a unit's rows in shared memory, and each of its waves walks a run of the unit's keys past them, the
// next 32 keys' rows on their way to registers meanwhile.  More rows than that take another turn over the run, which adds to what the last one wrote.
template <typename T, int OPT> __global__ __launch_bounds__(256, 2) void weights_few_kernel(WeightArgs a)
{
    constexpr int kPer = RowTile<T>::kRowsPerLoad, kRows = 65536 / RowTile<T>::kRowBytes;
    __shared__ __align__(16) char smem[65536];
    __shared__ WeightRow part[kRows];
    const CacheView &v = a.v;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
    const int unit = blockIdx.x, split = blockIdx.y, b = unit / v.g, kv = unit % v.g;
    const SeqSpan s = seq_span(v, b);
    const int prefix = a.o.prefix ? min(max(a.o.prefix[b], 0), s.len) : 0, rows = s.n << v.lg;
    const int64_t tiles = (s.len + 31) / 32, runs = (int64_t)a.nsplit * 4, run = split * 4 + wave;
    const int t0 = __builtin_amdgcn_readfirstlane((int)(tiles * run / runs)), t1 = __builtin_amdgcn_readfirstlane((int)(tiles * (run + 1) / runs));
    if (tiles * (split + 1) / a.nsplit == tiles * split / a.nsplit) return;   // nothing for any of the waves

    const int32_t *table = v.table + (size_t)b * v.max_pages;
    int e0 = -64;
    uint32_t page = 0, bad = 0;
    auto rows_of = [&](int t) -> uint32_t {
        const int key = min(t * 32 + (lane & 31), s.len - 1), e = key >> v.page_shift, last = min(t * 32 + 31, s.len - 1) >> v.page_shift;
        if (last >= e0 + 64 || (t * 32) >> v.page_shift < e0) {
            e0 = (t * 32) >> v.page_shift;
            page = (uint32_t)table[min(e0 + lane, v.max_pages - 1)];
            loads_landed<0>();
        }
        const uint32_t p = (uint32_t)__shfl((int)page, e - e0);
        bad = (uint32_t)__ballot(p >= v.num_pages || t * 32 + (lane & 31) >= s.len);
        return p < v.num_pages ? (uint32_t)((p * (uint64_t)v.g + kv) << v.page_shift) + (key & ((1 << v.page_shift) - 1)) : 0u;
    };
    const uint32_t lds0 = __builtin_amdgcn_readfirstlane(lds_at(smem));
    const size_t w0 = (size_t)unit * a.w_stride;
    const int mine = scattered_key(lane);
    int r0 = 0;
    do {
        const int have = min(rows - r0, kRows), blocks = (have + 31) / 32;
        // the tiles of the run that some of the rows see; the others' weights only decay
        const int tok0 = r0 >> v.lg, tok1 = (r0 + max(have, 1) - 1) >> v.lg;
        const int hi = have > 0 ? key_range(s, prefix, tok0, tok1).hi : 0;
        int lo = 0;
        if (a.o.first && have > 0) {
            lo = INT32_MAX;
            for (int i = tok0 + lane; i <= tok1; i += 64) lo = min(lo, max(a.o.first[s.c0 + i], 0));
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) lo = min(lo, __shfl_xor(lo, d));
            lo = __builtin_amdgcn_readfirstlane(lo);
        }
        const int all_hi = have > 0 ? key_range(s, prefix, tok0, tok1).all_hi : 0;
        const int s0 = max(t0, min(lo >> 5, t1)), s1 = max(s0, min(t1, (hi + 31) >> 5));
        Operand<T> k[1];
        uint32_t bad_now = 0;
        if (s0 < s1) {
            load_operand(k[0], (const T *)a.k_pages + (int64_t)rows_of(s0) * 128, half);
            bad_now = bad;
        }
        __syncthreads();
        for (int j = wave; j * kPer < 32 * blocks; j += 4) {   // (the last row again where they end)
            const int r = j * kPer + lane / RowTile<T>::kChunks, c = (lane % RowTile<T>::kChunks) ^ swz<T>(r), row = r0 + min(r, have - 1);
            row_to_lds(lds0 + j * kPer * RowTile<T>::kRowBytes,
                       (const char *)((const T *)a.q + (int64_t)(s.c0 + (row >> v.lg)) * a.q_stride + ((kv << v.lg) + (row & ((1 << v.lg) - 1))) * 128) + 16 * c);
        }
        bool left_out = false;
        for (int r = threadIdx.x; r < 32 * blocks; r += 256) {
            const WeightRow w = weight_row<OPT>(a, s, prefix, kv, r0 + r, rows);
            left_out |= r < have && w.nlse == -INFINITY;
            part[r] = w;
        }
        auto before_of = [&](int key) {
            if (r0 > 0) return key < s.len ? a.w_out[w0 + key] : 0.0f;
            return a.w_in && key < min(s.old, s.len) ? a.decay * a.w_in[w0 + key] : 0.0f;
        };
        if (r0 == 0) {
            for (int key = t0 * 32 + lane; key < min(s0 * 32, s.len); key += 64) a.w_out[w0 + key] = before_of(key);
            for (int key = s1 * 32 + lane; key < min(t1 * 32, s.len); key += 64) a.w_out[w0 + key] = before_of(key);
        }
        loads_landed<0>();
        const bool all_count = !__syncthreads_or(left_out);
        for (int t = s0; t < s1; ++t) {
            const int key = t * 32 + mine;
            const float before = before_of(key);
            Operand<T> next;
            if (sizeof(T) == 2 && t + 1 < s1) load_operand(next, (const T *)a.k_pages + (int64_t)rows_of(t + 1) * 128, half);
            const uint32_t bad_next = bad;
            f32x16_t sum[1] = {};
            if (sizeof(T) == 2 && all_count && !a.o.first && t * 32 + 32 <= all_hi && bad_now == 0) {
                if constexpr (sizeof(T) == 2) {
                    Operand<T> q;
                    tile_operand(q, smem, lane & 31, half);
                    f32x16_t sc = keys_dot(k[0], q);
                    for (int rb = 0; rb + 1 < blocks; ++rb) {
                        tile_operand(q, smem, 32 * (rb + 1) + (lane & 31), half);
                        const WeightRow w = part[32 * rb + (lane & 31)];
                        const f32x16_t ahead = keys_dot(k[0], q);
                        add_seen<OPT>(sum[0], sc, w, a.o, t * 32, half);
                        sc = ahead;
                    }
                    add_seen<OPT>(sum[0], sc, part[32 * (blocks - 1) + (lane & 31)], a.o, t * 32, half);
                }
            } else
            for (int rb = 0; rb < blocks; ++rb) {
                Operand<T> q;
                tile_operand(q, smem, 32 * rb + (lane & 31), half);
                add_weights<T, OPT, 1>(sum, k, q, part[32 * rb + (lane & 31)], a.o, t * 32, bad_now, half);
            }
            if (sizeof(T) == 4 && t + 1 < s1) load_operand(k[0], (const T *)a.k_pages + (int64_t)rows_of(t + 1) * 128, half);
            const float x = scattered_sum(sum[0], lane);
            if ((lane & 1) == 0 && key < s.len) a.w_out[w0 + key] = x + before;
            if constexpr (sizeof(T) == 2) {
                k[0] = next;
                bad_now = bad_next;
            } else {
                bad_now = bad;
            }
        }
        r0 += kRows;
    } while (r0 < rows);
}

// ---- append with rotary positions -----------------------------------------------------------------------
// Angles.  A pair's frequency is held as a 64-bit fraction of a turn, so that position times frequency modulo 2^64 is the angle modulo a
// turn, whatever the position, where a product in 32 bits would have lost it: a position of 2^31 is off by 2^-32 of a turn at most, and so much again goes with the low
// half of the product.  What is left, an eighth of a turn at most from a quarter, is rounded to fp32 (by 2^-28 of a turn at most).
struct RopeTable {
    uint64_t turn[64];
    uint8_t axis[64];
};
struct AppendArgs {
    CacheView v;
    RopeTable rope;
    const void *q, *k, *val;
    int64_t q_stride, k_stride, v_stride;
    const int32_t *positions;   // [axes][total] or null: the token's place in the cache on every axis
    void *q_out, *k_pages, *v_pages;
};

// sine and cosine of u / 2^32 turns: an eighth of a turn either side of a quarter, by their series (off by 2e-9)
__device__ __forceinline__ void sincos_turn(uint32_t u, float *sn, float *cs)
{
    const uint32_t quarter = (u + 0x20000000u) >> 30;
    const float x = (float)(int32_t)(u - (quarter << 30)) * 1.46291807926715968105e-9f, y = x * x;   // 2 pi / 2^32
    float s = fmaf(y, 2.7557319223985893e-6f, -1.9841269841269841e-4f);
    s = fmaf(y, s, 8.3333333333333333e-3f);
    s = fmaf(y, s, -1.6666666666666667e-1f);
    s = fmaf(x * y, s, x);
    float c = fmaf(y, -2.7557319223985888e-7f, 2.4801587301587302e-5f);
    c = fmaf(y, c, -1.3888888888888889e-3f);
    c = fmaf(y, c, 4.1666666666666667e-2f);
    c = fmaf(y, c, -0.5f);
    c = fmaf(y, c, 1.0f);
    const float a = (quarter & 1) ? c : s, b = (quarter & 1) ? s : c;
    *sn = (quarter & 2) ? -a : a;
    *cs = (quarter == 1 || quarter == 2) ? -b : b;
}

__device__ __forceinline__ void store_chunk(float *p, const float (&x)[8])
{
    reinterpret_cast<float4 *>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
    reinterpret_cast<float4 *>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
}
__device__ __forceinline__ void store_chunk(bf16_t *p, const float (&x)[8])
{
    bf16x8_t v;
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = (__bf16)x[i];
    *reinterpret_cast<bf16x8_t *>(p) = v;
}

// A wave's token: its sequence, slot and page, and the sines and cosines of the lane's pairs 8 (lane % 8) on.  Lane i turns pair i's angle, once for all heads.
struct AppendToken {
    int slot;
    uint32_t page;   // (of num_pages on: nothing is written)
    float cs[8], sn[8];
};
__device__ __forceinline__ bool append_token(const AppendArgs &a, int token, int lane, float2 *turn, AppendToken *at)
{
    const CacheView &v = a.v;
    if (token >= v.total) return false;
    // the token's sequence: the last one that begins at or before it
    int b = -1;
    for (int b0 = 0; b0 < v.batch; b0 += 64) {
        const bool before = b0 + lane < v.batch && v.cu[b0 + lane] <= token && v.cu[b0 + lane + 1] > token;
        const uint64_t hit = __ballot(before);
        if (hit) {
            b = b0 + __builtin_ctzll(hit);
            break;
        }
    }
    if (b < 0) return false;   // behind the last sequence
    const SeqSpan s = seq_span(v, b);
    const int slot = s.old + token - s.c0;
    const int pos = a.positions ? a.positions[(size_t)a.rope.axis[lane] * v.total + token] : slot;
    float2 t;
    sincos_turn((uint32_t)(((uint64_t)(int64_t)pos * a.rope.turn[lane]) >> 32), &t.y, &t.x);
    turn[lane] = t;
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    const int i8 = lane & 7;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float2 x = turn[8 * i8 + i];
        at->cs[i] = x.x;
        at->sn[i] = x.y;
    }
    const bool held = slot >= 0 && slot < s.len;
    at->slot = slot;
    at->page = held ? (uint32_t)v.table[(size_t)b * v.max_pages + (slot >> v.page_shift)] : 0xffffffffu;
    return true;
}

// A wave has a token, 8 lanes a row of it, the chunks i and i + 8 of 8 elements each.
template <typename T> __global__ __launch_bounds__(256) void append_kernel(AppendArgs a)
{
    __shared__ float2 turn[4][64];
    const CacheView &v = a.v;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, token = blockIdx.x * 4 + wave;
    AppendToken t;
    if (!append_token(a, token, lane, turn[wave], &t)) return;
    const int i8 = lane & 7;
    const int nq = a.q ? v.h : 0, nk = a.k ? v.g : 0, rows = nq + 2 * nk;
    for (int r = lane >> 3; r < rows; r += 8) {
        const int kv = r - nq;
        const T *from = r < nq ? (const T *)a.q + (int64_t)token * a.q_stride + r * 128
                        : kv < nk ? (const T *)a.k + (int64_t)token * a.k_stride + kv * 128
                                  : (const T *)a.val + (int64_t)token * a.v_stride + (kv - nk) * 128;
        const Chunk<T> lo = load_chunk_nt(from, i8), hi = load_chunk_nt(from, i8 + 8);   // (read once: 8192 tokens 49 -> 41 us)
        T *to;
        if (r < nq) {
            to = (T *)a.q_out + ((size_t)token * v.h + r) * 128;
        } else {
            if (t.page >= v.num_pages) continue;
            const int64_t row = (((int64_t)t.page * v.g + (kv < nk ? kv : kv - nk)) << v.page_shift) + (t.slot & ((1 << v.page_shift) - 1));
            to = (T *)(kv < nk ? a.k_pages : a.v_pages) + row * 128;
        }
        if (kv >= nk) {   // values as they are
            *reinterpret_cast<Chunk<T> *>(to + 8 * i8) = lo;
            *reinterpret_cast<Chunk<T> *>(to + 64 + 8 * i8) = hi;
            continue;
        }
        float x[8], y[8], p[8], q[8];
        unpack(lo, x);
        unpack(hi, y);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            p[i] = fmaf(x[i], t.cs[i], -(y[i] * t.sn[i]));
            q[i] = fmaf(y[i], t.cs[i], x[i] * t.sn[i]);
        }
        store_chunk(to + 8 * i8, p);
        store_chunk(to + 64 + 8 * i8, q);
    }
}

// ---- eviction ----------------------------------------------------------------------------------------------
struct EvictArgs {
    CacheView v;
    const float *w_in;     // [batch][g][w_stride]
    float *w_out;          // the same, or null
    int w_stride;
    int budget, n_init, n_local;
    int32_t *ids;          // [batch][g][budget]
    int32_t *lens;         // [batch], another array than v.cur (evict_lens_kernel: any), or null
    void *k_pages, *v_pages;
    int slices;
};

// a weight's rank: larger weights have larger words, -0 is +0; NaN comes last, with 1, and 0 is no key's
__device__ __forceinline__ uint32_t weight_rank(float w)
{
    const uint32_t u = __float_as_uint(w + 0.0f);
    const uint32_t r = u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
    return w == w ? r : 1;
}

constexpr int kBins = 2048;    // of a round over the ranks: 11, 11 and 10 bits, four counters each (lanes that agree in these bits wait for fewer others)
constexpr int kTied = 256;     // ranks of the deciding bin that a wave holds in shared memory

// The bin (from the largest down, two a thread) in which the want-th value lies, how many of that bin's are wanted, and how many it has
struct Found {
    uint32_t bin, want, has;
};
__device__ __forceinline__ Found find_bin(const uint4 *hist, uint32_t want, uint32_t *wave_sum, Found *found)
{
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const uint4 c0 = hist[kBins - 1 - 2 * tid], c1 = hist[kBins - 2 - 2 * tid];
    const uint32_t h0 = c0.x + c0.y + c0.z + c0.w, h1 = c1.x + c1.y + c1.z + c1.w;
    uint32_t upto = h0 + h1;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const uint32_t o = __shfl_up(upto, d);
        if (lane >= d) upto += o;
    }
    if (lane == 63) wave_sum[wave] = upto;
    __syncthreads();
    uint32_t above = upto - h0 - h1;
    for (int i = 0; i < wave; ++i) above += wave_sum[i];
    if (above < want && above + h0 >= want) *found = Found{(uint32_t)(kBins - 1 - 2 * tid), want - above, h0};
    else if (above + h0 < want && above + h0 + h1 >= want) *found = Found{(uint32_t)(kBins - 2 - 2 * tid), want - above - h0, h1};
    __syncthreads();
    return *found;
}
__device__ __forceinline__ uint32_t lanes_below(uint64_t mask)   // lanes of the mask before this one
{
    return __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
}

// One block a unit: the rank of the last weight that stays, found over the ranks of the keys that are free to go by their first 11 bits and then among those
// that share these, then the kept ids in order.  Each wave has a run of the keys, 64 at a time; with EACH > 0 that is 64 EACH keys whose ranks it holds, with 0
// they are read in every pass.  Lanes without a key hold rank 0, the lowest, which is never reached: more keys than are wanted have one above it.
// What bounds it is the instructions of the unit's one CU.
template <int EACH> __global__ __launch_bounds__(1024) void evict_select_kernel(EvictArgs a)
{
    __shared__ uint4 hist4[kBins];
    __shared__ uint32_t tied[16][kTied], wave_sum[16], many;
    __shared__ uint2 count[16];   // a wave's keys above the last rank, and at it
    __shared__ Found found;
    uint32_t *hist = reinterpret_cast<uint32_t *>(hist4);
    const CacheView &v = a.v;
    const int unit = blockIdx.x, b = unit / v.g, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), tid = threadIdx.x;
    const int len = min(max(v.cur[b], 0), v.max_pages << v.page_shift), keep = min(len, a.budget);
    int32_t *ids = a.ids + (size_t)unit * a.budget;
    const float *w = a.w_in + (size_t)unit * a.w_stride;
    if (a.lens && unit % v.g == 0 && tid == 0) a.lens[b] = keep;
    for (int j = keep + tid; j < a.budget; j += 1024) ids[j] = -1;
    if (keep == len) {
        for (int j = tid; j < len; j += 1024) ids[j] = j;
        return;
    }
    const int from = a.n_init, to = len - a.n_local, n = to - from;
    const int run = EACH ? 64 * EACH : ((n + 15) / 16 + 63) & ~63, my0 = from + wave * run, mine = min(max(to - my0, 0), run);
    const uint32_t all = keep - a.n_init - a.n_local;   // so many of them stay, fewer than n
    uint32_t rank[EACH ? EACH : 1];
    if constexpr (EACH > 0) {
#pragma unroll
        for (int i = 0; i < EACH; ++i)
            if (64 * i < mine) rank[i] = __float_as_uint(w[my0 + min(64 * i + lane, mine - 1)]);
    }
    for (int j = tid; j < a.n_init; j += 1024) ids[j] = j;
    for (int j = tid; j < a.n_local; j += 1024) ids[keep - a.n_local + j] = to + j;
    if (!all) return;
    hist4[tid] = hist4[tid + 1024] = uint4{};
    if (tid == 0) many = 0;
    __syncthreads();
    if constexpr (EACH > 0) {
#pragma unroll
        for (int i = 0; i < EACH; ++i)
            if (64 * i < mine) rank[i] = 64 * i + lane < mine ? weight_rank(__uint_as_float(rank[i])) : 0;
    }
    // f(rank, key), for all of the wave's keys
    auto each = [&](auto f) {
        if constexpr (EACH > 0) {
#pragma unroll
            for (int i = 0; i < EACH; ++i)
                if (64 * i < mine) f(rank[i], my0 + 64 * i + lane);
        } else {
            for (int i0 = 0; i0 < mine; i0 += 512) {   // (eight loads in flight)
                float x[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = w[my0 + min(i0 + 64 * i + lane, mine - 1)];
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (i0 + 64 * i < mine) f(i0 + 64 * i + lane < mine ? weight_rank(x[i]) : 0u, my0 + i0 + 64 * i + lane);
            }
        }
    };
    const uint32_t way = lane & 3;
    each([&](uint32_t r, int) { atomicAdd(&hist[(r >> 21) * 4 + way], 1u); });
    __syncthreads();
    const Found top = find_bin(hist4, all, wave_sum, &found);
    // the bin's ranks of each wave to shared memory, as far as there is room, and how many of the wave's keys are above it
    uint32_t over = 0, tie = 0, held = 0;
    each([&](uint32_t r, int) {
        over += __popcll(__ballot(r >> 21 > top.bin));
        const uint64_t in = __ballot(r >> 21 == top.bin);
        if (!in) return;
        const uint32_t at = held + lanes_below(in);
        if (r >> 21 == top.bin && at < kTied) tied[wave][at] = r;
        held += __popcll(in);
    });
    if (held > kTied) many = 1;
    uint32_t last = top.bin << 21, want = top.want;
    hist4[tid] = hist4[tid + 1024] = uint4{};
    __syncthreads();
    // the ranks that share the bin, from shared memory or where they are
    auto each_tied = [&](auto f) {
        if (!many) {
            for (uint32_t i = lane; i < held; i += 64) f(tied[wave][i]);
        } else {
            each([&](uint32_t r, int) {
                if (r >> 21 == top.bin) f(r);
            });
        }
    };
    if (want < top.has) {
        each_tied([&](uint32_t r) { atomicAdd(&hist[((r >> 10) & 2047) * 4 + way], 1u); });
        __syncthreads();
        const Found mid = find_bin(hist4, want, wave_sum, &found);
        last |= mid.bin << 10;
        want = mid.want;
        if (want < mid.has) {
            __syncthreads();
            hist4[tid] = hist4[tid + 1024] = uint4{};
            __syncthreads();
            each_tied([&](uint32_t r) {
                if ((r & ~1023u) == last) atomicAdd(&hist[(r & 1023) * 4 + way], 1u);
            });
            __syncthreads();
            const Found low = find_bin(hist4, want, wave_sum, &found);
            last |= low.bin;
            want = low.want;
            if (want == low.has) want = 0, last -= 1;
        } else {
            want = 0, last -= 1;
        }
    } else {
        want = 0, last -= 1;   // (a whole bin stays: what is above the rank before it)
    }
    // above `last` a weight stays, at it the first `want` do
    if (!many) {
        uint32_t x = 0, y = 0;
        for (uint32_t i = lane; i < held; i += 64) {
            const uint32_t r = tied[wave][i];
            x += r > last;
            y += r == last;
        }
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            x += __shfl_xor(x, d);
            y += __shfl_xor(y, d);
        }
        over += x;
        tie = y;
    } else {
        over = 0;
        each([&](uint32_t r, int) {
            over += __popcll(__ballot(r > last));
            tie += __popcll(__ballot(r == last));
        });
    }
    if (lane == 0) count[wave] = make_uint2(over, tie);
    __syncthreads();
    uint32_t ties = 0, at = a.n_init;
    for (int i = 0; i < wave; ++i) {
        at += count[i].x;
        ties += count[i].y;
    }
    at += min(ties, want);
    each([&](uint32_t r, int key) {
        uint64_t kept = __ballot(r > last);
        if (want) {
            const uint64_t here = __ballot(r == last);
            if (here) {
                kept |= __ballot(r == last && ties + lanes_below(here) < want);
                ties += __popcll(here);
            }
        }
        if (kept >> lane & 1) ids[at + lanes_below(kept)] = key;
        at += __popcll(kept);
    });
}

// The lengths after an eviction into the array that holds those before it: behind the other kernels, whose blocks all read them
static __global__ void evict_lens_kernel(EvictArgs a)
{
    const int b = blockIdx.x * blockDim.x + threadIdx.x;
    if (b < a.v.batch) a.lens[b] = min(min(max(a.v.cur[b], 0), a.v.max_pages << a.v.page_shift), a.budget);
}

// The kept rows to the front, in order and in place.  Row j comes from ids[j] >= j, so rounds of rows, read as a whole before the first of them is
// written, overwrite nothing that a later round reads; a block has 1 / slices of every row of its unit, which no other block touches.  A unit's
// slices share lines of its rows, so they are on one XCD where the units are a multiple of 8.
template <typename T> __global__ __launch_bounds__(1024) void evict_move_kernel(EvictArgs a)
{
    constexpr int kPieces = 2 * 128 * sizeof(T) / 16, kEach = 8;   // 16-byte pieces of a key's K and V rows
    const CacheView &v = a.v;
    const int unit = blockIdx.x, slice = blockIdx.y, b = unit / v.g, kv = unit % v.g;
    const int len = min(max(v.cur[b], 0), v.max_pages << v.page_shift), keep = min(len, a.budget);
    const int32_t *ids = a.ids + (size_t)unit * a.budget;
    const size_t w0 = (size_t)unit * a.w_stride;
    const bool weights = a.w_out && slice == 0;
    if (keep == len) {
        if (weights && a.w_out != a.w_in)
            for (int j = threadIdx.x; j < keep; j += 1024) a.w_out[w0 + j] = a.w_in[w0 + j];
        return;
    }
    const int wide = kPieces / a.slices, lane_rows = 1024 / wide, my = threadIdx.x / wide, piece = slice * wide + threadIdx.x % wide;
    char *pages = (char *)(piece < kPieces / 2 ? a.k_pages : a.v_pages) + 16 * (piece % (kPieces / 2));
    const int32_t *table = v.table + (size_t)b * v.max_pages;
    const int in_page = (1 << v.page_shift) - 1;
    const int round = lane_rows * kEach;
    uint32_t src[kEach], dst[kEach];
    // where the rows of the round from j0 on come from and go to
    auto look_up = [&](int j0) {
        int id[kEach];
#pragma unroll
        for (int i = 0; i < kEach; ++i) id[i] = ids[min(j0 + i * lane_rows + my, keep - 1)];
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            src[i] = (uint32_t)table[id[i] >> v.page_shift];
            dst[i] = (uint32_t)table[min(j0 + i * lane_rows + my, keep - 1) >> v.page_shift];
        }
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int j = j0 + i * lane_rows + my;
            const bool move = j < keep && id[i] != j && src[i] < v.num_pages && dst[i] < v.num_pages;
            src[i] = (uint32_t)((src[i] * (uint64_t)v.g + kv) << v.page_shift) + (id[i] & in_page);
            dst[i] = move ? (uint32_t)((dst[i] * (uint64_t)v.g + kv) << v.page_shift) + (j & in_page) : kNoRow;
        }
    };
    look_up(0);
    for (int j0 = 0; j0 < keep; j0 += round) {
        u32x4_t x[kEach];
        uint32_t to[kEach];
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            to[i] = dst[i];
            if (to[i] != kNoRow) x[i] = *reinterpret_cast<const u32x4_t *>(pages + (int64_t)src[i] * (128 * (int)sizeof(T)));
        }
        if (j0 + round < keep) look_up(j0 + round);   // in the shadow of the rows
        loads_landed<0>();
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kEach; ++i)
            if (to[i] != kNoRow) *reinterpret_cast<u32x4_t *>(pages + (int64_t)to[i] * (128 * (int)sizeof(T))) = x[i];
    }
    if (weights)
        for (int j0 = 0; j0 < keep; j0 += 1024) {
            const int j = j0 + threadIdx.x;
            const float x = j < keep ? a.w_in[w0 + ids[j]] : 0.0f;
            loads_landed<0>();
            __syncthreads();
            if (j < keep) a.w_out[w0 + j] = x;
        }
}

}  // namespace ctkvr
