// Pieces shared by the kernels of the paged key / value cache (cache.hip, paged_few.h, paged_many.h) and their launchers.
//
// A cache is four-dimensional, [pages, page_size, heads, head_size], any strides along the first three axes.  Position p of a sequence lies
// on page table[p / page_size], at place p % page_size of it.  An 8-bit cache holds codes, and a scale in 32 bits for each token and head: the
// value is code * scale.
#pragma once
#include "gemm_direct.h"
#include "paged_index.h"

namespace nt {

// How the cache's elements are held: in the type of the queries, or as codes of 8 bits.
enum CacheKind { CACHE_SAME = 0, CACHE_E4M3 = 1, CACHE_I8 = 2 };

typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2v __attribute__((ext_vector_type(2)));
typedef float float2v __attribute__((ext_vector_type(2)));
typedef float float4v __attribute__((ext_vector_type(4)));
typedef short short4v_p __attribute__((ext_vector_type(4)));
typedef unsigned short ushort2v __attribute__((ext_vector_type(2)));

// two fp32 values -> one register of two 16-bit values, round to nearest even
template <bool BF16>
__device__ __forceinline__ uint32_t pack_two(float a, float b)
{
    if constexpr (BF16) return __builtin_bit_cast(uint32_t, __builtin_convertvector(float2v{a, b}, bf16x2v));
    else return __builtin_bit_cast(uint32_t, half2v{(_Float16)a, (_Float16)b});
}

template <bool BF16>
__device__ __forceinline__ float4v mfma16(u32x4 a, u32x4 b, float4v c)
{
    if constexpr (BF16) return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bhalf8, a), __builtin_bit_cast(bhalf8, b), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8, a), __builtin_bit_cast(half8, b), c, 0, 0, 0);
}

// four codes -> four 16-bit values, exactly (e4m3 has 4 significant bits, int8 7 and a power of two)
template <bool BF16, int KIND>
__device__ __forceinline__ u32x2 widen4(uint32_t w)
{
    static_assert(KIND != CACHE_SAME, "codes");
    if constexpr (KIND == CACHE_E4M3) {
        if constexpr (BF16)
            return u32x2{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, false)),
                         __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.0f, true))};
        else
            return u32x2{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, false)),
                         __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.0f, true))};
    } else if constexpr (BF16) {
        // an integer of 8 bits as fp32 has its bits in the upper half: the two halves side by side, nothing to round
        float f[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = (float)(int8_t)(w >> (8 * i));
        return u32x2{__builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, f[1]), __builtin_bit_cast(uint32_t, f[0]), 0x07060302u),
                     __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, f[3]), __builtin_bit_cast(uint32_t, f[2]), 0x07060302u)};
    } else {
        // 0x6400 | u is 1024 + u: with u = code + 128, less 1152
        const uint32_t u = w ^ 0x80808080u;
        const half2v lo = __builtin_bit_cast(half2v, __builtin_amdgcn_perm(0x64646464u, u, 0x04010400u)) - half2v{(_Float16)1152.0f, (_Float16)1152.0f};
        const half2v hi = __builtin_bit_cast(half2v, __builtin_amdgcn_perm(0x64646464u, u, 0x04030402u)) - half2v{(_Float16)1152.0f, (_Float16)1152.0f};
        return u32x2{__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi)};
    }
}

template <bool BF16, int KIND>
__device__ __forceinline__ u32x4 widen8(u32x2 w)
{
    const u32x2 a = widen4<BF16, KIND>(w[0]), b = widen4<BF16, KIND>(w[1]);
    return u32x4{a[0], a[1], b[0], b[1]};
}

// infinities and NaN among eight 16-bit values: their exponent is all ones
template <bool BF16>
__device__ __forceinline__ bool any_not_finite(u32x4 v)
{
    constexpr uint32_t E = BF16 ? 0x7f80u : 0x7c00u;
    bool bad = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) bad = bad | ((v[i] & E) == E) | ((v[i] & (E << 16)) == (E << 16));
    return bad;
}

template <bool BF16>
__device__ __forceinline__ uint32_t without_not_finite(uint32_t w)
{
    constexpr uint32_t E = BF16 ? 0x7f80u : 0x7c00u;
    return ((w & E) == E ? 0u : w & 0xffffu) | ((w & (E << 16)) == (E << 16) ? 0u : w & 0xffff0000u);
}

template <bool BF16>
__device__ __forceinline__ u32x4 without_not_finite(u32x4 v)
{
    return u32x4{without_not_finite<BF16>(v[0]), without_not_finite<BF16>(v[1]), without_not_finite<BF16>(v[2]), without_not_finite<BF16>(v[3])};
}

template <bool BF16>
__device__ __forceinline__ float widen_one(uint32_t w, int upper)
{
    const uint32_t h = upper ? w >> 16 : w & 0xffffu;
    if constexpr (BF16) return __builtin_bit_cast(float, h << 16);
    else return (float)__builtin_bit_cast(_Float16, (uint16_t)h);
}

// What the rounding of two weights to `packed` left, packed alike.  The second product runs with both and adds up what the weights themselves would give, to
// 2^-17 of them in bf16, to 2^-23, or 2^-25 of a weight of 1, in fp16; one rounding is off by 2^-8 (2^-11), an error as large as that of the rounded result.
// SCALED: a weight times a value's scale.  That can be of any size beside its neighbours', beyond fp16's range either way, so that codes, which bf16 holds
// exactly too, are multiplied in bf16 whatever the queries' type.  (Scales may be infinite: then nothing is left, infinity less infinity is NaN.)
template <bool BF16, bool SCALED>
__device__ __forceinline__ uint32_t rest_of(uint32_t packed, float a, float b)
{
    float x = a - widen_one<BF16>(packed, 0), y = b - widen_one<BF16>(packed, 1);
    if constexpr (SCALED) {
        x = __builtin_fabsf(x) < INFINITY ? x : 0.f;
        y = __builtin_fabsf(y) < INFINITY ? y : 0.f;
    }
    return pack_two<BF16>(x, y);
}

// Two weights as the sums of two 16-bit numbers each, the first cut off, so that the rest is not negative: as long as both are more than 0 an infinity that they multiply stays
// one, which the rest of a rounded weight, of either sign or 0, makes NaN.  A rest below the type's smallest normal number (fp16: smallest of all, 2^-24) becomes that, and fp16 weights
// below 2^-24 are taken as 2^-24; of a weight of 0 both stay 0.  Off by 2^-16 of the weight in bf16, 2^-22 of it or 2^-24 in fp16, 2^-23 where it is below 2^-24.  These are to one side,
// and would add up over the keys (131072 beside one that weighs as much as twice all of them: 1e-3 of the result with a largest weight of 1): fp16 weights are such that a row's
// largest is 2^8 or more, 2^-24 then 2^-32 of it or less.  SCALED: as above; values then are codes, no infinities.
template <bool BF16, bool SCALED>
__device__ __forceinline__ void cut_two(float a, float b, uint32_t *first, uint32_t *rest)
{
    float x, y;
    if constexpr (BF16) {
        *first = __builtin_amdgcn_perm(__builtin_bit_cast(uint32_t, b), __builtin_bit_cast(uint32_t, a), 0x07060302u);
        x = a - __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, a) & 0xffff0000u);
        y = b - __builtin_bit_cast(float, __builtin_bit_cast(uint32_t, b) & 0xffff0000u);
    } else {
        if constexpr (!SCALED) {                                           // (2^100 a is above 2^-24 for every weight that is not 0)
            a = __builtin_amdgcn_fmed3f(a, a * 0x1p100f, 0x1p-24f);
            b = __builtin_amdgcn_fmed3f(b, b * 0x1p100f, 0x1p-24f);
        }
        *first = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_pkrtz(a, b));
        x = a - widen_one<false>(*first, 0);
        y = b - widen_one<false>(*first, 1);
    }
    constexpr float least = SCALED ? 0.f : BF16 ? 0x1p-126f : 0x1p-24f;    // (SCALED, a weight times a scale: of an infinite one 0 or as much, never of the other sign)
    x = __builtin_amdgcn_fmed3f(x, a, least);
    y = __builtin_amdgcn_fmed3f(y, b, least);
    *rest = pack_two<BF16>(x, y);
}

// v if it is an infinity or NaN, else 0
__device__ __forceinline__ float only_not_finite(float v) { return __builtin_fabsf(v) < INFINITY ? 0.f : v; }

// v, as something that the compiler knows nothing of: what is worked out from it stays where it is (a rare path's addresses, kept in registers around
// the loop that it lies in, cost the loop those registers)
__device__ __forceinline__ int here(int v)
{
    asm volatile("" : "+v"(v));
    return v;
}

// The same for a value that is the same in all lanes
__device__ __forceinline__ uint32_t here_scalar(uint32_t v)
{
    asm volatile("" : "+s"(v));
    return v;
}

// Largest and sum over lanes l, l ^ 16, l ^ 32 and l ^ 48 (BOTH) or over l and l ^ 32, in all of them: exchanges of rows and halves between registers, not by way of LDS
template <bool BOTH, typename F>
__device__ __forceinline__ float across(float v, F combine)
{
    const auto half = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, v), __builtin_bit_cast(uint32_t, v), false, false);
    v = combine(__builtin_bit_cast(float, (uint32_t)half[0]), __builtin_bit_cast(float, (uint32_t)half[1]));
    if constexpr (BOTH) {
        const auto row = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, v), __builtin_bit_cast(uint32_t, v), false, false);
        v = combine(__builtin_bit_cast(float, (uint32_t)row[0]), __builtin_bit_cast(float, (uint32_t)row[1]));
    }
    return v;
}
template <bool BOTH>
__device__ __forceinline__ float largest_across(float v)
{
    return across<BOTH>(v, [](float a, float b) { return fmaxf(a, b); });
}
template <bool BOTH>
__device__ __forceinline__ float sum_across(float v)
{
    return across<BOTH>(v, [](float a, float b) { return a + b; });
}

// Order of what one wavefront's lanes write to LDS and read of each other's: the hardware keeps it, the compiler has to
__device__ __forceinline__ void wavefront_fence()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// a * s, 32 by 64 bits
__device__ __forceinline__ int64_t times(uint32_t a, int64_t s)
{
    return (int64_t)((uint64_t)a * (uint32_t)s + ((uint64_t)(a * (uint32_t)((uint64_t)s >> 32)) << 32));
}

// ---- the attention kernels' arguments (strides in elements)
struct PagedArgs {
    const uint16_t *Q;
    uint16_t *O;
    const char *K, *V;
    const float *KS, *VS;              // scales (8-bit caches)
    const int32_t *table, *starts, *lengths;
    int64_t q_st, q_sh, o_st, o_sh;    // token, head
    int64_t k_sp, k_ss, k_sh, v_sp, v_ss, v_sh;         // page, place, head
    int64_t ks_sp, ks_ss, ks_sh, vs_sp, vs_ss, vs_sh;
    int64_t t_sb;                      // sequence
    int32_t T, B, Hq, Hkv, G;          // tokens, sequences, heads, G = Hq / Hkv query heads to a key head
    int32_t D;                         // head size
    int32_t width, pages;              // entries of a table row (that are in reach), pages of the cache
    int32_t tiles;                     // of query rows, all sequences together (paged_many)
    int32_t causal, window;            // window 0: none
    int32_t near;                      // offsets within 16 rows of a page are not negative and fit 32 bits
    int32_t uniform;                   // ... and 16 keys from a multiple of 16 on lie on one page
    int32_t aligned;                   // every row of the cache begins at a multiple of 16 bytes
    int32_t splits, split_keys;        // the keys of a tile are shared out over `splits` programs, split_keys each (the last: what is left)
    Divider page, group;               // by page_size, by G
    // trees of drafted tokens: a row of `words` words for each token, and its depth (windows)
    const uint64_t *masks;
    const int32_t *depths;
    int64_t m_st;
    int32_t words;
    int32_t parts;                     // programs that a sequence's rows are dealt out to,
    int32_t groups;                    // ... and that all sequences' keys are dealt out to (0: each sequence and head has one)
    int64_t *before;                   // blocks of the sequences before each, and of all
    float scale_log2e;                 // scale * log2(e): exponentials are taken in base 2
    // one program's share of a row (splits > 1): [token * Hq + head][split] of (reference, sum), and of D unnormalised outputs
    float *part_ml, *part_o;
};

__device__ __forceinline__ Sequence sequence_of(const PagedArgs &g, int b) { return sequence_at(g.starts, g.lengths, b, g.T); }

__device__ __forceinline__ KeyRange keys_of(const PagedArgs &g, const Sequence &q, int32_t i0, int32_t i1, int split, int32_t block)
{
    return key_range(q, i0, i1, g.causal, g.window, split, g.splits, g.split_keys, block, g.width * (int32_t)g.page.d);
}

// ---- where a block of keys lies in LDS: rows of SIZE 16-bit elements, their 16-byte chunks in an order that depends on the row, such that 16
// consecutive rows' same chunks (a fragment read of K, or lanes writing a column of rows) lie in 16 different groups of banks, and so do
// the 32 bytes of eight rows that a transposing read of V takes at a time.
template <int SIZE>
__device__ __forceinline__ uint32_t chunk_order(uint32_t row)
{
    static_assert(SIZE == 64 || SIZE == 128 || SIZE == 256, "built sizes");
    if constexpr (SIZE == 64) return (((row >> 1) & 1) << 2) | (((row >> 2) & 1) << 1) | ((row >> 3) & 1);
    else return ((row & 3) << 2) | (((row >> 2) & 1) << 1) | ((row >> 3) & 1);
}
template <int SIZE>
__device__ __forceinline__ uint32_t lds_at(uint32_t row, uint32_t chunk) { return row * (uint32_t)(SIZE * 2) + ((chunk ^ chunk_order<SIZE>(row)) << 4); }

__device__ __forceinline__ u32x2 lds_read_transposed(const char *smem, uint32_t addr)
{
    typedef short4v_p __attribute__((address_space(3))) *lds_s4;
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4)(smem + addr)));
}

// (not a number in either 16-bit type, twice: what a key reads as whose page the table does not name)
constexpr uint32_t kNanPair = 0x7fff7fffu;

nt_status launch_paged_64(const PagedArgs &a, int rows, int64_t programs, bool bf16, int kind, void *stream);
nt_status launch_paged_128(const PagedArgs &a, int rows, int64_t programs, bool bf16, int kind, void *stream);
nt_status launch_paged_256(const PagedArgs &a, int rows, int64_t programs, bool bf16, int kind, void *stream);
// sequences whose keys the tree kernel deals out evenly
constexpr int kTreeSequences = 1024;

nt_status launch_paged_tree_64(const PagedArgs &a, int rows, int64_t programs, bool bf16, int kind, void *stream);
nt_status launch_paged_tree_128(const PagedArgs &a, int rows, int64_t programs, bool bf16, int kind, void *stream);
nt_status launch_paged_tree_256(const PagedArgs &a, int rows, int64_t programs, bool bf16, int kind, void *stream);

}  // namespace nt
