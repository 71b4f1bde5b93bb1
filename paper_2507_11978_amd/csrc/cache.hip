// Writing a paged key / value cache, and reading it back.
//
// A token's head is a row of head_size elements.  In a cache of the tokens' type a write copies it.  In an 8-bit cache
//   s = up12(max |x| / L),  code = rne(x / s),   L = 448 (e4m3) or 127 (int8),
// with up12 rounding up to twelve significant bits, s at least 2^-100, and at most what keeps L s in fp16's range for fp16 tokens; reading gives
// code * s, rounded to 16 bits.  Rounded up, s never makes a code larger than L; and short, it leaves nothing between the quotient's border cases to
// be lost in 32 bits: a border t (the middle between two codes) has at most 8 significant bits, t s at most 20, x at most 11, so x / s is t exactly or
// differs from it by 2^-20 and more, far beyond the 2^-23 that the arithmetic may be off.  The codes are those of the
// real quotient, and code * s (8 x 12 bits) is exact in 32 bits.
// A row with an infinity or NaN has no scale: s is NaN, its codes are 0, and it reads as NaN.
//
// Both are bound by memory: a row's elements once in 16 bits and once as they are held.  A group of 8, 16 or 32 lanes has a row, 8 elements to a lane (16
// bytes of either tensor: K's and V's rows go through the same lanes), the largest magnitude from exchanges within the group.  Measured: 16384 tokens
// of 8 heads x 128 bf16 as int8 24.3 us written (4.15 TB/s), 18.6 read; 65536 read as e4m3 82 (4.9 TB/s, what a large copy reaches); calls of few tokens
// take the host's 3 to 4 us, the kernel 2 to 3 (a chain of launch, slot, row and store; dividing in 32 bits instead of 64 changes nothing).
#include "paged.h"

namespace nt {

struct CacheArgs {
    uint16_t *k, *v;                                          // the tokens' rows
    char *K, *V;                                              // the cache
    float *KS, *VS;
    const int64_t *slots;
    int64_t k_st, k_sh, v_st, v_sh;
    int64_t ck_sp, ck_ss, ck_sh, cv_sp, cv_ss, cv_sh;         // page, place, head
    int64_t ks_sp, ks_ss, ks_sh, vs_sp, vs_ss, vs_sh;
    int64_t rows, places;                                     // tokens * heads, pages * page_size
    int32_t heads, size, page_size;
};

template <bool BF16>
__device__ __forceinline__ void widen_row(u32x4 v, float (&f)[8])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = widen_one<BF16>(v[i], 0);
        f[2 * i + 1] = widen_one<BF16>(v[i], 1);
    }
}

// Codes and scale of the row that this group of LANES lanes holds, 8 elements each
template <bool BF16, int KIND, int LANES>
__device__ __forceinline__ u32x2 quantise(u32x4 x, float *scale)
{
    // the largest magnitude, as an integer: NaN is above infinity above every number
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t lo = x[i] & 0x7fffu, hi = (x[i] >> 16) & 0x7fffu;
        top = top > lo ? top : lo;
        top = top > hi ? top : hi;
    }
#pragma unroll
    for (int d = 1; d < LANES; d <<= 1) {
        const uint32_t other = __shfl_xor(top, d, 64);
        top = top > other ? top : other;
    }
    const float largest = widen_one<BF16>(top, 0);
    if (!(largest < INFINITY)) {
        *scale = __builtin_nanf("");
        return u32x2{0, 0};
    }
    // (a quotient by 448 or 127 of a number of at most 11 bits is on the 12-bit grid or 2^-19 and more away from it: its rounding to 32 bits changes nothing)
    const float q = largest / (KIND == CACHE_E4M3 ? 448.f : 127.f);
    float s = __builtin_bit_cast(float, (__builtin_bit_cast(uint32_t, q) + 0xfffu) & ~0xfffu);
    s = s < 0x1p-100f ? 0x1p-100f : s;
    // (the largest fp16 numbers: the next scale of twelve bits would take L * s past the type's range, and the quotient by this one still rounds to L)
    if constexpr (!BF16) s = fminf(s, KIND == CACHE_E4M3 ? 146.1875f : 515.75f);
    *scale = s;
    // x / s: the product with the reciprocal, then one correction by the remainder, which an exact quotient comes out of exactly
    const float r = 1.f / s;
    float f[8], y[8];
    widen_row<BF16>(x, f);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float y0 = f[i] * r;
        y[i] = __builtin_fmaf(__builtin_fmaf(-y0, s, f[i]), r, y0);
    }
    u32x2 code;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        if constexpr (KIND == CACHE_E4M3) {
            int c = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * i], y[4 * i + 1], 0, false);
            c = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * i + 2], y[4 * i + 3], c, true);
            code[i] = (uint32_t)c;
        } else {
            uint32_t c = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) c |= ((uint32_t)(int32_t)__builtin_rintf(y[4 * i + j]) & 0xffu) << (8 * j);
            code[i] = c;
        }
    }
    return code;
}

template <bool BF16, int KIND, int LANES>
__global__ __launch_bounds__(256) void cache_write_kernel(const CacheArgs g)
{
    const int64_t row = (int64_t)blockIdx.x * (256 / LANES) + threadIdx.x / LANES;
    const int d = 8 * (threadIdx.x % LANES);
    if (row >= g.rows) return;                                             // (all lanes of the group)
    const int64_t token = (uint32_t)row / (uint32_t)g.heads;               // (rows: below 2^31)
    const int h = (int)(row - token * g.heads);
    const int64_t slot = g.slots[token];
    u32x4 k{0, 0, 0, 0}, v{0, 0, 0, 0};
    const bool mine = d < g.size;
    if (mine) {                                                            // (ahead of the slot's wait)
        __builtin_memcpy(&k, g.k + token * g.k_st + h * g.k_sh + d, 16);
        __builtin_memcpy(&v, g.v + token * g.v_st + h * g.v_sh + d, 16);
    }
    if ((uint64_t)slot >= (uint64_t)g.places) return;
    const int64_t page = slot / g.page_size, at = slot - page * g.page_size;
    constexpr int ES = KIND == CACHE_SAME ? 2 : 1;
    char *K = g.K + (page * g.ck_sp + at * g.ck_ss + h * g.ck_sh + d) * ES, *V = g.V + (page * g.cv_sp + at * g.cv_ss + h * g.cv_sh + d) * ES;
    if constexpr (KIND == CACHE_SAME) {
        if (mine) {
            __builtin_memcpy(K, &k, 16);
            __builtin_memcpy(V, &v, 16);
        }
    } else {
        float sk, sv;
        const u32x2 ck = quantise<BF16, KIND, LANES>(k, &sk), cv = quantise<BF16, KIND, LANES>(v, &sv);
        if (mine) {
            __builtin_memcpy(K, &ck, 8);
            __builtin_memcpy(V, &cv, 8);
        }
        if (d == 0) {
            g.KS[page * g.ks_sp + at * g.ks_ss + h * g.ks_sh] = sk;
            g.VS[page * g.vs_sp + at * g.vs_ss + h * g.vs_sh] = sv;
        }
    }
}

// eight codes times the scale, in 16 bits
template <bool BF16, int KIND>
__device__ __forceinline__ u32x4 dequantise(u32x2 c, float s)
{
    u32x4 out;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        float f[4];
        if constexpr (KIND == CACHE_E4M3) {
            const float2v lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)c[i], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)c[i], true);
            f[0] = lo[0]; f[1] = lo[1]; f[2] = hi[0]; f[3] = hi[1];
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) f[j] = (float)(int8_t)(c[i] >> (8 * j));
        }
        out[2 * i] = pack_two<BF16>(f[0] * s, f[1] * s);
        out[2 * i + 1] = pack_two<BF16>(f[2] * s, f[3] * s);
    }
    return out;
}

template <bool BF16, int KIND, int LANES>
__global__ __launch_bounds__(256) void cache_read_kernel(const CacheArgs g)
{
    const int64_t row = (int64_t)blockIdx.x * (256 / LANES) + threadIdx.x / LANES;
    const int d = 8 * (threadIdx.x % LANES);
    if (row >= g.rows || d >= g.size) return;
    const int64_t token = (uint32_t)row / (uint32_t)g.heads;
    const int h = (int)(row - token * g.heads);
    const int64_t slot = g.slots[token];
    u32x4 k{0, 0, 0, 0}, v{0, 0, 0, 0};
    if ((uint64_t)slot < (uint64_t)g.places) {
        const int64_t page = slot / g.page_size, at = slot - page * g.page_size;
        constexpr int ES = KIND == CACHE_SAME ? 2 : 1;
        const char *K = g.K + (page * g.ck_sp + at * g.ck_ss + h * g.ck_sh + d) * ES, *V = g.V + (page * g.cv_sp + at * g.cv_ss + h * g.cv_sh + d) * ES;
        if constexpr (KIND == CACHE_SAME) {
            __builtin_memcpy(&k, K, 16);
            __builtin_memcpy(&v, V, 16);
        } else {
            u32x2 ck, cv;
            __builtin_memcpy(&ck, K, 8);
            __builtin_memcpy(&cv, V, 8);
            k = dequantise<BF16, KIND>(ck, g.KS[page * g.ks_sp + at * g.ks_ss + h * g.ks_sh]);
            v = dequantise<BF16, KIND>(cv, g.VS[page * g.vs_sp + at * g.vs_ss + h * g.vs_sh]);
        }
    }
    __builtin_memcpy(g.k + token * g.k_st + h * g.k_sh + d, &k, 16);
    __builtin_memcpy(g.v + token * g.v_st + h * g.v_sh + d, &v, 16);
}

template <bool BF16, int KIND, int LANES>
static nt_status launch_cache_lanes(bool write, const CacheArgs &a, hipStream_t s)
{
    const int64_t per = 256 / LANES, grid = (a.rows + per - 1) / per;
    if (grid > kMaxWorkgroups) return fail(NT_ERR_UNSUPPORTED, "tokens * heads too large for one launch");
    if (write) hipLaunchKernelGGL((cache_write_kernel<BF16, KIND, LANES>), dim3((unsigned)grid), dim3(256), 0, s, a);
    else hipLaunchKernelGGL((cache_read_kernel<BF16, KIND, LANES>), dim3((unsigned)grid), dim3(256), 0, s, a);
    return check_launch(write ? "cache_write_kernel" : "cache_read_kernel");
}

template <bool BF16, int KIND>
static nt_status launch_cache_kind(bool write, const CacheArgs &a, hipStream_t s)
{
    if (a.size <= 64) return launch_cache_lanes<BF16, KIND, 8>(write, a, s);
    if (a.size <= 128) return launch_cache_lanes<BF16, KIND, 16>(write, a, s);
    return launch_cache_lanes<BF16, KIND, 32>(write, a, s);
}

nt_status check_cache(const nt_paged_cache *c, int dtype, int *kind)
{
    if (!c || !c->dk || !c->dv) return fail(NT_ERR_INVALID_ARG, "null cache or descriptor");
    if (dtype != NT_F16 && dtype != NT_BF16) return fail(NT_ERR_UNSUPPORTED, "dtype must be NT_F16 or NT_BF16");
    if (c->dk->ndim != 4 || c->dv->ndim != 4) return fail(NT_ERR_SHAPE_MISMATCH, "cache tensors must be 4-D [pages, page_size, heads, head_size]");
    for (int i = 0; i < 4; ++i) {
        if (c->dk->size[i] < 0) return fail(NT_ERR_INVALID_ARG, "negative size");
        if (c->dk->size[i] != c->dv->size[i]) return fail(NT_ERR_SHAPE_MISMATCH, "the cache's K and V differ in size");
    }
    const int64_t pages = c->dk->size[0], page_size = c->dk->size[1], heads = c->dk->size[2], size = c->dk->size[3];
    if (size < 8 || size > 256 || size % 8 != 0) return fail(NT_ERR_UNSUPPORTED, "head_size must be a multiple of 8 up to 256");
    if (c->dk->stride[3] != 1 || c->dv->stride[3] != 1) return fail(NT_ERR_UNSUPPORTED, "the cache needs unit stride along head_size");
    if (page_size < 1 || page_size > (1 << 24)) return fail(NT_ERR_UNSUPPORTED, "page_size must be 1 to 2^24");
    if (heads < 1 || heads > 65535) return fail(NT_ERR_UNSUPPORTED, "1 to 65535 heads");
    if (pages > 0x7fffffffLL) return fail(NT_ERR_UNSUPPORTED, "more than 2^31 - 1 pages");
    if (c->dtype == (nt_dtype)dtype) *kind = CACHE_SAME;
    else if (c->dtype == NT_E4M3) *kind = CACHE_E4M3;
    else if (c->dtype == NT_I8) *kind = CACHE_I8;
    else return fail(NT_ERR_UNSUPPORTED, "the cache must have the tokens' type, NT_E4M3 or NT_I8");
    if (*kind == CACHE_SAME) {
        if (c->k_scale || c->v_scale) return fail(NT_ERR_INVALID_ARG, "scales belong to 8-bit caches only");
    } else {
        if (!c->dks || !c->dvs) return fail(NT_ERR_INVALID_ARG, "an 8-bit cache needs scales");
        if (c->dks->ndim != 3 || c->dvs->ndim != 3) return fail(NT_ERR_SHAPE_MISMATCH, "scales must be 3-D [pages, page_size, heads]");
        for (int i = 0; i < 3; ++i)
            if (c->dks->size[i] != c->dk->size[i] || c->dvs->size[i] != c->dk->size[i]) return fail(NT_ERR_SHAPE_MISMATCH, "scales and cache differ in size");
        if (pages && (!c->k_scale || !c->v_scale)) return fail(NT_ERR_INVALID_ARG, "null device pointer");
    }
    if (pages && (!c->k || !c->v)) return fail(NT_ERR_INVALID_ARG, "null device pointer");
    return NT_OK;
}

nt_status launch_cache(bool write, const nt_paged_cache *c, const void *k, const nt_tensor_desc *dk, const void *v, const nt_tensor_desc *dv,
                       const int64_t *slots, int dtype, void *stream)
{
    int kind = CACHE_SAME;
    const nt_status st = check_cache(c, dtype, &kind);
    if (st != NT_OK) return st;
    if (!dk || !dv) return fail(NT_ERR_INVALID_ARG, "null tensor descriptor");
    if (dk->ndim != 3 || dv->ndim != 3) return fail(NT_ERR_SHAPE_MISMATCH, "tokens must be 3-D [tokens, heads, head_size]");
    for (int i = 0; i < 3; ++i) {
        if (dk->size[i] < 0) return fail(NT_ERR_INVALID_ARG, "negative size");
        if (dk->size[i] != dv->size[i]) return fail(NT_ERR_SHAPE_MISMATCH, "K and V differ in size");
    }
    if (dk->size[1] != c->dk->size[2] || dk->size[2] != c->dk->size[3]) return fail(NT_ERR_SHAPE_MISMATCH, "tokens and cache differ in heads or head_size");
    if (dk->stride[2] != 1 || dv->stride[2] != 1) return fail(NT_ERR_UNSUPPORTED, "tokens need unit stride along head_size");
    if (dk->size[0] == 0) return NT_OK;
    if (!k || !v || !slots) return fail(NT_ERR_INVALID_ARG, "null device pointer");
    if (dk->size[0] > 0x7fffffffLL / dk->size[1]) return fail(NT_ERR_UNSUPPORTED, "tokens * heads must be below 2^31");
    CacheArgs a{};
    a.k = (uint16_t *)const_cast<void *>(k); a.v = (uint16_t *)const_cast<void *>(v);
    a.K = (char *)c->k; a.V = (char *)c->v;
    a.KS = c->k_scale; a.VS = c->v_scale;
    a.slots = slots;
    a.k_st = dk->stride[0]; a.k_sh = dk->stride[1];
    a.v_st = dv->stride[0]; a.v_sh = dv->stride[1];
    a.ck_sp = c->dk->stride[0]; a.ck_ss = c->dk->stride[1]; a.ck_sh = c->dk->stride[2];
    a.cv_sp = c->dv->stride[0]; a.cv_ss = c->dv->stride[1]; a.cv_sh = c->dv->stride[2];
    if (kind != CACHE_SAME) {
        a.ks_sp = c->dks->stride[0]; a.ks_ss = c->dks->stride[1]; a.ks_sh = c->dks->stride[2];
        a.vs_sp = c->dvs->stride[0]; a.vs_ss = c->dvs->stride[1]; a.vs_sh = c->dvs->stride[2];
    }
    a.rows = dk->size[0] * dk->size[1];
    a.places = c->dk->size[0] * c->dk->size[1];
    a.heads = (int32_t)dk->size[1]; a.size = (int32_t)dk->size[2]; a.page_size = (int32_t)c->dk->size[1];
    hipStream_t s = (hipStream_t)stream;
    const bool bf16 = dtype == NT_BF16;
    if (kind == CACHE_E4M3) return bf16 ? launch_cache_kind<true, CACHE_E4M3>(write, a, s) : launch_cache_kind<false, CACHE_E4M3>(write, a, s);
    if (kind == CACHE_I8) return bf16 ? launch_cache_kind<true, CACHE_I8>(write, a, s) : launch_cache_kind<false, CACHE_I8>(write, a, s);
    return launch_cache_kind<false, CACHE_SAME>(write, a, s);             // (copied as it is)
}

}  // namespace nt
