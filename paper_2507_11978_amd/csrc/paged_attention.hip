// Attention of new tokens over a paged key / value cache: checks, choice of kernel and shares, and the join of shared rows.
//
// Rows that see many keys while there are few programs have their keys shared out: each program leaves its reference m, sum l and unnormalised outputs o in the
// workspace, and a second launch joins them, O = sum_s 2^(m_s - M) o_s / sum_s 2^(m_s - M) l_s with M the largest m, in a fixed order.
#include <algorithm>

#include "paged_few.h"
#include "paged_many.h"
#include "workspace.h"

namespace nt {

// WAVES wavefronts per row (token, query head): groups of LANES lanes, 4 elements to a lane, take the shares in turn, eight of them in flight at a time; the
// groups' sums meet within a wavefront and then in LDS.  One wavefront has many rows to hide behind where the shares are few; four make the
// chain of 64 shares of a single long sequence short (2 x 32 rows of 128, 64 shares: 28 us with one, two of a group's loads in flight).  Where there are
// fewer shares than loads the rest are not made (12020 rows of 80 in 3 shares: 4 us less than with one share read again and again).
template <bool BF16, int LANES, int WAVES>
__global__ __launch_bounds__(256) void paged_join_kernel(const PagedArgs g)
{
    constexpr int PARTS = 64 / LANES * WAVES, AT_ONCE = 8;
    __shared__ __attribute__((aligned(16))) float4v red_o[WAVES > 1 ? WAVES : 1][LANES];
    __shared__ float red_m[WAVES], red_l[WAVES];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, part = (WAVES > 1 ? wave * (64 / LANES) : 0) + lane / LANES, d = 4 * (lane % LANES);
    const int64_t row = WAVES > 1 ? blockIdx.x : (int64_t)blockIdx.x * 4 + wave;
    if (row >= (int64_t)g.T * g.Hq) return;
    const int32_t token = (int32_t)((uint32_t)row / (uint32_t)g.Hq), head = (int32_t)(row - (int64_t)token * g.Hq);
    if (token < g.starts[0] || token >= g.starts[g.B]) return;             // (no sequence's: nobody has written its shares)
    const float *ml = g.part_ml + 2 * row * g.splits, *po = g.part_o + row * g.splits * g.D + (d < g.D ? d : 0);
    float m = -INFINITY, l = 0.f;
    float4v o{0.f, 0.f, 0.f, 0.f};
    for (int s0 = 0; s0 < g.splits; s0 += PARTS * AT_ONCE) {
        float2v f[AT_ONCE];
        float4v x[AT_ONCE];
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i) {
            if (s0 + i * PARTS >= g.splits) continue;                      // (wavefront-uniform)
            const int s = s0 + i * PARTS + part < g.splits ? s0 + i * PARTS + part : g.splits - 1;
            __builtin_memcpy(&f[i], ml + 2 * s, 8);
            __builtin_memcpy(&x[i], po + (int64_t)s * g.D, 16);
        }
        float top = m;
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i) {
            if (s0 + i * PARTS + part >= g.splits) f[i] = float2v{-INFINITY, 0.f};
            top = fmaxf(top, f[i][0]);
        }
        const float ref = top == -INFINITY ? 0.f : top, old = __builtin_amdgcn_exp2f(m - ref);
        m = top;
        l *= old;
        o = o * old;
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i) {
            if (s0 + i * PARTS + part >= g.splits) continue;               // (what is there once more may be an infinity)
            const float w = __builtin_amdgcn_exp2f(f[i][0] - ref);
            l = __builtin_fmaf(f[i][1], w, l);
#pragma unroll
            for (int v = 0; v < 4; ++v) o[v] = __builtin_fmaf(x[i][v], w, o[v]);
        }
    }
    float top = m;
#pragma unroll
    for (int x = LANES; x < 64; x <<= 1) top = fmaxf(top, __shfl_xor(top, x, 64));
    const float mine = __builtin_amdgcn_exp2f(m - (top == -INFINITY ? 0.f : top));
    l *= mine;
    o = o * mine;
#pragma unroll
    for (int x = LANES; x < 64; x <<= 1) {
        l += __shfl_xor(l, x, 64);
#pragma unroll
        for (int v = 0; v < 4; ++v) o[v] += __shfl_xor(o[v], x, 64);
    }
    if constexpr (WAVES > 1) {
        if (lane < LANES) red_o[wave][lane] = o;
        if (lane == 0) {
            red_m[wave] = top;
            red_l[wave] = l;
        }
        __syncthreads();
        if (wave) return;
        top = red_m[0];
#pragma unroll
        for (int i = 1; i < WAVES; ++i) top = fmaxf(top, red_m[i]);
        const float ref = top == -INFINITY ? 0.f : top;
        l = 0.f;
        o = float4v{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < WAVES; ++i) {
            const float w = __builtin_amdgcn_exp2f(red_m[i] - ref);
            l = __builtin_fmaf(red_l[i], w, l);
            const float4v x = red_o[i][lane % LANES];
#pragma unroll
            for (int v = 0; v < 4; ++v) o[v] = __builtin_fmaf(x[v], w, o[v]);
        }
    }
    if (lane >= LANES || d >= g.D) return;
    const float inv = l == 0.f ? 0.f : 1.0f / l;
    const u32x2 out{pack_two<BF16>(o[0] * inv, o[1] * inv), pack_two<BF16>(o[2] * inv, o[3] * inv)};
    __builtin_memcpy(g.O + (int64_t)token * g.o_st + (int64_t)head * g.o_sh + d, &out, 8);
}

template <bool BF16, int LANES>
static void launch_join(const PagedArgs &a, hipStream_t s)
{
    const int64_t rows = (int64_t)a.T * a.Hq;
    if (a.splits > 8 && rows <= kMaxWorkgroups) hipLaunchKernelGGL((paged_join_kernel<BF16, LANES, 4>), dim3((unsigned)rows), dim3(256), 0, s, a);
    else hipLaunchKernelGGL((paged_join_kernel<BF16, LANES, 1>), dim3((unsigned)((rows + 3) / 4)), dim3(256), 0, s, a);
}

static thread_local nt_paged_plan t_paged;
const nt_paged_plan &last_paged_plan() { return t_paged; }

nt_status launch_sdpa_paged(const void *q, const nt_tensor_desc *dq, const nt_paged_cache *c, const int32_t *table, const nt_tensor_desc *dt,
                            const int32_t *starts, const int32_t *lengths, void *out, const nt_tensor_desc *dout,
                            float scale, int causal, int64_t window, int64_t max_queries, int64_t max_length, int dtype, void *stream)
{
    t_paged = nt_paged_plan{};
    int kind = CACHE_SAME;
    const nt_status st = check_cache(c, dtype, &kind);
    if (st != NT_OK) return st;
    if (!dq || !dt || !dout) return fail(NT_ERR_INVALID_ARG, "null tensor descriptor");
    if (dq->ndim != 3 || dout->ndim != 3) return fail(NT_ERR_SHAPE_MISMATCH, "queries and output must be 3-D [tokens, heads, head_size]");
    if (dt->ndim != 2) return fail(NT_ERR_SHAPE_MISMATCH, "the page table must be 2-D [sequences, entries]");
    for (int i = 0; i < 3; ++i) {
        if (dq->size[i] < 0 || (i < 2 && dt->size[i] < 0)) return fail(NT_ERR_INVALID_ARG, "negative size");
        if (dq->size[i] != dout->size[i]) return fail(NT_ERR_SHAPE_MISMATCH, "queries and output differ in size");
    }
    const int64_t T = dq->size[0], Hq = dq->size[1], D = dq->size[2], B = dt->size[0], W = dt->size[1];
    const int64_t pages = c->dk->size[0], page_size = c->dk->size[1], Hkv = c->dk->size[2];
    if (D != c->dk->size[3]) return fail(NT_ERR_SHAPE_MISMATCH, "queries and cache differ in head_size");
    if (Hq < 1 || Hq % Hkv != 0) return fail(NT_ERR_SHAPE_MISMATCH, "the query heads must be a multiple of the cache's heads");
    if (dq->stride[2] != 1 || dout->stride[2] != 1) return fail(NT_ERR_UNSUPPORTED, "queries and output need unit stride along head_size");
    if (W > 1 && dt->stride[1] != 1) return fail(NT_ERR_UNSUPPORTED, "the page table needs unit stride along a sequence");
    if (window < 0 || max_queries < 0 || max_length < 0) return fail(NT_ERR_INVALID_ARG, "window, max_queries and max_length must not be negative");
    if (!(scale == scale)) return fail(NT_ERR_INVALID_ARG, "scale is NaN");
    if (T > (1 << 30) / Hq) return fail(NT_ERR_UNSUPPORTED, "tokens * query heads must be at most 2^30");
    if (W > 0x7fffffffLL || B > (1 << 24)) return fail(NT_ERR_UNSUPPORTED, "page table too large");
    if (T == 0 || B == 0) return NT_OK;
    if (!q || !out || !starts || !lengths || (W && !table)) return fail(NT_ERR_INVALID_ARG, "null device pointer");
    if (pages == 0) return fail(NT_ERR_INVALID_ARG, "the cache has no pages");

    PagedArgs a{};
    a.Q = (const uint16_t *)q; a.O = (uint16_t *)out;
    a.K = (const char *)c->k; a.V = (const char *)c->v;
    a.table = W ? table : starts;                                          // (no entries: something to read in their place)
    a.starts = starts; a.lengths = lengths;
    a.q_st = dq->stride[0]; a.q_sh = dq->stride[1];
    a.o_st = dout->stride[0]; a.o_sh = dout->stride[1];
    a.k_sp = c->dk->stride[0]; a.k_ss = c->dk->stride[1]; a.k_sh = c->dk->stride[2];
    a.v_sp = c->dv->stride[0]; a.v_ss = c->dv->stride[1]; a.v_sh = c->dv->stride[2];
    if (kind != CACHE_SAME) {
        a.KS = c->k_scale; a.VS = c->v_scale;
        a.ks_sp = c->dks->stride[0]; a.ks_ss = c->dks->stride[1]; a.ks_sh = c->dks->stride[2];
        a.vs_sp = c->dvs->stride[0]; a.vs_ss = c->dvs->stride[1]; a.vs_sh = c->dvs->stride[2];
    }
    a.t_sb = W ? dt->stride[0] : 0;
    a.T = (int32_t)T; a.B = (int32_t)B; a.Hq = (int32_t)Hq; a.Hkv = (int32_t)Hkv; a.G = (int32_t)(Hq / Hkv); a.D = (int32_t)D;
    a.width = entries_in_reach(W, (uint32_t)page_size); a.pages = (int32_t)pages;
    a.causal = causal ? 1 : 0;
    a.window = (int32_t)std::min<int64_t>(window, 0x7fffffff);              // (longer than any sequence)
    const int64_t es = kind == CACHE_SAME ? 2 : 1, most_bytes = (1LL << 31) - 4096;
    a.near = a.k_ss >= 0 && a.k_ss < most_bytes / (16 * es) && a.v_ss >= 0 && a.v_ss < most_bytes / (16 * es);
    a.uniform = a.near && page_size % 16 == 0;
    a.aligned = (((uintptr_t)a.K | (uintptr_t)a.V | (uint64_t)((a.k_sp | a.k_ss | a.k_sh | a.v_sp | a.v_ss | a.v_sh) * es)) & 15) == 0;
    a.page = divider_of((uint32_t)page_size);
    a.group = divider_of((uint32_t)a.G);
    a.scale_log2e = (scale == 0.f ? 1.0f / sqrtf((float)D) : scale) * 1.4426950408889634f;

    // Up to 32 rows per key head: the kernel whose wavefronts share the keys, else the one whose wavefronts share the rows (us, 8 heads x 128 bf16, 32 rows: 1 x 1000
    // keys 14.0, by the other 27.4, 1 x 8000 18.5 / 25.5, 32 x 2000 57.7 / 81.0; 4 x 16 heads x 64 f16, 8000 35.3 / 42.1).
    const int64_t most = max_queries && max_queries < T ? max_queries : T, group_rows = most * a.G;
    const int built = D <= 64 ? 64 : D <= 128 ? 128 : 256;
    const int rows = group_rows <= 16 ? 16 : group_rows <= 32 && built < 256 ? 32 : kManyRows;
    a.tiles = rows == kManyRows ? (int32_t)(T * a.G / kManyRows + B) : (int32_t)B;
    const int64_t base = (int64_t)a.tiles * Hkv;
    if (base > kMaxWorkgroups) return fail(NT_ERR_UNSUPPORTED, "too many programs for one launch");
    // ---- shares
    int64_t length = (int64_t)a.width * page_size;
    if (max_length) length = std::min(length, max_length);
    if (window) length = std::min(length, window + most);
    const int64_t block = rows == kManyRows ? many_keys(built) : few_trip(kind, built);
    int64_t splits;
    if (rows == kManyRows) {
        // Below 256 programs as many shares as make two for a unit at most, of 192 keys each and more; from 256 on, one program to a unit and more, none (us, graph replays, 32/8 heads x 128 bf16: 64 queries x 600 keys 22 unshared, 15.1 in 3 shares,
        // 1000 30 / 17.2 in 4, 20000 526 / 49.5 in 32; 200 x 4000 109 / 38.4 in 8, 60.3 in 16; 7 x 200 in windows of 512 29.6 / 29.1 in 3).
        splits = std::min(base >= 256 ? 1 : 512 / base, length / 192);
    } else {
        // As many programs as units at most, of 48 KB of K and V and more each (us, graph replays: 1 x 8 heads x 128 bf16, 500 keys 12.0 unshared, 9.5 in 6 shares, 2000 32.3 / 10.7
        // in 21, 32000 434 / 31.0 in 32, 31.2 in 63; 48 heads x 64 f16, 900 12.2 / 10.6 in 4, 12.3 in 3, 8000 60.0 / 24.5 in 4, 28.3 in 8; 300 9.1 / 9.7 in 3).
        const int64_t key_bytes = 2 * D * es, total = length * key_bytes;
        // Below 384 KB to a sequence's head not at all: the second launch and the workspace's event are 4 us of the host's time (48 x 900, called: 12.5 us, 13.2).
        splits = total < (384 << 10) ? 1 : std::min(256 / base, total / (48 << 10));
        // Where that leaves long programs, 256 KB each: sequences of different lengths fill the units more evenly (64 x 8 heads x 128 bf16, 17 to 4096 keys 154 us
        // unshared, 134 so, 143 with 512 KB; 2 x 8 heads x 131072 e4m3 135 with 1 MB, 130).
        if (total / std::max<int64_t>(1, splits) > (5 << 20) / 4) splits = total / (256 << 10);
    }
    splits = std::min(std::max<int64_t>(1, splits), kMaxWorkgroups / base);
    int64_t share = ((length + splits - 1) / splits + block - 1) / block * block;
    splits = share ? std::max<int64_t>(1, (length + share - 1) / share) : 1;
    WorkspaceLease lease;
    hipStream_t s = (hipStream_t)stream;
    if (splits > 1) {
        const size_t n = (size_t)(T * Hq * splits), n2 = 2 * n + 2 * (n & 1);             // (outputs begin at a multiple of 16 bytes)
        a.part_ml = (float *)lease.acquire((n2 + n * (size_t)D) * 4, s);
        if (a.part_ml) a.part_o = a.part_ml + n2;
        else splits = 1;                                                   // (no room: unshared)
    }
    a.splits = (int32_t)splits;
    a.split_keys = (int32_t)std::min<int64_t>(share, 0x7fffffff / 2);
    const bool bf16 = dtype == NT_BF16;
    auto launch = built == 64 ? launch_paged_64 : built == 128 ? launch_paged_128 : launch_paged_256;
    nt_status rc = launch(a, rows, base * splits, bf16, kind, stream);
    if (rc != NT_OK) return rc;
    if (splits > 1) {
        if (built == 64) bf16 ? launch_join<true, 16>(a, s) : launch_join<false, 16>(a, s);
        else if (built == 128) bf16 ? launch_join<true, 32>(a, s) : launch_join<false, 32>(a, s);
        else bf16 ? launch_join<true, 64>(a, s) : launch_join<false, 64>(a, s);
        rc = check_launch("paged_join_kernel");
        if (rc != NT_OK) return rc;
    }
    t_paged = nt_paged_plan{rows, (int32_t)splits, splits > 1 ? a.split_keys : 0};
    return NT_OK;
}

}  // namespace nt
