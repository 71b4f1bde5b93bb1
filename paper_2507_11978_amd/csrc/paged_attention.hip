// Attention of new tokens over a paged key / value cache: checks, choice of kernel and shares, and the join of shared rows.
//
// Rows that see many keys while there are few programs have their keys shared out: each program leaves its reference m, sum l and unnormalised outputs o in the
// workspace, and a second launch joins them, O = sum_s 2^(m_s - M) o_s / sum_s 2^(m_s - M) l_s with M the largest m, in a fixed order.
#include <algorithm>

#include "paged_few.h"
#include "paged_many.h"
#include "workspace.h"

namespace nt {

// One wavefront per row (token, query head): lanes / LANES groups take the shares in turn, LANES lanes have 4 elements each.
template <bool BF16, int LANES>
__global__ __launch_bounds__(256) void paged_join_kernel(const PagedArgs g)
{
    const int lane = threadIdx.x & 63, part = lane / LANES, d = 4 * (lane % LANES);
    const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (row >= (int64_t)g.T * g.Hq) return;
    const int32_t token = (int32_t)((uint32_t)row / (uint32_t)g.Hq), head = (int32_t)(row - (int64_t)token * g.Hq);
    if (token < g.starts[0] || token >= g.starts[g.B]) return;             // (no sequence's: nobody has written its shares)
    const float *ml = g.part_ml + 2 * row * g.splits;
    float top = -INFINITY;
    for (int s = lane; s < g.splits; s += 64) top = fmaxf(top, ml[2 * s]);
#pragma unroll
    for (int x = 1; x < 64; x <<= 1) top = fmaxf(top, __shfl_xor(top, x, 64));
    const float ref = top == -INFINITY ? 0.f : top;
    float sum = 0.f;
    float4v o{0.f, 0.f, 0.f, 0.f};
    for (int s = part; s < g.splits; s += 64 / LANES) {
        const float f = __builtin_amdgcn_exp2f(ml[2 * s] - ref);
        sum = __builtin_fmaf(ml[2 * s + 1], f, sum);
        if (d < g.D) {
            float4v x;
            __builtin_memcpy(&x, g.part_o + (row * g.splits + s) * g.D + d, 16);
#pragma unroll
            for (int v = 0; v < 4; ++v) o[v] = __builtin_fmaf(x[v], f, o[v]);
        }
    }
#pragma unroll
    for (int x = LANES; x < 64; x <<= 1) {
        sum += __shfl_xor(sum, x, 64);
#pragma unroll
        for (int v = 0; v < 4; ++v) o[v] += __shfl_xor(o[v], x, 64);
    }
    if (part != 0 || d >= g.D) return;
    const float inv = sum == 0.f ? 0.f : 1.0f / sum;
    const u32x2 out{pack_two<BF16>(o[0] * inv, o[1] * inv), pack_two<BF16>(o[2] * inv, o[3] * inv)};
    __builtin_memcpy(g.O + (int64_t)token * g.o_st + (int64_t)head * g.o_sh + d, &out, 8);
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
    a.table = table; a.starts = starts; a.lengths = lengths;
    a.q_st = dq->stride[0]; a.q_sh = dq->stride[1];
    a.o_st = dout->stride[0]; a.o_sh = dout->stride[1];
    a.k_sp = c->dk->stride[0]; a.k_ss = c->dk->stride[1]; a.k_sh = c->dk->stride[2];
    a.v_sp = c->dv->stride[0]; a.v_ss = c->dv->stride[1]; a.v_sh = c->dv->stride[2];
    if (kind != CACHE_SAME) {
        a.KS = c->k_scale; a.VS = c->v_scale;
        a.ks_sp = c->dks->stride[0]; a.ks_ss = c->dks->stride[1]; a.ks_sh = c->dks->stride[2];
        a.vs_sp = c->dvs->stride[0]; a.vs_ss = c->dvs->stride[1]; a.vs_sh = c->dvs->stride[2];
    }
    a.t_sb = dt->stride[0];
    a.T = (int32_t)T; a.B = (int32_t)B; a.Hq = (int32_t)Hq; a.Hkv = (int32_t)Hkv; a.G = (int32_t)(Hq / Hkv); a.D = (int32_t)D;
    a.width = (int32_t)W; a.pages = (int32_t)pages;
    a.causal = causal ? 1 : 0;
    a.window = (int32_t)std::min<int64_t>(window, 1 << 30);
    const int64_t es = kind == CACHE_SAME ? 2 : 1, most_bytes = (1LL << 31) - 4096;
    a.uniform = page_size % 16 == 0 && a.k_ss >= 0 && a.k_ss < most_bytes / (16 * es) && a.v_ss >= 0 && a.v_ss < most_bytes / (16 * es);
    a.page = divider_of((uint32_t)page_size);
    a.group = divider_of((uint32_t)a.G);
    a.scale_log2e = (scale == 0.f ? 1.0f / sqrtf((float)D) : scale) * 1.4426950408889634f;

    // Up to 32 rows per key head: the kernel whose wavefronts share the keys, else the one whose wavefronts share the rows.
    const int64_t most = max_queries && max_queries < T ? max_queries : T, group_rows = most * a.G;
    const int rows = group_rows <= 16 ? 16 : group_rows <= 32 ? 32 : kManyRows;
    a.tiles = rows == kManyRows ? (int32_t)(T * a.G / kManyRows + B) : (int32_t)B;
    const int64_t base = (int64_t)a.tiles * Hkv;
    if (base > kMaxWorkgroups) return fail(NT_ERR_UNSUPPORTED, "too many programs for one launch");
    // ---- shares
    const int built = D <= 64 ? 64 : D <= 128 ? 128 : 256;
    int64_t length = W * page_size;
    if (max_length) length = std::min(length, max_length);
    if (window) length = std::min(length, window + most);
    const int64_t block = rows == kManyRows ? many_keys(built) : few_trip(kind, built);
    const int64_t wanted = rows == kManyRows ? (base >= 256 ? 1 : 512 / base) : (1024 + base - 1) / base;
    int64_t splits = std::max<int64_t>(1, std::min(wanted, length / (rows == kManyRows ? 512 : 256)));
    splits = std::min<int64_t>(splits, kMaxWorkgroups / base);
    int64_t share = ((length + splits - 1) / splits + block - 1) / block * block;
    splits = share ? std::max<int64_t>(1, (length + share - 1) / share) : 1;
    WorkspaceLease lease;
    hipStream_t s = (hipStream_t)stream;
    if (splits > 1) {
        const size_t n = (size_t)(T * Hq * splits);
        a.part_ml = (float *)lease.acquire(n * (size_t)(D + 2) * 4, s);
        if (a.part_ml) a.part_o = a.part_ml + 2 * n;
        else splits = 1;                                                   // (no room: unshared)
    }
    a.splits = (int32_t)splits;
    a.split_keys = (int32_t)std::min<int64_t>(share, 0x7fffffff / 2);
    const bool bf16 = dtype == NT_BF16;
    auto launch = D <= 64 ? launch_paged_64 : D <= 128 ? launch_paged_128 : launch_paged_256;
    nt_status rc = launch(a, rows, base * splits, bf16, kind, stream);
    if (rc != NT_OK) return rc;
    if (splits > 1) {
        const unsigned grid = (unsigned)((T * Hq + 3) / 4);
        auto join = [&](auto kern) { hipLaunchKernelGGL(kern, dim3(grid), dim3(256), 0, s, a); };
        if (D <= 64) bf16 ? join(paged_join_kernel<true, 16>) : join(paged_join_kernel<false, 16>);
        else if (D <= 128) bf16 ? join(paged_join_kernel<true, 32>) : join(paged_join_kernel<false, 32>);
        else bf16 ? join(paged_join_kernel<true, 64>) : join(paged_join_kernel<false, 64>);
        rc = check_launch("paged_join_kernel");
        if (rc != NT_OK) return rc;
    }
    t_paged = nt_paged_plan{rows, (int32_t)splits, splits > 1 ? a.split_keys : 0};
    return NT_OK;
}

}  // namespace nt
