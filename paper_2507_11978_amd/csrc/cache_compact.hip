// The tokens of a drafted tree that stand, moved to the places behind the past: in every layer's cache at once.
//
// Sequence b has lengths[b] tokens with the accepted[b] that stand, so that position p = lengths[b] - accepted[b] is where the first of them belongs; token path[b][k] of the
// tree, at position p + path[b][k], goes to p + k.  Paths ascend, path[k] >= k: a place that is written was read before, or is read by no one.  Each lane keeps to
// 8 elements of one head of one cache and takes the tokens in order, so that no other lane's reads matter to it: loads of several tokens go out together, ahead of
// their stores, and none is behind a store to the place that it reads (path[j] > path[k] >= k).
//
// Bound by memory, and where few tokens move by the chain path, table, row, store: 64 sequences of 1 to 32 tokens, 16 layers of 8 heads x 128 bf16 7.0 us for 20 MB (2.9 TB/s), one
// sequence, 4 layers 3.0.  (Token after token, with a branch around what is in place already, 21 us.)
#include "paged.h"

namespace nt {

constexpr int kCompactCaches = 32, kCompactAhead = 4;

struct CompactArgs {
    char *K[kCompactCaches], *V[kCompactCaches];
    float *KS[kCompactCaches], *VS[kCompactCaches];
    const int32_t *table, *lengths, *path, *accepted;
    int64_t t_sb, p_sb;
    int64_t ck_sp, ck_ss, ck_sh, cv_sp, cv_ss, cv_sh;         // page, place, head
    int64_t ks_sp, ks_ss, ks_sh, vs_sp, vs_ss, vs_sh;
    int64_t rows;                                             // sequences * heads
    int32_t heads, size, pages, width, moves;                 // entries of a table row, of a path
    Divider page;
};

template <typename Piece>
__device__ __forceinline__ Piece piece_at(const char *p)
{
    Piece v;
    __builtin_memcpy(&v, p, sizeof(Piece));
    return v;
}

template <int BYTES, int LANES>
__global__ __launch_bounds__(256) void cache_compact_kernel(const CompactArgs g)
{
    typedef typename std::conditional<BYTES == 2, u32x4, u32x2>::type Piece;                       // 8 elements
    const int64_t row = (int64_t)blockIdx.x * (256 / LANES) + threadIdx.x / LANES;
    const int cache = blockIdx.y, d = 8 * (threadIdx.x % LANES);
    if (row >= g.rows || d >= g.size) return;
    const int32_t b = (int32_t)((uint32_t)row / (uint32_t)g.heads), h = (int32_t)(row - (int64_t)b * g.heads);
    const int32_t *path = g.path + b * g.p_sb, *pages = g.table + b * g.t_sb;
    const int32_t count = clamp_i32(g.accepted[b], 0, g.moves);
    const int64_t past = (int64_t)g.lengths[b] - g.accepted[b];
    char *K = g.K[cache] + (h * g.ck_sh + d) * BYTES, *V = g.V[cache] + (h * g.cv_sh + d) * BYTES;
    float *KS = BYTES == 1 ? g.KS[cache] + h * g.ks_sh : nullptr, *VS = BYTES == 1 ? g.VS[cache] + h * g.vs_sh : nullptr;
    for (int32_t k0 = 0; k0 < count; k0 += kCompactAhead) {
        Piece kr[kCompactAhead], vr[kCompactAhead];
        float ks[kCompactAhead], vs[kCompactAhead];
        int32_t to[kCompactAhead], at[kCompactAhead];          // page (-1: nothing to move) and place
        int32_t from[kCompactAhead], place[kCompactAhead], id[2][kCompactAhead];
        uint32_t fe[kCompactAhead], te[kCompactAhead];
        bool moves[kCompactAhead];
        // (step by step for all of them, so that the loads of a step are on their way together; what is not to be moved is looked up at its own place)
#pragma unroll
        for (int i = 0; i < kCompactAhead; ++i) from[i] = path[k0 + i < count ? k0 + i : k0];
#pragma unroll
        for (int i = 0; i < kCompactAhead; ++i) {
            const int64_t f = past + from[i], t = past + k0 + i;
            moves[i] = k0 + i < count && from[i] > k0 + i && t >= 0 && f < kMostKeys;            // (not in place already; of a position)
            fe[i] = divide(moves[i] ? (uint32_t)f : 0, g.page);
            te[i] = divide(moves[i] ? (uint32_t)t : 0, g.page);
            place[i] = (int32_t)((uint32_t)f - fe[i] * g.page.d);
            at[i] = (int32_t)((uint32_t)t - te[i] * g.page.d);
            id[0][i] = pages[entry_read(fe[i], g.width)];
            id[1][i] = pages[entry_read(te[i], g.width)];
        }
#pragma unroll
        for (int i = 0; i < kCompactAhead; ++i) {
            const bool ok = moves[i] && names_page(fe[i], id[0][i], g.width, g.pages) && names_page(te[i], id[1][i], g.width, g.pages);
            to[i] = ok ? id[1][i] : -1;
            const int64_t fp = ok ? id[0][i] : 0, p = ok ? place[i] : 0;   // (nothing to move: the cache's first row, for nothing)
            kr[i] = piece_at<Piece>(K + (fp * g.ck_sp + p * g.ck_ss) * BYTES);
            vr[i] = piece_at<Piece>(V + (fp * g.cv_sp + p * g.cv_ss) * BYTES);
            if constexpr (BYTES == 1) {
                ks[i] = KS[fp * g.ks_sp + p * g.ks_ss];
                vs[i] = VS[fp * g.vs_sp + p * g.vs_ss];
            }
        }
#pragma unroll
        for (int i = 0; i < kCompactAhead; ++i) {
            if (to[i] < 0) continue;
            __builtin_memcpy(K + (to[i] * g.ck_sp + at[i] * g.ck_ss) * BYTES, &kr[i], sizeof(Piece));
            __builtin_memcpy(V + (to[i] * g.cv_sp + at[i] * g.cv_ss) * BYTES, &vr[i], sizeof(Piece));
            if constexpr (BYTES == 1)
                if (d == 0) {
                    KS[to[i] * g.ks_sp + at[i] * g.ks_ss] = ks[i];
                    VS[to[i] * g.vs_sp + at[i] * g.vs_ss] = vs[i];
                }
        }
    }
}

template <int BYTES>
static void launch_compact_bytes(const CompactArgs &a, int caches, hipStream_t s)
{
    const int lanes = a.size <= 64 ? 8 : a.size <= 128 ? 16 : 32;
    const dim3 grid((unsigned)((a.rows + 256 / lanes - 1) / (256 / lanes)), caches);
    if (lanes == 8) hipLaunchKernelGGL((cache_compact_kernel<BYTES, 8>), grid, dim3(256), 0, s, a);
    else if (lanes == 16) hipLaunchKernelGGL((cache_compact_kernel<BYTES, 16>), grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL((cache_compact_kernel<BYTES, 32>), grid, dim3(256), 0, s, a);
}

static bool same_layout(const nt_tensor_desc *a, const nt_tensor_desc *b, int ndim)
{
    for (int i = 0; i < ndim; ++i)
        if (a->size[i] != b->size[i] || a->stride[i] != b->stride[i]) return false;
    return true;
}

nt_status launch_cache_compact(const nt_paged_cache *caches, int64_t n, const int32_t *table, const nt_tensor_desc *dt, const int32_t *lengths, const int32_t *path,
                               const nt_tensor_desc *dp, const int32_t *accepted, void *stream)
{
    if (n < 0) return fail(NT_ERR_INVALID_ARG, "negative size");
    if (n && !caches) return fail(NT_ERR_INVALID_ARG, "null cache or descriptor");
    int kind = CACHE_SAME;
    for (int64_t i = 0; i < n; ++i) {
        const nt_paged_cache &c = caches[i];
        // (tokens of a 16-bit cache are of its type; those of an 8-bit one do not matter here)
        const nt_status st = check_cache(&c, c.dtype == NT_E4M3 || c.dtype == NT_I8 ? NT_F16 : c.dtype, &kind);
        if (st != NT_OK) return st;
        if (c.dtype != caches[0].dtype) return fail(NT_ERR_SHAPE_MISMATCH, "the caches must share one type");
        if (!same_layout(c.dk, caches[0].dk, 4) || !same_layout(c.dv, caches[0].dv, 4) ||
            (kind != CACHE_SAME && (!same_layout(c.dks, caches[0].dks, 3) || !same_layout(c.dvs, caches[0].dvs, 3))))
            return fail(NT_ERR_SHAPE_MISMATCH, "the caches must share one layout");
    }
    if (!dt || !dp) return fail(NT_ERR_INVALID_ARG, "null tensor descriptor");
    if (dt->ndim != 2 || dp->ndim != 2) return fail(NT_ERR_SHAPE_MISMATCH, "page table and paths must be 2-D");
    for (int i = 0; i < 2; ++i)
        if (dt->size[i] < 0 || dp->size[i] < 0) return fail(NT_ERR_INVALID_ARG, "negative size");
    if (dt->size[0] != dp->size[0]) return fail(NT_ERR_SHAPE_MISMATCH, "page table and paths differ in sequences");
    if ((dt->size[1] > 1 && dt->stride[1] != 1) || (dp->size[1] > 1 && dp->stride[1] != 1)) return fail(NT_ERR_UNSUPPORTED, "page table and paths need unit stride along a sequence");
    if (dt->size[0] > (1 << 24) || dt->size[1] > 0x7fffffffLL || dp->size[1] > 0x7fffffffLL) return fail(NT_ERR_UNSUPPORTED, "page table or paths too large");
    if (n == 0 || dt->size[0] == 0 || dt->size[1] == 0 || dp->size[1] == 0 || caches[0].dk->size[0] == 0) return NT_OK;
    if (!table || !lengths || !path || !accepted) return fail(NT_ERR_INVALID_ARG, "null device pointer");
    const nt_paged_cache &c = caches[0];
    CompactArgs a{};
    a.table = table; a.lengths = lengths; a.path = path; a.accepted = accepted;
    a.t_sb = dt->stride[0]; a.p_sb = dp->stride[0];
    a.ck_sp = c.dk->stride[0]; a.ck_ss = c.dk->stride[1]; a.ck_sh = c.dk->stride[2];
    a.cv_sp = c.dv->stride[0]; a.cv_ss = c.dv->stride[1]; a.cv_sh = c.dv->stride[2];
    if (kind != CACHE_SAME) {
        a.ks_sp = c.dks->stride[0]; a.ks_ss = c.dks->stride[1]; a.ks_sh = c.dks->stride[2];
        a.vs_sp = c.dvs->stride[0]; a.vs_ss = c.dvs->stride[1]; a.vs_sh = c.dvs->stride[2];
    }
    a.rows = dt->size[0] * c.dk->size[2];
    a.heads = (int32_t)c.dk->size[2]; a.size = (int32_t)c.dk->size[3]; a.pages = (int32_t)c.dk->size[0];
    a.page = divider_of((uint32_t)c.dk->size[1]);
    a.width = entries_in_reach(dt->size[1], a.page.d); a.moves = (int32_t)dp->size[1];
    if (a.rows > kMaxWorkgroups) return fail(NT_ERR_UNSUPPORTED, "too many sequences and heads for one launch");
    // (moved twice at a time, a cache's rows could be read after they were written)
    for (int64_t i = 0; i < n; ++i)
        for (int64_t j = 0; j < i; ++j)
            if (caches[i].k == caches[j].k || caches[i].k == caches[j].v || caches[i].v == caches[j].k || caches[i].v == caches[j].v)
                return fail(NT_ERR_INVALID_ARG, "a cache is listed twice");
    for (int64_t i = 0; i < n; i += kCompactCaches) {
        const int m = (int)(n - i < kCompactCaches ? n - i : kCompactCaches);
        for (int j = 0; j < m; ++j) {
            a.K[j] = (char *)caches[i + j].k; a.V[j] = (char *)caches[i + j].v;
            a.KS[j] = caches[i + j].k_scale; a.VS[j] = caches[i + j].v_scale;
        }
        if (kind == CACHE_SAME) launch_compact_bytes<2>(a, m, (hipStream_t)stream);
        else launch_compact_bytes<1>(a, m, (hipStream_t)stream);
        const nt_status st = check_launch("cache_compact_kernel");
        if (st != NT_OK) return st;
    }
    return NT_OK;
}

}  // namespace nt
