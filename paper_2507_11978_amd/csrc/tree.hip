// Trees of drafted tokens: who is whose ancestor, and which drafts stand.
//
// A sequence's new tokens are a tree, each token behind its parent: parents[t] is the parent's number within the sequence, -1 for none.
//
// Masks.  A token's mask has the bits of itself and its ancestors, its depth is their number less one.  A thread walks up from its token, with the parents in LDS; a word of
// the mask is written when the walk, whose numbers fall, leaves it.
//
// Verification.  With p the target's row at a node, q the draft's, u and r given random numbers in [0, 1): w = p, m = 1; for each child in order, x its token,
//   stands if u q(x) m < w(x)  (the walk goes on from there);  if not,  w = max(w / m - q, 0),  m = sum w.
// Where no child stands the next token is the first t with w(0) + .. + w(t) > r sum w.  Without q the drafts are taken as certain: stands if u m < w(x); if not, m -= w(x),
// w(x) = 0.  (The next token is then distributed as the target's row would have it, whatever was drafted: a child is tried with the probability that what is left
// of p gives it over the probability that it was drafted with, and what is left is p less what was tried.)  Sums and comparisons in 64 bits: a token changes where they are off.
#include <type_traits>

#include "gemm_fast.h"
#include "kernels.h"
#include "paged_index.h"

namespace nt {

// ------------------------------------------------------------------------------------------------------------ masks
constexpr int kParentsHere = 2048;                                         // of a sequence, in LDS

struct MasksArgs {
    const int32_t *parents, *starts, *lengths;
    uint64_t *masks;
    int32_t *depths, *positions;
    int64_t m_st;
    int32_t T, words, window;
};

__global__ __launch_bounds__(256) void tree_masks_kernel(const MasksArgs g)
{
    __shared__ int32_t near[kParentsHere];
    const int b = blockIdx.x;
    const int32_t first = clamp_i32(g.starts[b], 0, g.T), count = clamp_i32(g.starts[b + 1], first, g.T) - first;
    const int32_t *parents = g.parents + first;
    for (int i = threadIdx.x; i < count && i < kParentsHere; i += blockDim.x) near[i] = parents[i];
    __syncthreads();
    for (int32_t i = threadIdx.x; i < count; i += blockDim.x) {
        uint64_t *mask = g.masks + (int64_t)(first + i) * g.m_st, bits = 0;
        int32_t depth = 0, word = g.words - 1;
        for (int32_t j = i;; ++depth) {
            if (!g.window || depth < g.window) {
                for (; word > (j >> 6); --word) {
                    mask[word] = bits;
                    bits = 0;
                }
                if (word == (j >> 6)) bits |= 1ull << (j & 63);            // (not where the masks have too few words)
            }
            const int32_t p = j < kParentsHere ? near[j] : parents[j];
            if (p < 0 || p >= j) break;
            j = p;
        }
        for (; word >= 0; --word) {
            mask[word] = bits;
            bits = 0;
        }
        g.depths[first + i] = depth;
        if (g.positions) g.positions[first + i] = g.lengths[b] - count + depth;
    }
}

nt_status launch_tree_masks(const int32_t *parents, const int32_t *starts, int64_t sequences, uint64_t *masks, const nt_tensor_desc *dm, int32_t *depths,
                            const int32_t *lengths, int32_t *positions, int64_t window, void *stream)
{
    if (!dm) return fail(NT_ERR_INVALID_ARG, "null tensor descriptor");
    if (dm->ndim != 2) return fail(NT_ERR_SHAPE_MISMATCH, "masks must be 2-D [tokens, words]");
    if (sequences < 0 || dm->size[0] < 0) return fail(NT_ERR_INVALID_ARG, "negative size");
    if (dm->size[1] < 1 || dm->size[1] > (1 << 20)) return fail(NT_ERR_UNSUPPORTED, "masks must have 1 to 2^20 words");
    if (dm->size[1] > 1 && dm->stride[1] != 1) return fail(NT_ERR_UNSUPPORTED, "masks need unit stride along a token's words");
    if (window < 0) return fail(NT_ERR_INVALID_ARG, "window must not be negative");
    if (sequences > kMaxWorkgroups || dm->size[0] > (1 << 30)) return fail(NT_ERR_UNSUPPORTED, "too many sequences or tokens");
    if ((positions != nullptr) != (lengths != nullptr)) return fail(NT_ERR_INVALID_ARG, "positions need lengths, and lengths are for positions");
    if (sequences == 0 || dm->size[0] == 0) return NT_OK;
    if (!parents || !starts || !masks || !depths) return fail(NT_ERR_INVALID_ARG, "null device pointer");
    const MasksArgs a{parents, starts, lengths, masks, depths, positions, dm->stride[0], (int32_t)dm->size[0], (int32_t)dm->size[1],
                      (int32_t)(window < 0x7fffffff ? window : 0x7fffffff)};
    hipLaunchKernelGGL(tree_masks_kernel, dim3((unsigned)sequences), dim3(256), 0, (hipStream_t)stream, a);
    return check_launch("tree_masks_kernel");
}

// ----------------------------------------------------------------------------------------------------- verification
constexpr int kVerifyThreads = 1024, kVerifyWaves = kVerifyThreads / 64;
constexpr int kMostTried = 64;                                             // children of a node

struct VerifyArgs {
    const void *target, *draft;
    const int64_t *ids;
    const int32_t *parents, *starts, *lengths;
    const float *uniform, *last_uniform;
    int32_t *path, *accepted, *new_lengths;
    int64_t *next;
    int64_t t_st, d_st, p_sb;
    int32_t T, V, moves;
};

// What is not a positive finite number has no weight
__device__ __forceinline__ double weight_of(float v) { return v > 0.f && v < INFINITY ? (double)v : 0.0; }

template <typename T>
__device__ __forceinline__ float as_float(T v)
{
    if constexpr (std::is_same<T, float>::value) return v;
    else return (float)v;
}

// A node's row as the walk leaves it: what is left of p after `tried` rejections
template <typename T, bool DRAFT>
struct Left {
    static constexpr int N = 16 / sizeof(T);                               // elements of one load
    const T *p, *q;
    const double *mass;                                                    // (DRAFT) m before rejection number j
    const int64_t *gone;                                                   // (not DRAFT) tokens whose weight is 0
    int32_t tried;

    __device__ __forceinline__ double one(float pv, float qv, int32_t t) const
    {
        double w = weight_of(pv);
        if constexpr (DRAFT) {
            const double q1 = weight_of(qv);
            for (int j = 0; j < tried; ++j) {
                const double m = mass[j];
                w = m > 0.0 ? (j ? w / m : w) - q1 : 0.0;                  // (m is 1 at first)
                w = w > 0.0 ? w : 0.0;
            }
        } else {
            for (int j = 0; j < tried; ++j) w = gone[j] == t ? 0.0 : w;
        }
        return w;
    }
    // weights of N elements from t on, those from `hi` on are 0
    __device__ __forceinline__ void load(int32_t t, int32_t hi, double (&w)[N]) const
    {
        T pv[N], qv[N];
        if (t + N <= hi) {
            __builtin_memcpy(pv, p + t, 16);
            if (DRAFT && tried) __builtin_memcpy(qv, q + t, 16);
#pragma unroll
            for (int i = 0; i < N; ++i) w[i] = one(as_float(pv[i]), DRAFT && tried ? as_float(qv[i]) : 0.f, t + i);
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) w[i] = t + i < hi ? one(as_float(p[t + i]), DRAFT && tried ? as_float(q[t + i]) : 0.f, t + i) : 0.0;
        }
    }
    // this lane's part of the sum over [lo, hi), `lanes` lanes side by side
    __device__ __forceinline__ double sum(int32_t lo, int32_t hi, int lane, int lanes) const
    {
        double s = 0.0;
        for (int64_t t = lo + (int64_t)lane * N; t < hi; t += (int64_t)lanes * N) {
            double w[N];
            load((int32_t)t, hi, w);
#pragma unroll
            for (int i = 0; i < N; ++i) s += w[i];
        }
        return s;
    }
};

__device__ __forceinline__ double wave_sum(double v)
{
#pragma unroll
    for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d, 64);
    return v;
}

// Sum over the workgroup, in all threads, added in a fixed order
__device__ __forceinline__ double group_sum(double v, double *scratch)
{
    v = wave_sum(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) scratch[threadIdx.x >> 6] = v;
    __syncthreads();
    double s = 0.0;
#pragma unroll
    for (int w = 0; w < kVerifyWaves; ++w) s += scratch[w];
    return s;
}

// The first element of [lo, hi) whose weight brings the sum, `before` ahead of lo, above `goal`; rounding may leave none: then the last with a weight, -1 if there is
// none.  A sixteenth of the range to a wavefront until it is short.
template <typename T, bool DRAFT>
__device__ int32_t find_above(const Left<T, DRAFT> &left, int32_t lo, int32_t hi, double before, double goal, double *scratch, int32_t *found)
{
    constexpr int N = Left<T, DRAFT>::N;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    while (hi - lo > kVerifyThreads * N) {
        const int32_t part = ((hi - lo + kVerifyWaves - 1) / kVerifyWaves + 64 * N - 1) / (64 * N) * (64 * N);
        const int64_t at = lo + (int64_t)wave * part;
        const int32_t end = at + part < hi ? (int32_t)(at + part) : hi;
        const double s = wave_sum(at < end ? left.sum((int32_t)at, end, lane, 64) : 0.0);
        __syncthreads();
        if (lane == 0) scratch[wave] = s;
        __syncthreads();
        int chosen = -1, last = -1;
        double run = before, at_chosen = before, at_last = before;
        for (int w = 0; w < kVerifyWaves; ++w) {
            const double next = run + scratch[w];
            if (scratch[w] > 0.0) {
                last = w;
                at_last = run;
            }
            if (chosen < 0 && next > goal) {
                chosen = w;
                at_chosen = run;
            }
            run = next;
        }
        if (chosen < 0) {
            chosen = last;
            at_chosen = at_last;
        }
        if (chosen < 0) return -1;
        lo += chosen * part;
        hi = lo + (int64_t)part < hi ? lo + part : hi;
        before = at_chosen;
    }
    double w[N], mine = 0.0;
    const int32_t t = lo + tid * N;
    if (t < hi) {
        left.load(t, hi, w);
#pragma unroll
        for (int i = 0; i < N; ++i) mine += w[i];
    }
    double upto = mine;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const double other = __shfl_up(upto, d, 64);
        if (lane >= d) upto += other;
    }
    __syncthreads();
    if (lane == 63) scratch[wave] = upto;
    if (tid == 0) {
        found[0] = 0x7fffffff;
        found[1] = -1;
    }
    __syncthreads();
    double run = before + (upto - mine);
    for (int i = 0; i < wave; ++i) run += scratch[i];
    int32_t above = 0x7fffffff, last = -1;
    if (t < hi) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            run += w[i];
            if (w[i] > 0.0) {
                last = t + i;
                if (run > goal && above == 0x7fffffff) above = t + i;
            }
        }
    }
    if (above != 0x7fffffff) atomicMin(&found[0], above);
    if (last >= 0) atomicMax(&found[1], last);
    __syncthreads();
    const int32_t a = found[0], l = found[1];
    __syncthreads();
    return a != 0x7fffffff ? a : l;
}

// A workgroup to a sequence: the walk, which every wavefront makes for itself (a token to a lane, its numbers loaded ahead of it), and the next token.
template <typename T, bool DRAFT>
__global__ __launch_bounds__(kVerifyThreads) void verify_tree_kernel(const VerifyArgs g)
{
    __shared__ double scratch[kVerifyWaves], mass[kMostTried];
    __shared__ int64_t gone[kMostTried];
    __shared__ int32_t found[2];
    const int tid = threadIdx.x, lane = tid & 63, b = blockIdx.x;
    const int32_t first = clamp_i32(g.starts[b], 0, g.T), count = clamp_i32(g.starts[b + 1], first, g.T) - first;
    int32_t *path = g.path + b * g.p_sb;
    auto target_row = [&](int32_t node) { return (const T *)g.target + (int64_t)(first + node) * g.t_st; };
    auto draft_row = [&](int32_t node) { return DRAFT ? (const T *)g.draft + (int64_t)(first + node) * g.d_st : nullptr; };

    int32_t node = 0, accepted = count && g.moves ? 1 : 0, tried = 0, known = 0;        // known: rejections that m is of
    double m = 1.0;
    if (tid == 0 && accepted) path[0] = 0;
    for (int32_t c = 0; c < count && accepted && accepted < g.moves; c += 64) {
        const int32_t i = c + lane, t = first + (i < count ? i : 0);
        const int32_t parent = i < count && i > 0 ? g.parents[t] : -1;
        const int64_t x = g.ids[t];
        const float u = g.uniform[t];
        const bool real = parent >= 0 && parent < i && x >= 0 && x < g.V;  // (a token of no vocabulary is passed over)
        const double p = real ? weight_of(as_float(target_row(parent)[x])) : 0.0, q = DRAFT ? (real ? weight_of(as_float(draft_row(parent)[x])) : 0.0) : 1.0;
        uint64_t behind = ~0ull;                                           // those behind the last one that was tried
        while (accepted < g.moves) {
            const uint64_t children = __ballot(real && parent == node) & behind;
            if (!children || tried == kMostTried) break;
            const int l = __builtin_ctzll(children);
            behind = l == 63 ? 0 : ~0ull << (l + 1);
            const double pl = __shfl(p, l, 64), ql = __shfl(q, l, 64);
            const float ul = __shfl(u, l, 64);
            const int64_t xl = __shfl(x, l, 64);
            const Left<T, DRAFT> left{target_row(node), draft_row(node), mass, gone, tried};
            if (DRAFT && known < tried) {
                m = group_sum(left.sum(0, g.V, tid, kVerifyThreads), scratch);
                known = tried;
            }
            // (p and q have been through weight_of: once more changes nothing)
            double w = pl;
            if constexpr (DRAFT) {
                for (int j = 0; j < tried; ++j) {
                    const double d = mass[j];
                    w = d > 0.0 ? (j ? w / d : w) - ql : 0.0;
                    w = w > 0.0 ? w : 0.0;
                }
            } else {
                for (int j = 0; j < tried; ++j) w = gone[j] == xl ? 0.0 : w;
            }
            if ((double)ul * ql * m < w) {
                node = c + l;
                if (tid == 0) path[accepted] = node;
                ++accepted;
                tried = known = 0;
                m = 1.0;
            } else {
                __syncthreads();                                           // (all wavefronts are here: they walk alike; what is written below may still be read)
                if (tid == 0) {
                    if (DRAFT) mass[tried] = m;
                    else gone[tried] = xl;
                }
                __syncthreads();
                if (!DRAFT) m = m - w > 0.0 ? m - w : 0.0;
                ++tried;
            }
        }
    }

    int64_t next = -1;
    if (count > 0) {
        Left<T, DRAFT> left{target_row(node), draft_row(node), mass, gone, tried};
        double total = group_sum(left.sum(0, g.V, tid, kVerifyThreads), scratch);
        if (!(total > 0.0) && tried) {                                     // (nothing is left: the target's row as it is)
            left.tried = 0;
            total = group_sum(left.sum(0, g.V, tid, kVerifyThreads), scratch);
        }
        const float r = g.last_uniform[b];
        if (total > 0.0) next = find_above(left, 0, g.V, 0.0, r > 0.f ? (double)r * total : 0.0, scratch, found);
    }
    for (int32_t k = accepted + tid; k < g.moves; k += kVerifyThreads) path[k] = -1;
    if (tid == 0) {
        g.accepted[b] = accepted;
        g.next[b] = next;
        if (g.new_lengths) g.new_lengths[b] = g.lengths[b] - count + accepted;
    }
}

template <typename T>
static void launch_verify_type(const VerifyArgs &a, int64_t sequences, hipStream_t s)
{
    if (a.draft) hipLaunchKernelGGL((verify_tree_kernel<T, true>), dim3((unsigned)sequences), dim3(kVerifyThreads), 0, s, a);
    else hipLaunchKernelGGL((verify_tree_kernel<T, false>), dim3((unsigned)sequences), dim3(kVerifyThreads), 0, s, a);
}

nt_status launch_verify_tree(const void *target, const nt_tensor_desc *dt, const void *draft, const nt_tensor_desc *dd, const int64_t *ids, const int32_t *parents,
                             const int32_t *starts, int64_t sequences, const float *uniform, const float *last_uniform, int32_t *path, const nt_tensor_desc *dp,
                             int32_t *accepted, int64_t *next, const int32_t *lengths, int32_t *new_lengths, int dtype, void *stream)
{
    if (dtype != NT_F32 && dtype != NT_F16 && dtype != NT_BF16) return fail(NT_ERR_UNSUPPORTED, "dtype must be NT_F32, NT_F16 or NT_BF16");
    if (!dt || !dp || (draft && !dd)) return fail(NT_ERR_INVALID_ARG, "null tensor descriptor");
    if (dt->ndim != 2 || (dd && dd->ndim != 2)) return fail(NT_ERR_SHAPE_MISMATCH, "probabilities must be 2-D [tokens, vocabulary]");
    if (dp->ndim != 2) return fail(NT_ERR_SHAPE_MISMATCH, "paths must be 2-D [sequences, tokens]");
    if (sequences < 0) return fail(NT_ERR_INVALID_ARG, "negative size");
    for (int i = 0; i < 2; ++i) {
        if (dt->size[i] < 0 || dp->size[i] < 0) return fail(NT_ERR_INVALID_ARG, "negative size");
        if (dd && dd->size[i] != dt->size[i]) return fail(NT_ERR_SHAPE_MISMATCH, "the target's and the draft's probabilities differ in size");
    }
    if (dp->size[0] != sequences) return fail(NT_ERR_SHAPE_MISMATCH, "paths and starts differ in sequences");
    if (dp->size[1] < 1) return fail(NT_ERR_SHAPE_MISMATCH, "paths must have room for a token");
    const auto unit = [](const nt_tensor_desc *d) { return d->size[1] < 2 || d->stride[1] == 1; };
    if (!unit(dt) || (dd && !unit(dd)) || !unit(dp)) return fail(NT_ERR_UNSUPPORTED, "probabilities and paths need unit stride along a row");
    if (dt->size[0] > (1 << 30) || dt->size[1] > 0x7fffffffLL - 65536 || dp->size[1] > 0x7fffffffLL || sequences > (1 << 22))
        return fail(NT_ERR_UNSUPPORTED, "too many tokens or sequences, or too large a vocabulary");
    if ((lengths != nullptr) != (new_lengths != nullptr)) return fail(NT_ERR_INVALID_ARG, "lengths and new lengths, or neither");
    if (sequences == 0) return NT_OK;
    if (!starts || !last_uniform || !path || !accepted || !next || (dt->size[0] && (!ids || !parents || !uniform)) || (dt->size[0] && dt->size[1] && !target))
        return fail(NT_ERR_INVALID_ARG, "null device pointer");
    const VerifyArgs a{target, draft, ids, parents, starts, lengths, uniform, last_uniform, path, accepted, new_lengths, next,
                       dt->stride[0], dd ? dd->stride[0] : 0, dp->stride[0], (int32_t)dt->size[0], (int32_t)dt->size[1], (int32_t)dp->size[1]};
    hipStream_t s = (hipStream_t)stream;
    if (dtype == NT_F32) launch_verify_type<float>(a, sequences, s);
    else if (dtype == NT_F16) launch_verify_type<_Float16>(a, sequences, s);
    else launch_verify_type<__bf16>(a, sequences, s);
    return check_launch("verify_tree_kernel");
}

}  // namespace nt
