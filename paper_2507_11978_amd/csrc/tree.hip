// Trees of drafted tokens: who is whose ancestor, and which drafts stand.
//
// A sequence's new tokens are a tree, each token behind its parent: parents[t] is the parent's number within the sequence, -1 for none.
//
// Masks.  A token's mask has the bits of itself and its ancestors, its depth is their number less one.  A thread walks up from its token, with the parents in LDS; a word of
// the mask is written when the walk, whose numbers fall, leaves it.  A launch, a load, LDS: 1.9 us for a chain of 8, 3.2 for 128 trees of 100.  Bound
// by the longest walk, a chain of reads: 128 chains of 100 13.8 us, one of 2000 1260, of 8000, whose parents are read from memory, 25 ms.
//
// Verification.  With p the target's row at a node, q the draft's, u and r given random numbers in [0, 1): w = p, m = 1; for each child in order, x its token,
//   stands if u q(x) m < w(x)  (the walk goes on from there);  if not,  w = max(w / m - q, 0),  m = sum w.
// Where no child stands the next token is the first t with w(0) + .. + w(t) > r sum w.  Without q the drafts are taken as certain: stands if u m < w(x); if not, m -= w(x),
// w(x) = 0.  (The next token is then distributed as the target's row would have it, whatever was drafted: a child is tried with the probability that what is left
// of p gives it over the probability that it was drafted with, and what is left is p less what was tried.)  Sums and comparisons in 64 bits: a token changes where they are off.
//
// What has to be read are a few numbers of each draft, and the rows p and q of the node where the walk ends (and of those where more than one child is tried, for m).  One unit reads
// 128000 words of both in 20 us, the chip 64 of them in 14: the rows are summed in chunks by all of it, then the chunk is searched in which the sum passes its goal.
// Measured: 64 trees of 24 drafts, 128000 words fp32 61 to 131 us, by the random numbers (walks meet two or three such nodes, in the longest five or more: what is behind the rounds is one unit's work; in a call of 85 40 us of sums, the chain of launches and loads the rest), one chain of 6, 32000
// words, 11.4 us: walk 3.1, sums 1.9, search 4.8 us, each a chain of loads.
#include <algorithm>
#include <type_traits>

#include "gemm_fast.h"
#include "kernels.h"
#include "paged_index.h"
#include "workspace.h"

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
    if (count <= kParentsHere)
        for (int i = threadIdx.x; i < count; i += blockDim.x) near[i] = parents[i];
    __syncthreads();
    // (from LDS or from memory, not from either: a load that may be of both is as slow as the slower)
    const auto walks = [&](const int32_t *from) __attribute__((always_inline)) {
        for (int32_t i = threadIdx.x; i < count; i += blockDim.x) {
            uint64_t *mask = g.masks + (int64_t)(first + i) * g.m_st, bits = 0;
            int32_t depth = 0, word = g.words - 1;
            for (int32_t j = i;; ++depth) {
                if (!g.window || depth < g.window) {
                    for (; word > (j >> 6); --word) {
                        mask[word] = bits;
                        bits = 0;
                    }
                    if (word == (j >> 6)) bits |= 1ull << (j & 63);        // (not where the masks have too few words)
                }
                const int32_t p = from[j];
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
    };
    if (count <= kParentsHere) walks(near);
    else walks(parents);
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
constexpr int kMostChunks = 256;                                           // of a row

struct VerifyArgs {
    const void *target, *draft;
    const int64_t *ids;
    const int32_t *parents, *starts, *lengths;
    const float *uniform, *last_uniform;
    int32_t *path, *accepted, *new_lengths;
    int64_t *next;
    int64_t t_st, d_st, p_sb;
    int32_t T, V, moves;
    // in rounds: where each walk is, and sums of its row in chunks
    struct VerifyState *state;
    double *sums;
    int32_t chunk, chunks;
};

struct Walk {
    int32_t node, accepted, tried, at;                                     // tokens before `at` have been passed
};

// A sum m and 1 / m, rounded to nearest; 0 and 0 where m is 0
struct Sum {
    double m, inverse;
};
__device__ __forceinline__ Sum sum_and_inverse(double m) { return Sum{m, m > 0.0 ? 1.0 / m : 0.0}; }

// w / m, rounded to nearest, 0 where m is 0.  w times the inverse is within two last places; one correction by the remainder makes it one of the two neighbours, from which the
// next gives the nearest (Markstein's theorem: an inverse rounded to nearest, a remainder without rounding).  64 trees of 24, 128000 words 90.5 us so, 109 with divisions, each of which
// finds the inverse anew, 87 with one correction.  81 with products by the inverse alone: but then w / m that is q leaves something or not by how the inverse was rounded.
__device__ __forceinline__ double quotient(double w, const Sum &s)
{
    double q = w * s.inverse;
    q = __builtin_fma(__builtin_fma(-q, s.m, w), s.inverse, q);
    return __builtin_fma(__builtin_fma(-q, s.m, w), s.inverse, q);
}

struct VerifyState {
    Walk walk;
    int32_t done, summed;                                                  // the walk has ended; the sums are of where it did
    Sum over[kMostTried];
    int64_t gone[kMostTried];
};

// What is not a positive finite number has no weight
__device__ __forceinline__ double weight_of(float v)
{
    constexpr int POSITIVE_SUBNORMAL = 1 << 7, POSITIVE_NORMAL = 1 << 8;
    return (double)(__builtin_amdgcn_classf(v, POSITIVE_SUBNORMAL | POSITIVE_NORMAL) ? v : 0.f);
}

template <typename T>
__device__ __forceinline__ float as_float(T v)
{
    if constexpr (std::is_same<T, float>::value) return v;
    else return (float)v;
}

// A node's row as the walk leaves it: what is left of p after `tried` rejections
template <typename T, bool DRAFT>
struct Left {
    static constexpr int N = 16 / sizeof(T), DEEP = 16 / N;                // elements of one load, loads of a row on their way
    struct Piece {
        T v[N];
    };
    const T *p, *q;
    const Sum *over;                                                       // (DRAFT) m before rejection number j
    const int64_t *gone;                                                   // (not DRAFT) tokens whose weight is 0
    int32_t tried;

    // FEW: of no rejections, or of one (DRAFT; m is 1 at first)
    static constexpr int ANY = 2;
    template <int FEW>
    __device__ __forceinline__ double one(float pv, float qv, int32_t t) const
    {
        double w = weight_of(pv);
        if constexpr (FEW == 0) return w;
        if constexpr (DRAFT) {
            const double q1 = weight_of(qv);
            w = __builtin_fmax(w - q1, 0.0);
            if constexpr (FEW != 1)
                for (int j = 1; j < tried; ++j) w = __builtin_fmax(quotient(w, over[j]) - q1, 0.0);
        } else if constexpr (FEW == ANY) {
            for (int j = 0; j < tried; ++j) w = gone[j] == t ? 0.0 : w;
        }
        return w;
    }
    // whether one of N tokens from t on is gone
    __device__ __forceinline__ bool any_gone(int64_t t) const
    {
        bool any = false;
        if constexpr (!DRAFT)
            for (int j = 0; j < tried; ++j) any = any | ((uint64_t)(gone[j] - t) < (uint64_t)N);
        return any;
    }
    __device__ __forceinline__ double weight(float pv, float qv, int32_t t) const { return tried ? one<ANY>(pv, qv, t) : one<0>(pv, qv, t); }

    // weights of N elements from t on, those from `hi` on are 0
    __device__ __forceinline__ void load(int32_t t, int32_t hi, double (&w)[N]) const
    {
        Piece pv, qv;
        if (t + N <= hi) {
            __builtin_memcpy(&pv, p + t, 16);
            if (DRAFT) __builtin_memcpy(&qv, q + t, 16);
#pragma unroll
            for (int i = 0; i < N; ++i) w[i] = weight(as_float(pv.v[i]), DRAFT ? as_float(qv.v[i]) : 0.f, t + i);
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) w[i] = t + i < hi ? weight(as_float(p[t + i]), DRAFT ? as_float(q[t + i]) : 0.f, t + i) : 0.0;
        }
    }
    template <int FEW>
    __device__ __forceinline__ double sum_of(int32_t lo, int32_t hi, int lane, int lanes) const
    {
        constexpr bool BOTH = DRAFT && FEW > 0;
        double s[DEEP] = {};
        int64_t t = lo + (int64_t)lane * N;
        const int64_t step = (int64_t)lanes * N;
        for (; t + (DEEP - 1) * step + N <= hi; t += DEEP * step) {
            Piece pv[DEEP], qv[BOTH ? DEEP : 1];
#pragma unroll
            for (int d = 0; d < DEEP; ++d) __builtin_memcpy(&pv[d], p + t + d * step, 16);
            if constexpr (BOTH)
#pragma unroll
                for (int d = 0; d < DEEP; ++d) __builtin_memcpy(&qv[d], q + t + d * step, 16);
#pragma unroll
            for (int d = 0; d < DEEP; ++d) {
                if (!DRAFT && FEW > 0 && any_gone(t + d * step)) {
                    double w[N];
                    load((int32_t)(t + d * step), hi, w);
#pragma unroll
                    for (int i = 0; i < N; ++i) s[d] += w[i];
                    continue;
                }
#pragma unroll
                for (int i = 0; i < N; ++i) s[d] += one<DRAFT ? FEW : 0>(as_float(pv[d].v[i]), BOTH ? as_float(qv[BOTH ? d : 0].v[i]) : 0.f, (int32_t)(t + d * step) + i);
            }
        }
        for (; t < hi; t += step) {
            double w[N];
            load((int32_t)t, hi, w);
#pragma unroll
            for (int i = 0; i < N; ++i) s[0] += w[i];
        }
        double all = s[0];
#pragma unroll
        for (int d = 1; d < DEEP; ++d) all += s[d];
        return all;
    }
    // this lane's part of the sum over [lo, hi), `lanes` lanes side by side
    __device__ __forceinline__ double sum(int32_t lo, int32_t hi, int lane, int lanes) const
    {
        return tried == 0 ? sum_of<0>(lo, hi, lane, lanes) : DRAFT && tried == 1 ? sum_of<1>(lo, hi, lane, lanes) : sum_of<ANY>(lo, hi, lane, lanes);
    }
};

__device__ __forceinline__ double wave_sum(double v)
{
#pragma unroll
    for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d, 64);
    return v;
}

// Sum over the workgroup of THREADS, in all threads, added in a fixed order
template <int THREADS>
__device__ __forceinline__ double group_sum(double v, double *scratch)
{
    v = wave_sum(v);
    if constexpr (THREADS > 64) {
        __syncthreads();
        if ((threadIdx.x & 63) == 0) scratch[threadIdx.x >> 6] = v;
        __syncthreads();
        v = 0.0;
#pragma unroll
        for (int w = 0; w < THREADS / 64; ++w) v += scratch[w];
    }
    return v;
}

// The first element of [lo, hi) whose weight brings the sum, `before` ahead of lo, above `goal`; rounding may leave none: then the last with a weight, -1 if there is
// none.  (What has no weight is never chosen: sums of the same numbers in another order may put `before` itself above the goal.)  A sixteenth of the range to a wavefront until it is short.
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
            if (chosen < 0 && scratch[w] > 0.0 && next > goal) {
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
    // (one lane of a wavefront: its first, its last; 1024 atomics to one place take 6 us)
    const uint64_t some = __ballot(above != 0x7fffffff), any = __ballot(last >= 0);
    if (some && lane == __builtin_ctzll(some)) atomicMin(&found[0], above);
    if (any && lane == 63 - __builtin_clzll(any)) atomicMax(&found[1], last);
    __syncthreads();
    const int32_t a = found[0], l = found[1];
    __syncthreads();
    return a != 0x7fffffff ? a : l;
}

// The walk, which every wavefront makes for itself (a token to a lane, its numbers loaded ahead of it).  m: after the `tried` rejections, if known.  False: m is needed and not known
// (SELF: worked out here).
template <typename T, bool DRAFT, bool SELF, int THREADS>
__device__ __forceinline__ bool walk_tree(const VerifyArgs &g, const int32_t first, const int32_t count, int32_t *path, Walk &s, double m, bool known, Sum *over, int64_t *gone,
                                          double *scratch)
{
    const int tid = threadIdx.x, lane = tid & 63;
    auto target_row = [&](int32_t node) { return (const T *)g.target + (int64_t)(first + node) * g.t_st; };
    auto draft_row = [&](int32_t node) { return DRAFT ? (const T *)g.draft + (int64_t)(first + node) * g.d_st : nullptr; };
    while (s.at < count && s.accepted < g.moves) {
        const int32_t c = s.at & ~63, i = c + lane, t = first + (i < count ? i : 0);
        const int32_t parent = i < count && i > 0 ? g.parents[t] : -1;
        const int64_t x = g.ids[t];
        const float u = g.uniform[t];
        const bool real = parent >= 0 && parent < i && x >= 0 && x < g.V;  // (a token of no vocabulary is passed over)
        const float p = real ? as_float(target_row(parent)[x]) : 0.f, q = DRAFT && real ? as_float(draft_row(parent)[x]) : 0.f;
        while (s.accepted < g.moves) {
            const uint64_t children = __ballot(real && parent == s.node && i >= s.at);
            if (!children || s.tried == kMostTried) break;
            const int l = __builtin_ctzll(children);
            const float pl = __shfl(p, l, 64), ql = __shfl(q, l, 64), ul = __shfl(u, l, 64);
            const int64_t xl = __shfl(x, l, 64);
            const Left<T, DRAFT> left{target_row(s.node), draft_row(s.node), over, gone, s.tried};
            if (DRAFT && !known) {
                if constexpr (!SELF) return false;
                m = group_sum<THREADS>(left.sum(0, g.V, tid, THREADS), scratch);
                known = true;
            }
            const double w = left.weight(pl, ql, (int32_t)xl);
            s.at = c + l + 1;
            if ((double)ul * (DRAFT ? weight_of(ql) : 1.0) * m < w) {
                s.node = c + l;
                if (tid == 0) path[s.accepted] = s.node;
                ++s.accepted;
                s.tried = 0;
                m = 1.0;
            } else {
                __syncthreads();                                           // (all wavefronts are here: they walk alike; what is written below may still be read)
                if (tid == 0) {
                    if (DRAFT) over[s.tried] = sum_and_inverse(m);
                    else gone[s.tried] = xl;
                }
                __syncthreads();
                if (DRAFT) known = false;
                else m = m - w > 0.0 ? m - w : 0.0;
                ++s.tried;
            }
        }
        s.at = s.at > c + 64 ? s.at : c + 64;
    }
    return true;
}

// What is told of a sequence where its walk ends
__device__ __forceinline__ void tell(const VerifyArgs &g, int b, int32_t count, const Walk &s, int threads)
{
    for (int64_t k = s.accepted + (int64_t)threadIdx.x; k < g.moves; k += threads) g.path[b * g.p_sb + k] = -1;
    if (threadIdx.x == 0) {
        g.accepted[b] = s.accepted;
        if (g.new_lengths) g.new_lengths[b] = g.lengths[b] - count + s.accepted;
    }
}

// The next token, from the node's row as it is left, `total` its sum and `before` that ahead of lo; where nothing is left the target's row as it is
template <typename T, bool DRAFT>
__device__ __forceinline__ int64_t next_token(const VerifyArgs &g, int b, Left<T, DRAFT> left, int32_t lo, int32_t hi, double before, double total, double *scratch, int32_t *found)
{
    if (!(total > 0.0) && left.tried) {
        left.tried = 0;
        lo = 0;
        hi = g.V;
        before = 0.0;
        total = group_sum<kVerifyThreads>(left.sum(0, g.V, threadIdx.x, kVerifyThreads), scratch);
    }
    const float r = g.last_uniform[b];
    return total > 0.0 ? find_above(left, lo, hi, before, r > 0.f ? (double)r * total : 0.0, scratch, found) : -1;
}

__device__ __forceinline__ int32_t first_of(const VerifyArgs &g, int b) { return clamp_i32(g.starts[b], 0, g.T); }
__device__ __forceinline__ int32_t count_of(const VerifyArgs &g, int b) { return clamp_i32(g.starts[b + 1], first_of(g, b), g.T) - first_of(g, b); }

// A workgroup to a sequence: short rows
template <typename T, bool DRAFT>
__global__ __launch_bounds__(kVerifyThreads) void verify_tree_kernel(const VerifyArgs g)
{
    __shared__ double scratch[kVerifyWaves];
    __shared__ Sum over[kMostTried];
    __shared__ int64_t gone[kMostTried];
    __shared__ int32_t found[2];
    const int b = blockIdx.x;
    const int32_t first = first_of(g, b), count = count_of(g, b);
    int32_t *path = g.path + b * g.p_sb;
    Walk s{0, count ? 1 : 0, 0, 1};
    if (threadIdx.x == 0 && count) path[0] = 0;
    if (count) walk_tree<T, DRAFT, true, kVerifyThreads>(g, first, count, path, s, 1.0, true, over, gone, scratch);
    int64_t next = -1;
    if (count) {
        const int64_t row = first + s.node;
        const Left<T, DRAFT> left{(const T *)g.target + row * g.t_st, DRAFT ? (const T *)g.draft + row * g.d_st : nullptr, over, gone, s.tried};
        const double total = group_sum<kVerifyThreads>(left.sum(0, g.V, threadIdx.x, kVerifyThreads), scratch);
        next = next_token(g, b, left, 0, g.V, 0.0, total, scratch, found);
    }
    tell(g, b, count, s, kVerifyThreads);
    if (threadIdx.x == 0) g.next[b] = next;
}

// ---- the same in rounds: a walk goes as far as it knows m, and the sums of the rows that it needs are dealt out over the chip
// A sequence's sums of chunks: PER side by side to a lane, in every wavefront alike
struct Chunks {
    static constexpr int PER = kMostChunks / 64;
    double v[PER], before = 0.0;

    __device__ __forceinline__ Chunks(const VerifyArgs &g, int b)
    {
        const int c = PER * (threadIdx.x & 63);
#pragma unroll
        for (int i = 0; i < PER; ++i) v[i] = c + i < g.chunks ? g.sums[(int64_t)b * g.chunks + c + i] : 0.0;
    }
    // their sum; and the first chunk that brings it above share * sum (the last that has anything, if rounding leaves none; -1: none has), `before` what is ahead of it
    __device__ __forceinline__ int find(double share, double *total)
    {
        const int lane = threadIdx.x & 63;
        double mine = 0.0;
#pragma unroll
        for (int i = 0; i < PER; ++i) mine += v[i];
        double upto = mine;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const double other = __shfl_up(upto, d, 64);
            if (lane >= d) upto += other;
        }
        *total = __shfl(upto, 63, 64);
        const double goal = share * *total;
        int above = -1, last = -1;
        double run = upto - mine, at_above = 0.0, at_last = 0.0;
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            if (above < 0 && v[i] > 0.0 && run + v[i] > goal) {
                above = i;
                at_above = run;
            }
            if (v[i] > 0.0) {
                last = i;
                at_last = run;
            }
            run += v[i];
        }
        const uint64_t some = __ballot(above >= 0), any = __ballot(last >= 0);
        if (!any) return -1;
        const int l = some ? __builtin_ctzll(some) : 63 - __builtin_clzll(any);
        before = __shfl(some ? at_above : at_last, l, 64);
        return PER * l + __shfl(some ? above : last, l, 64);
    }
};

template <typename T, bool DRAFT, bool FIRST, bool LAST>
__global__ __launch_bounds__(LAST ? kVerifyThreads : 64) void verify_walk_kernel(const VerifyArgs g)
{
    constexpr int THREADS = LAST ? kVerifyThreads : 64;
    __shared__ double scratch[kVerifyWaves];
    __shared__ Sum over[kMostTried];
    __shared__ int64_t gone[kMostTried];
    const int b = blockIdx.x, tid = threadIdx.x;
    const int32_t first = first_of(g, b), count = count_of(g, b);
    VerifyState *state = g.state + b;
    int32_t *path = g.path + b * g.p_sb;
    Walk s{0, count ? 1 : 0, 0, 1};
    double m = 1.0;
    if constexpr (FIRST) {
        if (tid == 0 && count) path[0] = 0;
    } else {
        if (state->done) {
            if (tid == 0) state->summed = 1;
            return;
        }
        s = state->walk;
        if (DRAFT && tid < s.tried) over[tid] = state->over[tid];
        Chunks(g, b).find(0.0, &m);
        __syncthreads();
    }
    const bool done = !count || walk_tree<T, DRAFT, LAST, THREADS>(g, first, count, path, s, m, true, over, gone, scratch);
    __syncthreads();
    if (tid < s.tried) {
        if constexpr (DRAFT) state->over[tid] = over[tid];
        else state->gone[tid] = gone[tid];
    }
    if (tid == 0) {
        state->walk = s;
        state->done = done;
        state->summed = 0;
    }
    if (done) tell(g, b, count, s, THREADS);
}

template <typename T, bool DRAFT>
__global__ __launch_bounds__(256) void verify_sums_kernel(const VerifyArgs g)
{
    __shared__ double scratch[4];
    const int b = blockIdx.x / g.chunks, c = blockIdx.x - b * g.chunks;
    const VerifyState *state = g.state + b;
    const int32_t count = count_of(g, b);
    if (state->summed || !count) return;
    const int64_t row = first_of(g, b) + state->walk.node;
    const Left<T, DRAFT> left{(const T *)g.target + row * g.t_st, DRAFT ? (const T *)g.draft + row * g.d_st : nullptr, state->over, state->gone, state->walk.tried};
    const int32_t lo = c * g.chunk, hi = g.V - lo < g.chunk ? g.V : lo + g.chunk;
    const double sum = group_sum<256>(left.sum(lo, hi, threadIdx.x, 256), scratch);
    if (threadIdx.x == 0) g.sums[(int64_t)b * g.chunks + c] = sum;
}

template <typename T, bool DRAFT>
__global__ __launch_bounds__(kVerifyThreads) void verify_pick_kernel(const VerifyArgs g)
{
    __shared__ double scratch[kVerifyWaves];
    __shared__ int32_t found[2];
    const int b = blockIdx.x, tid = threadIdx.x;
    const VerifyState *state = g.state + b;
    int64_t next = -1;
    if (count_of(g, b)) {
        Chunks sums(g, b);
        const float r = g.last_uniform[b];
        double total;
        const int found_at = sums.find(r > 0.f ? (double)r : 0.0, &total), chosen = found_at < 0 ? 0 : found_at;
        const int64_t row = first_of(g, b) + state->walk.node;
        const Left<T, DRAFT> left{(const T *)g.target + row * g.t_st, DRAFT ? (const T *)g.draft + row * g.d_st : nullptr, state->over, state->gone, state->walk.tried};
        const int32_t lo = chosen * g.chunk, hi = g.V - lo < g.chunk ? g.V : lo + g.chunk;
        next = next_token(g, b, left, lo, hi, sums.before, total, scratch, found);
    }
    if (tid == 0) g.next[b] = next;
}

template <typename T, bool DRAFT>
static nt_status launch_verify_kind(VerifyArgs &a, int64_t sequences, hipStream_t s)
{
    const dim3 each((unsigned)sequences);
    constexpr int N = 16 / sizeof(T);
    // Chunks for some 2048 workgroups in all, of whole rounds of loads
    const int64_t least = 256 * N, wanted = std::max<int64_t>(1, std::min<int64_t>(kMostChunks, 2048 / sequences));
    const int64_t chunk = std::max(least, ((a.V + wanted - 1) / wanted + least - 1) / least * least), chunks = (a.V + chunk - 1) / chunk;
    // A unit reads some 40 GB/s: of rows of 64 KB (both) and less one has enough (1 sequence, 8000 words 10.3 us, 10.8 in three launches; 32000 15.1, 11.4; 128000 30.9, 11.3).  Rounds
    // before the last, whose sums are a unit's own work, are 3 us each where no walk needs one: only for long rows of trees that are likely to (us, means of ten sets of random numbers, 64 trees of 24, 128000 words: none 137,
    // four 80, 131 at most, six 78, 89 at most; 64000 88, 67 with four; 32000 49, 51; chains of 6, 128000: 13.8, 18.0 with one).
    const int64_t row_bytes = (int64_t)a.V * (int64_t)sizeof(T) * (DRAFT ? 2 : 1);
    const int rounds = DRAFT && row_bytes > (256 << 10) ? (int)std::min<int64_t>(4, std::max<int64_t>(0, (a.T / sequences - 3) / 5)) : 0;
    WorkspaceLease lease;
    char *ws = nullptr;
    if (row_bytes > (64 << 10) && sequences * chunks <= kMaxWorkgroups) ws = (char *)lease.acquire((size_t)sequences * (sizeof(VerifyState) + (size_t)chunks * 8), s);
    if (!ws) {
        hipLaunchKernelGGL((verify_tree_kernel<T, DRAFT>), each, dim3(kVerifyThreads), 0, s, a);
        return check_launch("verify_tree_kernel");
    }
    a.state = (VerifyState *)ws;
    a.sums = (double *)(ws + (size_t)sequences * sizeof(VerifyState));
    a.chunk = (int32_t)chunk;
    a.chunks = (int32_t)chunks;
    const dim3 all((unsigned)(sequences * chunks));
    if (rounds) {
        hipLaunchKernelGGL((verify_walk_kernel<T, DRAFT, true, false>), each, dim3(64), 0, s, a);
        for (int i = 1; i <= rounds; ++i) {
            hipLaunchKernelGGL((verify_sums_kernel<T, DRAFT>), all, dim3(256), 0, s, a);
            if (i < rounds) hipLaunchKernelGGL((verify_walk_kernel<T, DRAFT, false, false>), each, dim3(64), 0, s, a);
            else hipLaunchKernelGGL((verify_walk_kernel<T, DRAFT, false, true>), each, dim3(kVerifyThreads), 0, s, a);
        }
    } else {
        hipLaunchKernelGGL((verify_walk_kernel<T, DRAFT, true, true>), each, dim3(kVerifyThreads), 0, s, a);
    }
    hipLaunchKernelGGL((verify_sums_kernel<T, DRAFT>), all, dim3(256), 0, s, a);
    hipLaunchKernelGGL((verify_pick_kernel<T, DRAFT>), each, dim3(kVerifyThreads), 0, s, a);
    return check_launch("verify_walk_kernel");
}

template <typename T>
static nt_status launch_verify_type(VerifyArgs &a, int64_t sequences, hipStream_t s)
{
    return a.draft ? launch_verify_kind<T, true>(a, sequences, s) : launch_verify_kind<T, false>(a, sequences, s);
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
    VerifyArgs a{target, draft, ids, parents, starts, lengths, uniform, last_uniform, path, accepted, new_lengths, next,
                 dt->stride[0], dd ? dd->stride[0] : 0, dp->stride[0], (int32_t)dt->size[0], (int32_t)dt->size[1], (int32_t)dp->size[1], nullptr, nullptr, 0, 0};
    hipStream_t s = (hipStream_t)stream;
    if (dtype == NT_F32) return launch_verify_type<float>(a, sequences, s);
    if (dtype == NT_F16) return launch_verify_type<_Float16>(a, sequences, s);
    return launch_verify_type<__bf16>(a, sequences, s);
}

}  // namespace nt
