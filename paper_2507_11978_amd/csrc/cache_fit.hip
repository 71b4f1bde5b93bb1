// Pages, slots and positions of a step's new tokens, from the sequences' lengths.
//
// With n = lengths[b] + counts[b] sequence b wants ceil(n / page_size) pages, as many as a table row has entries at most, and has held[b].  What it has beyond that goes back
// onto the stack of free pages, what it lacks comes from the stack's top: surplus page number a of all (counted by sequence, then entry) lands at top - 1 - a, and missing
// page number k is taken from top - 1 - k, where top counts the returned pages in.  Sums of counts, surplus and missing pages before a sequence are three scans.
//
// One workgroup does it, a sequence to a thread, 1024 at a time; the pages that move are dealt out to all threads (a bisection tells whose each is), so that a long prompt's
// pages are not one thread's.  Then a thread to a token.
//
// Bound by its chain, not by bytes: lengths, scan, stack or table, starts, page, slot, one waiting for the other.  256 sequences that get a token each 5.9 us; 96 of them, a third
// new prompts and a third that end, 51000 tokens 6.2 us and 3.6 of the second launch (16.2 called).  Three scans one after the other instead of one took 2.6 us more.
#include "gemm_fast.h"
#include "kernels.h"
#include "paged_index.h"

namespace nt {

constexpr int kFitThreads = 1024, kFitHere = 4096;                        // (tokens that the first launch gives their slots itself)

struct FitArgs {
    const int32_t *lengths, *counts;
    int32_t *table, *held, *free_pages, *free_count, *starts, *new_lengths, *positions;
    int64_t *slots;
    int64_t t_sb, tokens, capacity;
    int32_t B, width;
    Divider page;
};

struct Need {
    int32_t count, after, want, held;
};

__device__ __forceinline__ Need need_of(const FitArgs &g, int32_t b)
{
    if (b >= g.B) return Need{0, 0, 0, 0};
    const int32_t n = g.lengths[b] > 0 ? g.lengths[b] : 0, m = g.counts[b] > 0 ? g.counts[b] : 0;
    const int32_t after = m < 0x7fffffff - n ? n + m : 0x7fffffff;
    const int32_t pages = after ? (int32_t)divide(after - 1, g.page) + 1 : 0;
    return Need{after - n, after, pages < g.width ? pages : g.width, clamp_i32(g.held[b], 0, g.width)};
}

// Of three numbers of each thread: the sums of the threads before this one
struct Sums {
    int64_t surplus, missing, count;
};
__device__ __forceinline__ Sums operator+(const Sums &a, const Sums &b) { return Sums{a.surplus + b.surplus, a.missing + b.missing, a.count + b.count}; }
__device__ __forceinline__ Sums operator-(const Sums &a, const Sums &b) { return Sums{a.surplus - b.surplus, a.missing - b.missing, a.count - b.count}; }

__device__ __forceinline__ Sums shuffled(const Sums &v, int lane) { return Sums{__shfl(v.surplus, lane, 64), __shfl(v.missing, lane, 64), __shfl(v.count, lane, 64)}; }

__device__ __forceinline__ Sums sums_before(const Sums &v, Sums *scratch, Sums *all)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    Sums upto = v;
    const auto scan = [lane](Sums x, int lanes) {
#pragma unroll
        for (int d = 1; d < lanes; d <<= 1) {
            const Sums other = shuffled(x, lane - d);
            if (lane >= d) x = x + other;
        }
        return x;
    };
    upto = scan(upto, 64);
    __syncthreads();                                                       // (what was there has been read)
    if (lane == 63) scratch[wave] = upto;
    __syncthreads();
    constexpr int WAVES = kFitThreads / 64;
    const Sums waves = scan(lane < WAVES ? scratch[lane] : Sums{0, 0, 0}, WAVES);
    *all = shuffled(waves, WAVES - 1);
    const Sums before = shuffled(waves, wave - 1);
    return (wave ? before + upto : upto) - v;
}

// The last of 1024 ascending numbers, the first of them 0, that is not above j (0 <= j)
__device__ __forceinline__ int whose(const int64_t *first, int64_t j)
{
    int at = 0;
#pragma unroll
    for (int step = kFitThreads / 2; step; step >>= 1)
        if (first[at + step] <= j) at += step;
    return at;
}

// Token t's slot and position.  `starts`: of all sequences (LDS or global memory); n: tokens there are; length_of(b), pages_of(b): what sequence b has with them
template <typename Length, typename Pages>
__device__ __forceinline__ void place_token(const FitArgs &g, int64_t t, const int32_t *starts, int32_t n, Length length_of, Pages pages_of)
{
    int64_t slot = -1;
    int32_t pos = 0;
    if (t < n) {
        int32_t b = 0;                                                     // the last sequence that begins at or before the token
        for (int32_t up = g.B; up - b > 1;) {
            const int32_t at = b + (up - b) / 2;
            if (starts[at] <= t) b = at;
            else up = at;
        }
        pos = length_of(b) - (b + 1 < g.B ? starts[b + 1] : n) + (int32_t)t;
        const uint32_t entry = divide(pos, g.page);
        const int32_t id = entry < (uint32_t)pages_of(b) ? g.table[b * g.t_sb + entry] : -1;
        if (id >= 0) slot = (int64_t)id * g.page.d + (pos - entry * g.page.d);
    }
    g.slots[t] = slot;
    g.positions[t] = pos;
}

__global__ __launch_bounds__(kFitThreads) void cache_fit_kernel(const FitArgs g)
{
    __shared__ Sums scratch[kFitThreads / 64];
    __shared__ int64_t first[kFitThreads];
    __shared__ int32_t from[kFitThreads], starts[kFitThreads], after[kFitThreads], pages[kFitThreads];
    const int tid = threadIdx.x;
    const bool one = g.B <= kFitThreads;                                   // ... chunk of sequences
    const int32_t stack = *g.free_count;
    const auto lacks_of = [](const Need &n) { return Sums{n.held > n.want ? n.held - n.want : 0, n.want > n.held ? n.want - n.held : 0, n.count}; };
    Need n = need_of(g, tid);
    Sums all, before = sums_before(lacks_of(n), scratch, &all);
    int64_t back = all.surplus;
    for (int32_t c = kFitThreads; c < g.B; c += kFitThreads) {
        Sums more;
        sums_before(lacks_of(need_of(g, c + tid)), scratch, &more);
        back += more.surplus;
    }
    const int64_t top = (int64_t)clamp_i32(stack, 0, (int32_t)g.capacity) + back;

    // ---- pages that go back
    if (back) {
        int64_t done = 0;
        for (int32_t c = 0; c < g.B; c += kFitThreads) {
            if (!one) {
                n = need_of(g, c + tid);
                before = sums_before(lacks_of(n), scratch, &all);
            }
            first[tid] = before.surplus;
            from[tid] = n.want;
            __syncthreads();
            for (int64_t j = tid; j < all.surplus; j += kFitThreads) {
                const int s = whose(first, j);
                const int64_t at = top - 1 - (done + j);
                if (at < g.capacity) g.free_pages[at] = g.table[(c + s) * g.t_sb + from[s] + (j - first[s])];
            }
            done += all.surplus;
            __syncthreads();
        }
    }

    // ---- pages that are taken, and what the sequences have then
    int64_t tokens = 0, taken = 0;
    for (int32_t c = 0; c < g.B; c += kFitThreads) {
        if (!one) {
            n = need_of(g, c + tid);
            before = sums_before(lacks_of(n), scratch, &all);
        }
        const int64_t left = top - taken - before.missing, lacks = n.want > n.held ? n.want - n.held : 0, start = tokens + before.count;     // left: pages there are for this sequence
        const int32_t held = (n.held < n.want ? n.held : n.want) + (int32_t)(left <= 0 ? 0 : left < lacks ? left : lacks);
        starts[tid] = (int32_t)(start < 0x7fffffff ? start : 0x7fffffff);
        after[tid] = n.after;
        pages[tid] = held;
        if (all.missing) {
            first[tid] = before.missing;
            from[tid] = n.held;
            __syncthreads();
            for (int64_t j = tid; j < all.missing; j += kFitThreads) {
                const int s = whose(first, j);
                const int64_t at = top - 1 - (taken + j);
                g.table[(c + s) * g.t_sb + from[s] + (j - first[s])] = at >= 0 && at < g.capacity ? g.free_pages[at] : -1;
            }
        }
        if (c + tid < g.B) {
            g.held[c + tid] = held;
            g.new_lengths[c + tid] = n.after;
            g.starts[c + tid] = starts[tid];
        }
        taken += all.missing;
        tokens += all.count;
        __syncthreads();
    }
    const int32_t count = (int32_t)(tokens < 0x7fffffff ? tokens : 0x7fffffff);
    if (tid == 0) {
        const int64_t left = top - taken;
        *g.free_count = (int32_t)(left > g.capacity ? g.capacity : left < -0x7fffffff ? -0x7fffffff : left);
        g.starts[g.B] = count;
    }
    if (g.tokens > kFitHere || !one) return;
    for (int64_t t = tid; t < g.tokens; t += kFitThreads)
        place_token(g, t, starts, count, [&](int32_t b) { return after[b]; }, [&](int32_t b) { return pages[b]; });
}

// (starts of up to kStartsHere sequences in LDS: a bisection in memory is a chain of as many loads as it has steps)
constexpr int kStartsHere = 4096;
template <bool NEAR>
__global__ __launch_bounds__(256) void cache_slots_kernel(const FitArgs g)
{
    __shared__ int32_t near[NEAR ? kStartsHere : 1];
    if constexpr (NEAR) {
        for (int i = threadIdx.x; i < g.B; i += 256) near[i] = g.starts[i];
        __syncthreads();
    }
    const int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (t < g.tokens) place_token(g, t, NEAR ? near : g.starts, g.starts[g.B], [&](int32_t b) { return g.new_lengths[b]; }, [&](int32_t b) { return g.held[b]; });
}

nt_status launch_cache_fit(const int32_t *lengths, const int32_t *counts, int64_t sequences, int64_t page_size, int32_t *table, const nt_tensor_desc *dt, int32_t *held,
                           int32_t *free_pages, int64_t capacity, int32_t *free_count, int32_t *starts, int32_t *new_lengths, int64_t *slots, int32_t *positions,
                           int64_t tokens, void *stream)
{
    if (!dt) return fail(NT_ERR_INVALID_ARG, "null tensor descriptor");
    if (dt->ndim != 2) return fail(NT_ERR_SHAPE_MISMATCH, "the page table must be 2-D [sequences, entries]");
    if (sequences < 0 || capacity < 0 || tokens < 0 || dt->size[0] < 0 || dt->size[1] < 0) return fail(NT_ERR_INVALID_ARG, "negative size");
    if (dt->size[0] != sequences) return fail(NT_ERR_SHAPE_MISMATCH, "lengths and page table differ in sequences");
    if (dt->size[1] > 1 && dt->stride[1] != 1) return fail(NT_ERR_UNSUPPORTED, "the page table needs unit stride along a sequence");
    if (page_size < 1 || page_size > (1 << 24)) return fail(NT_ERR_UNSUPPORTED, "page_size must be 1 to 2^24");
    if (sequences > (1 << 24) || dt->size[1] > 0x7fffffffLL) return fail(NT_ERR_UNSUPPORTED, "page table too large");
    if (capacity > 0x7fffffffLL) return fail(NT_ERR_UNSUPPORTED, "more than 2^31 - 1 pages");
    if (tokens > 0x7fffffffLL) return fail(NT_ERR_UNSUPPORTED, "more than 2^31 - 1 tokens");
    if (!starts || !free_count || (sequences && (!lengths || !counts || !held || !new_lengths)) || (sequences && dt->size[1] && !table) || (capacity && !free_pages) ||
        (tokens && (!slots || !positions)))
        return fail(NT_ERR_INVALID_ARG, "null device pointer");
    const FitArgs a{lengths, counts, table, held, free_pages, free_count, starts, new_lengths, positions, slots, dt->stride[0], tokens, capacity,
                    (int32_t)sequences, (int32_t)dt->size[1], divider_of((uint32_t)page_size)};
    hipStream_t s = (hipStream_t)stream;
    hipLaunchKernelGGL(cache_fit_kernel, dim3(1), dim3(kFitThreads), 0, s, a);
    const nt_status st = check_launch("cache_fit_kernel");
    if (st != NT_OK || tokens == 0 || (tokens <= kFitHere && sequences <= kFitThreads)) return st;
    const dim3 grid((unsigned)((tokens + 255) / 256));
    if (sequences <= kStartsHere) hipLaunchKernelGGL(cache_slots_kernel<true>, grid, dim3(256), 0, s, a);
    else hipLaunchKernelGGL(cache_slots_kernel<false>, grid, dim3(256), 0, s, a);
    return check_launch("cache_slots_kernel");
}

}  // namespace nt
