// Attention for trees of drafted tokens over a paged cache: who walks which keys, and the launches for one built head size.
//
// Tiles of 128 or 64 rows (token, query head of the group) of one sequence and key head, walked as in paged_many.h; with 64 rows two wavefronts share them and two groups of
// wavefronts the keys of a block, so that all four SIMDs multiply.  Fewer rows go the same way: paged_few.h with masks took 76 us, 67 so, for 32 sequences of 17 to 4096 keys, 16 rows
// of 128 bf16 a key head, 118 and 72 with 32 rows (its shares are of one length, and write and join more); 15.3 against 17.4 for one sequence of 900, 48 heads x 64.
//
// Measured, join included, f16 or bf16 unless codes are named: 32 sequences of 17 to 4096 keys x 32/8 heads x 128, 16 tokens each 90 us = 3.6 TB/s of keys and values (equally long ones 4.4 to 4.9: where a
// run passes into another sequence it begins anew); 2 of 100000 to 131072 int8 keys, 64 tokens each 460, of 16 up to 3000 e4m3 keys x 20/5 heads x 80, 26 tokens 34.5;
// one of 900 x 48 heads x 64, 8 tokens 17.4 to 18.3 (14.4 and the join's 4.0, both chains of loads).
//
// Sequences of a serving batch are of every age, and a program to each is done when the oldest is.  So the blocks of keys of all sequences and heads, one behind the other, are
// dealt out to as many programs as the units hold, each the same number.  Where a program's run ends inside a sequence's head it leaves its share (reference m, sum l and
// unnormalised outputs o) in the workspace: one at the beginning of its run at most, and one at its end.  A second launch joins them, in the order of the keys:
// O = sum 2^(m_i - M) o_i / sum 2^(m_i - M) l_i.
#pragma once
#include "paged_many.h"

namespace nt {

// A sequence's beginning costs a program as much as so many blocks (its rows, its first pages and keys one after the other), and is dealt out along with them:
// us, graph replays, 32 x 17 to 4096 keys x 32/8 heads x 128 bf16, 16 tokens each: 99.5 with 0, 94.3 with 2, 90.5 with 4, 91 with 6 and 8; 128 x 500 to 1000 97.6 / 88.5 / 89 / 88.
constexpr int kTreeBegin = 4;

// Blocks to a program, beginnings among them but for the first sequence's (every program has one at its own start).  Short runs go to half of the programs, one to a unit, where
// the sequences are few: less shares to join (4 x 2048 to 4096 keys 34.4 us with all, 28.8; 1 x 4096 50.9, 33.1; but 16 x 1 to 3000 keys 37.0, 40.3).
__device__ __forceinline__ int64_t tree_run(const PagedArgs &g, int64_t all)
{
    const int64_t shared = all - kTreeBegin, run = (shared + g.groups - 1) / g.groups, half = g.groups / 2;
    return run < 12 && half > 4 * g.B ? (shared + half - 1) / half : run;
}

// The same in all lanes: in scalar registers
__device__ __forceinline__ int32_t uniform(int32_t v) { return __builtin_amdgcn_readfirstlane(v); }
__device__ __forceinline__ int64_t uniform(int64_t v) { return (int64_t)((uint64_t)(uint32_t)uniform((int32_t)v) | (uint64_t)(uint32_t)uniform((int32_t)(v >> 32)) << 32); }

template <bool BF16, int KIND, int SIZE, bool FAST, bool FULL, int GROUPS>
__global__ __launch_bounds__(64 * kManyWaves, many_resident(KIND, SIZE)) void paged_tree_kernel(const PagedArgs g)
{
    constexpr int ROWS = kManyRows / GROUPS, KB = many_keys(SIZE), PER = kTreeSequences / 64;
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    const int32_t capacity = g.width * (int32_t)g.page.d;

    // A sequence's heads and row parts on one XCD (workgroups go to the XCDs in turn), near each other in time: what they read lies side by side, or is the same
    const uint32_t x = blockIdx.x & 7, per_xcd = gridDim.x >> 3, more = gridDim.x & 7;
    const uint32_t program = x * per_xcd + (x < more ? x : more) + (blockIdx.x >> 3);
    const uint32_t inner = (uint32_t)g.Hkv * g.parts, which = program % inner, part = which % g.parts, group = program / inner;
    const int32_t h = which / g.parts;

    // ---- the blocks of each sequence, and before a lane's first: up to PER of them side by side to a lane.  Every wavefront finds and writes the same, and reads what it wrote
    __shared__ int32_t blocks[PER][64];
    __shared__ int64_t before[64];
    const int lane = threadIdx.x & 63, per = (g.B + 63) / 64;
    int64_t start = 0, end = 1, run = 1;
    if (g.groups) {
        Sequence seq[PER];
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            if (i < per) seq[i] = sequence_of(g, per * lane + i < g.B ? per * lane + i : g.B - 1);
        }
        int64_t upto = 0;
#pragma unroll
        for (int i = 0; i < PER; ++i)
            if (i < per) {
                const int32_t n = per * lane + i < g.B ? tree_blocks(seq[i], g.window, KB, capacity) : 0;
                blocks[i][lane] = n ? n + kTreeBegin : 0;
                upto += n ? n + kTreeBegin : 0;
            }
        int64_t sum = -upto;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int64_t other = __shfl_up(upto, d, 64);
            if (lane >= d) upto += other;
        }
        sum += upto;
        before[lane] = sum;
        const int64_t all = uniform(__shfl(upto, 63, 64));
        run = tree_run(g, all);
        start = kTreeBegin + group * run;
        end = start + run < all ? start + run : all;
        if (blockIdx.x == 0 && threadIdx.x < 64) {                         // (for the join)
            for (int i = 0; i < per; ++i) {
                if (per * lane + i < g.B) g.before[per * lane + i] = sum;
                sum += blocks[i][lane];
            }
            if (lane == 0) g.before[g.B] = all;
        }
    }

    for (int64_t at = start; at < end;) {
        int32_t b = group;
        int64_t ahead = 0;                                                 // blocks before sequence b
        if (g.groups) {
            // the last sequence that begins at or before the block, of those that have any: in the last lane that begins there with any
            int64_t sum = before[lane], mine = 0;
            int32_t which = -1;
            for (int i = 0; i < per; ++i) {
                const int32_t n = blocks[i][lane];
                if (n && sum <= at) {
                    which = per * lane + i;
                    mine = sum;
                }
                sum += n;
            }
            const int l = 63 - __builtin_clzll(__ballot(which >= 0));
            b = uniform(__shfl(which, l, 64));
            ahead = uniform(__shfl(mine, l, 64));
        }
        const Sequence in_memory = sequence_of(g, b), seq{uniform(in_memory.first), uniform(in_memory.count), uniform(in_memory.length)};
        const KeyRange keys = tree_range(seq, g.window, capacity);
        const int32_t n = tree_blocks(seq, g.window, KB, capacity);
        const int64_t inside = g.groups ? at - ahead : kTreeBegin;
        if (!g.groups) end = n;
        const int32_t from = inside > kTreeBegin ? (int32_t)(inside - kTreeBegin) : 0;
        const int64_t until = end - at + inside - kTreeBegin;
        const int32_t to = until < n ? (int32_t)until : n;
        at += n + kTreeBegin - inside;
        const int64_t slot = (2 * (int64_t)program + (inside <= kTreeBegin && ahead + kTreeBegin != start)) * ROWS, rows = (int64_t)seq.count * g.G;
        // Rows beyond the caller's bound on new tokens: not shared, tiles of all keys, dealt out to the programs that have blocks of this sequence
        int64_t sharers = 1, mine = 0;
        if (g.groups && rows > (int64_t)g.parts * ROWS) {
            sharers = (ahead + n - 1) / run - ahead / run + 1;
            mine = (int64_t)group - ahead / run;
        }
        int64_t tile = 0;
        for (int64_t r0 = (int64_t)part * ROWS; r0 < rows; r0 += (int64_t)g.parts * ROWS, ++tile) {
            if (tile ? tile % sharers != mine : to <= from) continue;      // (workgroup-uniform)
            const bool share = tile == 0 && (from > 0 || to < n);
            paged_many_tile<BF16, KIND, SIZE, FAST, FULL, true, GROUPS>(g, smem, b, h, seq, (int)r0, 0, tile ? keys : tree_part(keys, KB, n, from, to),
                                                                        share ? g.part_ml + slot * 2 : nullptr, share ? g.part_o + slot * g.D : nullptr);
            __syncthreads();
        }
    }
}

// 16 rows of a sequence, key head and row part to a workgroup, LANES lanes to a row with 4 elements each
template <bool BF16, int LANES, int ROWS>
__global__ __launch_bounds__(256) void paged_tree_join_kernel(const PagedArgs g)
{
    constexpr int AT_ONCE = 8;
    const uint32_t inner = (uint32_t)g.Hkv * g.parts, which = blockIdx.x % inner, part = which % g.parts, h = which / g.parts, b = blockIdx.x / inner;
    const Sequence seq = sequence_of(g, b);
    const int64_t rows = (int64_t)seq.count * g.G, r0 = (int64_t)part * ROWS;
    if (r0 + 16 * blockIdx.y >= rows) return;
    const int64_t first = g.before[b], run = tree_run(g, g.before[g.B]), g0 = first / run, g1 = (g.before[b + 1] - 1 - kTreeBegin) / run;
    if (g0 == g1) return;                                                  // (one program has had it all)
    const int d = 4 * (threadIdx.x % LANES);
    if (d >= g.D) return;
    for (int row = 16 * blockIdx.y + threadIdx.x / LANES; row < 16 * ((int)blockIdx.y + 1) && r0 + row < rows; row += 256 / LANES) {
        // share number j: its row among all that the workspace holds
        auto at = [&](int64_t j) { return (2 * (j * inner + which) + (j == g0 && first != g0 * run)) * ROWS + row; };
        float m = -INFINITY, l = 0.f;
        float4v o{0.f, 0.f, 0.f, 0.f};
        for (int64_t j0 = g0; j0 <= g1; j0 += AT_ONCE) {
            float2v f[AT_ONCE];
            float4v v[AT_ONCE];
#pragma unroll
            for (int i = 0; i < AT_ONCE; ++i) {
                if (j0 + i > g1) continue;                                 // (workgroup-uniform)
                const int64_t r = at(j0 + i);
                __builtin_memcpy(&f[i], g.part_ml + 2 * r, 8);
                __builtin_memcpy(&v[i], g.part_o + r * g.D + d, 16);
            }
            float top = m;
#pragma unroll
            for (int i = 0; i < AT_ONCE; ++i) {
                if (j0 + i > g1) f[i] = float2v{-INFINITY, 0.f};
                top = fmaxf(top, f[i][0]);
            }
            const float ref = top == -INFINITY ? 0.f : top, old = __builtin_amdgcn_exp2f(m - ref);
            m = top;
            l *= old;
            o = o * old;
#pragma unroll
            for (int i = 0; i < AT_ONCE; ++i) {
                if (j0 + i > g1) continue;
                const float w = __builtin_amdgcn_exp2f(f[i][0] - ref);
                l = __builtin_fmaf(f[i][1], w, l);
#pragma unroll
                for (int e = 0; e < 4; ++e) o[e] = __builtin_fmaf(v[i][e], w, o[e]);
            }
        }
        const uint32_t i = divide((uint32_t)(r0 + row), g.group), head = h * g.G + ((uint32_t)(r0 + row) - i * g.group.d);
        const int64_t token = seq.first + (int32_t)i;
        const float inv = l == 0.f ? 0.f : 1.0f / l;
        const u32x2 out{pack_two<BF16>(o[0] * inv, o[1] * inv), pack_two<BF16>(o[2] * inv, o[3] * inv)};
        __builtin_memcpy(g.O + token * g.o_st + (int64_t)head * g.o_sh + d, &out, 8);
    }
}

template <int SIZE, bool BF16, int KIND, int GROUPS>
static nt_status launch_paged_tree_rows(const PagedArgs &a, int64_t programs, hipStream_t s)
{
    static DeviceOnce c[3];
    constexpr int ROWS = kManyRows / GROUPS;
    const bool together = a.near && a.aligned && a.page.d % many_together(KIND, SIZE) == 0 && a.D % many_piece(KIND) == 0;
    auto launch = [&](auto kernel, DeviceOnce &configured) -> nt_status {
        if (many_lds(SIZE) > 65536 && !configured.done()) {
            const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)many_lds(SIZE));
            if (e != hipSuccess) return fail(NT_ERR_DEVICE, std::string("hipFuncSetAttribute: ") + hipGetErrorString(e));
            configured.set();
        }
        hipLaunchKernelGGL(kernel, dim3((unsigned)programs), dim3(256), many_lds(SIZE), s, a);
        return check_launch("paged_tree_kernel");
    };
    nt_status st;
    if (together && a.D == SIZE) st = launch(paged_tree_kernel<BF16, KIND, SIZE, true, true, GROUPS>, c[0]);
    else if (together) st = launch(paged_tree_kernel<BF16, KIND, SIZE, true, false, GROUPS>, c[1]);
    else st = launch(paged_tree_kernel<BF16, KIND, SIZE, false, false, GROUPS>, c[2]);
    if (st != NT_OK || a.groups == 0) return st;
    hipLaunchKernelGGL((paged_tree_join_kernel<BF16, SIZE / 4, ROWS>), dim3((unsigned)((int64_t)a.B * a.Hkv * a.parts), ROWS / 16), dim3(256), 0, s, a);
    return check_launch("paged_tree_join_kernel");
}

template <int SIZE, bool BF16, int KIND>
static nt_status launch_paged_tree_kind(const PagedArgs &a, int rows, int64_t programs, hipStream_t s)
{
    if constexpr (SIZE < 256)
        if (rows == kManyRows / 2) return launch_paged_tree_rows<SIZE, BF16, KIND, 2>(a, programs, s);
    return launch_paged_tree_rows<SIZE, BF16, KIND, 1>(a, programs, s);
}

// rows: to a tile, kManyRows or half of them
template <int SIZE>
static nt_status launch_paged_tree_size(const PagedArgs &a, int rows, int64_t programs, bool bf16, int kind, void *stream)
{
    hipStream_t s = (hipStream_t)stream;
    if (kind == CACHE_E4M3) return bf16 ? launch_paged_tree_kind<SIZE, true, CACHE_E4M3>(a, rows, programs, s) : launch_paged_tree_kind<SIZE, false, CACHE_E4M3>(a, rows, programs, s);
    if (kind == CACHE_I8) return bf16 ? launch_paged_tree_kind<SIZE, true, CACHE_I8>(a, rows, programs, s) : launch_paged_tree_kind<SIZE, false, CACHE_I8>(a, rows, programs, s);
    return bf16 ? launch_paged_tree_kind<SIZE, true, CACHE_SAME>(a, rows, programs, s) : launch_paged_tree_kind<SIZE, false, CACHE_SAME>(a, rows, programs, s);
}

}  // namespace nt
