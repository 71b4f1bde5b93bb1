// Attention over a paged cache for many query rows: chunks of new tokens, whole prompts.
//
// A tile is 128 rows (token, query head of the group) of one sequence and key head, 32 to a wavefront, so that what the group shares is loaded once; the
// program walks the keys that some row sees in blocks of 64 (32 at head size 256).  Arithmetic and layout are those of attention.hip: everything
// transposed, S^T = K Q^T with the query on the lane axis, weights against a reference M that lags behind the running maximum (raised when a
// block holds a score 15 above it), packed weights as they are for O^T += V^T P^T.  Blocks that every row of a wavefront sees are not masked; those that none
// sees are not computed.  With an 8-bit cache the codes are widened on their way to LDS, a key's scale multiplies its scores in fp32 and a value's scale
// its weight, so that nothing is rounded but the weights, as in a 16-bit cache.
//
// Weights are rounded to 16 bits once, and over 16-bit caches their sum is that of the rounded ones.  In two parts, as in paged_few.h, they would cost a second set of
// products where products are the bound (1024 queries x 8000 keys x 32/8 heads x 128 bf16 212 us, 276 with two; 4 x 1024 x 48 heads x 64 f16 64, 98).  fp16 queries
// over codes have no choice, see rest_of (20 us of the 365 that 1024 x 8000 e4m3 take).
//
// FAST (rows at addresses that are multiples of 16 bytes, and pages that hold the 2 to 16 rows that a wavefront moves with one load or a multiple of
// them, so that these lie on one page): the table is read and the addresses are made by one lane for all.  A 16-bit cache then travels straight into
// LDS, one block ahead, codes through registers, 16 at a time.  Other caches: 8 elements to a lane through registers, every lane with an address of its own.
//
// Measured: 2048 queries of 32/8 heads x 128 bf16 over 18500 keys 620 to 650 us = 0.90 to 0.94 PFLOP/s (a large matrix product reaches 1.18), 1024 queries x 8000 211, over
// e4m3 290 to 297, int8 304 to 310 (each lane widens 64 elements of a block and scales 64 scores and weights), fp16 over them 365 and 376.  A block of 64 keys is
// 32 matrix instructions of 32 cycles and 4 of 16 to a wavefront beside 32 exponentials, the multiplications and packs that feed them; the matrix pipe is busy for
// 44 % of the cycles, LDS has no conflicts.  Two wavefronts to a SIMD (128; three at 64) are what the registers allow, and where both weigh their blocks the pipe
// waits.  Tried: the next block's products between this block's exponentials (K two blocks ahead, two sets of scores): 629 us with all 256 registers, but 7.5 %
// slower at head size 64 and half again as long where registers ran out; blocks of 32 keys: 775.  Hidden keys of codes told by their weight in every block, not
// by position in those that have any: 8 % longer.
#pragma once
#include "paged.h"

namespace nt {

constexpr int kManyWaves = 4, kManyRows = 32 * kManyWaves;
constexpr int many_keys(int size) { return size == 256 ? 32 : 64; }
// elements that a lane moves at a time (FAST), and the rows that a wavefront then moves with one load
constexpr int many_piece(int kind) { return kind == CACHE_SAME ? 8 : 16; }
constexpr int many_together(int kind, int size) { return 64 * many_piece(kind) / size; }
constexpr size_t many_block(int size) { return (size_t)many_keys(size) * size * 2; }
// [K0][K1][V0][V1], scales of two blocks (K's, then V's), three flags
constexpr size_t many_lds(int size) { return 4 * many_block(size) + 2 * 2 * many_keys(size) * 4 + 16; }

// Wavefronts per SIMD that the registers are shared out for.  Codes at head size 64 do better with more registers (2 x 1024 queries x 8000 keys x 16 heads f16 over int8
// 396 us with three, 349 when that was measured, 316 since; bf16, half of that, 119, 113), 16-bit caches use 168.
constexpr int many_resident(int kind, int size) { return size == 256 ? 1 : size == 128 || kind != CACHE_SAME ? 2 : 3; }

// FULL: rows of SIZE elements (the switched-off lanes of others cost 5 % where none is: 1024 queries x 8000 keys x 32/8 heads x 128 bf16 217 us, 228)
template <bool BF16, int KIND, int SIZE, bool FAST, bool FULL>
__global__ __launch_bounds__(64 * kManyWaves, many_resident(KIND, SIZE)) void paged_many_kernel(const PagedArgs g)
{
    constexpr bool DMA = FAST && KIND == CACHE_SAME;
    constexpr int EPL = FAST ? many_piece(KIND) : 8;
    constexpr int KB = many_keys(SIZE), JB = KB / 32, CH = SIZE / EPL, PER = KB * CH / 256, RSTEP = 256 / CH;
    constexpr int ES = KIND == CACHE_SAME ? 2 : 1;
    constexpr uint32_t BLK = many_block(SIZE);
    constexpr bool VB = BF16 || KIND != CACHE_SAME;                        // the second product's type is bf16,
    constexpr bool SPLIT = VB && !BF16;                                    // ... where that is not the queries', with weights in two parts: see rest_of
    constexpr int DEEP = 4;                                                // products that a fragment of K or V is read ahead of its own
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    float *const scales = reinterpret_cast<float *>(smem + 4 * BLK);
    int *const flags = reinterpret_cast<int *>(scales + 4 * KB);
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), l32 = lane & 31, hi = lane >> 5;

    // ---- which tile: head fastest (a head's tiles on one XCD, where the heads are a multiple of 8), then share, then tile, the sequences' last first: they
    // see the most keys.
    int w = blockIdx.x;
    const int h = w % g.Hkv;
    w /= g.Hkv;
    const int split = w % g.splits, number = g.tiles - 1 - w / g.splits;
    auto tiles_before = [&](int b) { return first_tile(g.starts, b, g.T, g.G, kManyRows); };
    int b = 0;
    for (int up = g.B; up - b > 1;) {                                      // 64 sequences at a time: the last whose tiles begin at or before this one
        const int step = (up - b + 63) / 64, at = b + lane * step;
        const uint64_t below = __ballot(at < up && tiles_before(at < up ? at : b) <= number);
        const int found = below ? 63 - __builtin_clzll(below) : 0;
        b += found * step;
        up = b + step < up ? b + step : up;
    }
    const Sequence seq = sequence_of(g, b);
    const int64_t r0_64 = (int64_t)(number - tiles_before(b)) * kManyRows;
    const int rows_all = seq.count * g.G;
    if (r0_64 < 0 || r0_64 >= rows_all) return;                            // (workgroup-uniform)
    const int r0 = (int)r0_64, tile_last = r0 + kManyRows < rows_all ? r0 + kManyRows - 1 : rows_all - 1;
    const int32_t *pages = g.table + (int64_t)b * g.t_sb;
    const char *Kh = g.K + (int64_t)h * g.k_sh * ES, *Vh = g.V + (int64_t)h * g.v_sh * ES;
    const int32_t tile_i0 = (int32_t)divide(r0, g.group), tile_i1 = (int32_t)divide(tile_last, g.group);
    const KeyRange keys = keys_of(g, seq, tile_i0, tile_i1, split, KB);
    // keys that every row of the tile sees: [seen_lo, seen_hi)
    const int32_t seen_lo = keys_seen(seq, tile_i1, g.causal, g.window).lo, seen_hi = keys_seen(seq, tile_i0, g.causal, g.window).hi;

    // ---- this lane's row and its keys [row_lo, row_hi); the wavefront's: seen by some row [wave_lo, wave_hi), by all [all_lo, all_hi)
    const int row = r0 + 32 * wave + l32;
    const bool real = row < rows_all;
    const bool busy = r0 + 32 * wave < rows_all;                           // wavefront-uniform
    const uint32_t rc = real ? row : tile_last, mine = divide(rc, g.group), head = h * g.G + (rc - mine * g.group.d);
    const KeyRange row_keys = keys_seen(seq, (int32_t)mine, g.causal, g.window);
    const int32_t row_lo = row_keys.lo, row_hi = row_keys.hi;
    const int32_t all_lo = __builtin_amdgcn_readlane(row_lo, 31), all_hi = __builtin_amdgcn_readlane(row_hi, 0);
    const int32_t wave_lo = __builtin_amdgcn_readlane(row_lo, 0), wave_hi = __builtin_amdgcn_readlane(row_hi, 31);
    const int64_t token = seq.first + (int32_t)mine;

    u32x4 qf[SIZE / 16];
    {
        const uint16_t *q = g.Q + token * g.q_st + (int64_t)head * g.q_sh;
#pragma unroll
        for (int ks = 0; ks < SIZE / 16; ++ks) {
            qf[ks] = u32x4{0, 0, 0, 0};
            if (16 * ks + 8 * hi < g.D) __builtin_memcpy(&qf[ks], q + 16 * ks + 8 * hi, 16);
        }
    }

    // ---- a block on its way: thread tid moves piece tid % CH of rows tid / CH + u * RSTEP, a wavefront RSTEP / 4 rows from row wave * RSTEP / 4 on
    const int ch = tid % CH, row0 = tid / CH;
    typedef typename std::conditional<EPL * ES == 16, u32x4, u32x2>::type Piece;
    Piece kr[DMA ? 1 : PER], vr[DMA ? 1 : PER];
    float sc = 0.f;
    int32_t id[PER], sid = -1;                                             // the table's entries for the block that is fetched next; sid: for the thread's scale
    uint32_t named = 0;                                                    // bit u: a page is named for the thread's row u (of the block that was fetched last)
    // FAST: lane u has what is the same for all of a wavefront's row u: its table entry and its address in K, lane PER + u that in V
    const bool of_v = (lane / PER) & 1;
    const int64_t lane_sp = of_v ? g.v_sp : g.k_sp, lane_ss = of_v ? g.v_ss : g.k_ss;
    const char *const lane_base = of_v ? Vh : Kh;
    auto row_of = [&](int kb, int u) { return (uint32_t)(kb * KB + u * RSTEP + (FAST ? wave * (RSTEP / 4) : row0)); };
    auto find = [&](int kb) {
#pragma unroll
        for (int u = 0; u < (FAST ? 1 : PER); ++u) id[u] = pages[entry_read(divide(row_of(kb, FAST ? lane % PER : u), g.page), g.width)];
        if constexpr (KIND != CACHE_SAME) sid = pages[entry_read(divide((uint32_t)(kb * KB + tid % KB), g.page), g.width)];
    };
    // byte offsets within the wavefront's rows (FAST).  Straight into LDS: a lane's 16 bytes land at lane * 16, so it fetches the piece that belongs there; of
    // rows that lie 8 apart (head size 256) the order of the pieces differs in its last bit.
    const int lane_row = FAST ? lane / CH : 0;
    const uint32_t at_piece = DMA ? (uint32_t)(lane % CH) ^ chunk_order<SIZE>((uint32_t)(wave * (RSTEP / 4) + lane_row)) : (uint32_t)(lane % CH);
    // (codes beyond the head size: the row's last ones, see stash; 16-bit elements beyond it are not fetched)
    const uint32_t piece = DMA || FULL || at_piece < (uint32_t)g.D / EPL ? at_piece : (uint32_t)g.D / EPL - 1;
    const uint32_t kl = FAST ? (uint32_t)(lane_row * (int32_t)g.k_ss * ES) + 16 * piece : 0, vl = FAST ? (uint32_t)(lane_row * (int32_t)g.v_ss * ES) + 16 * piece : 0;
    // whether the lane's piece of the wavefront's row u holds elements (DMA; at head size 256 odd u have the pieces in another order)
    auto holds = [&](int u) { return FULL || 8 * (at_piece ^ (uint32_t)(RSTEP == 8 && (u & 1))) < (uint32_t)g.D; };
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)smem;
    auto fetch = [&](int kb, uint32_t copy) {
        named = 0;
        const char *address[FAST ? 1 : PER][2];
#pragma unroll
        for (int u = 0; u < (FAST ? 1 : PER); ++u) {
            const uint32_t key = row_of(kb, FAST ? lane % PER : u), index = divide(key, g.page), at = key - index * g.page.d;
            const bool ok = names_page(index, id[u], g.width, g.pages);
            const uint32_t page = ok ? id[u] : 0;
            if constexpr (FAST) {
                named = (uint32_t)__ballot(ok) & ((1u << PER) - 1);
                address[0][0] = lane_base + (times(page, lane_sp) + times(at, lane_ss)) * ES;
            } else {
                named |= (ok ? 1u : 0u) << u;
                address[u][0] = Kh + (times(page, g.k_sp) + times(at, g.k_ss)) * ES;
                address[u][1] = Vh + (times(page, g.v_sp) + times(at, g.v_ss)) * ES;
            }
        }
        auto of_lane = [&](int l) {
            const uint64_t p = reinterpret_cast<uint64_t>(address[0][0]);
            return reinterpret_cast<const char *>((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)p, l) | (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(p >> 32), l) << 32);
        };
        if constexpr (DMA) {
            const uint32_t to = lds0 + copy * BLK + (uint32_t)(wave * (RSTEP / 4) * SIZE * 2);
            auto flip = [&](int u) { return RSTEP == 8 && (u & 1) ? (at_piece & 1 ? 0u - 16u : 16u) : 0u; };
            if constexpr (FULL) {
#pragma unroll
                for (int u = 0; u < PER; ++u) {
                    dma16(of_lane(u), kl + flip(u), to + (uint32_t)(u * RSTEP * SIZE * 2));
                    dma16(of_lane(PER + u), vl + flip(u), to + (uint32_t)(u * RSTEP * SIZE * 2) + 2 * BLK);
                }
            } else {
                const char *from[2 * PER];                                 // (in scalar registers before lanes are switched off)
#pragma unroll
                for (int u = 0; u < 2 * PER; ++u) from[u] = of_lane(u);
#pragma unroll
                for (int u = 0; u < PER; ++u)
                    if (holds(u)) {
                        dma16(from[u], kl + flip(u), to + (uint32_t)(u * RSTEP * SIZE * 2));
                        dma16(from[PER + u], vl + flip(u), to + (uint32_t)(u * RSTEP * SIZE * 2) + 2 * BLK);
                    }
            }
        }
#pragma unroll
        for (int u = 0; u < (DMA ? 0 : PER); ++u) {
            if constexpr (FAST) {
                __builtin_memcpy(&kr[u], of_lane(u) + kl, 16);
                __builtin_memcpy(&vr[u], of_lane(PER + u) + vl, 16);
            } else {
                const int d = 8 * ch <= g.D - 8 ? 8 * ch : g.D - 8;        // (no elements there: the row's last ones, see stash)
                __builtin_memcpy(&kr[u], address[u][0] + d * ES, sizeof(Piece));
                __builtin_memcpy(&vr[u], address[u][1] + d * ES, sizeof(Piece));
            }
        }
        if constexpr (KIND != CACHE_SAME) {
            const uint32_t key = kb * KB + tid % KB, index = divide(key, g.page), at = key - index * g.page.d;
            const uint32_t page = names_page(index, sid, g.width, g.pages) ? sid : 0;
            sc = tid < KB ? g.KS[times(page, g.ks_sp) + times(at, g.ks_ss) + (int64_t)h * g.ks_sh] : g.VS[times(page, g.vs_sp) + times(at, g.vs_ss) + (int64_t)h * g.vs_sh];
        }
    };
    // The fetched block is where the other wavefronts read it, in LDS copy `copy`, once they have passed a barrier behind this.  Keys that no page is named for
    // become NaN, their values, and those of keys outside the range, zeros (see paged_few.h)
    auto stash = [&](int kb, uint32_t copy) {
        const bool hidden = kb * KB < seen_lo || kb * KB + KB > seen_hi;   // from some row
        if constexpr (DMA) {
            NT_WAIT_VMCNT(0);
            asm volatile("" ::: "memory");
            if (hidden || kb * KB < keys.lo || kb * KB + KB > keys.hi || named != (1u << PER) - 1) {           // wavefront-uniform
                bool odd = false;
#pragma unroll 1
                for (int u = 0; u < PER; ++u) {
                    const int32_t r = u * RSTEP + wave * (RSTEP / 4) + here(lane) / CH, key = kb * KB + r;
                    const uint32_t at = copy * BLK + (uint32_t)((u * RSTEP + wave * (RSTEP / 4)) * SIZE * 2 + here(lane) * 16);
                    if (!((named >> u) & 1) && holds(u)) lds_write16(smem, at, u32x4{kNanPair, kNanPair, kNanPair, kNanPair});
                    if (!((named >> u) & 1) || key < keys.lo || key >= keys.hi) lds_write16(smem, at + 2 * BLK, u32x4{0, 0, 0, 0});
                    else if (hidden) odd = odd | any_not_finite<BF16>(lds_read16(smem, at + 2 * BLK));
                }
                if (odd) flags[kb % 3] = 1;
            }
        } else {
            bool odd = false;
#pragma unroll
            for (int u = 0; u < PER; ++u) {
                const uint32_t r = u * RSTEP + row0;
                const int32_t key = kb * KB + (int32_t)r;
                const bool page = (named >> u) & 1, good = page && key >= keys.lo && key < keys.hi;
#pragma unroll
                for (int half = 0; half < EPL / 8; ++half) {
                    u32x4 k, v;
                    if constexpr (KIND == CACHE_SAME) {
                        k = kr[u];
                        v = vr[u];
                    } else if constexpr (FAST) {
                        k = widen8<BF16, KIND>(u32x2{kr[u][2 * half], kr[u][2 * half + 1]});
                        v = widen8<VB, KIND>(u32x2{vr[u][2 * half], vr[u][2 * half + 1]});
                    } else {
                        k = widen8<BF16, KIND>(u32x2{kr[u][0], kr[u][1]});
                        v = widen8<VB, KIND>(u32x2{vr[u][0], vr[u][1]});
                    }
                    if (!FULL && EPL * ch >= g.D) k = v = u32x4{0, 0, 0, 0};
                    k = page ? k : u32x4{kNanPair, kNanPair, kNanPair, kNanPair};
                    v = good ? v : u32x4{0, 0, 0, 0};
                    if (hidden) odd = odd | any_not_finite<VB>(v);
                    const uint32_t at = lds_at<SIZE>(r, EPL / 8 * ch + half);
                    lds_write16(smem, copy * BLK + at, k);
                    lds_write16(smem, (2 + copy) * BLK + at, v);
                }
            }
            if constexpr (KIND != CACHE_SAME)
                if (tid < 2 * KB) scales[copy * 2 * KB + tid] = sc;
            if (odd) flags[kb % 3] = 1;
        }
    };

    float16v ot[SIZE / 32];
#pragma unroll
    for (int db = 0; db < SIZE / 32; ++db)
#pragma unroll
        for (int v = 0; v < 16; ++v) ot[db][v] = 0.f;
    float m_ref = -INFINITY, l_run = 0.f;                                  // reference (-inf: none yet) and sum (8-bit caches: of this lane's keys)
    bool pending = true;                                                   // wavefront-uniform: some row has no reference
    const uint32_t one_pair = ((lane >> 4) & 1) == ((lane >> 2) & 1) ? (BF16 ? 0x3f803f80u : 0x3c003c00u) : 0u;
    const u32x4 ones{one_pair, one_pair, one_pair, one_pair};              // (the sum of query lane % 32 in every lane: see attention.hip)
    const int gq = lane >> 4, li = lane & 15;
    const uint32_t v_key = 4 * (gq >> 1) + (li >> 2), v_chunk = 2 * (gq & 1) + ((li >> 1) & 1), v_half = (li & 1) * 8;

    u32x4 pk[JB][2];                                                       // a block's weights, packed (8-bit caches: times the values' scales)
    u32x4 rest[SPLIT ? JB : 1][2];                                         // ... and what their rounding left
    auto weigh = [&](const int kb, const uint32_t copy) __attribute__((always_inline)) {
        const int base = kb * KB;
        const char *ks_lds = smem + copy * BLK;
        // ---- S^T: st[jb][v] <-> key 32 jb + 8 (v / 4) + 4 hi + v % 4, query l32
        float16v st[JB];
#pragma unroll
        for (int jb = 0; jb < JB; ++jb)
#pragma unroll
            for (int v = 0; v < 16; ++v) st[jb][v] = 0.f;
        // (product by product, in an order that is pinned: left to itself the compiler reads a fragment when it is due and waits for it, 666 us against 643
        // for 2048 queries of 32 heads over 18500 keys; DEEP 6: 642)
        constexpr int PRODUCTS = SIZE / 16 * JB;
        auto fragment = [&](int i) __attribute__((always_inline)) { return lds_read16(ks_lds, lds_at<SIZE>(32 * (i % JB) + l32, 2 * (i / JB) + hi)); };
        u32x4 f[DEEP];
#pragma unroll
        for (int i = 0; i < DEEP; ++i) f[i] = fragment(i);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < PRODUCTS; ++i) {
            st[i % JB] = mfma32<BF16>(f[i % DEEP], qf[i / JB], st[i % JB]);
            if (i + DEEP < PRODUCTS) f[i % DEEP] = fragment(i + DEEP);
            __builtin_amdgcn_sched_barrier(0);
        }
        if constexpr (KIND != CACHE_SAME) {
#pragma unroll
            for (int jb = 0; jb < JB; ++jb)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const float4v k4 = *reinterpret_cast<const float4v *>(&scales[copy * 2 * KB + 32 * jb + 8 * q + 4 * hi]);
#pragma unroll
                    for (int e = 0; e < 4; ++e) st[jb][4 * q + e] *= k4[e];
                }
        }
        const bool hidden = base < all_lo || base + KB > all_hi;          // wavefront-uniform: from some row
        if (hidden) {
            const float out = g.scale_log2e >= 0.f ? -INFINITY : INFINITY;
            const uint32_t from = here(base + 4 * hi) - row_lo, count = row_hi > row_lo ? row_hi - row_lo : 0;      // (keys before row_lo: far beyond count)
#pragma unroll
            for (int jb = 0; jb < JB; ++jb)
#pragma unroll
                for (int v = 0; v < 16; ++v) st[jb][v] = from + (uint32_t)(32 * jb + 8 * (v / 4) + v % 4) < count ? st[jb][v] : out;
        }
        // ---- weights and their sum
        float rs;
        auto exponentials = [&](const float m) {
            float sum = 0.f;
#pragma unroll
            for (int jb = 0; jb < JB; ++jb)
#pragma unroll
                for (int s2 = 0; s2 < 2; ++s2)
#pragma unroll
                    for (int q = 0; q < 2; ++q) {
                        float p[4];
#pragma unroll
                        for (int e = 0; e < 4; ++e) p[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(st[jb][8 * s2 + 4 * q + e], g.scale_log2e, -m));
                        if constexpr (KIND != CACHE_SAME) {
                            sum += (p[0] + p[1]) + (p[2] + p[3]);
                            const float4v v4 = *reinterpret_cast<const float4v *>(&scales[copy * 2 * KB + KB + 32 * jb + 16 * s2 + 8 * q + 4 * hi]);
#pragma unroll
                            for (int e = 0; e < 4; ++e) p[e] *= v4[e];
                        }
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            const uint32_t w = pack_two<VB>(p[2 * i], p[2 * i + 1]);
                            pk[jb][s2][2 * q + i] = w;
                            if constexpr (SPLIT) rest[jb][s2][2 * q + i] = rest_of<VB, true>(w, p[2 * i], p[2 * i + 1]);
                        }
                    }
            if constexpr (KIND != CACHE_SAME) rs = sum;
        };
        // the sums of the packed weights on the matrix pipe; `apart`: queries 0 .. 15 and 16 .. 31 by instructions of their own (0 * NaN is NaN: what
        // one holds would reach the other; the sums are the same bits either way)
        auto matrix_sum = [&](bool apart) {
            float4v sum[2]{};
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                if (half && !apart) break;
#pragma unroll
                for (int jb = 0; jb < JB; ++jb)
#pragma unroll
                    for (int s2 = 0; s2 < 2; ++s2)
                        sum[half] = mfma16<BF16>(ones, !apart || (l32 >> 4) == half ? pk[jb][s2] : u32x4{0, 0, 0, 0}, sum[half]);
            }
            return apart && l32 >= 16 ? sum[1][0] : sum[0][0];
        };
        // A row's weights, sum and reference depend on that row alone, also where a neighbour in the wavefront needs its reference raised.
        bool accept = false;
        if (!pending) {
            exponentials(m_ref);
            if constexpr (KIND == CACHE_SAME) rs = matrix_sum(false);
            accept = __all(rs < 32768.f);
        }
        if (!accept) {                                                     // wavefront-uniform: a row without reference, or a score far above M
            bool keep = false;                                             // this row's reference is close enough
            if (__any(m_ref != -INFINITY)) {
                exponentials(m_ref == -INFINITY ? 0.f : m_ref);
                if constexpr (KIND == CACHE_SAME) rs = matrix_sum(true);
                keep = m_ref != -INFINITY && rs < 32768.f;
                if constexpr (KIND != CACHE_SAME) {
                    const float other = __shfl_xor(rs, 32, 64);            // the row's other lane (exchanged by all: a lane that is switched off reads as 0)
                    keep = keep && other < 32768.f;
                }
            }
            float mx = -INFINITY;
#pragma unroll
            for (int jb = 0; jb < JB; ++jb)
#pragma unroll
                for (int v = 0; v < 16; ++v) mx = fmaxf(mx, st[jb][v] * g.scale_log2e);
            mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
            const float m_new = keep ? m_ref : fmaxf(m_ref, mx), m_use = m_new == -INFINITY ? 0.f : m_new;
            const float alpha = __builtin_amdgcn_exp2f(m_ref - m_use);
            exponentials(m_use);
            if constexpr (KIND == CACHE_SAME) rs = matrix_sum(true);
            l_run *= alpha;
#pragma unroll
            for (int db = 0; db < SIZE / 32; ++db)
#pragma unroll
                for (int v = 0; v < 16; ++v) ot[db][v] *= alpha;
            m_ref = m_new;
            pending = __any(m_new == -INFINITY);
        }
        l_run += rs;
        if (KIND != CACHE_SAME && hidden) {                                // (the scale of a hidden key may be anything; a seen one's NaN shows whatever its weight)
            const uint32_t from = here(base + 4 * hi) - row_lo, count = row_hi > row_lo ? row_hi - row_lo : 0;
#pragma unroll
            for (int i = 0; i < 8 * JB; ++i) {                             // pair i: key 8 (i / 2) + 4 hi + 2 (i % 2) of the block and the next
                const uint32_t j = from + (uint32_t)(8 * (i / 2) + 2 * (i % 2));
                const uint32_t seen = (j < count ? 0xffffu : 0u) | (j + 1 < count ? 0xffff0000u : 0u);
                pk[i / 8][i / 4 % 2][i % 4] &= seen;
                if constexpr (SPLIT) rest[i / 8][i / 4 % 2][i % 4] &= seen;
            }
        }
    };
    // ---- O^T += V^T P^T: k step (jb, s2) lists its 16 keys as 32 jb + 16 s2 + 8 part + 4 hi + 0 .. 3
    auto add_values = [&](const uint32_t copy) __attribute__((always_inline)) {
        const char *vs_lds = smem + (2 + copy) * BLK;
        constexpr int DB = SIZE / 32, PRODUCTS = 2 * JB * DB;
        auto fragment = [&](int i) __attribute__((always_inline)) {
            const int key = 16 * (i / DB), chunk = 4 * (i % DB);
            const u32x2 a = lds_read_transposed(vs_lds, lds_at<SIZE>(key + v_key, chunk + v_chunk) + v_half);
            const u32x2 c = lds_read_transposed(vs_lds, lds_at<SIZE>(key + 8 + v_key, chunk + v_chunk) + v_half);
            return u32x4{a[0], a[1], c[0], c[1]};
        };
        u32x4 f[DEEP];
#pragma unroll
        for (int i = 0; i < DEEP; ++i) f[i] = fragment(i);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < PRODUCTS; ++i) {
            ot[i % DB] = mfma32<VB>(f[i % DEEP], pk[i / DB / 2][i / DB % 2], ot[i % DB]);
            if constexpr (SPLIT) ot[i % DB] = mfma32<VB>(f[i % DEEP], rest[i / DB / 2][i / DB % 2], ot[i % DB]);
            if (i + DEEP < PRODUCTS) f[i % DEEP] = fragment(i + DEEP);
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    // Infinities and NaN of keys that only some rows see: added to those rows alone (a weight of 0 does not silence them)
    auto add_not_finite = [&](const int kb, const uint32_t copy) {
        const char *vs_lds = smem + (2 + copy) * BLK;
        const int half = here(hi);
#pragma unroll 1
        for (int j = 0; j < KB; ++j) {
            const bool sees = kb * KB + j >= row_lo && kb * KB + j < row_hi;
#pragma unroll
            for (int db = 0; db < SIZE / 32; ++db)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    u32x2 v;
                    __builtin_memcpy(&v, vs_lds + lds_at<SIZE>(j, 4 * db + q) + half * 8, 8);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float x = only_not_finite(widen_one<VB>(v[e >> 1], e & 1));
                        ot[db][4 * q + e] += sees ? x : 0.f;
                    }
                }
        }
    };

    const int k_end = keys.lo < keys.hi ? (keys.hi + KB - 1) / KB : 0;
    int kb = keys.lo < keys.hi ? keys.lo / KB : 0;
    if (tid < 3) flags[tid] = 0;
    if (DMA && !FULL)                                                      // what no load writes
        for (uint32_t i = here(tid); i < 4 * BLK / 16; i += 256) lds_write16(smem, 16 * i, u32x4{0, 0, 0, 0});
    __syncthreads();
    if (kb < k_end) {                                                      // (workgroup-uniform, as the loop's count)
        find(kb);
        fetch(kb, 0);
        find(kb + 1);
        // (Q is waited for here: inside the loop the wait would be one for everything in flight)
#pragma unroll
        for (int ks = 0; ks < SIZE / 16; ++ks) asm volatile("" : "+v"(qf[ks]));
        stash(kb, 0);
    }
    __syncthreads();
    for (uint32_t copy = 0; kb < k_end; ++kb, copy ^= 1) {
        const bool more = kb + 1 < k_end;
        if (more) {
            fetch(kb + 1, copy ^ 1);
            find(kb + 2);
        }
        const bool act = busy && kb * KB < wave_hi && kb * KB + KB > wave_lo;
        if (act) weigh(kb, copy);
        if ((kb * KB < seen_lo || kb * KB + KB > seen_hi) && flags[kb % 3] != 0) {         // (workgroup-uniform; rare)
            if (act) add_not_finite(kb, copy);
            __syncthreads();
            for (int i = here(tid); i < KB * (SIZE / 8); i += 256) {       // ... and taken out of the block
                const uint32_t at = (2 + copy) * BLK + 16 * i;
                lds_write16(smem, at, without_not_finite<VB>(lds_read16(smem, at)));
            }
            __syncthreads();
        }
        if (act) add_values(copy);
        if (tid == 0) flags[(kb + 2) % 3] = 0;                             // (read in the pass before this one, set in the next)
        if (more) stash(kb + 1, copy ^ 1);
        __syncthreads();
    }

    // ---- O = O^T / l, stored along d: after the half-wavefronts trade register groups a lane owns d = 32 db + 16 hi .. + 15 of its row
    const float total = KIND == CACHE_SAME ? l_run : l_run + __shfl_xor(l_run, 32, 64);
    const float factor = g.splits > 1 ? 1.f : total == 0.f ? 0.f : 1.0f / total;
    const int64_t at = (token * g.Hq + head) * g.splits + split;
    if (g.splits > 1 && real && hi == 0) *reinterpret_cast<float2v *>(g.part_ml + 2 * at) = float2v{m_ref, total};
#pragma unroll
    for (int db = 0; db < SIZE / 32; ++db) {
#pragma unroll
        for (int v = 0; v < 16; ++v) ot[db][v] *= factor;
        uint32_t o[16];
        gather_row16(ot[db], o);                                           // (all lanes take part)
        const int d = 32 * db + 16 * hi;
        if (!real || d >= g.D) continue;
        if (g.splits > 1) {
            float *dst = g.part_o + at * g.D + d;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (d + 4 * i < g.D) __builtin_memcpy(dst + 4 * i, &o[4 * i], 16);
        } else {
            uint16_t *dst = g.O + token * g.o_st + (int64_t)head * g.o_sh + d;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                u32x4 x;
#pragma unroll
                for (int j = 0; j < 4; ++j) x[j] = pack_two<BF16>(__builtin_bit_cast(float, o[8 * i + 2 * j]), __builtin_bit_cast(float, o[8 * i + 2 * j + 1]));
                if (d + 8 * i < g.D) __builtin_memcpy(dst + 8 * i, &x, 16);
            }
        }
    }
}

}  // namespace nt
