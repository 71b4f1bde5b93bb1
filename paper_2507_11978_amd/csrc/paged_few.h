// Attention over a paged cache for few query rows per key head: a decoding step, or a few tokens of each sequence.
//
// One program per (sequence, key head, share of the keys) has the rows (token, query head of the group) of that sequence, 16 or 32 at a time, so that
// K and V are read once for all query heads that share them.  Its wavefronts take the keys in turn, tiles of 32, each with a running maximum m (base-2
// units), sum l and accumulator of its own:
//   S^T = K Q^T;  p = 2^(c S - m);  l += sum p;  O^T += V^T P^T,
// brought to a common maximum at the end.  16 x 16 x 32 matrix instructions with the query on the lane axis (lane % 16): the four scores that a lane holds
// of each 16 keys are, packed, its part of the second product's operand, if the other operand lists the keys in the same order.
//
// K goes from memory straight into the operand's registers (a lane holds its key's elements).  V has to be turned: through registers into LDS, a region per
// wavefront, and out with transposing reads; no barrier in the loop.  A trip takes as many tiles as make 16 KB of K and V, all of them in flight at once: K's
// loads for the next trip go out once the scores are there, V's as its registers empty into LDS.
//
// Weights multiply V as the sum of two 16-bit numbers each (rest_of): the second half of the products hides behind the loads (64 x 4096 bf16 134 us either way, 2 x
// 131072 e4m3 128 and 129), but for two sets of 16 rows over codes (8 x 8 queries x 4000 keys x 32/8 heads x 128 e4m3 30.7 us, 32.8).  Rounded once they would be off
// by as much as the rounded result.
//
// Bound by reading K and V: 64 sequences of 17 to 4096 tokens, 32/8 heads x 128 bf16 134 us = 4.15 TB/s (a large copy reaches 4.84), 2 of 131072 in e4m3 129 us =
// 4.3 TB/s, 32 of 2047 with 48 heads x 64 in int8 63.6 us = 4.5 TB/s; the matrix pipe is busy for 4 to 8 % of the cycles, 1.03 of their bytes are read.  One of 900
// 12.5 us, most of it the host's call and one wavefront's chain of loads.
#pragma once
#include "paged.h"

namespace nt {

constexpr int kFewWaves = 4;                                             // (8 measured no gain: 48 heads x 900 f16 12.2 us with four, 13.1)
constexpr size_t few_lds(int size, int mb) { return (size_t)kFewWaves * mb * 64 * size; }        // V's 32 keys (64 * size bytes), later 16 * mb rows of fp32 outputs
// 32-key tiles of a trip, which a wavefront has in flight: two, or one where a tile of K and V is 16 KB
constexpr int few_tiles(int kind, int size) { return size * (kind == CACHE_SAME ? 2 : 1) >= 256 ? 1 : 2; }
constexpr int few_trip(int kind, int size) { return 32 * few_tiles(kind, size); }        // keys

// Wavefronts per SIMD that the registers are shared out for: three at head size 64, whose trips are half as long (32 x 48 heads x 2047 int8 72 us with two, 63).
// At 128 three do not help (64 x 8 heads x 4096 bf16 134 us with two, 144): 128 KB in flight per unit are enough, and more only wait for each other.
constexpr int few_resident(int size, int mb) { return mb == 1 && size == 64 ? 3 : size * mb <= 128 ? 2 : 1; }

// UNIFORM: page_size is a multiple of 16, so that 16 keys that begin at a multiple of 16 lie on one page: the table is read and the addresses are made
// once for a wavefront, on the scalar unit, and a lane's part is an offset that never changes.
template <bool BF16, int KIND, int SIZE, int MB, bool UNIFORM, bool FULL>
__global__ __launch_bounds__(64 * kFewWaves, few_resident(SIZE, MB)) void paged_few_kernel(const PagedArgs g)
{
    constexpr int KS = SIZE / 32;                                          // k steps of the first product
    constexpr int NV = KIND == CACHE_SAME ? SIZE / 32 : SIZE / 64;         // 16-byte loads per lane, 16 keys and tensor
    constexpr int ES = KIND == CACHE_SAME ? 2 : 1;
    constexpr int NT = few_tiles(KIND, SIZE), NG = 2 * NT, TRIP = 32 * NT;   // tiles of 32 and groups of 16 keys in a trip
    constexpr bool VB = BF16 || KIND != CACHE_SAME;                        // the second product's type is bf16 (see rest_of)
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    __shared__ float red_m[kFewWaves][16 * MB], red_l[kFewWaves][16 * MB];
    __shared__ __attribute__((aligned(16))) float scales[KIND == CACHE_SAME ? 1 : kFewWaves][KIND == CACHE_SAME ? 4 : 2 * TRIP];     // K's, V's
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), c16 = lane & 15, g4 = lane >> 4;
    char *vt = smem + wave * (64 * SIZE * MB);

    // Consecutive programs go to different XCDs (number mod 8).  The heads of one share lie side by side in memory: one XCD has them, one after the other, and
    // the pages of an eighth of the shares, not an eighth of all pages' bytes
    const uint32_t w = blockIdx.x, heads = g.Hkv, items = (uint32_t)g.B * g.splits, whole = (items & ~7u) * heads;
    uint32_t item, h;
    if (w < whole) {
        const uint32_t j = w >> 3;
        const uint32_t group = j / heads;
        item = group * 8 + ((w + group) & 7);
        h = j % heads;
    } else {
        item = w / heads;
        h = w % heads;
    }
    const int split = item % g.splits, b = item / g.splits;
    typedef const __attribute__((address_space(4))) int32_t *ScalarTable;
    const int32_t *pages = g.table + (int64_t)b * g.t_sb;
    const char *Kh = g.K + (int64_t)h * g.k_sh * ES, *Vh = g.V + (int64_t)h * g.v_sh * ES;
    const float *KSh = g.KS + (int64_t)h * g.ks_sh, *VSh = g.VS + (int64_t)h * g.vs_sh;

    // ---- loads: lane (c16, g4) has key c16 of each 16 and a quarter of its elements
    u32x4 kr[NG][NV], vr[NG][NV];
    float sc[NT];                                                          // lanes 0 .. 31: the scale of key lane's K of a tile, 32 .. 63: of key lane - 32's V
    int32_t id[NG];                                                        // the table's entries for the trip that is fetched next
    int64_t k_at[NG], v_at[NG];                                            // ... and byte offsets of this lane's keys (UNIFORM: of the 16 keys' first)
    uint32_t named[NG];                                                    // bit i: a page is named for key i of the 16 (of the trip in kr, vr)
    // a lane's own byte offset: its elements' (FULL), its key's (UNIFORM; they fit 32 bits)
    const int32_t mine = FULL ? 16 * g4 : 0, kl = mine + (UNIFORM ? (int32_t)(c16 * g.k_ss) * ES : 0), vl = mine + (UNIFORM ? (int32_t)(c16 * g.v_ss) * ES : 0);
    auto find = [&](int t) {
#pragma unroll
        for (int u = 0; u < NG; ++u) {
            const uint32_t index = divide((uint32_t)t * TRIP + 16 * u + (UNIFORM ? 0 : c16), g.page);
            const uint32_t entry = entry_read(index, g.width);
            id[u] = UNIFORM ? ((ScalarTable)pages)[entry] : pages[entry];
        }
    };
    auto locate = [&](int t, uint32_t (&has)[NG]) {
        uint32_t page[NG];
#pragma unroll
        for (int u = 0; u < NG; ++u) {
            const uint32_t key = (uint32_t)t * TRIP + 16 * u + (UNIFORM ? 0 : c16), index = divide(key, g.page), at = key - index * g.page.d;
            const bool ok = names_page(index, id[u], g.width, g.pages);
            page[u] = ok ? id[u] : 0;
            has[u] = UNIFORM ? (ok ? 0xffffu : 0u) : (uint32_t)__ballot(ok) & 0xffffu;
            k_at[u] = (times(page[u], g.k_sp) + times(at, g.k_ss)) * ES;
            v_at[u] = (times(page[u], g.v_sp) + times(at, g.v_ss)) * ES;
        }
        if constexpr (KIND != CACHE_SAME) {
#pragma unroll
            for (int s = 0; s < NT; ++s) {
                const uint32_t key = (uint32_t)t * TRIP + 32 * s + (lane & 31), at = key - divide(key, g.page) * g.page.d;
                const uint32_t p0 = page[2 * s], p1 = page[2 * s + 1], p = (lane & 16) ? p1 : p0;
                sc[s] = lane < 32 ? KSh[times(p, g.ks_sp) + times(at, g.ks_ss)] : VSh[times(p, g.vs_sp) + times(at, g.vs_ss)];
            }
        }
    };
    // 64 bytes of a row to a load of four lanes; a head size below SIZE: where there are no elements, the row's last ones once more (codes: 8 at a time)
    auto load_rows = [&](u32x4 (&to)[NV], const char *p, int32_t lane_off) {
        if constexpr (FULL) {
#pragma unroll
            for (int n = 0; n < NV; ++n) __builtin_memcpy(&to[n], p + (uint32_t)lane_off + 64 * n, 16);
        } else {
            const int q = here(16 * g4), end = (g.D - 8) * ES;
#pragma unroll
            for (int n = 0; n < NV; ++n) {
                const int at = 64 * n + q;
                if constexpr (KIND == CACHE_SAME) {
                    __builtin_memcpy(&to[n], p + (uint32_t)(lane_off + (at < end ? at : end)), 16);
                } else {
                    u32x2 lo, hi;
                    __builtin_memcpy(&lo, p + (uint32_t)(lane_off + (at < end ? at : end)), 8);
                    __builtin_memcpy(&hi, p + (uint32_t)(lane_off + (at + 8 < end ? at + 8 : end)), 8);
                    to[n] = u32x4{lo[0], lo[1], hi[0], hi[1]};
                }
            }
        }
    };
    // (`more` false: nothing is needed any more.  The loads go out all the same, from one address: a branch around them would make the waits behind it wait
    // for everything, since the number of loads in flight would not be known)
    auto load_k = [&](bool more) {
#pragma unroll
        for (int u = 0; u < NG; ++u) load_rows(kr[u], Kh + (UNIFORM || more ? k_at[u] : 0), more ? kl : 0);
    };
    auto load_v = [&](int u, bool more) { load_rows(vr[u], Vh + (UNIFORM || more ? v_at[u] : 0), more ? vl : 0); };

    // Without a window a share begins where it does whatever the sequence's length is: its first pages are looked up along with that.
    const int t_first = g.window ? -1 : (int)((int64_t)split * g.split_keys / TRIP) + wave;
    if (t_first >= 0) find(t_first);
    const Sequence seq = sequence_of(g, b);
    const int rows_all = seq.count * g.G;

    for (int r0 = 0; r0 < rows_all; r0 += 16 * MB) {                       // (one pass, unless the caller's bound on new tokens was too low)
        const int last = r0 + 16 * MB < rows_all ? r0 + 16 * MB - 1 : rows_all - 1;
        const KeyRange keys = keys_of(g, seq, (int32_t)divide(r0, g.group), (int32_t)divide(last, g.group), split, TRIP);

        const int t_end = keys.lo < keys.hi ? (keys.hi + TRIP - 1) / TRIP : 0;
        int t = keys.lo / TRIP + wave;

        // ---- this lane's rows (row c16 of each 16): their keys [row_lo, row_hi), and Q as the first product's operand
        int32_t row_lo[MB], row_hi[MB];
        u32x4 qf[MB][KS];
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) {
            const int r = r0 + 16 * mb + c16;
            const bool real = r < rows_all;
            const uint32_t rc = real ? r : last, i = divide(rc, g.group), head = h * g.G + (rc - i * g.group.d);
            const KeyRange sees = keys_seen(seq, (int32_t)i, g.causal, g.window);
            row_lo[mb] = real ? sees.lo : INT32_MIN;                       // (rows past the last are not stored: nothing to hide from them)
            row_hi[mb] = real ? sees.hi : INT32_MAX;
            const uint16_t *q = g.Q + (int64_t)(seq.first + (int32_t)i) * g.q_st + (int64_t)head * g.q_sh;
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
                const int d = KIND == CACHE_SAME ? 32 * ks + 8 * g4 : 64 * (ks >> 1) + 16 * g4 + 8 * (ks & 1);
                qf[mb][ks] = u32x4{0, 0, 0, 0};
                if (d < g.D) __builtin_memcpy(&qf[mb][ks], q + d, 16);
            }
        }

        // (behind Q's loads: those have landed where these have)
        if (t < t_end) {
            if (t != t_first || r0 > 0) find(t);
            locate(t, named);
            load_k(true);
#pragma unroll
            for (int u = 0; u < NG; ++u) load_v(u, true);
            find(t + kFewWaves);
        }

        // Q is waited for here: at its first use inside the loop the wait would be one for everything in flight, in every trip
#pragma unroll
        for (int mb = 0; mb < MB; ++mb)
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) asm volatile("" : "+v"(qf[mb][ks]));

        float m[MB], l[MB];
        float4v acc[MB][SIZE / 16];
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) {
            m[mb] = -INFINITY;
            l[mb] = 0.f;
#pragma unroll
            for (int db = 0; db < SIZE / 16; ++db) acc[mb][db] = float4v{0.f, 0.f, 0.f, 0.f};
        }

        for (; t < t_end; t += kFewWaves) {
            const int base = t * TRIP, next = t + kFewWaves;
            const bool more = next < t_end;
            // ---- S^T: lane (c16, g4) gets query c16, keys 16 u + 4 g4 + 0 .. 3
            float4v st[MB][NG];
#pragma unroll
            for (int mb = 0; mb < MB; ++mb)
#pragma unroll
                for (int u = 0; u < NG; ++u) st[mb][u] = float4v{0.f, 0.f, 0.f, 0.f};
            if constexpr (!FULL) {                                         // (Q has zeros there, but 0 * infinity is NaN)
                const int g4 = here(lane) >> 4;
#pragma unroll
                for (int u = 0; u < NG; ++u)
#pragma unroll
                    for (int n = 0; n < NV; ++n) {
                        if constexpr (KIND == CACHE_SAME) {
                            kr[u][n] = 32 * n + 8 * g4 < g.D ? kr[u][n] : u32x4{0, 0, 0, 0};
                        } else {
                            const bool lo = 64 * n + 16 * g4 < g.D, hi = 64 * n + 16 * g4 + 8 < g.D;
                            kr[u][n] = u32x4{lo ? kr[u][n][0] : 0u, lo ? kr[u][n][1] : 0u, hi ? kr[u][n][2] : 0u, hi ? kr[u][n][3] : 0u};
                        }
                    }
            }
#pragma unroll
            for (int u = 0; u < NG; ++u)
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) {
                    u32x4 kf;
                    if constexpr (KIND == CACHE_SAME) {
                        kf = kr[u][ks];
                    } else {
                        const u32x4 raw = kr[u][ks >> 1];
                        kf = widen8<BF16, KIND>((ks & 1) ? u32x2{raw[2], raw[3]} : u32x2{raw[0], raw[1]});
                    }
#pragma unroll
                    for (int mb = 0; mb < MB; ++mb) st[mb][u] = mfma16<BF16>(kf, qf[mb][ks], st[mb][u]);
                }
            if constexpr (KIND != CACHE_SAME) {
                wavefront_fence();                                         // (the reads of the trip before are done)
#pragma unroll
                for (int s = 0; s < NT; ++s) scales[wave][(lane < 32 ? 0 : TRIP) + 32 * s + (lane & 31)] = sc[s];
                wavefront_fence();
            }
            // ---- the next trip's K, into registers that are free now
            uint32_t named_next[NG];
            locate(next, named_next);
            load_k(more);
            find(next + kFewWaves);
            // ---- keys that no page is named for have the score NaN: a row that sees one shows it.  V's rows are zeros there, and for keys outside the range: what
            // lies there may be anything, and a weight of 0 does not silence an infinity.
            uint32_t good[NG], all = 0xffffu;
            bool clear = true;                                             // every row sees every key of the trip
#pragma unroll
            for (int u = 0; u < NG; ++u) {
                const int32_t from = keys.lo - base - 16 * u, to = keys.hi - base - 16 * u;        // the range, from the first of the 16 on
                const uint32_t below = from <= 0 ? 0u : from >= 16 ? 0xffffu : (1u << from) - 1, under = to <= 0 ? 0u : to >= 16 ? 0xffffu : (1u << to) - 1;
                good[u] = named[u] & under & ~below;
                all &= good[u];
            }
#pragma unroll
            for (int mb = 0; mb < MB; ++mb) clear = clear && row_lo[mb] <= base && base + TRIP <= row_hi[mb];
            clear = __all(clear);
            bool careful = false;                                          // (codes: some row does not see a NaN)
            if (all != 0xffffu || !clear) {                                // wavefront-uniform
                bool odd = false;
#pragma unroll
                for (int u = 0; u < NG; ++u)
#pragma unroll
                    for (int n = 0; n < NV; ++n) {
                        vr[u][n] = (good[u] >> c16) & 1 ? vr[u][n] : u32x4{0, 0, 0, 0};
                        if constexpr (KIND == CACHE_E4M3)                  // (0x7f, the type's one NaN)
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                const uint32_t x = vr[u][n][i] & 0x7f7f7f7fu;
                                odd = odd | (((x + 0x01010101u) & 0x80808080u) != 0);
                            }
                    }
                careful = !clear && __any(odd);
            }

            // ---- weights
            u32x4 pk[MB][NT], rest[MB][NT];
#pragma unroll
            for (int mb = 0; mb < MB; ++mb) {
                float s[4 * NG];
#pragma unroll
                for (int u = 0; u < NG; ++u)
#pragma unroll
                    for (int v = 0; v < 4; ++v) s[4 * u + v] = st[mb][u][v] * g.scale_log2e;
                if constexpr (KIND != CACHE_SAME) {
#pragma unroll
                    for (int u = 0; u < NG; ++u) {
                        const float4v k4 = *reinterpret_cast<const float4v *>(&scales[wave][16 * u + 4 * g4]);
#pragma unroll
                        for (int v = 0; v < 4; ++v) s[4 * u + v] *= k4[v];
                    }
                }
                if (all != 0xffffu || !clear) {
                    const int q = here(4 * g4);
#pragma unroll
                    for (int u = 0; u < NG; ++u)
#pragma unroll
                        for (int v = 0; v < 4; ++v) {
                            const int32_t key = base + 16 * u + q + v;
                            const float x = (named[u] >> (q + v)) & 1 ? s[4 * u + v] : __builtin_nanf("");
                            s[4 * u + v] = key >= row_lo[mb] && key < row_hi[mb] ? x : -INFINITY;        // (shares begin and end between trips)
                        }
                }
                float top = s[0];
#pragma unroll
                for (int j = 1; j < 4 * NG; ++j) top = fmaxf(top, s[j]);
                top = largest_across<true>(top);
                const float m_new = fmaxf(m[mb], top), ref = m_new == -INFINITY ? 0.f : m_new;
                const float alpha = __builtin_amdgcn_exp2f(m[mb] - ref);
                m[mb] = m_new;
                float p[4 * NG], sum = 0.f;
#pragma unroll
                for (int j = 0; j < 4 * NG; ++j) {
                    p[j] = __builtin_amdgcn_exp2f(s[j] - ref);
                    sum += p[j];
                }
                l[mb] = __builtin_fmaf(l[mb], alpha, sum);
                if (!__all(alpha == 1.f)) {
#pragma unroll
                    for (int db = 0; db < SIZE / 16; ++db) acc[mb][db] = acc[mb][db] * alpha;
                }
                if constexpr (KIND != CACHE_SAME) {
#pragma unroll
                    for (int u = 0; u < NG; ++u) {
                        const float4v v4 = *reinterpret_cast<const float4v *>(&scales[wave][TRIP + 16 * u + 4 * g4]);
#pragma unroll
                        for (int v = 0; v < 4; ++v) p[4 * u + v] *= v4[v];
                    }
                    if (!clear) {                                          // (the scale of a hidden key may be anything; a seen one's NaN shows whatever its weight)
                        const int32_t first = here(base + 4 * g4);
#pragma unroll
                        for (int j = 0; j < 4 * NG; ++j) {
                            const int32_t key = first + 16 * (j / 4) + j % 4;
                            p[j] = key >= row_lo[mb] && key < row_hi[mb] ? p[j] : 0.f;
                        }
                    }
                }
#pragma unroll
                for (int i = 0; i < NT; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float a = p[8 * i + 2 * j], b = p[8 * i + 2 * j + 1];
                        pk[mb][i][j] = pack_two<VB>(a, b);
                        rest[mb][i][j] = rest_of<VB, KIND != CACHE_SAME>(pk[mb][i][j], a, b);
                    }
            }
            // ---- O^T += V^T P^T, 32 keys at a time: V into LDS (its registers take the next trip's), then lane (c16, g4) supplies d = 16 db + c16 and keys
            // 4 g4 + 0 .. 3, 16 + 4 g4 + 0 .. 3; lane i of a group of 16 points the transposing read at key i / 4 of its four, 8 bytes i % 4 of the 32
#pragma unroll
            for (int i = 0; i < NT; ++i) {
                wavefront_fence();                                         // (the reads of the tile before are done)
                ushort2v top{0, 0};                                        // largest magnitude among this lane's values, as integers: infinities and NaN above all numbers
#pragma unroll
                for (int u = 0; u < 2; ++u) {
#pragma unroll
                    for (int n = 0; n < NV; ++n) {
                        const uint32_t row = 16 * u + c16;
                        const u32x4 x = vr[2 * i + u][n];
                        if constexpr (KIND == CACHE_SAME) {
                            lds_write16(vt, lds_at<SIZE>(row, 4 * n + g4), x);
#pragma unroll
                            for (int w = 0; w < 4; ++w) top = __builtin_elementwise_max(top, __builtin_bit_cast(ushort2v, x[w] & 0x7fff7fffu));
                        } else {
                            lds_write16(vt, lds_at<SIZE>(row, 8 * n + 2 * g4), widen8<VB, KIND>(u32x2{x[0], x[1]}));
                            lds_write16(vt, lds_at<SIZE>(row, 8 * n + 2 * g4 + 1), widen8<VB, KIND>(u32x2{x[2], x[3]}));
                        }
                    }
                    load_v(2 * i + u, more);
                }
                wavefront_fence();
                constexpr uint16_t ABOVE = BF16 ? 0x7f80 : 0x7c00;
                if (KIND == CACHE_SAME ? __any(top[0] >= ABOVE || top[1] >= ABOVE) : careful) {
                    // infinities and NaN: added to the rows that see their keys alone, and taken out of the tile (a weight of 0 does not silence them, and with one in
                    // two parts an infinity would become infinity less infinity)
                    const int lane_here = here(lane), c = lane_here & 15, q = lane_here >> 4;
#pragma unroll 1
                    for (int j = 0; j < 32; ++j)
#pragma unroll
                        for (int db = 0; db < SIZE / 16; ++db) {
                            u32x2 v;
                            __builtin_memcpy(&v, vt + lds_at<SIZE>(j, 2 * db + (q >> 1)) + (q & 1) * 8, 8);
                            const int32_t key = base + 32 * i + j;
#pragma unroll
                            for (int mb = 0; mb < MB; ++mb) {
                                const bool sees = key >= row_lo[mb] && key < row_hi[mb];
#pragma unroll
                                for (int e = 0; e < 4; ++e) {
                                    const float x = only_not_finite(widen_one<VB>(v[e >> 1], e & 1));
                                    acc[mb][db][e] += sees ? x : 0.f;
                                }
                            }
                        }
                    wavefront_fence();
#pragma unroll 1
                    for (int j = 0; j < SIZE / 16; ++j) {                  // (each lane has SIZE / 16 of the tile's 16-byte pieces)
                        const uint32_t at = lds_at<SIZE>(16 * (j & 1) + c, (j >> 1) * 4 + q);
                        lds_write16(vt, at, without_not_finite<VB>(lds_read16(vt, at)));
                    }
                    wavefront_fence();
                }
                // (four blocks' reads are on their way while the four before them are multiplied)
                const uint32_t row = 4 * g4 + (c16 >> 2), half = (c16 & 1) * 8;
                u32x2 frag[2][4][2];
                auto read_four = [&](int q) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const uint32_t chunk = 2 * (4 * q + j) + ((c16 >> 1) & 1);
                        frag[q & 1][j][0] = lds_read_transposed(vt, lds_at<SIZE>(row, chunk) + half);
                        frag[q & 1][j][1] = lds_read_transposed(vt, lds_at<SIZE>(row + 16, chunk) + half);
                    }
                };
                read_four(0);
#pragma unroll
                for (int q = 0; q < SIZE / 64; ++q) {
                    if (q + 1 < SIZE / 64) read_four(q + 1);
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int part = 0; part < 2; ++part)
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const u32x2 a = frag[q & 1][j][0], c = frag[q & 1][j][1];
#pragma unroll
                            for (int mb = 0; mb < MB; ++mb)
                                acc[mb][4 * q + j] = mfma16<VB>(u32x4{a[0], a[1], c[0], c[1]}, part ? rest[mb][i] : pk[mb][i], acc[mb][4 * q + j]);
                        }
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
#pragma unroll
            for (int u = 0; u < NG; ++u) named[u] = named_next[u];
        }

        // ---- the wavefronts' results to a common maximum: through LDS, row by row
        float *ex = reinterpret_cast<float *>(vt);
        const int tid = here(threadIdx.x), lane16 = tid & 15, lane4 = (tid >> 4) & 3;
        wavefront_fence();
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) {
            l[mb] = sum_across<true>(l[mb]);
            if (lane4 == 0) {
                red_m[wave][16 * mb + lane16] = m[mb];
                red_l[wave][16 * mb + lane16] = l[mb];
            }
#pragma unroll
            for (int db = 0; db < SIZE / 16; ++db)
                *reinterpret_cast<float4v *>(ex + (16 * mb + lane16) * SIZE + 16 * db + 4 * lane4) = acc[mb][db];
        }
        __syncthreads();
        for (int e = tid; e < 16 * MB * (SIZE / 4); e += 64 * kFewWaves) {
            const int row = e / (SIZE / 4), d = 4 * (e % (SIZE / 4));
            const uint32_t r = r0 + row;
            if (r >= (uint32_t)rows_all || d >= g.D) continue;
            float top = red_m[0][row];
#pragma unroll
            for (int i = 1; i < kFewWaves; ++i) top = fmaxf(top, red_m[i][row]);
            const float ref = top == -INFINITY ? 0.f : top;
            float sum = 0.f;
            float4v o{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int i = 0; i < kFewWaves; ++i) {
                const float f = __builtin_amdgcn_exp2f(red_m[i][row] - ref);
                sum = __builtin_fmaf(red_l[i][row], f, sum);
                const float4v x = *reinterpret_cast<const float4v *>(smem + i * (64 * SIZE * MB) + (row * SIZE + d) * 4);
#pragma unroll
                for (int v = 0; v < 4; ++v) o[v] = __builtin_fmaf(x[v], f, o[v]);
            }
            const uint32_t i = divide(r, g.group), head = h * g.G + (r - i * g.group.d);
            const int64_t token = seq.first + (int32_t)i;
            if (g.splits > 1) {
                const int64_t at = (token * g.Hq + head) * g.splits + split;
                *reinterpret_cast<float4v *>(g.part_o + at * g.D + d) = o;
                if (d == 0) *reinterpret_cast<float2v *>(g.part_ml + 2 * at) = float2v{top, sum};
            } else {
                const float inv = sum == 0.f ? 0.f : 1.0f / sum;           // (a row that sees nothing: zeros)
                const u32x2 out{pack_two<BF16>(o[0] * inv, o[1] * inv), pack_two<BF16>(o[2] * inv, o[3] * inv)};
                __builtin_memcpy(g.O + token * g.o_st + (int64_t)head * g.o_sh + d, &out, 8);
            }
        }
        __syncthreads();                                                   // (before the next rows' tiles go where the results lie)
    }
}

}  // namespace nt
