// Attention over a paged cache for few query rows per key head: a decoding step, or a few tokens of each sequence.
//
// One program per (sequence, key head, share of the keys) has the rows (token, query head of the group) of that sequence, 16 or 32 at a time, so that
// K and V are read once for all query heads that share them.  Its four wavefronts take tiles of 32 keys in turn, each with a running maximum m (base-2
// units), sum l and accumulator of its own:
//   S^T = K Q^T;  p = 2^(c S - m);  l += sum p;  O^T += V^T P^T,
// brought to a common maximum at the end.  16 x 16 x 32 matrix instructions with the query on the lane axis (lane % 16): the four scores that a lane holds
// of each 16 keys are, packed, its part of the second product's operand, if the other operand lists the keys in the same order.
//
// K goes from memory straight into the operand's registers (a lane holds its key's elements).  V has to be turned: through registers into LDS, a region per
// wavefront, and out with transposing reads; no barrier in the loop.  The next tile's loads are issued as soon as this one's registers are free, before
// its exponentials and the second product.  What bounds it is memory: per tile a wavefront has some 150 vector instructions and 16 matrix
// instructions for 16 KB (128 elements of 16 bits), a tenth of the time that the unit's share of memory takes to bring them.
#pragma once
#include "paged.h"

namespace nt {

constexpr int kFewWaves = 4, kFewKeys = 32;
constexpr size_t few_lds(int size, int mb) { return (size_t)kFewWaves * mb * 64 * size; }        // V's tile (64 * size bytes), later 16 * mb rows of fp32 outputs

template <bool BF16, int KIND, int SIZE, int MB>
__global__ __launch_bounds__(64 * kFewWaves, SIZE * MB <= 128 ? 2 : 1) void paged_few_kernel(const PagedArgs g)
{
    constexpr int KS = SIZE / 32;                                          // k steps of the first product
    constexpr int NV = KIND == CACHE_SAME ? SIZE / 32 : SIZE / 64;         // 16-byte loads per lane, 16 keys and tensor
    constexpr int ES = KIND == CACHE_SAME ? 2 : 1;
    constexpr bool NORM = KIND != CACHE_SAME && !BF16;                     // weights times scales may leave fp16's range: see `unit`
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    __shared__ float red_m[kFewWaves][16 * MB], red_l[kFewWaves][16 * MB];
    __shared__ __attribute__((aligned(16))) float scales[KIND == CACHE_SAME ? 1 : kFewWaves][2 * kFewKeys];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), c16 = lane & 15, g4 = lane >> 4;
    char *vt = smem + wave * (64 * SIZE * MB);

    int w = blockIdx.x;
    const int h = w % g.Hkv;                                               // (consecutive programs, on different XCDs, have different heads)
    w /= g.Hkv;
    const int split = w % g.splits, b = w / g.splits;
    const Sequence seq = sequence_of(g, b);
    const int32_t *pages = g.table + (int64_t)b * g.t_sb;
    const int rows_all = seq.count * g.G;
    const char *Kh = g.K + (int64_t)h * g.k_sh * ES, *Vh = g.V + (int64_t)h * g.v_sh * ES;

    for (int r0 = 0; r0 < rows_all; r0 += 16 * MB) {                       // (one pass, unless the caller's bound on new tokens was too low)
        const int last = r0 + 16 * MB < rows_all ? r0 + 16 * MB - 1 : rows_all - 1;
        const KeyRange keys = keys_of(g, seq, (int32_t)divide(r0, g.group), (int32_t)divide(last, g.group), split, kFewKeys);

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

        float m[MB], l[MB];
        float4v acc[MB][SIZE / 16];
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) {
            m[mb] = -INFINITY;
            l[mb] = 0.f;
#pragma unroll
            for (int db = 0; db < SIZE / 16; ++db) acc[mb][db] = float4v{0.f, 0.f, 0.f, 0.f};
        }
        // NORM: a row's accumulator is held in units of a power of two that follows the largest scale it has seen, so that weight * scale / unit is at
        // most 1 and in fp16's range whatever the size of the values
        float unit[MB], per_unit[MB];
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) unit[mb] = per_unit[mb] = 0.f;

        // ---- loads: lane (c16, g4) has key c16 of either 16 and a quarter of its elements
        u32x4 kr[2][NV], vr[2][NV];
        float sc = 0.f;                                                    // lanes 0 .. 31: the scale of key lane's K, 32 .. 63: of key lane - 32's V
        int32_t id[2];                                                     // page of the tile that is fetched next
        bool named[2], inside[2];                                          // of the tile in kr, vr: the table names its page; the key is in `keys`
        auto find = [&](int t) {
#pragma unroll
            for (int u = 0; u < 2; ++u) id[u] = page_at(pages, divide((uint32_t)(t * kFewKeys + 16 * u + c16), g.page), g.width, g.pages);
        };
        auto fetch = [&](int t) {
            int64_t page[2], at[2];
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const int32_t key = t * kFewKeys + 16 * u + c16;
                named[u] = id[u] >= 0;
                inside[u] = key >= keys.lo && key < keys.hi;
                page[u] = named[u] ? id[u] : 0;
                at[u] = (uint32_t)key - divide((uint32_t)key, g.page) * g.page.d;
                const char *kp = Kh + (page[u] * g.k_sp + at[u] * g.k_ss) * ES, *vp = Vh + (page[u] * g.v_sp + at[u] * g.v_ss) * ES;
#pragma unroll
                for (int n = 0; n < NV; ++n) {
                    const int d = KIND == CACHE_SAME ? 32 * n + 8 * g4 : 64 * n + 16 * g4;
                    kr[u][n] = vr[u][n] = u32x4{0, 0, 0, 0};
                    if (d + 16 / ES <= g.D) {
                        __builtin_memcpy(&kr[u][n], kp + d * ES, 16);
                        __builtin_memcpy(&vr[u][n], vp + d * ES, 16);
                    } else if (KIND != CACHE_SAME && d < g.D) {             // (a head size is a multiple of 8)
                        __builtin_memcpy(&kr[u][n], kp + d, 8);
                        __builtin_memcpy(&vr[u][n], vp + d, 8);
                    }
                }
            }
            if constexpr (KIND != CACHE_SAME) {
                const int64_t p = (lane & 16) ? page[1] : page[0], a = (lane & 16) ? at[1] : at[0];
                sc = lane < 32 ? g.KS[p * g.ks_sp + a * g.ks_ss + (int64_t)h * g.ks_sh] : g.VS[p * g.vs_sp + a * g.vs_ss + (int64_t)h * g.vs_sh];
            }
        };

        const int t_end = (keys.hi + kFewKeys - 1) / kFewKeys;
        int t = keys.lo / kFewKeys + wave;
        if (keys.lo == keys.hi) t = t_end;
        if (t < t_end) {
            find(t);
            fetch(t);
            find(t + kFewWaves);
        }
        for (; t < t_end; t += kFewWaves) {
            // ---- keys that no page is named for read as NaN: a row that sees one shows it.  V's are zeros, as are those of keys outside the range: what lies
            // there may be anything, and a weight of 0 does not silence an infinity.
            if (!__all(named[0] && named[1] && inside[0] && inside[1])) {
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const bool good = named[u] && inside[u];
#pragma unroll
                    for (int n = 0; n < NV; ++n) vr[u][n] = good ? vr[u][n] : u32x4{0, 0, 0, 0};
                }
            }
            // ---- S^T: lane (c16, g4) gets query c16, keys 16 u + 4 g4 + 0 .. 3
            float4v st[MB][2];
#pragma unroll
            for (int mb = 0; mb < MB; ++mb)
#pragma unroll
                for (int u = 0; u < 2; ++u) st[mb][u] = float4v{0.f, 0.f, 0.f, 0.f};
            const bool all_named = __all(named[0] && named[1]);
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) {
                    u32x4 kf;
                    if constexpr (KIND == CACHE_SAME) {
                        kf = kr[u][ks];
                    } else {
                        const u32x4 raw = kr[u][ks >> 1];
                        kf = widen8<BF16, KIND>((ks & 1) ? u32x2{raw[2], raw[3]} : u32x2{raw[0], raw[1]});
                    }
                    if (!all_named) kf = named[u] ? kf : u32x4{kNanPair, kNanPair, kNanPair, kNanPair};
#pragma unroll
                    for (int mb = 0; mb < MB; ++mb) st[mb][u] = mfma16<BF16>(kf, qf[mb][ks], st[mb][u]);
                }
            // ---- V and the scales into LDS
            bool odd = false;                                              // (an infinity or NaN among this lane's values)
            const int base = t * kFewKeys;
            bool clear = true;                                             // every row sees every key of the tile
#pragma unroll
            for (int mb = 0; mb < MB; ++mb) clear = clear && row_lo[mb] <= base && base + kFewKeys <= row_hi[mb];
            clear = __all(clear);
            wavefront_fence();                                             // (the reads of the tile before are done)
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int n = 0; n < NV; ++n) {
                    const uint32_t row = 16 * u + c16;
                    if constexpr (KIND == CACHE_SAME) {
                        if (!clear) odd = odd || any_not_finite<BF16>(vr[u][n]);
                        lds_write16(vt, lds_at<SIZE>(row, 4 * n + g4), vr[u][n]);
                    } else {
                        const u32x4 lo = widen8<BF16, KIND>(u32x2{vr[u][n][0], vr[u][n][1]}), hi = widen8<BF16, KIND>(u32x2{vr[u][n][2], vr[u][n][3]});
                        if (!clear) odd = odd || any_not_finite<BF16>(lo) || any_not_finite<BF16>(hi);
                        lds_write16(vt, lds_at<SIZE>(row, 8 * n + 2 * g4), lo);
                        lds_write16(vt, lds_at<SIZE>(row, 8 * n + 2 * g4 + 1), hi);
                    }
                }
            if constexpr (KIND != CACHE_SAME) {
                scales[wave][lane] = sc;
            }
            const bool careful = !clear && __any(odd);
            wavefront_fence();
            const int next = t + kFewWaves;
            if (next < t_end) {
                fetch(next);
                find(next + kFewWaves);
            }

            // ---- weights
            u32x4 pk[MB];
#pragma unroll
            for (int mb = 0; mb < MB; ++mb) {
                float s[8];
#pragma unroll
                for (int u = 0; u < 2; ++u)
#pragma unroll
                    for (int v = 0; v < 4; ++v) s[4 * u + v] = st[mb][u][v] * g.scale_log2e;
                if constexpr (KIND != CACHE_SAME) {
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        const float4v k4 = *reinterpret_cast<const float4v *>(&scales[wave][16 * u + 4 * g4]);
#pragma unroll
                        for (int v = 0; v < 4; ++v) s[4 * u + v] *= k4[v];
                    }
                }
                if (!clear) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const int32_t key = base + 16 * (j >> 2) + 4 * g4 + (j & 3);
                        s[j] = key >= row_lo[mb] && key < row_hi[mb] ? s[j] : -INFINITY;     // (shares begin and end between tiles)
                    }
                }
                float top = s[0];
#pragma unroll
                for (int j = 1; j < 8; ++j) top = fmaxf(top, s[j]);
                top = fmaxf(top, __shfl_xor(top, 16, 64));
                top = fmaxf(top, __shfl_xor(top, 32, 64));
                const float m_new = fmaxf(m[mb], top), ref = m_new == -INFINITY ? 0.f : m_new;
                const float alpha = __builtin_amdgcn_exp2f(m[mb] - ref);
                m[mb] = m_new;
                float p[8], sum = 0.f;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    p[j] = __builtin_amdgcn_exp2f(s[j] - ref);
                    sum += p[j];
                }
                l[mb] = __builtin_fmaf(l[mb], alpha, sum);
                if constexpr (NORM) {
                    float most = 0.f;                                      // the largest scale that the row sees (fmax passes over NaN)
#pragma unroll
                    for (int u = 0; u < 2; ++u)
#pragma unroll
                        for (int v = 0; v < 4; ++v)
                            if (s[4 * u + v] != -INFINITY) most = fmaxf(most, __builtin_fabsf(scales[wave][kFewKeys + 16 * u + 4 * g4 + v]));
                    most = fmaxf(most, __shfl_xor(most, 16, 64));
                    most = fmaxf(most, __shfl_xor(most, 32, 64));
                    if (__any(most > unit[mb])) {
                        const float grown = most > unit[mb] ? unit_above(most) : unit[mb], shrink = unit[mb] == 0.f ? 0.f : unit[mb] / grown;
                        unit[mb] = grown;
                        per_unit[mb] = grown == 0.f ? 0.f : 1.f / grown;
#pragma unroll
                        for (int db = 0; db < SIZE / 16; ++db) acc[mb][db] = acc[mb][db] * shrink;
                    }
                }
                if (!__all(alpha == 1.f)) {
#pragma unroll
                    for (int db = 0; db < SIZE / 16; ++db) acc[mb][db] = acc[mb][db] * alpha;
                }
                if constexpr (KIND != CACHE_SAME) {
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        const float4v v4 = *reinterpret_cast<const float4v *>(&scales[wave][kFewKeys + 16 * u + 4 * g4]);
#pragma unroll
                        for (int v = 0; v < 4; ++v) {
                            const float x = p[4 * u + v] * (NORM ? v4[v] * per_unit[mb] : v4[v]);
                            p[4 * u + v] = s[4 * u + v] == -INFINITY ? 0.f : x;        // (the scale of a hidden key may be anything)
                        }
                    }
                }
                pk[mb] = u32x4{pack_two<BF16>(p[0], p[1]), pack_two<BF16>(p[2], p[3]), pack_two<BF16>(p[4], p[5]), pack_two<BF16>(p[6], p[7])};
            }
            // ---- O^T += V^T P^T: lane (c16, g4) supplies d = 16 db + c16 and keys 4 g4 + 0 .. 3, 16 + 4 g4 + 0 .. 3; lane i of a group of 16 points the
            // transposing read at key i / 4 of its four, 8 bytes i % 4 of the 32
#pragma unroll
            for (int db = 0; db < SIZE / 16; ++db) {
                const uint32_t row = 4 * g4 + (c16 >> 2), chunk = 2 * db + ((c16 >> 1) & 1), half = (c16 & 1) * 8;
                u32x2 a = lds_read_transposed(vt, lds_at<SIZE>(row, chunk) + half), c = lds_read_transposed(vt, lds_at<SIZE>(row + 16, chunk) + half);
                if (careful) {
                    a = u32x2{without_not_finite<BF16>(a[0]), without_not_finite<BF16>(a[1])};
                    c = u32x2{without_not_finite<BF16>(c[0]), without_not_finite<BF16>(c[1])};
                }
#pragma unroll
                for (int mb = 0; mb < MB; ++mb) acc[mb][db] = mfma16<BF16>(u32x4{a[0], a[1], c[0], c[1]}, pk[mb], acc[mb][db]);
            }
            if (careful) {
                // infinities and NaN of keys that only some rows see: added to those rows alone
#pragma unroll 1
                for (int key = 0; key < kFewKeys; ++key)
#pragma unroll
                    for (int db = 0; db < SIZE / 16; ++db) {
                        u32x2 v;
                        __builtin_memcpy(&v, vt + lds_at<SIZE>(key, 2 * db + (g4 >> 1)) + (g4 & 1) * 8, 8);
#pragma unroll
                        for (int mb = 0; mb < MB; ++mb) {
                            const bool sees = base + key >= row_lo[mb] && base + key < row_hi[mb];
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const float x = only_not_finite(widen_one<BF16>(v[e >> 1], e & 1));
                                acc[mb][db][e] += sees ? x : 0.f;
                            }
                        }
                    }
            }
        }

        // ---- the wavefronts' results to a common maximum: through LDS, row by row
        float *ex = reinterpret_cast<float *>(vt);
        wavefront_fence();
#pragma unroll
        for (int mb = 0; mb < MB; ++mb) {
            l[mb] += __shfl_xor(l[mb], 16, 64);
            l[mb] += __shfl_xor(l[mb], 32, 64);
            if (lane < 16) {
                red_m[wave][16 * mb + lane] = m[mb];
                red_l[wave][16 * mb + lane] = l[mb];
            }
#pragma unroll
            for (int db = 0; db < SIZE / 16; ++db) {
                float4v v = acc[mb][db];
                if constexpr (NORM) v = v * unit[mb];
                *reinterpret_cast<float4v *>(ex + (16 * mb + c16) * SIZE + 16 * db + 4 * g4) = v;
            }
        }
        __syncthreads();
        for (int e = threadIdx.x; e < 16 * MB * (SIZE / 4); e += 64 * kFewWaves) {
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
