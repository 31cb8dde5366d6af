// lamp_cache_few.h -- attention over the 8-bit paged cache for few query rows of
// one sequence and kv head: single tokens and short chunks (the mathematics in
// lamp_cache_attn.hip; library-internal, device code).
#pragma once
#include "lamp_cache_plan.h"

namespace lamp {
namespace {

// One unit: FewRows::ROWS query rows (row = token * G + head of the group) of one
// sequence and kv head against one piece of its keys; the waves take key
// tiles of KT in turn, each with its own m, l and o, and join them at the end.
//
// The transposed products S^T = K Q^T and O^T = V^T P^T (16x16x32) leave a
// lane (row n = lane % 16, g = lane / 16) with the logits of the KT/4
// consecutive keys from g KT/4, which is what it then holds as P^T's operand:
// P moves through no LDS.  For that, row m of the K operand t is key
// (m / 4) KT/4 + 4 t + m % 4, and both products take their summed axis in the
// order that makes a lane's bytes contiguous: K's channels g D/4 .. of a key,
// V's KT/4 keys of a channel (V is stored transposed within its page).  Codes
// go from global memory straight to registers in 16-byte loads; the next
// tile's are requested as soon as this tile's have been used.  Bound by HBM
// (32 x 8192 keys, d = 128: 537 MB in 97 us, 5.5 TB/s where a large copy reaches
// 5.1), for one sequence by the latencies of lengths, table and codes, one after
// another (20011 keys, 41 MB: 13 us; 37 tokens: 6).  Tiles of 64 keys (32 at d =
// 256, for registers): with tiles of 32 the 32 x 8192 keys take 6 % longer; with
// three workgroups a CU instead of two registers spill (62 %).
template <int D, int WAVES>
struct FewShared {
    float o[WAVES * 16 * (D + 4)];
    float ml[WAVES * 16 * 2];
    uint32_t marks[FewRows::ROWS][D / 32];   // rows and channels that see NaN values (mark_nan)
};

template <int D, int KT, int WAVES>
__device__ __forceinline__ void cache_few(const CacheAttnParams &p, int x, FewShared<D, WAVES> &sh)
{
    constexpr int NT = KT / 16;        // K operands of a tile
    constexpr int KPL = KT / 4;        // keys of a lane
    constexpr int KW = D / 16;         // words of a lane's channels of one key
    constexpr int VW = KPL / 4;        // words of a lane's keys of one channel
    constexpr int DT = D / 16;         // 16-channel tiles of o
    constexpr int OS = D + 4;          // row stride of the joining buffer
    float *obuf = sh.o, *ml = sh.ml;

    const int G = p.Hq / p.b.Hkv;
    const Unit u = find_unit<FewRowsOf<WAVES>>(p, G, x);
    if (u.s < 0) return;
    const SeqPlan sq = seq_plan<FewRows>(p, u.s, G);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), n = lane & 15, g = lane >> 4;
    if (threadIdx.x < FewRows::ROWS * (D / 32)) sh.marks[0][threadIdx.x] = 0;
    __syncthreads();
    const int rows = sq.n * G;
    const int r0 = u.tile * FewRows::ROWS, rlast = (r0 + FewRows::ROWS < rows ? r0 + FewRows::ROWS : rows) - 1;
    write_info<FewRows>(p, u, sq.a, r0, rlast + 1 - r0);
    const int row = r0 + n < rows ? r0 + n : rlast;   // (missing rows repeat the last, and are not written)
    const int tok = row / G, qh = u.head * G + row - tok * G;
    const int pos = sq.pos0 + tok;                    // may be negative: sees nothing
    const int pmin = sq.pos0 + r0 / G, pmax = sq.pos0 + rlast / G;
    // keys that a position sees: this row's, those that some row sees, that every row sees
    auto upto = [&](int x) { return p.causal ? (x + 1 < sq.len ? x + 1 : sq.len) : sq.len; };
    auto from = [&](int x) { return p.window > 0 && x - p.window + 1 > 0 ? x - p.window + 1 : 0; };
    const int hi = upto(pos), lo = from(pos);
    const int hi_any = upto(pmax), lo_any = from(pmin), hi_all = upto(pmin), lo_all = from(pmax);
    const int t0 = lo_any / KT, t1 = hi_any > lo_any ? (hi_any + KT - 1) / KT : t0;
    const int beg = __builtin_amdgcn_readfirstlane(t0 + (int)((int64_t)(t1 - t0) * u.piece / u.pieces));
    const int end = __builtin_amdgcn_readfirstlane(t0 + (int)((int64_t)(t1 - t0) * (u.piece + 1) / u.pieces));

    bf16x8 qf[D / 32];
    {
        const uint16_t *q = p.q + (int64_t)(sq.a + tok) * p.q_st + (int64_t)qh * p.q_sh + g * (D / 4);
#pragma unroll
        for (int k = 0; k < D / 32; ++k) qf[k] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4 *>(q + 8 * k));
    }

    const int *table = p.b.table + u.s * p.b.table_stride;
    const int ps = p.b.page_shift, pmask = (1 << ps) - 1;
    // page of the KPL keys from `key` (a page holds them whole): as the table has it (not looked at before its first use, a tile
    // on), or UNSEEN by every row
    constexpr int UNSEEN = INT_MIN;
    auto page_at = [&](int key) {
        int pg = UNSEEN;
        if (key < hi_any && key + KPL > lo_any) pg = table[key >> ps];
        return pg;
    };
    auto held = [&](int pg) { return pg >= 0 && pg < p.b.pages; };   // (otherwise UNSEEN or missing)
    const int kgrp = ((n >> 2) * KPL);   // the lane's key group as a row of K, its first key in the tile
    uint32_t kreg[NT][KW], vreg[DT][VW];
    float kscale = 0.0f, vscale = 0.0f;
    int pgk, pgv;
    bool bad = false;   // the lane's keys (of V) are in a missing page

    auto load_k = [&](int t) {
        const int key = t * KT + kgrp + (n & 3);
        const uint8_t *c = p.kc + ((int64_t)(held(pgk) ? pgk : 0) * p.b.Hkv + u.head) * ((int64_t)D << ps)
                           + (int64_t)(key & pmask) * D + g * (D / 4);
#pragma unroll
        for (int i = 0; i < NT; ++i)
#pragma unroll
            for (int w = 0; w < KW; w += 4) {
                const u32x4 x = *reinterpret_cast<const u32x4 *>(c + 4 * i * D + 4 * w);
#pragma unroll
                for (int e = 0; e < 4; ++e) kreg[i][w + e] = x[e];
            }
    };
    auto load_v = [&](int t) {
        const bool is = held(pgv);
        const int64_t at = (int64_t)(is ? pgv : 0) * p.b.Hkv + u.head;
        bad = !is && pgv != UNSEEN;
        kscale = p.ks[at] * p.scale_log2;
        vscale = is ? p.vs[at] : 1.0f;   // (its probabilities are 0 or NaN)
        const uint8_t *c = p.vc + at * ((int64_t)D << ps) + (int64_t)n * (1 << ps) + ((t * KT + g * KPL) & pmask);
#pragma unroll
        for (int i = 0; i < DT; ++i) {
            const uint8_t *ci = c + ((int64_t)(16 * i) << ps);
            if constexpr (VW == 4) {
                const u32x4 x = *reinterpret_cast<const u32x4 *>(ci);
#pragma unroll
                for (int e = 0; e < 4; ++e) vreg[i][e] = x[e];
            } else {
                const u32x2 x = *reinterpret_cast<const u32x2 *>(ci);
                vreg[i][0] = x[0];
                vreg[i][1] = x[1];
            }
        }
    };

    f32x4 o[DT];
#pragma unroll
    for (int i = 0; i < DT; ++i) o[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
    // l: of this lane's keys.  A row that sees keys beyond the table's reach is NaN.
    float m = hi > lo ? LOWEST : NEG_INF, l = (p.causal && pos + 1 < sq.all ? pos + 1 : sq.all) > sq.len ? __builtin_nanf("") : 0.0f;

    int t = beg + wave;
    if (t < end) {
        pgk = page_at(t * KT + kgrp);
        pgv = page_at(t * KT + g * KPL);
        load_k(t);
        load_v(t);
    }
    for (; t < end; t += WAVES) {
        const int next = t + WAVES;
        if (next < end) {
            pgk = page_at(next * KT + kgrp);
            pgv = page_at(next * KT + g * KPL);
        }
        f32x4 acc[NT];
#pragma unroll
        for (int i = 0; i < NT; ++i) {
            acc[i] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int k = 0; k < D / 32; ++k)
                acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen(kreg[i][2 * k], kreg[i][2 * k + 1]), qf[k], acc[i], 0, 0, 0);
        }
        if (next < end) load_k(next);
        const int key0 = t * KT + g * KPL;   // the lane's keys: key0 + 4 i + e
        const bool partial = t * KT < lo_all || t * KT + KT > hi_all || __ballot(bad) != 0;   // (of the whole wave)
        float x[KPL];
#pragma unroll
        for (int i = 0; i < NT; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) x[4 * i + e] = acc[i][e] * kscale;
        if (partial) {
#pragma unroll
            for (int i = 0; i < KPL; ++i) {
                const int key = key0 + i;
                x[i] = key < lo || key >= hi ? NEG_INF : (bad ? __builtin_nanf("") : x[i]);
            }
        }
        float mt = x[0];
#pragma unroll
        for (int i = 1; i < KPL; ++i) mt = fmaxf(mt, x[i]);
        mt = fmaxf(mt, __shfl_xor(mt, 16, 64));
        mt = fmaxf(mt, __shfl_xor(mt, 32, 64));
        const float mn = fmaxf(m, mt);
        const float ms = mn == NEG_INF ? 0.0f : mn;   // (a row that has seen no key yet)
        const float alpha = __builtin_amdgcn_exp2f(m - ms);
        m = mn;
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < KPL; ++i) {
            x[i] = __builtin_amdgcn_exp2f(x[i] - ms);
            sum += x[i];
        }
        l = l * alpha + sum;
        if (__ballot(alpha != 1.0f)) {
#pragma unroll
            for (int i = 0; i < DT; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[i][e] *= alpha;
        }
        bf16x8 pf[KPL / 8];
#pragma unroll
        for (int k = 0; k < KPL / 8; ++k) {
            u32x4 w;
#pragma unroll
            for (int e = 0; e < 4; ++e) w[e] = pack2(x[8 * k + 2 * e] * vscale, x[8 * k + 2 * e + 1] * vscale);
            pf[k] = __builtin_bit_cast(bf16x8, w);
        }
        if (partial) {
            // Values that no row sees (behind the sequence's end, before the
            // window, of a missing page) are whatever memory holds: zeroed, as
            // 0 * NaN is NaN; NaN that some rows see is marked.
            uint32_t some = 0;
#pragma unroll
            for (int w = 0; w < VW; ++w) {
                const uint32_t see = bad ? 0u : byte_mask(key0 + 4 * w, lo_any, hi_any);
#pragma unroll
                for (int i = 0; i < DT; ++i) {
                    vreg[i][w] &= see;
                    some |= nan_bytes(vreg[i][w]);
                }
            }
            if (some) {
#pragma unroll
                for (int i = 0; i < DT; ++i)
#pragma unroll
                    for (int w = 0; w < VW; ++w) {
                        const uint32_t nan = nan_bytes(vreg[i][w]);
                        mark_nan<D>(sh.marks, nan, 16 * i + n, key0 + 4 * w, rlast + 1 - r0, [&](int r, int key) {
                            const int rp = sq.pos0 + (r0 + r) / G;
                            return key >= from(rp) && key < upto(rp);
                        });
                        vreg[i][w] &= ~((nan >> 7) * 0xFFu);
                    }
            }
        }
#pragma unroll
        for (int i = 0; i < DT; ++i)
#pragma unroll
            for (int k = 0; k < KPL / 8; ++k)
                o[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen(vreg[i][2 * k], vreg[i][2 * k + 1]), pf[k], o[i], 0, 0, 0);
        if (next < end) {
            load_v(next);
        }
    }

    // join the waves
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);
    if (g == 0) {
        ml[(wave * 16 + n) * 2] = m;
        ml[(wave * 16 + n) * 2 + 1] = l;
    }
#pragma unroll
    for (int i = 0; i < DT; ++i) *reinterpret_cast<f32x4 *>(&obuf[(wave * 16 + n) * OS + 16 * i + 4 * g]) = o[i];
    __syncthreads();
    for (int at = threadIdx.x * 4; at < 16 * D; at += 256 * WAVES) {
        const int r = at / D, d = at - r * D;
        if (r0 + r >= rows) continue;
        float mx = NEG_INF;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) mx = fmaxf(mx, ml[(w * 16 + r) * 2]);
        const float ms = mx == NEG_INF ? 0.0f : mx;
        float sum = 0.0f;
        f32x4 v = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const float f = __builtin_amdgcn_exp2f(ml[(w * 16 + r) * 2] - ms);
            sum += ml[(w * 16 + r) * 2 + 1] * f;
            const f32x4 ow = *reinterpret_cast<const f32x4 *>(&obuf[(w * 16 + r) * OS + d]);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] += ow[e] * f;
        }
        const uint32_t nan = sh.marks[r][d >> 5] >> (d & 31);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = nan >> e & 1u ? __builtin_nanf("") : v[e];
        if (u.pieces > 1) {
            const int64_t at_row = (int64_t)u.slot * FewRows::ROWS + r;
            *reinterpret_cast<f32x4 *>(p.part[0] + at_row * D + d) = v;
            if (d == 0) {
                p.part_ml[0][at_row * 2] = mx;
                p.part_ml[0][at_row * 2 + 1] = sum;
            }
        } else {
            const int gr = r0 + r, i = gr / G;
            const int64_t orow = (int64_t)(sq.a + i) * p.Hq + u.head * G + gr - i * G;
            const float inv = finish(mx, sum);
            *reinterpret_cast<u32x2 *>(p.o + orow * D + d) = u32x2{pack2(v[0] * inv, v[1] * inv), pack2(v[2] * inv, v[3] * inv)};
            if (d == 0) p.lse[orow] = finish_lse(mx, sum);
        }
    }
}

} // namespace
} // namespace lamp
