// lamp_cache_attn.hip -- attention of a ragged batch of new tokens over the
// 8-bit paged cache.
//
// Row (token i of sequence s, head h) sees keys j < kv_lens[s] with, causal,
// j <= p and, windowed, j > p - window, p the token's position:
//   l_j = scale ks_j (q . kcode_j),  P = softmax(l),  o = sum_j P_j vs_j vcode_j,
// ks_j, vs_j the scales of the key's page.  e4m3 codes are exact in bf16, so
// q.k and P.v run on the bf16 matrix cores with fp32 accumulation and the
// scales apply to the fp32 logits and probabilities.  One pass with the running
// maximum m and sum l of the softmax in fp32 (base-2 exponentials of logits
// pre-multiplied by log2 e).  P_j vs_j is rounded to bf16 for the matrix cores
// (at most 2^-9 relative per term, below the bf16 output's own 2^-9); the sum l
// is of the unrounded probabilities.
#include <hip/hip_runtime.h>

#include "lamp_serve.h"

namespace lamp {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr float NEG_INF = -__builtin_inff();
constexpr int TILE = 64;       // keys of the plan's tiles
constexpr int MIN_TILES = 4;   // least tiles of a piece (one a wave)
constexpr int TARGET = 512;    // workgroups that fill the 256 CUs (two fit in each one's registers)

// The key range of one sequence is cut in pieces when its row tiles alone do
// not fill the device: with `total` the key tiles of all (sequence, row tile,
// kv head) triples, pieces hold about total / TARGET tiles.  Every workgroup
// works the plan out for itself from the lengths (no planning launch, and a
// captured graph follows lengths that change).
struct Unit {
    int s;           // sequence (-1: none)
    int tile, head;  // row tile, kv head
    int piece, pieces;
    int slot;        // partial output (first piece's slot + piece) where pieces > 1
};

struct SeqPlan {
    int a, n;        // first new token, new tokens
    int all, len;    // keys, and those in the table's reach
    int pos0;        // position of the first new token
    int tiles;       // row tiles
    int kt;          // key tiles that a row tile visits at most
};

__device__ __forceinline__ SeqPlan seq_plan(const CacheAttnParams &p, int s, int G)
{
    SeqPlan r;
    r.a = p.b.q_start ? p.b.q_start[s] : s;
    const int e = p.b.q_start ? p.b.q_start[s + 1] : s + 1;
    const int len = p.b.kv_lens[s] > 0 ? p.b.kv_lens[s] : 0;
    r.n = r.a >= 0 && e <= p.b.T && e > r.a ? e - r.a : 0;
    r.pos0 = len - r.n;
    const int64_t reach = (int64_t)p.b.width << p.b.page_shift;
    r.all = len;
    r.len = len < reach ? len : (int)reach;
    r.tiles = (int)(((int64_t)r.n * G + CACHE_ROWS - 1) / CACHE_ROWS);
    r.kt = (r.len + TILE - 1) / TILE;
    if (p.window > 0) {
        const int64_t span = ((int64_t)p.window + CACHE_ROWS - 1 + TILE - 1) / TILE + 1;
        if (span < r.kt) r.kt = (int)span;
    }
    return r;
}

__device__ __forceinline__ int64_t wave_sum(int64_t v)
{
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) v += __shfl_xor(v, m, 64);
    return v;
}

// Tiles of a piece, from the lengths of every sequence (by one wave).
__device__ int piece_tiles(const CacheAttnParams &p, int G)
{
    int64_t total = 0;
    for (int s = threadIdx.x & 63; s < p.b.S; s += 64) {
        const SeqPlan r = seq_plan(p, s, G);
        total += (int64_t)r.tiles * r.kt;
    }
    total = wave_sum(total) * p.b.Hkv;
    const int64_t c = (total + TARGET - 1) / TARGET;
    return (int)(c < MIN_TILES ? MIN_TILES : (c < 1 << 24 ? c : 1 << 24));
}

// Unit x of the plan; with `joined`, unit x among the (row tile, kv head) pairs
// of split sequences instead (piece 0, slot of the first piece).
__device__ Unit find_unit(const CacheAttnParams &p, int G, int64_t x, bool joined)
{
    const int lane = threadIdx.x & 63;
    const int chunk = piece_tiles(p, G);
    int64_t units = 0, slots = 0;   // of the sequences before this round of 64
    for (int s0 = 0; s0 < p.b.S; s0 += 64) {
        const int s = s0 + lane;
        int64_t pairs = 0;
        int c = 1;
        if (s < p.b.S) {
            const SeqPlan r = seq_plan(p, s, G);
            pairs = (int64_t)r.tiles * p.b.Hkv;
            c = (r.kt + chunk - 1) / chunk;
            c = c < 1 ? 1 : c;
        }
        const int64_t u = joined ? (c > 1 ? pairs : 0) : pairs * c, sl = c > 1 ? pairs * c : 0;
        int64_t ui = u, si = sl;   // inclusive prefix sums
#pragma unroll
        for (int m = 1; m < 64; m <<= 1) {
            const int64_t a = __shfl_up(ui, m, 64), b = __shfl_up(si, m, 64);
            if (lane >= m) ui += a, si += b;
        }
        const uint64_t hit = __ballot(x < units + ui);
        if (hit) {
            const int l = __builtin_ctzll(hit);   // the first sequence that ends behind x
            const int64_t local = x - (units + __shfl(ui - u, l, 64));
            const int64_t slot0 = slots + __shfl(si - sl, l, 64);
            const int cs = __shfl(c, l, 64);
            Unit r;
            r.s = s0 + l;
            r.pieces = cs;
            r.piece = joined ? 0 : (int)(local % cs);
            const int64_t pair = joined ? local : local / cs;
            r.head = (int)(pair % p.b.Hkv);
            r.tile = (int)(pair / p.b.Hkv);
            const int64_t slot = slot0 + pair * cs + r.piece;
            if (cs > 1 && slot + (joined ? cs : 1) > p.slots) break;   // (lengths that break the contract)
            r.slot = (int)slot;
            return r;
        }
        units += __shfl(ui, 63, 64);
        slots += __shfl(si, 63, 64);
    }
    return {-1, 0, 0, 0, 0, 0};
}

__device__ __forceinline__ uint32_t pack2(float a, float b)
{
    bf16x2 v;
    v[0] = (__bf16)a;
    v[1] = (__bf16)b;
    return __builtin_bit_cast(uint32_t, v);
}

// 8 codes as bf16 (exact).
__device__ __forceinline__ bf16x8 widen(uint32_t lo, uint32_t hi)
{
    u32x4 r;
    r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false));
    r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true));
    r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false));
    r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true));
    return __builtin_bit_cast(bf16x8, r);
}

// The high bit of each byte that holds the NaN code (0x7F or 0xFF).
__device__ __forceinline__ uint32_t nan_bytes(uint32_t c)
{
    return ((c & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u;
}

// Bytes of a word of 4 keys from `k` that lie in [lo, hi).
__device__ __forceinline__ uint32_t byte_mask(int k, int lo, int hi)
{
    const int a = lo - k, e = hi - k;
    const uint32_t below = e >= 4 ? ~0u : (e <= 0 ? 0u : (1u << (8 * e)) - 1u);
    const uint32_t from = a <= 0 ? ~0u : (a >= 4 ? 0u : ~0u << (8 * a));
    return below & from;
}

// One unit: CACHE_ROWS query rows (row = token * G + head of the group) of one
// sequence and kv head against one piece of its keys; the 4 waves take key
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
// tile's are requested as soon as this tile's have been used.
template <int D, int KT>
__global__ __launch_bounds__(256) void cache_attn_kernel(CacheAttnParams p)
{
    constexpr int NT = KT / 16;        // K operands of a tile
    constexpr int KPL = KT / 4;        // keys of a lane
    constexpr int KW = D / 16;         // words of a lane's channels of one key
    constexpr int VW = KPL / 4;        // words of a lane's keys of one channel
    constexpr int DT = D / 16;         // 16-channel tiles of o
    constexpr int OS = D + 4;          // row stride of the joining buffer
    __shared__ float obuf[4 * 16 * OS];
    __shared__ float ml[4 * 16 * 2];

    const int G = p.Hq / p.b.Hkv;
    const Unit u = find_unit(p, G, blockIdx.x, false);
    if (u.s < 0) return;
    const SeqPlan sq = seq_plan(p, u.s, G);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = lane & 15, g = lane >> 4;
    const int rows = sq.n * G;
    const int r0 = u.tile * CACHE_ROWS, rlast = (r0 + CACHE_ROWS < rows ? r0 + CACHE_ROWS : rows) - 1;
    const int row = r0 + n < rows ? r0 + n : rlast;   // (missing rows repeat the last, and are not written)
    const int tok = row / G, qh = u.head * G + row - tok * G;
    const int pos = sq.pos0 + tok;                    // may be negative: sees nothing
    const int pmin = sq.pos0 + r0 / G, pmax = sq.pos0 + rlast / G;
    // keys that this row sees, that some row sees, that every row sees
    const int hi = p.causal ? (pos + 1 < sq.len ? pos + 1 : sq.len) : sq.len;
    const int lo = p.window > 0 && pos - p.window + 1 > 0 ? pos - p.window + 1 : 0;
    const int hi_any = p.causal ? (pmax + 1 < sq.len ? pmax + 1 : sq.len) : sq.len;
    const int lo_any = p.window > 0 && pmin - p.window + 1 > 0 ? pmin - p.window + 1 : 0;
    const int hi_all = p.causal ? (pmin + 1 < sq.len ? pmin + 1 : sq.len) : sq.len;
    const int lo_all = p.window > 0 && pmax - p.window + 1 > 0 ? pmax - p.window + 1 : 0;
    const int t0 = lo_any / KT, t1 = hi_any > lo_any ? (hi_any + KT - 1) / KT : t0;
    const int beg = t0 + (int)((int64_t)(t1 - t0) * u.piece / u.pieces);
    const int end = t0 + (int)((int64_t)(t1 - t0) * (u.piece + 1) / u.pieces);

    bf16x8 qf[D / 32];
    {
        const uint16_t *q = p.q + (int64_t)(sq.a + tok) * p.q_st + (int64_t)qh * p.q_sh + g * (D / 4);
#pragma unroll
        for (int k = 0; k < D / 32; ++k) qf[k] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4 *>(q + 8 * k));
    }

    const int *table = p.b.table + u.s * p.b.table_stride;
    const int ps = p.b.page_shift, pmask = (1 << ps) - 1;
    // page of the KPL keys from `key` (a page holds them whole): UNSEEN by every row, or MISSING where the table names none
    constexpr int UNSEEN = -2, MISSING = -1;
    auto page_at = [&](int key) {
        if (key >= hi_any || key + KPL <= lo_any) return UNSEEN;
        const int pg = table[key >> ps];
        return pg >= 0 && pg < p.b.pages ? pg : MISSING;
    };
    const int kgrp = ((n >> 2) * KPL);   // the lane's key group as a row of K, its first key in the tile
    uint32_t kreg[NT][KW], vreg[DT][VW];
    float kscale = 0.0f, vscale = 0.0f;
    int pgk, pgv;

    auto load_k = [&](int t) {
        const int key = t * KT + kgrp + (n & 3);
        const uint8_t *c = p.kc + ((int64_t)(pgk < 0 ? 0 : pgk) * p.b.Hkv + u.head) * ((int64_t)D << ps)
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
        const int64_t at = (int64_t)(pgv < 0 ? 0 : pgv) * p.b.Hkv + u.head;
        kscale = p.ks[at] * p.scale_log2;
        vscale = pgv < 0 ? 1.0f : p.vs[at];   // (its probabilities are 0 or NaN)
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
    float m = NEG_INF, l = (p.causal && pos + 1 < sq.all ? pos + 1 : sq.all) > sq.len ? __builtin_nanf("") : 0.0f;

    int t = beg + wave;
    bool bad = false;
    if (t < end) {
        pgk = page_at(t * KT + kgrp);
        pgv = page_at(t * KT + g * KPL);
        load_k(t);
        load_v(t);
        bad = pgv == MISSING;
    }
    for (; t < end; t += 4) {
        const int next = t + 4;
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
            // window, of a missing page) are whatever memory holds: zero them,
            // as 0 * NaN is NaN.  Values that some rows see may hold NaN for
            // the others: those are zeroed too and counted by row and channel.
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
            if (__ballot(some != 0)) {
                bf16x8 vis[KPL / 8];
#pragma unroll
                for (int k = 0; k < KPL / 8; ++k) {
                    u32x4 w;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int key = key0 + 8 * k + 2 * e;
                        w[e] = (key >= lo && key < hi ? 0x3F80u : 0u) | (key + 1 >= lo && key + 1 < hi ? 0x3F800000u : 0u);
                    }
                    vis[k] = __builtin_bit_cast(bf16x8, w);
                }
#pragma unroll
                for (int i = 0; i < DT; ++i) {
                    f32x4 count = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
                    for (int k = 0; k < KPL / 8; ++k) {
                        uint32_t one[2];
#pragma unroll
                        for (int w = 0; w < 2; ++w) {
                            const uint32_t b = nan_bytes(vreg[i][2 * k + w]);
                            one[w] = (b >> 7) * 0x38u;   // e4m3 1.0 where NaN
                            vreg[i][2 * k + w] &= ~((b >> 7) * 0xFFu);
                        }
                        count = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen(one[0], one[1]), vis[k], count, 0, 0, 0);
                    }
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[i][e] = count[e] > 0.0f ? __builtin_nanf("") : o[i][e];
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
            bad = pgv == MISSING;
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
    for (int at = threadIdx.x * 4; at < 16 * D; at += 1024) {
        const int r = at / D, d = at - r * D;
        if (r0 + r >= rows) continue;
        float mx = NEG_INF;
#pragma unroll
        for (int w = 0; w < 4; ++w) mx = fmaxf(mx, ml[(w * 16 + r) * 2]);
        const float ms = mx == NEG_INF ? 0.0f : mx;
        float sum = 0.0f;
        f32x4 v = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const float f = __builtin_amdgcn_exp2f(ml[(w * 16 + r) * 2] - ms);
            sum += ml[(w * 16 + r) * 2 + 1] * f;
            const f32x4 ow = *reinterpret_cast<const f32x4 *>(&obuf[(w * 16 + r) * OS + d]);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] += ow[e] * f;
        }
        if (u.pieces > 1) {
            const int64_t at_row = (int64_t)u.slot * CACHE_ROWS + r;
            *reinterpret_cast<f32x4 *>(p.part + at_row * D + d) = v;
            if (d == 0) {
                p.part_ml[at_row * 2] = mx;
                p.part_ml[at_row * 2 + 1] = sum;
            }
        } else {
            const int gr = r0 + r, i = gr / G;
            const int64_t orow = (int64_t)(sq.a + i) * p.Hq + u.head * G + gr - i * G;
            const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
            *reinterpret_cast<u32x2 *>(p.o + orow * D + d) = u32x2{pack2(v[0] * inv, v[1] * inv), pack2(v[2] * inv, v[3] * inv)};
            if (d == 0) p.lse[orow] = sum == 0.0f ? NEG_INF : (mx + __builtin_amdgcn_logf(sum)) * 0.6931471805599453f;
        }
    }
}

// The pieces of one row tile and kv head joined; 4 rows to a workgroup, one a
// wave, whose lanes hold D/64 channels each.
template <int D>
__global__ __launch_bounds__(256) void cache_join_kernel(CacheAttnParams p)
{
    constexpr int C = D / 64;
    const int G = p.Hq / p.b.Hkv;
    const Unit u = find_unit(p, G, blockIdx.x, true);
    if (u.s < 0) return;
    const SeqPlan sq = seq_plan(p, u.s, G);
    const int lane = threadIdx.x & 63, r = (int)blockIdx.y * 4 + (threadIdx.x >> 6), gr = u.tile * CACHE_ROWS + r;
    if (gr >= sq.n * G) return;
    const int64_t base = (int64_t)u.slot * CACHE_ROWS + r;
    float mx = NEG_INF;
    for (int c = lane; c < u.pieces; c += 64) mx = fmaxf(mx, p.part_ml[(base + (int64_t)c * CACHE_ROWS) * 2]);
#pragma unroll
    for (int k = 1; k < 64; k <<= 1) mx = fmaxf(mx, __shfl_xor(mx, k, 64));
    const float ms = mx == NEG_INF ? 0.0f : mx;
    float sum = 0.0f, v[C] = {};
    for (int c = 0; c < u.pieces; ++c) {
        const int64_t at = base + (int64_t)c * CACHE_ROWS;
        const float f = __builtin_amdgcn_exp2f(p.part_ml[at * 2] - ms);
        sum += p.part_ml[at * 2 + 1] * f;
#pragma unroll
        for (int k = 0; k < C; ++k) v[k] += p.part[at * D + 64 * k + lane] * f;
    }
    const int i = gr / G;
    const int64_t orow = (int64_t)(sq.a + i) * p.Hq + u.head * G + gr - i * G;
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
#pragma unroll
    for (int k = 0; k < C; ++k) {
        const uint32_t b = pack2(v[k] * inv, 0.0f);
        p.o[orow * D + 64 * k + lane] = (uint16_t)b;
    }
    if (lane == 0) p.lse[orow] = sum == 0.0f ? NEG_INF : (mx + __builtin_amdgcn_logf(sum)) * 0.6931471805599453f;
}

// Row tiles times kv heads that the batch can have at most.
int64_t max_pairs(const CacheAttnParams &p)
{
    const int G = p.Hq / p.b.Hkv;
    return ((int64_t)p.b.T * G / CACHE_ROWS + p.b.S) * p.b.Hkv;
}

// A sequence of kt key tiles and `pairs` row tiles times heads is cut in
// c = ceil(kt / chunk) < 1 + kt / chunk pieces, and sum(pairs kt) / chunk <=
// TARGET: below max_pairs + TARGET units in all.
template <int D, int KT>
hipError_t launch(const CacheAttnParams &p, hipStream_t s)
{
    const int64_t pairs = max_pairs(p);
    cache_attn_kernel<D, KT><<<dim3((unsigned)(p.slots ? pairs + TARGET : pairs)), 256, 0, s>>>(p);
    if (p.slots) {
        const dim3 grid((unsigned)(pairs < TARGET ? pairs : TARGET), CACHE_ROWS / 4);
        cache_join_kernel<D><<<grid, 256, 0, s>>>(p);
    }
    return hipGetLastError();
}

} // namespace

// Where c >= 2, c < 2 kt / chunk: below 2 TARGET partial outputs, of below
// TARGET row tiles times heads.  Sequences of one piece need none.
int cache_attn_slots(int64_t keys)
{
    return (keys + TILE - 1) / TILE > MIN_TILES ? 2 * TARGET : 0;
}

hipError_t launch_cache_attn(int D, const CacheAttnParams &p, hipStream_t s)
{
    switch (D) {
    case 64: return launch<64, 64>(p, s);
    case 128: return launch<128, 64>(p, s);
    default: return launch<256, 32>(p, s);
    }
}

} // namespace lamp
