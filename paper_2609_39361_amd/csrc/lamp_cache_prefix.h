// lamp_cache_prefix.h -- attention over the 8-bit paged cache where all query rows see
// a whole range of keys: the new tokens of a group of sequences and their shared
// prefix (the mathematics in lamp_cache_attn.hip; library-internal, device code).
#pragma once
#include "lamp_cache_plan.h"

namespace lamp {
namespace {

// One unit: 32 query rows of a group and kv head against one piece of the prefix;
// the 4 waves take key tiles of KT in turn, each with its own m, l and o, and join
// them at the end.
//
// The transposed products S^T = K Q^T and O^T = V^T P^T (32x32x16) leave a lane
// (row n = lane % 32, h = lane / 32) with the logits of the KT/2 consecutive keys
// from h KT/2, 8 for each step of 16 keys of the second product, which is what it
// holds as P^T's operand.  For that, row m of the K operand b is key key_of(m, b),
// and both products take their summed axis in the order that makes a lane's bytes
// contiguous: K's channels h D/2 .. of a key, V's KT/2 keys of a channel.
//
// A wave loads a tile's codes in the order of memory (64 lanes, 1 KB), keeps them in
// registers until they are due, and passes them through a stretch of LDS of its own, K
// first, then V, with rows a 16-byte unit longer than their bytes (and the upper half
// of the keys 64 bytes on), so that 8 lanes reading a unit of their rows use all
// banks.  No barrier is needed until the waves join: a wave's accesses of LDS are
// executed in order, and the compiler is kept to it.  Nothing is masked but whole
// groups of 16 keys behind the prefix's end, which is a page's.
//
// Bound by issue (d = 128): a tile's 290 vector and 32 matrix instructions take a wave
// 1.85 us alone on its SIMD and 2.8 beside another (lanes that read rows of their own
// straight into operands: 3.0), whatever the caches hold: touching L2 a tile ahead
// gained nothing.  64 tokens of 32/8 heads behind 8192 shared keys and 20 to 1500 of
// their own: 33 us with the form for few rows beside it (all in that form: 51).
template <int D, int KT>
struct PrefixShared {
    static constexpr int DC = D == 128 ? 128 : 64;      // channels joined at a time (two workgroups a CU hold theirs)
    static constexpr int KROW = D + 16, VROW = KT + 16; // bytes of a row
    static constexpr int STAGE = KT * KROW + 64 > D * VROW ? KT * KROW + 64 : D * VROW;
    union {
        u32x4 stage[4][STAGE / 16];
        float o[4 * 32 * (DC + 4)];
    };
    float ml[4 * 32 * 2];
    u32x4 q[D > 128 ? D / 16 : 1][D > 128 ? 64 : 1];    // d = 256: the operands of the queries (registers hold the rest)
};

// NPG: pages of a tile (1: a page holds whole tiles).
template <int D, int KT, int NPG>
__device__ __forceinline__ void cache_prefix(const SharedAttnParams &p, int x, PrefixShared<D, KT> &sh)
{
    typedef PrefixShared<D, KT> SH;
    constexpr int WAVES = 4, NB = KT / 32, DB = D / 32, KS = D / 16, DC = SH::DC, OS = DC + 4;
    constexpr int NL = KT * D / 1024;              // loads of K, and of V, of a tile
    constexpr int PAGE = KT / NPG;                 // keys of a page, where a tile has several
    constexpr bool QLDS = D > 128;
    constexpr float LAZY = 8.0f;                   // the running maximum is raised when a logit passes it by this (as in lamp_cache_many.h)
    const int G = p.Hq / p.b.Hkv;
    Unit u;
    SeqPlan sq;
    locate<PrefixRows>(p, G, x, u, sq);
    if (u.s < 0) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), n = lane & 31, h = lane >> 5;
    auto same = [](int v) { return __builtin_amdgcn_readfirstlane(v); };
    const int len = same(sq.len), rows = sq.n * G, r0 = u.tile * PrefixRows::ROWS;
    const int here = rows - r0 < PrefixRows::ROWS ? rows - r0 : PrefixRows::ROWS;
    write_info<PrefixRows>(p, u, sq, r0, here);
    const int row = r0 + (n < here ? n : here - 1);   // (missing rows repeat the last, and are not written)
    const int tok = row / G, qh = u.head * G + row - tok * G;
    const int tiles = (len + KT - 1) / KT;
    const int beg = same((int)((int64_t)tiles * u.piece / u.pieces)), end = same((int)((int64_t)tiles * (u.piece + 1) / u.pieces));

    // --- staging.  Tiles beyond the last repeat it (and are not used).
    const int *table = p.b.table + (int64_t)same(sq.row) * p.b.table_stride;
    const int ps = p.b.page_shift, pmask = (1 << ps) - 1;
    // read with scalar loads, as the same for all lanes, which the waits for codes do not wait for
    auto scalar = [](auto *a) {
        typedef __attribute__((address_space(4))) const std::remove_reference_t<decltype(*a)> *constant;
        return *(constant)(uintptr_t)a;
    };
    auto held = [&](int pg) { return pg >= 0 && pg < p.b.pages; };
    auto first_key = [&](int t, int g) {   // of page g of tile t, or of the last page
        const int key = (t < end ? t : end - 1) * KT + g * PAGE;
        return key < len ? key : len - 1;
    };
    int page[NPG];                         // of the next tile to load
    float ks[NPG], vs[NPG];                // scales of the tile in vr
    bool is[NPG];
    u32x4 kr[NL], vr[NL];
    auto look_up = [&](int t) {
#pragma unroll
        for (int g = 0; g < NPG; ++g) page[g] = scalar(table + (first_key(t, g) >> ps));
    };
    auto page_row = [&](int pg) { return ((int64_t)(held(pg) ? pg : 0) * p.b.Hkv + u.head) << ps; };
    auto load_k = [&](int t) {
#pragma unroll
        for (int i = 0; i < NL; ++i) {
            const int g = i * NPG / NL;
            const uint8_t *c = p.kc + (page_row(page[g]) + (NPG == 1 ? first_key(t, 0) & pmask & ~(KT - 1) : 0)) * D + 1024 * (i - g * (NL / NPG));
            kr[i] = *reinterpret_cast<const u32x4 *>(c + (uint32_t)(16 * lane));
        }
    };
    auto load_v = [&](int t) {
#pragma unroll
        for (int g = 0; g < NPG; ++g) {
            const int64_t at = (int64_t)(held(page[g]) ? page[g] : 0) * p.b.Hkv + u.head;
            is[g] = held(page[g]);
            ks[g] = scalar(p.ks + at);
            vs[g] = scalar(p.vs + at);
        }
#pragma unroll
        for (int i = 0; i < NL; ++i) {
            const int g = i * NPG / NL;
            const uint8_t *c = p.vc + page_row(page[g]) * D;
            if constexpr (NPG == 1)   // KT/16 units of each channel
                c += (first_key(t, 0) & pmask & ~(KT - 1)) + ((int64_t)(i * (1024 / KT)) << ps) + (uint32_t)((lane / (KT / 16) << ps) + 16 * (lane % (KT / 16)));
            else c += 1024 * (i - g * (NL / NPG)) + (uint32_t)(16 * lane);
            vr[i] = *reinterpret_cast<const u32x4 *>(c);
        }
    };
    char *stage = reinterpret_cast<char *>(sh.stage[wave]);
    // unit 64 i + lane of K, in the order of memory; and of V
    auto store_k = [&]() {
        char *s = stage + lane / (D / 16) * SH::KROW + lane % (D / 16) * 16;
#pragma unroll
        for (int i = 0; i < NL; ++i)
            *reinterpret_cast<u32x4 *>(s + i * (1024 / D) * SH::KROW + (i * (1024 / D) >= KT / 2 ? 64 : 0)) = kr[i];
    };
    auto store_v = [&]() {
        char *s = stage + 16 * lane / PAGE * SH::VROW + 16 * lane % PAGE;
#pragma unroll
        for (int i = 0; i < NL; ++i) {
            const int g = i * NPG / NL;
            *reinterpret_cast<u32x4 *>(s + (i - g * (NL / NPG)) * (1024 / PAGE) * SH::VROW + g * PAGE) = vr[i];
        }
    };
    // What lanes have stored is there for the others of the wave, and what they have read may be stored over.  (The
    // compiler looks at one lane, whose loads and stores could be told apart.  No instruction comes of it.)
    auto in_order = [] {
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "local");
    };
    // the lane's key in the tile as row n of the K operand b; its keys of V and of logits, 16 for each b
    auto key_of = [&](int b) { return (KT / 2) * (n >> 2 & 1) + 16 * b + 8 * (n >> 4) + 4 * (n >> 3 & 1) + (n & 3); };
    auto group_of = [&](int b) { return (KT / 2) * h + 16 * b; };
    const char *k_at = stage + key_of(0) * SH::KROW + (n >> 2 & 1) * 64 + h * (D / 2);
    const char *v_at = stage + n * SH::VROW + h * (KT / 2);

    int t = beg + wave;
    if (t < end) {
        look_up(t);
        load_k(t);
        load_v(t);
        look_up(t + WAVES);
    }
    bf16x8 qf[QLDS ? 1 : KS];
    {
        const uint16_t *q = p.q + (int64_t)(sq.a + tok) * p.q_st + (int64_t)qh * p.q_sh + h * (D / 2);
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            u32x4 w = *reinterpret_cast<const u32x4 *>(q + 8 * k);
            if (p.scale_log2 < 0.0f) w ^= 0x80008000u;   // (a negative scale as a negated query: factors of logits stay non-negative)
            if constexpr (QLDS) {
                if (wave == 0) sh.q[k][lane] = w;
            } else {
                qf[k] = __builtin_bit_cast(bf16x8, w);
            }
        }
        if constexpr (QLDS) __syncthreads();
    }
    const float scale = fabsf(p.scale_log2);

    f32x16 o[DB];
#pragma unroll
    for (int i = 0; i < DB; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[i][e] = 0.0f;
    float m = LOWEST, l = 0.0f;   // (l: of this lane's keys)
    for (; t < end; t += WAVES) {
        in_order();
        store_k();
        in_order();
        load_k(t + WAVES);
        f32x16 s[NB];
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int e = 0; e < 16; ++e) s[b][e] = 0.0f;
#pragma unroll
        for (int w = 0; w < D / 32; ++w)
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                const u32x4 y = *reinterpret_cast<const u32x4 *>(k_at + 16 * b * SH::KROW + 16 * w);
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    bf16x8 q;
                    if constexpr (QLDS) q = __builtin_bit_cast(bf16x8, sh.q[2 * w + k][lane]);
                    else q = qf[2 * w + k];
                    s[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(widen(y[2 * k], y[2 * k + 1]), q, s[b], 0, 0, 0);
                }
            }
        // factors of the lane's logits and of its values, of its 16 keys b
        float c[NB], v[NB];
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            auto of = [&](int hh, bool values) {
                const int g = NPG == 1 ? 0 : ((KT / 2) * hh + 16 * b) / PAGE;
                return values ? (is[g] ? vs[g] : 1.0f) : (is[g] ? ks[g] * scale : __builtin_nanf(""));   // (logits of a missing page)
            };
            c[b] = NPG == 1 ? of(0, false) : (h ? of(1, false) : of(0, false));
            v[b] = NPG == 1 ? of(0, true) : (h ? of(1, true) : of(0, true));
        }
        const bool ends = NPG > 1 && (t + 1) * KT > len;   // (a page that holds tiles holds whole ones)
        if (ends) {   // groups behind the end: hidden
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                const bool see = t * KT + group_of(b) < len;
#pragma unroll
                for (int e = 0; e < 16; ++e) s[b][e] = see ? s[b][e] * c[b] : NEG_INF;
                c[b] = 1.0f;
            }
        }
        float mt = NEG_INF;
#pragma unroll
        for (int b = 0; b < NB; ++b) {
            float mg = NEG_INF;
#pragma unroll
            for (int e = 0; e < 16; e += 2) mg = fmaxf(fmaxf(mg, s[b][e]), s[b][e + 1]);
            mt = fmaxf(mt, mg * c[b]);
        }
        {
            const auto halves = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, mt), __builtin_bit_cast(uint32_t, mt), false, false);
            mt = fmaxf(__builtin_bit_cast(float, (uint32_t)halves[0]), __builtin_bit_cast(float, (uint32_t)halves[1]));
        }
        in_order();
        store_v();
        in_order();
        load_v(t + WAVES);
        look_up(t + 2 * WAVES);
        if (__ballot(mt > m + LAZY)) {
            const float mn = fmaxf(m, mt), alpha = __builtin_amdgcn_exp2f(m - mn);
            m = mn;
            l *= alpha;
#pragma unroll
            for (int i = 0; i < DB; ++i)
#pragma unroll
                for (int e = 0; e < 16; ++e) o[i][e] *= alpha;
        }
        bf16x8 pf[KT / 16];
        // probabilities exp2(s c - ref), summed into l times `unit`, times v in the operand
        auto exponentials = [&](float ref, float unit, bool scaled) {
#pragma unroll
            for (int k = 0; k < KT / 16; ++k) {
                const int b = k / 2;
                float y[8], sum = 0.0f;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    y[j] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][8 * (k & 1) + j], c[b], -ref));
                    sum += y[j];
                }
                l = __builtin_fmaf(sum, unit, l);
                u32x4 w;
#pragma unroll
                for (int e = 0; e < 4; ++e) w[e] = scaled ? pack2(y[2 * e], y[2 * e + 1]) : pack2(y[2 * e] * v[b], y[2 * e + 1] * v[b]);
                pf[k] = __builtin_bit_cast(bf16x8, w);
            }
        };
        // one value scale for the tile goes into the exponent (as in lamp_cache_many.h)
        if (NPG == 1 && v[0] > 0x1p-64f && v[0] < 0x1p64f) exponentials(m - __builtin_amdgcn_logf(v[0]), __builtin_amdgcn_rcpf(v[0]), true);
        else exponentials(m, 1.0f, false);
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int i = 0; i < DB; ++i) {
                u32x4 y = *reinterpret_cast<const u32x4 *>(v_at + 32 * i * SH::VROW + 16 * b);
                if (ends && t * KT + group_of(b) >= len) y = u32x4{0, 0, 0, 0};   // (whatever memory holds: 0 * NaN is NaN)
#pragma unroll
                for (int k = 0; k < 2; ++k)
                    o[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(widen(y[2 * k], y[2 * k + 1]), pf[2 * b + k], o[i], 0, 0, 0);
            }
    }

    // join the waves
    l += __shfl_xor(l, 32, 64);
    if (h == 0) {
        sh.ml[(wave * 32 + n) * 2] = m;
        sh.ml[(wave * 32 + n) * 2 + 1] = l;
    }
#pragma unroll
    for (int d0 = 0; d0 < D; d0 += DC) {
        __syncthreads();   // (the stretches of LDS, or what was joined before, have been read)
#pragma unroll
        for (int i = 0; i < DC / 32; ++i)
#pragma unroll
            for (int a = 0; a < 4; ++a)
                *reinterpret_cast<f32x4 *>(&sh.o[(wave * 32 + n) * OS + 32 * i + 8 * a + 4 * h]) =
                    f32x4{o[d0 / 32 + i][4 * a], o[d0 / 32 + i][4 * a + 1], o[d0 / 32 + i][4 * a + 2], o[d0 / 32 + i][4 * a + 3]};
        __syncthreads();
        for (int at = threadIdx.x * 4; at < 32 * DC; at += 256 * WAVES) {
            const int r = at / DC, d = at - r * DC;
            if (r >= here) continue;
            float mx = LOWEST, sum = 0.0f;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) mx = fmaxf(mx, sh.ml[(w * 32 + r) * 2]);
            f32x4 y = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                const float f = __builtin_amdgcn_exp2f(sh.ml[(w * 32 + r) * 2] - mx);
                sum += sh.ml[(w * 32 + r) * 2 + 1] * f;
                const f32x4 ow = *reinterpret_cast<const f32x4 *>(&sh.o[(w * 32 + r) * OS + d]);
#pragma unroll
                for (int e = 0; e < 4; ++e) y[e] += ow[e] * f;
            }
            const int64_t at_row = (int64_t)u.slot * PrefixRows::ROWS + r;
            *reinterpret_cast<f32x4 *>(p.part[2] + at_row * D + d0 + d) = y;
            if (d0 + d == 0) {
                p.part_ml[2][at_row * 2] = mx;
                p.part_ml[2][at_row * 2 + 1] = sum;
            }
        }
    }
}

} // namespace
} // namespace lamp
