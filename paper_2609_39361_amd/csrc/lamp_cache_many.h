// lamp_cache_many.h -- attention over the 8-bit paged cache for many query rows
// of one sequence and kv head: prompts and their chunks (the mathematics as in
// lamp_cache_attn.hip; library-internal, device code).
//
// A workgroup of 8 waves takes 256 query rows, 32 a wave, and walks over key
// tiles.  Its threads widen the tile's codes to bf16 once for all rows and lay
// them out in LDS.  The transposed products S^T = K Q^T and
// O^T = V^T P^T (32x32x16) leave a lane (row n = lane % 32, half = lane / 32)
// with the logits of half of the row's keys, which is also the operand of the
// second product: row m of a 32-key operand of K is key swap(m), m with bits 2
// and 3 exchanged, so that a lane's logits 8 s .. 8 s + 7 are the keys 16 s + 8
// half + 0 .. 7, the operand V^T is read in.  The softmax needs one exchange
// between the two halves a tile.
//
// Both LDS layouts are rows of 16-byte units (K: 8 channels of a key, keys in
// operand order; V: 8 keys of a channel) with one unit of padding, so that the
// lanes reading one unit of consecutive rows use all banks, at addresses that
// differ by constants.
//
// A wave alternates between a phase for the matrix cores (o += V^T P^T of the
// tile before, then S^T of this one, with the widening and storing of its share
// of the next tile between the products) and one for the vector unit (the
// softmax of this tile).  There is one barrier a tile, which the lower four
// waves meet after the softmax and the upper four, which share the four SIMDs
// with them, after the products: between two barriers the lower half multiplies
// for tile t and then exponentiates, the upper exponentiates for tile t - 1 and
// then multiplies for t, so that the two waves of a SIMD are at different units.
// The products of tile t read K of tile t and V of t - 1 and store K of t + 1 and
// V of t, in buffers whose former tiles were read before the last barrier: two
// of each do.
//
// Bound by the issue of products and vector instructions together.  An 8K prompt
// (32/8 heads, d = 128) takes 520 us a call back to back (562 the median
// in a trace, 534 the least), 1.06 PFLOP/s, where a large bf16 product reaches
// 1.28: by its counters a tile of 64 keys takes a SIMD's two waves 4260
// cycles, the matrix cores being busy for 2050 of them and the vector unit for
// 2340 (no LDS bank conflicts).  Both waves in the same phase: 589 us instead of
// 557; 64 rows a wave, one wave a SIMD: registers spill, 8 times as long.  For
// d = 256 half of the queries' operands come from LDS as well (registers hold o
// and the other half).
#pragma once
#include "lamp_cache_few.h"

namespace lamp {
namespace {

constexpr int WAVES = 8, THREADS = 64 * WAVES;

// The running maximum is raised only when a logit (times log2 e) passes it by
// LAZY: probabilities stay below 2^LAZY, far inside fp32 and bf16, and o is
// rescaled a few times a row instead of at every tile.
constexpr float LAZY = 8.0f;

__device__ __forceinline__ int swap23(int m)
{
    return (m & ~12) | ((m & 4) << 1) | ((m & 8) >> 1);
}

// Operands of the queries that are read from LDS: at d = 256 registers hold
// half of them beside o.
template <int D>
constexpr int Q_LDS = D > 128 ? D / 32 : 0;

template <int D, int KT>
struct PromptShared {
    u32x4 q[WAVES][Q_LDS<D> ? Q_LDS<D> : 1][Q_LDS<D> ? 64 : 1];
    u32x4 k[2][KT * (D / 8 + 1)];
    u32x4 v[2][D * (KT / 8 + 1)];
    float meta[4][KT / 16][2];                        // of each 16 keys: logit factor (scale, log2 e, key scale), value scale
    uint32_t marks[ManyRows::ROWS][D / 32];           // rows and channels that see NaN values (mark_nan)
    int marked;
};

// WIDE: a page holds whole tiles, so that a tile's page, scales and addresses
// are the same for all threads (otherwise for each group of 16 keys).
template <int D, int KT, bool WIDE, class P>
__device__ __forceinline__ void cache_prompt(const P &p, int x, PromptShared<D, KT> &sh)
{
    constexpr int NB = KT / 32;                 // 32-key operands of K
    constexpr int DB = D / 32;                  // 32-channel tiles of o
    constexpr int KU = D / 8, VU = KT / 8;      // 16-byte units of a row of K and V in LDS
    constexpr auto k_at = [](int m, int unit) { return m * (KU + 1) + unit; };   // of row m
    constexpr auto v_at = [](int d, int unit) { return d * (VU + 1) + unit; };
    constexpr int NG = KT / 16;                 // groups of 16 keys (each in one page)
    constexpr int CH = KT * D / 16;             // 16-byte chunks of codes of one tile of K (and of V)
    constexpr int PER = (CH + THREADS - 1) / THREADS;   // chunks of K of a thread, and of V

    const int G = p.Hq / p.b.Hkv;
    Unit u;
    SeqPlan sq;
    locate<ManyRows>(p, G, x, u, sq);
    if (u.s < 0) return;
    const int tid = (int)threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n = lane & 31, half = lane >> 5;
    const int rows = sq.n * G, r0 = u.tile * ManyRows::ROWS;
    const int rend = r0 + ManyRows::ROWS < rows ? r0 + ManyRows::ROWS : rows;
    write_info<ManyRows>(p, u, sq, r0, rend - r0);
    // keys that a position sees; those that some row sees, that every row sees
    auto upto = [&](int pos) { return sq.causal ? (pos + 1 < sq.len ? pos + 1 : sq.len) : sq.len; };
    auto from = [&](int pos) { return p.window > 0 && pos - p.window + 1 > 0 ? pos - p.window + 1 : sq.lo; };
    const int pmin = sq.pos0 + r0 / G, pmax = sq.pos0 + (rend - 1) / G;
    const int hi_any = upto(pmax), lo_any = from(pmin), hi_all = upto(pmin), lo_all = from(pmax);
    const int t0 = lo_any / KT, t1 = hi_any > lo_any ? (hi_any + KT - 1) / KT : t0;
    const int beg = __builtin_amdgcn_readfirstlane(t0 + (int)((int64_t)(t1 - t0) * u.piece / u.pieces));
    const int end = __builtin_amdgcn_readfirstlane(t0 + (int)((int64_t)(t1 - t0) * (u.piece + 1) / u.pieces));

    // this wave's rows (missing ones repeat the last and are not written)
    const int w0 = r0 + 32 * wave, wlast = w0 + 31 < rend ? w0 + 31 : rend - 1;
    const bool active = w0 < rend;
    const int row = w0 + n < rend ? w0 + n : rend - 1;
    const int tok = row / G, qh = u.head * G + row - tok * G, pos = sq.pos0 + tok;
    const int hi = upto(pos), lo = from(pos);
    const int wpmin = sq.pos0 + w0 / G, wpmax = sq.pos0 + wlast / G;
    const int whi_any = upto(wpmax), wlo_any = from(wpmin), whi_all = upto(wpmin), wlo_all = from(wpmax);

    constexpr int QR = D / 16 - Q_LDS<D>;       // operands in registers
    // operands in flight from LDS (8K prompt, d = 128, side by side: with one 564 us, two 540, eight 543; d = 256, 8K: two 446,
    // four 427)
    constexpr int AHEAD = D > 128 ? 4 : 2;
    bf16x8 qf[QR];
    {
        const uint16_t *q = p.q + (int64_t)(sq.a + tok) * p.q_st + (int64_t)qh * p.q_sh + 8 * half;
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
            u32x4 w = *reinterpret_cast<const u32x4 *>(q + 16 * k);
            // a negative scale as a negated query: factors of logits stay non-negative
            if (p.scale_log2 < 0.0f) w ^= 0x80008000u;
            if (k < QR) qf[k] = __builtin_bit_cast(bf16x8, w);
            else sh.q[wave][k - QR][lane] = w;
        }
    }
    const float scale = fabsf(p.scale_log2);

    // --- staging.  Straight-line code, so that no load is waited for before it
    // is used: tiles beyond the last repeat it (nothing reads what that stores),
    // places beyond the table's width read its last entry (no row sees them).
    const int *table = p.b.table + sq.row * p.b.table_stride;
    const int ps = p.b.page_shift, pmask = (1 << ps) - 1;
    auto entry = [&](int key) {   // of the table, for the 16 keys from `key`
        const int at = key >> ps;
        return table[at < p.b.width ? at : p.b.width - 1];
    };
    auto held = [&](int pg) { return pg >= 0 && pg < p.b.pages; };
    auto seen = [&](int key) { return key < hi_any && key + 16 > lo_any; };   // by some row
    auto tile = [&](int t) { return t < end ? t : end - 1; };
    // chunk i of K: 16 channels of a key; of V: 16 keys of a channel (two threads share one where a tile has fewer than threads)
    int kkey[PER], kch[PER], vch[PER], vgr[PER];
    // their bytes in a page, but for the tile's place in it (a tile is part of a page or holds whole ones)
    int koff[PER], voff[PER];
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int c = (tid + i * THREADS) % CH;
        kkey[i] = c / (D / 16);
        kch[i] = c % (D / 16);
        vch[i] = c / NG;
        vgr[i] = c % NG;
        koff[i] = (kkey[i] & pmask) * D + 16 * kch[i];
        voff[i] = (vch[i] << ps) + (16 * vgr[i] & pmask);
    }
    u32x4 kraw[PER], vraw[PER];
    // Table entries of the next tiles to load, and (vp, mp) those of the tiles
    // in vraw and in mk, mv, the scales of a tile's group tid % NG; WIDE: the
    // pages of tiles t, t + 1 and t + 2 in iteration t, and the entry of t + 3.
    int kpage[PER], vpage[PER], mpage, vp[PER], mp;
    int page0 = 0, page1 = 0, page2 = 0, ahead;
    float mk, mv;
    auto uniform = [](int v) { return __builtin_amdgcn_readfirstlane(v); };
    auto look_up_k = [&](int t) {
#pragma unroll
        for (int i = 0; i < PER; ++i) kpage[i] = entry(tile(t) * KT + (kkey[i] & ~15));
    };
    auto look_up_v = [&](int t) {
#pragma unroll
        for (int i = 0; i < PER; ++i) vpage[i] = entry(tile(t) * KT + 16 * vgr[i]);
    };
    auto look_up_meta = [&](int t) { mpage = entry(tile(t) * KT + 16 * (tid % NG)); };
    auto look_up = [&](int t) { ahead = entry(tile(t) * KT); };
    // of the page's codes for this head, the tile's part
    auto page_row = [&](int pg) { return ((int64_t)(held(pg) ? pg : 0) * p.b.Hkv + u.head) << ps; };
    auto k_base = [&](int pg, int t) { return p.kc + (page_row(pg) + (tile(t) * KT & pmask)) * D; };
    auto v_base = [&](int pg, int t) { return p.vc + (page_row(pg) * D + (tile(t) * KT & pmask)); };
    auto load_k = [&](int t, int pg) {
#pragma unroll
        for (int i = 0; i < PER; ++i) kraw[i] = *reinterpret_cast<const u32x4 *>(k_base(WIDE ? pg : kpage[i], t) + (uint32_t)koff[i]);
    };
    auto load_v = [&](int t, int pg) {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            vraw[i] = *reinterpret_cast<const u32x4 *>(v_base(WIDE ? pg : vpage[i], t) + (uint32_t)voff[i]);
            vp[i] = WIDE ? pg : vpage[i];
        }
    };
    auto load_meta = [&](int pg) {
        mp = WIDE ? pg : mpage;
        const int64_t at = (int64_t)(held(mp) ? mp : 0) * p.b.Hkv + u.head;
        mk = p.ks[at];
        mv = p.vs[at];
    };
    auto row_sees = [&](int r, int key) {
        const int rp = sq.pos0 + (r0 + r) / G;
        return key >= from(rp) && key < upto(rp);
    };
    // unit `second` of the thread's two of each chunk (the lower half of a row's lanes store their even unit first, the upper
    // their odd one: all banks each time)
    auto store_k = [&](int b, int second) {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int m = (kkey[i] & ~31) | swap23(kkey[i] & 31), c = kch[i];
            const bool odd = (c >= D / 32) != (second != 0);
            const uint32_t w0 = odd ? kraw[i][2] : kraw[i][0], w1 = odd ? kraw[i][3] : kraw[i][1];
            sh.k[b][k_at(m, 2 * c + odd)] = __builtin_bit_cast(u32x4, widen(w0, w1));
        }
    };
    // Values of tile t that no row sees are whatever memory holds: zeroed, as
    // 0 * NaN is NaN; only in a tile that not every row sees whole.
    auto mask_v = [&](int t) {
        const int key0 = tile(t) * KT;
        if (key0 >= lo_all && key0 + KT <= hi_all) return;
#pragma unroll
        for (int i = 0; i < PER; ++i)
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const int key = key0 + 16 * vgr[i] + 4 * w;
                uint32_t x = vraw[i][w] & byte_mask(key, lo_any, hi_any);
                const uint32_t nan = held(vp[i]) ? nan_bytes(x) : 0u;
                if (nan) {
                    sh.marked = 1;
                    mark_nan<D>(sh.marks, nan, vch[i], key, rend - r0, row_sees);
                    x &= ~((nan >> 7) * 0xFFu);
                }
                vraw[i][w] = x;
            }
    };
    auto store_v = [&](int b, int second) {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const uint32_t keep = held(vp[i]) ? ~0u : 0u;
            const bf16x8 x = widen(vraw[i][2 * second] & keep, vraw[i][2 * second + 1] & keep);
            sh.v[b][v_at(vch[i], 2 * vgr[i] + second)] = __builtin_bit_cast(u32x4, x);
        }
    };
    // The factor of a group's logits (scale, log2 e, key scale) and the scale of
    // its values: logits of a missing page are NaN, keys that no row sees are masked.
    float tc = 0.0f, tv = 1.0f;   // WIDE: those of tile t in iteration t
    auto store_meta = [&](int t) {
        if constexpr (WIDE) {
            tc = held(mp) ? mk * scale : __builtin_nanf("");
            tv = held(mp) ? mv : 1.0f;
        } else {   // (every thread stores its group's, the same ones)
            const int key = tile(t) * KT + 16 * (tid % NG);
            const bool is = held(mp), see = seen(key);
            sh.meta[t & 3][tid % NG][0] = is ? mk * scale : (see ? __builtin_nanf("") : 0.0f);
            sh.meta[t & 3][tid % NG][1] = is && see ? mv : 1.0f;
        }
    };

    f32x16 o[DB];
#pragma unroll
    for (int i = 0; i < DB; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[i][e] = 0.0f;
    // m: the reference of the exponentials; l: of this lane's keys.  A row that sees keys beyond the table's reach is NaN.
    float m = hi > lo ? LOWEST : NEG_INF, l = (sq.causal && pos + 1 < sq.all ? pos + 1 : sq.all) > sq.len ? __builtin_nanf("") : 0.0f;

    for (int i = tid; i < ManyRows::ROWS * (D / 32); i += THREADS) sh.marks[0][i] = 0;
    if (tid == 0) sh.marked = 0;
    // what the products of the first tile's predecessor read
    for (int i = tid; i < D * (VU + 1); i += THREADS) sh.v[(beg + 1) & 1][i] = u32x4{0, 0, 0, 0};
    __syncthreads();
    if (beg < end) {
        if constexpr (WIDE) {
            const int first = entry(tile(beg) * KT), second = entry(tile(beg + 1) * KT);
            look_up(beg + 2);
            page0 = uniform(first);
            page1 = uniform(second);
            load_k(beg, page0);
            load_v(beg, page0);
            load_meta(page0);
            store_k(beg & 1, 0);
            store_k(beg & 1, 1);
            load_k(beg + 1, page1);
            mask_v(beg);
        } else {
            look_up_k(beg);
            look_up_v(beg);
            look_up_meta(beg);
            load_k(beg, 0);
            load_v(beg, 0);
            load_meta(0);
            look_up_k(beg + 1);
            look_up_v(beg + 1);
            look_up_meta(beg + 1);
            store_k(beg & 1, 0);
            store_k(beg & 1, 1);
            store_meta(beg);
            load_k(beg + 1, 0);
            load_meta(0);
            look_up_k(beg + 2);
            look_up_meta(beg + 2);
            mask_v(beg);
        }
    }
    __syncthreads();
    const bool behind = wave >= WAVES / 2;

    f32x16 s[NB];
    bf16x8 pf[NG];
    // the stores of iteration t and the loads of the next one's, in pieces
    constexpr int PIECES = 9;
    auto stage = [&](int t, int piece) {
        switch (piece) {
        case 0: store_v(t & 1, 0); break;
        case 1: store_v(t & 1, 1); break;
        case 2: store_k(t + 1 & 1, 0); break;
        case 3: store_k(t + 1 & 1, 1); break;
        case 4:
            store_meta(WIDE ? t : t + 1);
            if (WIDE) page2 = uniform(ahead);
            break;
        case 5: load_v(t + 1, page1); break;
        case 6: load_k(t + 2, page2); break;
        case 7: load_meta(page1); break;
        default:
            if constexpr (WIDE) {
                page0 = page1;
                page1 = page2;
                look_up(t + 3);
            } else {
                look_up_v(t + 2), look_up_k(t + 3), look_up_meta(t + 3);
            }
        }
    };
    // whether some row of the wave sees some key of the tile
    auto visible = [&](int t) { return active && t * KT < whi_any && t * KT + KT > wlo_any; };
#pragma unroll
    for (int g = 0; g < NG; ++g) pf[g] = __builtin_bit_cast(bf16x8, u32x4{0, 0, 0, 0});
    for (int t = beg; t <= end && beg < end; ++t) {
        const bool now = t < end && visible(t);
        // (Also for tiles that no row of the wave sees: their logits are left unused, their probabilities 0, and their values
        // hold no NaN, as not every row sees them.)
        {
            // Operands come from LDS AHEAD products before they are used;
            // neighbouring products are on different accumulators.  The phase
            // has priority: its few instructions keep the matrix cores busy
            // (8K prompt: 557 us with it, 587 without, 608 the other way round).
            __builtin_amdgcn_s_setprio(1);
            constexpr int OV = DB * NG, ALL = OV + NB * D / 16, EVERY = ALL / PIECES;
            bf16x8 a[AHEAD], q[AHEAD];
            auto read = [&](int i) {
                const int k = (i - OV) / NB;
                a[i % AHEAD] = __builtin_bit_cast(bf16x8, i < OV ? sh.v[t + 1 & 1][v_at(32 * (i % DB) + n, 2 * (i / DB) + half)]
                                                                 : sh.k[t & 1][k_at(32 * ((i - OV) % NB) + n, 2 * k + half)]);
                if (i >= OV && k >= QR) q[i % AHEAD] = __builtin_bit_cast(bf16x8, sh.q[wave][k - QR][lane]);
            };
#pragma unroll
            for (int i = 0; i < NB; ++i)
#pragma unroll
                for (int e = 0; e < 16; ++e) s[i][e] = 0.0f;
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) read(i);
#pragma unroll
            for (int i = 0; i < ALL; ++i) {
                const int k = (i - OV) / NB, at = i % AHEAD, b = (i - OV) % NB;
                if (i < OV) o[i % DB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[at], pf[i / DB], o[i % DB], 0, 0, 0);
                else s[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[at], k < QR ? qf[k < QR ? k : 0] : q[at], s[b], 0, 0, 0);
                if (i + AHEAD < ALL) read(i + AHEAD);
                if (i % EVERY == EVERY - 1 && i / EVERY < PIECES) stage(t, i / EVERY);
                __builtin_amdgcn_sched_barrier(0x0006);   // (only vector and scalar arithmetic may move past)
            }
        }
        __builtin_amdgcn_s_setprio(0);
        if (behind) __syncthreads();
        if (now) {
            const int key0 = t * KT;
            constexpr int CG = WIDE ? 1 : NG;   // groups with factors of their own
            float c[CG], vs[CG];
#pragma unroll
            for (int g = 0; g < CG; ++g) {
                c[g] = WIDE ? tc : sh.meta[t & 3][g][0];
                vs[g] = WIDE ? tv : sh.meta[t & 3][g][1];
            }
            // logits of group g: s[g / 2][8 (g % 2) + j], key 16 g + 8 half + j
            if (key0 < wlo_all || key0 + KT > whi_all) {
#pragma unroll
                for (int g = 0; g < NG; ++g)
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const int key = key0 + 16 * g + 8 * half + j;
                        const float y = s[g / 2][8 * (g & 1) + j] * c[g % CG];
                        s[g / 2][8 * (g & 1) + j] = key < lo || key >= hi ? NEG_INF : y;
                    }
#pragma unroll
                for (int g = 0; g < CG; ++g) c[g] = 1.0f;
            }
            float mt = NEG_INF;
#pragma unroll
            for (int g = 0; g < CG; ++g) {
                float mg = NEG_INF;
#pragma unroll
                for (int j = 0; j < KT / 2 / CG; j += 2) {
                    const int e = KT / 2 / CG * g + j;
                    mg = fmaxf(fmaxf(mg, s[e / 16][e % 16]), s[e / 16][e % 16 + 1]);
                }
                mt = fmaxf(mt, mg * c[g]);
            }
            mt = fmaxf(mt, __shfl_xor(mt, 32, 64));
            if (__ballot(mt > m + LAZY)) {
                const float mn = fmaxf(m, mt), alpha = __builtin_amdgcn_exp2f(m - (mn == NEG_INF ? 0.0f : mn));
                m = mn;
                l *= alpha;
#pragma unroll
                for (int i = 0; i < DB; ++i)
#pragma unroll
                    for (int e = 0; e < 16; ++e) o[i][e] *= alpha;
            }
            const float ms = m == NEG_INF ? 0.0f : m;   // (a row that has seen no key yet)
            // probabilities of all groups: exp2(s c - ref), summed into l times `unit`, times vs in the operand
            auto exponentials = [&](float ref, float unit, bool scaled) {
#pragma unroll
                for (int g = 0; g < NG; ++g) {
                    float y[8], sum = 0.0f;
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        y[j] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[g / 2][8 * (g & 1) + j], c[g % CG], -ref));
                        sum += y[j];
                    }
                    l = __builtin_fmaf(sum, unit, l);
                    u32x4 w;
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        w[e] = scaled ? pack2(y[2 * e], y[2 * e + 1]) : pack2(y[2 * e] * vs[g % CG], y[2 * e + 1] * vs[g % CG]);
                    pf[g] = __builtin_bit_cast(bf16x8, w);
                }
            };
            // One value scale for the tile goes into the exponent (a power of
            // two, so that the sum has it divided out exactly), if it leaves
            // the smallest probabilities that count (2^-60) far above fp32's.
            // The reference is rounded once more for it, to fp32: as the logits
            // are, half a step of a number of their size.
            if (WIDE && vs[0] > 0x1p-64f && vs[0] < 0x1p64f)
                exponentials(ms - __builtin_amdgcn_logf(vs[0]), __builtin_amdgcn_rcpf(vs[0]), true);
            else
                exponentials(ms, 1.0f, false);
        }
        if (!now) {
#pragma unroll
            for (int g = 0; g < NG; ++g) pf[g] = __builtin_bit_cast(bf16x8, u32x4{0, 0, 0, 0});
        }
        mask_v(t + 1);
        if (!behind) __syncthreads();
    }
    if (!active) return;
    l += __shfl_xor(l, 32, 64);
    if (w0 + n >= rend) return;
    if (sh.marked) {
#pragma unroll
        for (int i = 0; i < DB; ++i) {
            const uint32_t nan = sh.marks[32 * wave + n][i] >> (4 * half);
#pragma unroll
            for (int e = 0; e < 16; ++e) o[i][e] = nan >> (8 * (e >> 2) + (e & 3)) & 1u ? __builtin_nanf("") : o[i][e];
        }
    }
    // o[i][4 a + e]: channel 32 i + 8 a + 4 half + e
    if (joined(p, sq, u.pieces)) {
        const int64_t at = (int64_t)u.slot * ManyRows::ROWS + 32 * wave + n;
#pragma unroll
        for (int i = 0; i < DB; ++i)
#pragma unroll
            for (int a = 0; a < 4; ++a)
                *reinterpret_cast<f32x4 *>(p.part[1] + at * D + 32 * i + 8 * a + 4 * half) =
                    f32x4{o[i][4 * a], o[i][4 * a + 1], o[i][4 * a + 2], o[i][4 * a + 3]};
        if (half == 0) {
            p.part_ml[1][at * 2] = m;
            p.part_ml[1][at * 2 + 1] = l;
        }
        return;
    }
    const int64_t orow = (int64_t)(sq.a + tok) * p.Hq + qh;
    const float inv = finish(m, l);
#pragma unroll
    for (int i = 0; i < DB; ++i)
#pragma unroll
        for (int a = 0; a < 4; ++a)
            *reinterpret_cast<u32x2 *>(p.o + orow * D + 32 * i + 8 * a + 4 * half) =
                u32x2{pack2(o[i][4 * a] * inv, o[i][4 * a + 1] * inv), pack2(o[i][4 * a + 2] * inv, o[i][4 * a + 3] * inv)};
    if (half == 0) p.lse[orow] = finish_lse(m, l);
}

} // namespace
} // namespace lamp
