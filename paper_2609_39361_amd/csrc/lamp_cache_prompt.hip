// lamp_cache_prompt.hip -- attention over the 8-bit paged cache for many query
// rows of one sequence and kv head: prompts and their chunks (the mathematics as
// in lamp_cache_attn.hip).
//
// A workgroup of 8 waves takes 256 query rows, 32 a wave, and walks over key
// tiles.  Its threads widen the tile's codes to bf16 once for all rows and lay
// them out in LDS (two buffers: the next tile is written while this one is
// used, one barrier a tile).  The transposed products S^T = K Q^T and
// O^T = V^T P^T (32x32x16) leave a lane (row n = lane % 32, half = lane / 32)
// with the logits of half of the row's keys, which is also the operand of the
// second product: row m of a 32-key operand of K is key swap(m), m with bits 2
// and 3 exchanged, so that a lane's logits 8 s .. 8 s + 7 are the keys 16 s + 8
// half + 0 .. 7, the operand V^T is read in.  The softmax needs one exchange
// between the two halves a tile.
//
// Both LDS layouts are rows of 16-byte units (K: 8 channels of a key, keys in
// operand order; V: 8 keys of a channel), the unit's place exchanged with the
// row's low bits, so that the lanes reading one unit of consecutive rows use
// all banks.
#include <hip/hip_runtime.h>

#include "lamp_cache_plan.h"

namespace lamp {
namespace {

constexpr int WAVES = 8, THREADS = 64 * WAVES;

// The running maximum is raised only when a logit passes it by 2^LAZY (in
// units of log2): probabilities stay below 2^LAZY, far inside fp32 and bf16,
// and o is rescaled a few times a row instead of at every tile.
constexpr float LAZY = 8.0f;

__device__ __forceinline__ int swap23(int m)
{
    return (m & ~12) | ((m & 4) << 1) | ((m & 8) >> 1);
}

template <int D, int KT>
__global__ __launch_bounds__(THREADS, 2) void cache_prompt_kernel(CacheAttnParams p)
{
    constexpr int NB = KT / 32;                 // 32-key operands of K
    constexpr int DB = D / 32;                  // 32-channel tiles of o
    constexpr int KU = D / 8, VU = KT / 8;      // 16-byte units of a row of K and V in LDS
    // the unit's place in row m of K, d of V (8 units fill the banks once: 2 rows of V where it has 4)
    auto k_at = [](int m, int unit) { return m * KU + (unit ^ (m & (KU < 16 ? KU - 1 : 15))); };
    auto v_at = [](int d, int unit) { return d * VU + (unit ^ (VU < 8 ? (d >> 1) & (VU - 1) : d & (VU - 1))); };
    constexpr int NG = KT / 16;                 // groups of 16 keys (each in one page)
    constexpr int CH = KT * D / 16;             // 16-byte chunks of codes of one tile of K (and of V)
    constexpr int PER = (CH + THREADS - 1) / THREADS;   // chunks of K of a thread, and of V
    __shared__ u32x4 kbuf[2][KT * KU];
    __shared__ u32x4 vbuf[2][D * VU];
    __shared__ float meta[2][NG][2];            // logit factor (scale, log2 e, key scale) and value scale of each group
    __shared__ uint32_t marks[ManyRows::ROWS][D / 32];   // rows and channels that see NaN values (mark_nan)
    __shared__ int marked;

    const int G = p.Hq / p.b.Hkv;
    const Unit u = find_unit<ManyRows>(p, G, blockIdx.x, false);
    if (u.s < 0) return;
    const SeqPlan sq = seq_plan<ManyRows>(p, u.s, G);
    const int tid = (int)threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n = lane & 31, half = lane >> 5;
    const int rows = sq.n * G, r0 = u.tile * ManyRows::ROWS;
    const int rend = r0 + ManyRows::ROWS < rows ? r0 + ManyRows::ROWS : rows;
    // keys that rows from ra to rb (inclusive) see: some of them [lo, hi), all of them [lo_all, hi_all)
    auto upto = [&](int pos) { return p.causal ? (pos + 1 < sq.len ? pos + 1 : sq.len) : sq.len; };
    auto from = [&](int pos) { return p.window > 0 && pos - p.window + 1 > 0 ? pos - p.window + 1 : 0; };
    const int pmin = sq.pos0 + r0 / G, pmax = sq.pos0 + (rend - 1) / G;
    const int hi_any = upto(pmax), lo_any = from(pmin), hi_all = upto(pmin), lo_all = from(pmax);
    const int t0 = lo_any / KT, t1 = hi_any > lo_any ? (hi_any + KT - 1) / KT : t0;
    const int beg = t0 + (int)((int64_t)(t1 - t0) * u.piece / u.pieces);
    const int end = t0 + (int)((int64_t)(t1 - t0) * (u.piece + 1) / u.pieces);

    // this wave's rows (missing ones repeat the last and are not written)
    const int w0 = r0 + 32 * wave, wlast = w0 + 31 < rend ? w0 + 31 : rend - 1;
    const bool active = w0 < rend;
    const int row = w0 + n < rend ? w0 + n : rend - 1;
    const int tok = row / G, qh = u.head * G + row - tok * G, pos = sq.pos0 + tok;
    const int hi = upto(pos), lo = from(pos);
    const int wpmin = sq.pos0 + w0 / G, wpmax = sq.pos0 + wlast / G;
    const int whi_any = upto(wpmax), wlo_any = from(wpmin), whi_all = upto(wpmin), wlo_all = from(wpmax);

    bf16x8 qf[D / 16];
    {
        const uint16_t *q = p.q + (int64_t)(sq.a + tok) * p.q_st + (int64_t)qh * p.q_sh + 8 * half;
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
            u32x4 w = *reinterpret_cast<const u32x4 *>(q + 16 * k);
            // a negative scale as a negated query: factors of logits stay non-negative
            if (p.scale_log2 < 0.0f) w ^= 0x80008000u;
            qf[k] = __builtin_bit_cast(bf16x8, w);
        }
    }
    const float scale = fabsf(p.scale_log2);

    // --- staging: this thread's chunks of a tile
    const int *table = p.b.table + u.s * p.b.table_stride;
    const int ps = p.b.page_shift, pmask = (1 << ps) - 1;
    constexpr int UNSEEN = -2, MISSING = -1;
    auto page_at = [&](int key) {   // of the 16 keys from `key`
        if (key >= hi_any || key + 16 <= lo_any) return UNSEEN;
        const int pg = table[key >> ps];
        return pg >= 0 && pg < p.b.pages ? pg : MISSING;
    };
    // chunk i of K: key, 16 channels; of V: channel, 16 keys
    auto k_key = [&](int i) { return (tid + i * THREADS) / (D / 16); };
    auto k_chunk = [&](int i) { return (tid + i * THREADS) % (D / 16); };
    auto v_chan = [&](int i) { return (tid + i * THREADS) / NG; };
    auto v_group = [&](int i) { return (tid + i * THREADS) % NG; };
    auto mine = [&](int i) { return CH % THREADS == 0 || tid + i * THREADS < CH; };
    u32x4 kraw[PER], vraw[PER];
    int kpage[PER], vpage[PER], mpage = UNSEEN;   // pages of the next tile to load
    auto look_up = [&](int t) {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            if (!mine(i)) continue;
            kpage[i] = page_at(t * KT + (k_key(i) & ~15));
            vpage[i] = page_at(t * KT + 16 * v_group(i));
        }
        if (tid < NG) mpage = page_at(t * KT + 16 * tid);
    };
    float mk = 0.0f, mv = 0.0f;   // the scales of group `tid`
    int vp[PER], mp = UNSEEN;     // pages of the tile in kraw, vraw
    auto load = [&](int t) {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            if (!mine(i)) continue;
            const int64_t ka = (int64_t)(kpage[i] < 0 ? 0 : kpage[i]) * p.b.Hkv + u.head;
            kraw[i] = *reinterpret_cast<const u32x4 *>(p.kc + (ka << ps) * D + (int64_t)((t * KT + k_key(i)) & pmask) * D + 16 * k_chunk(i));
            const int64_t va = (int64_t)(vpage[i] < 0 ? 0 : vpage[i]) * p.b.Hkv + u.head;
            vraw[i] = *reinterpret_cast<const u32x4 *>(p.vc + (va << ps) * D + ((int64_t)v_chan(i) << ps) + ((t * KT + 16 * v_group(i)) & pmask));
            vp[i] = vpage[i];
        }
        if (tid < NG) {
            mp = mpage;
            const int64_t a = (int64_t)(mp < 0 ? 0 : mp) * p.b.Hkv + u.head;
            mk = p.ks[a];
            mv = p.vs[a];
        }
    };
    auto sees = [&](int r, int key) {
        const int rp = sq.pos0 + (r0 + r) / G;
        return key >= from(rp) && key < upto(rp);
    };
    // a tile that not every row of the workgroup sees whole
    auto partial_tile = [&](int t) { return t * KT < lo_all || t * KT + KT > hi_all; };
    auto store = [&](int t, int b) {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            if (!mine(i)) continue;
            const int key = k_key(i), m = (key & ~31) | swap23(key & 31), c = k_chunk(i);
            u32x4 x = kraw[i];
            kbuf[b][k_at(m, 2 * c)] = __builtin_bit_cast(u32x4, widen(x[0], x[1]));
            kbuf[b][k_at(m, 2 * c + 1)] = __builtin_bit_cast(u32x4, widen(x[2], x[3]));
            x = vraw[i];
            const int d = v_chan(i), g = v_group(i);
            // values that no row sees are whatever memory holds: zeroed, as 0 * NaN is NaN
            if (vp[i] < 0) {
                x = u32x4{0, 0, 0, 0};
            } else if (partial_tile(t)) {
                const int k0 = t * KT + 16 * g;
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    x[w] &= byte_mask(k0 + 4 * w, lo_any, hi_any);
                    const uint32_t nan = nan_bytes(x[w]);
                    if (nan) {
                        marked = 1;
                        mark_nan<D>(marks, nan, d, k0 + 4 * w, rend - r0, sees);
                        x[w] &= ~((nan >> 7) * 0xFFu);
                    }
                }
            }
            vbuf[b][v_at(d, 2 * g)] = __builtin_bit_cast(u32x4, widen(x[0], x[1]));
            vbuf[b][v_at(d, 2 * g + 1)] = __builtin_bit_cast(u32x4, widen(x[2], x[3]));
        }
        if (tid < NG) {
            // logits of a missing page are NaN; unseen groups are masked
            meta[b][tid][0] = mp == MISSING ? __builtin_nanf("") : (mp == UNSEEN ? 0.0f : mk * scale);
            meta[b][tid][1] = mp < 0 ? 1.0f : mv;
        }
    };

    f32x16 o[DB];
#pragma unroll
    for (int i = 0; i < DB; ++i)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[i][e] = 0.0f;
    // m: the reference of the exponentials; l: of this lane's keys.  A row that sees keys beyond the table's reach is NaN.
    float m = NEG_INF, l = (p.causal && pos + 1 < sq.all ? pos + 1 : sq.all) > sq.len ? __builtin_nanf("") : 0.0f;

    for (int i = tid; i < ManyRows::ROWS * (D / 32); i += THREADS) marks[0][i] = 0;
    if (tid == 0) marked = 0;
    __syncthreads();
    if (beg < end) {
        look_up(beg);
        load(beg);
        if (beg + 1 < end) look_up(beg + 1);
        store(beg, 0);
        if (beg + 1 < end) {
            load(beg + 1);
            if (beg + 2 < end) look_up(beg + 2);
        }
        __syncthreads();
    }
    for (int t = beg; t < end; ++t) {
        const int b = (t - beg) & 1;
        if (t + 1 < end) {
            store(t + 1, b ^ 1);
            if (t + 2 < end) {
                load(t + 2);
                if (t + 3 < end) look_up(t + 3);
            }
        }
        const int key0 = t * KT;
        if (active && key0 < whi_any && key0 + KT > wlo_any) {
            f32x16 s[NB];
#pragma unroll
            for (int i = 0; i < NB; ++i) {
#pragma unroll
                for (int e = 0; e < 16; ++e) s[i][e] = 0.0f;
                const int r = 32 * i + n;
#pragma unroll
                for (int k = 0; k < D / 16; ++k) {
                    const bf16x8 a = __builtin_bit_cast(bf16x8, kbuf[b][k_at(r, 2 * k + half)]);
                    s[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, qf[k], s[i], 0, 0, 0);
                }
            }
            float c[NG], vs[NG];
#pragma unroll
            for (int g = 0; g < NG; ++g) {
                c[g] = meta[b][g][0];
                vs[g] = meta[b][g][1];
            }
            const bool partial = key0 < wlo_all || key0 + KT > whi_all;
            // logits of group g: s[g / 2][8 (g % 2) + j], key 16 g + 8 half + j
            if (partial) {
#pragma unroll
                for (int g = 0; g < NG; ++g) {
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        const int key = key0 + 16 * g + 8 * half + j;
                        const float x = s[g / 2][8 * (g & 1) + j] * c[g];
                        s[g / 2][8 * (g & 1) + j] = key < lo || key >= hi ? NEG_INF : x;
                    }
                    c[g] = 1.0f;
                }
            }
            float mt = NEG_INF;
#pragma unroll
            for (int g = 0; g < NG; ++g) {
                float mg = s[g / 2][8 * (g & 1)];
#pragma unroll
                for (int j = 1; j < 8; ++j) mg = fmaxf(mg, s[g / 2][8 * (g & 1) + j]);
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
            bf16x8 pf[NG];
#pragma unroll
            for (int g = 0; g < NG; ++g) {
                float x[8], sum = 0.0f;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    x[j] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[g / 2][8 * (g & 1) + j], c[g], -ms));
                    sum += x[j];
                }
                l += sum;
                u32x4 w;
#pragma unroll
                for (int e = 0; e < 4; ++e) w[e] = pack2(x[2 * e] * vs[g], x[2 * e + 1] * vs[g]);
                pf[g] = __builtin_bit_cast(bf16x8, w);
            }
#pragma unroll
            for (int i = 0; i < DB; ++i) {
                const int d = 32 * i + n;
#pragma unroll
                for (int g = 0; g < NG; ++g) {
                    const bf16x8 a = __builtin_bit_cast(bf16x8, vbuf[b][v_at(d, 2 * g + half)]);
                    o[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, pf[g], o[i], 0, 0, 0);
                }
            }
        }
        __syncthreads();
    }
    if (!active) return;
    l += __shfl_xor(l, 32, 64);
    if (w0 + n >= rend) return;
    if (marked) {
#pragma unroll
        for (int i = 0; i < DB; ++i) {
            const uint32_t nan = marks[32 * wave + n][i] >> (4 * half);
#pragma unroll
            for (int e = 0; e < 16; ++e) o[i][e] = nan >> (8 * (e >> 2) + (e & 3)) & 1u ? __builtin_nanf("") : o[i][e];
        }
    }
    // o[i][4 a + e]: channel 32 i + 8 a + 4 half + e
    if (u.pieces > 1) {
        const int64_t at = (int64_t)u.slot * ManyRows::ROWS + 32 * wave + n;
#pragma unroll
        for (int i = 0; i < DB; ++i)
#pragma unroll
            for (int a = 0; a < 4; ++a)
                *reinterpret_cast<f32x4 *>(p.part + at * D + 32 * i + 8 * a + 4 * half) =
                    f32x4{o[i][4 * a], o[i][4 * a + 1], o[i][4 * a + 2], o[i][4 * a + 3]};
        if (half == 0) {
            p.part_ml[at * 2] = m;
            p.part_ml[at * 2 + 1] = l;
        }
        return;
    }
    const int64_t orow = (int64_t)(sq.a + tok) * p.Hq + qh;
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
    for (int i = 0; i < DB; ++i)
#pragma unroll
        for (int a = 0; a < 4; ++a)
            *reinterpret_cast<u32x2 *>(p.o + orow * D + 32 * i + 8 * a + 4 * half) =
                u32x2{pack2(o[i][4 * a] * inv, o[i][4 * a + 1] * inv), pack2(o[i][4 * a + 2] * inv, o[i][4 * a + 3] * inv)};
    if (half == 0) p.lse[orow] = l == 0.0f ? NEG_INF : (m + __builtin_amdgcn_logf(l)) * LN2;
}

} // namespace

hipError_t launch_cache_prompt(int D, const CacheAttnParams &p, hipStream_t s)
{
    const dim3 grid((unsigned)max_units<ManyRows>(p));
    switch (D) {
    case 64: cache_prompt_kernel<64, 64><<<grid, THREADS, 0, s>>>(p); break;
    case 128: cache_prompt_kernel<128, 64><<<grid, THREADS, 0, s>>>(p); break;
    default: cache_prompt_kernel<256, 32><<<grid, THREADS, 0, s>>>(p); break;
    }
    return hipGetLastError();
}

} // namespace lamp
