// lamp_cache_plan.h -- the cache attention's division of work and the pieces its
// kernels share (library-internal, device code).
#pragma once
#include <hip/hip_runtime.h>

#include <limits.h>

#include <type_traits>

#include "lamp_search.h"
#include "lamp_serve.h"

namespace lamp {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr float NEG_INF = -__builtin_inff();
constexpr float LN2 = 0.6931471805599453f;
// Where the running maximum of a row that sees keys starts: below every finite
// logit, so that -infinity is left to the rows that see none.
constexpr float LOWEST = -3.4028234663852886e38f;
constexpr int TILE = 64;       // keys of the plan's tiles

// The two forms of the attention.  ROWS: query rows of a workgroup (row = token
// * G + head of the group); TARGET: workgroups that fill the 256 CUs; MIN_TILES:
// least key tiles of a piece.
template <int WAVES>
struct FewRowsOf {     // single tokens and short chunks (lamp_cache_few.h): 8 waves fill a CU's registers, a tile for each wave
    static constexpr int ROWS = 16, TARGET = 2048 / WAVES, MIN_TILES = WAVES, FORM = 0;
};
using FewRows = FewRowsOf<4>;
struct ManyRows {      // prompts (lamp_cache_prompt.hip; 32 row tiles' window of 1024: 31 us with pieces of 5 tiles at least, 37 of 8)
    static constexpr int ROWS = 256, TARGET = 256, MIN_TILES = 5, FORM = 1;
};

// The key range of one sequence is cut in pieces when its row tiles alone do
// not fill the device: with `total` the key tiles of all (sequence, row tile,
// kv head) triples of a form, pieces hold about total / TARGET tiles.  Up to
// PLAN_ALONE sequences every wave works the plan out for itself from the lengths
// (one load a lane, no launch more); for more, a launch of its own leaves it in
// the workspace (cache_plan_kernel).  Either way the lengths are read on the
// device, and a captured graph follows them.
constexpr int PLAN_ALONE = 256;

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
    float mean;      // and on average
};

// Row tiles whose mean is this part of the longest at least count as even.
constexpr float EVEN = 0.75f;

template <class F>
__device__ __forceinline__ SeqPlan seq_plan(const CacheAttnParams &p, int s, int G)
{
    SeqPlan r;
    r.a = p.b.q_start ? p.b.q_start[s] : s;
    const int e = p.b.q_start ? p.b.q_start[s + 1] : s + 1;
    const int len = p.b.kv_lens[s] > 0 ? p.b.kv_lens[s] : 0;
    r.n = r.a >= 0 && e <= p.b.T && e > r.a ? e - r.a : 0;
    r.pos0 = len - r.n;
    const int reach = p.b.width << p.b.page_shift;   // (at most 2^30)
    r.all = len;
    r.len = len < reach ? len : reach;
    const int rows = r.n * G;                        // (at most 2^27)
    r.tiles = rows > p.rows_above[F::FORM] && rows <= p.rows_upto[F::FORM] ? (rows + F::ROWS - 1) / F::ROWS : 0;
    r.kt = (r.len + TILE - 1) / TILE;
    if (p.window > 0) {
        const int span = (p.window + F::ROWS - 1 + TILE - 1) / TILE + 1;
        if (span < r.kt) r.kt = span;
    }
    r.mean = p.causal ? fminf((float)r.kt, ((float)r.len - 0.5f * (float)r.n) * (1.0f / TILE)) : (float)r.kt;
    return r;
}

// Inclusive sum over the wave's lanes; and maximum, of numbers >= 0.
template <class T, class OP>
__device__ __forceinline__ T wave_scan_by(T v, OP op)
{
    const T zero = 0;
    auto step = [&](auto ctrl, auto rows) {
        const int x = __builtin_amdgcn_update_dpp(__builtin_bit_cast(int, zero), __builtin_bit_cast(int, v), decltype(ctrl)::value,
                                                  decltype(rows)::value, 0xf, false);
        v = op(v, __builtin_bit_cast(T, x));
    };
    step(std::integral_constant<int, 0x111>{}, std::integral_constant<int, 0xf>{});   // row_shr:1
    step(std::integral_constant<int, 0x112>{}, std::integral_constant<int, 0xf>{});   // row_shr:2
    step(std::integral_constant<int, 0x114>{}, std::integral_constant<int, 0xf>{});   // row_shr:4
    step(std::integral_constant<int, 0x118>{}, std::integral_constant<int, 0xf>{});   // row_shr:8
    step(std::integral_constant<int, 0x142>{}, std::integral_constant<int, 0xa>{});   // row_bcast:15
    step(std::integral_constant<int, 0x143>{}, std::integral_constant<int, 0xc>{});   // row_bcast:31
    return v;
}

template <class T>
__device__ __forceinline__ T wave_scan(T v)
{
    return wave_scan_by(v, [](T a, T b) { return a + b; });
}

__device__ __forceinline__ float wave_scan_max(float v)
{
    return wave_scan_by(v, [](float a, float b) { return fmaxf(a, b); });
}

__device__ __forceinline__ int lane_value(int v, int lane)
{
    return __builtin_amdgcn_readlane(v, lane);
}

// Units and partial outputs of the sequences before one (workspace).
struct Before {
    int units, slots;
};

// What is known of a sequence (a lane's) to find a unit in it.
struct Share {
    int tiles, c, units, slots;   // row tiles, pieces of each, and theirs of all kv heads
};

// How row tiles are cut: those of kt key tiles in kt / each pieces, rounded down,
// but in `least` where that is above 1, and no shorter than `tiles`.
struct Split {
    float each;
    int least, tiles;
};

template <class F>
__device__ __forceinline__ Share share_of(const CacheAttnParams &p, const SeqPlan &r, Split split)
{
    const float x = (float)r.kt * (1.0f / split.each) + 0.01f;   // (an even share stays one under the sums' rounding)
    const int c = x > 1.02f && x < 2.0f ? split.least : (int)x, most = r.kt / split.tiles, fit = c < most ? c : most;
    const int pieces = fit < 1 ? 1 : fit, units = r.tiles * p.b.Hkv * pieces;
    return {r.tiles, pieces, units, pieces > 1 ? units : 0};
}

// Sums over a form's row tiles (of one head): their number, the key tiles they
// visit at most and on average; and the most that one visits.
struct Work {
    float tiles, most, mean, longest;
};

__device__ __forceinline__ void add(Work &w, const SeqPlan &r)
{
    const float t = (float)r.tiles;
    w.tiles += t;
    w.most += t * (float)r.kt;
    w.mean += t * r.mean;
    w.longest = fmaxf(w.longest, r.tiles ? (float)r.kt : 0.0f);
}

// An even share of the work is `each` key tiles.  Pieces are no shorter, so that
// they fill the device once and not a little more: 80 row tiles of 6640 keys
// take 86 us, with pieces no longer than the share 119; nine single tokens of
// 8000 keys 41 instead of 48.  But where prompts' row tiles visit unlike numbers
// of keys, those longer than the share are cut in two (prompts of 300 to 1300
// tokens together: 100 us instead of 123).  In the launch of both forms pieces
// are of 8 tiles at least, as if single tokens' units, which that launch is for,
// filled the rest of the device (512 tokens after 1000 keys beside 15 single
// tokens: 71 us, of 5 tiles 76).
template <class F>
__device__ __forceinline__ Split split_of(const CacheAttnParams &p, const Work &w)
{
    const int tiles = F::FORM && p.units[0] && !p.apart ? 8 : F::MIN_TILES;
    const float each = fmaxf(w.most * (float)p.b.Hkv * (1.0f / F::TARGET), (float)tiles);
    return {each, F::FORM && w.mean < EVEN * w.tiles * w.longest ? 2 : 1, tiles};
}

// Unit `local` of sequence s, whose partial outputs start at `slots`.  (Tables
// that break their rules may count past the bounds: such units are left out.)
template <class F>
__device__ __forceinline__ Unit unit_of(const CacheAttnParams &p, int s, int tiles, int c, int local, int slots)
{
    const int pair = local / c, slot = slots + local;
    if (local < 0 || pair >= tiles * p.b.Hkv || (c > 1 && (slot < 0 || slot >= p.slots[F::FORM]))) return {-1, 0, 0, 0, 0, 0};
    // (causal: the last row tiles see most keys, and start first)
    return {s, tiles - 1 - pair / p.b.Hkv, pair % p.b.Hkv, local - pair * c, c, slot};
}

// Of the wave's lanes together.
__device__ __forceinline__ Work wave_work(Work w)
{
    auto last = [](float v) { return __builtin_bit_cast(float, lane_value(__builtin_bit_cast(int, v), 63)); };
    w = {wave_scan(w.tiles), wave_scan(w.most), wave_scan(w.mean), wave_scan_max(w.longest)};
    return {last(w.tiles), last(w.most), last(w.mean), last(w.longest)};
}

// Unit x, by a wave that plans for itself: lane l has the EACH sequences from
// EACH l.
template <class F, int EACH>
__device__ __forceinline__ Unit plan_alone(const CacheAttnParams &p, int G, int x)
{
    const int lane = threadIdx.x & 63;
    SeqPlan r[EACH];
    Work w = {};
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        const int s = EACH * lane + i;
        r[i] = s < p.b.S ? seq_plan<F>(p, s, G) : SeqPlan{};
        add(w, r[i]);
    }
    const Split split = split_of<F>(p, wave_work(w));
    Share h[EACH];
    int units = 0, slots = 0;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        h[i] = share_of<F>(p, r[i], split);
        units += h[i].units;
        slots += h[i].slots;
    }
    const int ui = wave_scan(units), si = wave_scan(slots);
    if (x == 0 && p.slots[F::FORM] && threadIdx.x == 0) p.counts[F::FORM] = lane_value(si, 63);
    const uint64_t hit = __ballot(x >= ui - units && x < ui);
    if (!hit) return {-1, 0, 0, 0, 0, 0};
    const int l = __builtin_ctzll(hit);
    int local = x - lane_value(ui - units, l), before = lane_value(si - slots, l), i = 0;
    Share at = {lane_value(h[0].tiles, l), lane_value(h[0].c, l), lane_value(h[0].units, l), lane_value(h[0].slots, l)};
#pragma unroll
    for (int k = 1; k < EACH; ++k) {
        if (i == k - 1 && local >= at.units) {
            local -= at.units;
            before += at.slots;
            at = {lane_value(h[k].tiles, l), lane_value(h[k].c, l), lane_value(h[k].units, l), lane_value(h[k].slots, l)};
            i = k;
        }
    }
    return unit_of<F>(p, EACH * l + i, at.tiles, at.c, local, before);
}

template <class F>
__device__ __forceinline__ Unit unit_at(const CacheAttnParams &p, int G, int x)
{
    if (p.b.S == 1) {
        const SeqPlan r = seq_plan<F>(p, 0, G);
        Work w = {};
        add(w, r);
        const Share h = share_of<F>(p, r, split_of<F>(p, w));
        if (x == 0 && p.slots[F::FORM] && threadIdx.x == 0) p.counts[F::FORM] = h.slots;
        return unit_of<F>(p, 0, h.tiles, h.c, x, 0);
    }
    if (p.b.S <= 64) return plan_alone<F, 1>(p, G, x);
    if (p.b.S <= PLAN_ALONE) return plan_alone<F, PLAN_ALONE / 64>(p, G, x);
    const Before *before = static_cast<const Before *>(p.before[F::FORM]);
    const int s = last_at_most(p.b.S, x, [&](int i) { return (int64_t)before[i].units; });
    const Share h = share_of<F>(p, seq_plan<F>(p, s, G), static_cast<const Split *>(p.split)[F::FORM]);
    return unit_of<F>(p, s, h.tiles, h.c, x - before[s].units, before[s].slots);
}

// Unit x of form F, the same in each of the workgroup's waves (in scalar
// registers, whatever it was worked out in).
template <class F>
__device__ __forceinline__ Unit find_unit(const CacheAttnParams &p, int G, int x)
{
    const Unit u = unit_at<F>(p, G, x);
    auto same = [](int v) { return __builtin_amdgcn_readfirstlane(v); };
    return {same(u.s), same(u.tile), same(u.head), same(u.piece), same(u.pieces), same(u.slot)};
}

// What cache_join_kernel needs to know of a partial output; each unit writes its own.
struct PartInfo {
    int token, row0, rows, head;   // first token of the sequence, rows [row0, row0 + rows) of it
    int piece, pieces, unused[2];
};

template <class F>
__device__ __forceinline__ void write_info(const CacheAttnParams &p, const Unit &u, int token, int row0, int rows)
{
    if (u.pieces > 1 && threadIdx.x == 0) {
        PartInfo *i = static_cast<PartInfo *>(p.info[F::FORM]) + u.slot;
        *i = {token, row0, rows, u.head, u.piece, u.pieces, {0, 0}};
    }
}

// The factor that finishes o, and lse, from a row's maximum m and sum l of
// exponentials (l == 0: the row saw no key, and is 0, or only logits of
// -infinity, and is 0/0).
__device__ __forceinline__ float finish(float m, float l)
{
    return l != 0.0f ? 1.0f / l : (m == NEG_INF ? 0.0f : __builtin_nanf(""));
}

__device__ __forceinline__ float finish_lse(float m, float l)
{
    return l == 0.0f ? NEG_INF : (m + __builtin_amdgcn_logf(l)) * LN2;
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

// NaN among the values of keys that only some rows of a workgroup see: the
// matrix product takes them as 0 (0 * NaN would reach every row), and a bit for
// each row and channel in LDS makes those that see one NaN at the end.
// `nan`: nan_bytes of the word of 4 keys from `key`, of channel d; sees(r, key):
// whether row r of the workgroup's `rows` does.
template <int D, class SEES>
__device__ __forceinline__ void mark_nan(uint32_t (*marks)[D / 32], uint32_t nan, int d, int key, int rows, SEES sees)
{
    for (; nan; nan &= nan - 1) {
        const int k = key + (__builtin_ctz(nan) >> 3);
        for (int r = 0; r < rows; ++r)
            if (sees(r, k)) atomicOr(&marks[r][d >> 5], 1u << (d & 31));
    }
}

} // namespace
} // namespace lamp
