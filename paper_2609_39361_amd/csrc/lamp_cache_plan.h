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
struct ManyRows {      // prompts (lamp_cache_many.h; 32 row tiles' window of 1024: 31 us with pieces of 5 tiles at least, 37 of 8)
    static constexpr int ROWS = 256, TARGET = 256, MIN_TILES = 5, FORM = 1;
};

// A group's rows over their shared prefix (lamp_cache_prefix.h).  Two workgroups fill a
// CU's registers, but share its issue: units for one a CU (behind 8192 shared keys, without
// others of their own: 32 tokens 20 us, 64 tokens 27, 250 tokens 73; for two 26, 32 and 80).
struct PrefixRows {
    static constexpr int ROWS = 32, TARGET = 256, MIN_TILES = 8, FORM = 2;
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
    int row;         // of the table
    int lo, causal;  // first key of the range; whether a row sees none behind its own position
};

// Row tiles whose mean is this part of the longest at least count as even.
constexpr float EVEN = 0.75f;

template <class F>
__device__ __forceinline__ SeqPlan seq_plan(const CacheAttnParams &p, int s, int G)
{
    SeqPlan r;
    r.row = s;
    r.lo = 0;
    r.causal = p.causal;
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

// Groups of sequences with a shared prefix (lamp_cache_shared.hip): what is
// planned is each group's new tokens over the prefix (in the forms 1 and 2), then each
// sequence's over the keys behind it (in the forms 0 and 1).
// (Without branches: the loads of several sequences do not wait for each other.)
template <class F>
__device__ __forceinline__ SeqPlan seq_plan(const SharedAttnParams &p, int v, int G)
{
    SeqPlan r;
    const bool group = F::FORM == 2 || (F::FORM == 1 && v < p.groups);
    const int at = group ? v : 0, g0 = F::FORM == 0 ? 0 : p.group_start[at], g1 = F::FORM == 0 ? 0 : p.group_start[at + 1];
    const int s = group ? g0 : (F::FORM == 0 ? v : v - p.groups), s1 = group ? g1 : s + 1;
    const bool is = s >= 0 && s1 <= p.b.S && s < s1;
    const int i = is ? s : 0, i1 = is ? s1 : 0;
    const int a = p.b.q_start ? p.b.q_start[i] : i, e = p.b.q_start ? p.b.q_start[i1] : i1;
    const int keys = p.b.kv_lens[i], said = p.prefix_lens[i], page = 1 << p.b.page_shift, reach = p.b.width << p.b.page_shift;   // (at most 2^30)
    const int whole = said > 0 ? said & ~(page - 1) : 0, prefix = whole < reach ? whole : reach, len = keys > 0 ? keys : 0;
    r.row = i;
    r.a = a;
    r.n = is && a >= 0 && e <= p.b.T && e > a && (!group || prefix > 0) ? e - a : 0;
    r.causal = !group;
    r.lo = group ? 0 : prefix;
    r.pos0 = group ? 0 : len - r.n;
    r.all = group ? prefix : len;
    r.len = r.all < reach ? r.all : reach;
    const int rows = r.n * G;                        // (at most 2^27)
    const int above = group ? p.group_above[F::FORM] : p.rows_above[F::FORM], upto = group ? p.group_upto[F::FORM] : p.rows_upto[F::FORM];
    r.tiles = rows > above && rows <= upto ? (rows + F::ROWS - 1) / F::ROWS : 0;
    const int span = r.len > r.lo ? r.len - r.lo : 0;
    r.kt = (span + TILE - 1) / TILE;
    r.mean = group ? 1.0f : 0.0f;                    // (what split_of counts here)
    return r;
}

// A token and its list of pages: planned from the sizes alone.
constexpr int PAGES_LISTED = 1024;   // entries of a piece

template <class F>
__device__ __forceinline__ SeqPlan seq_plan(const PagesAttnParams &p, int t, int)
{
    SeqPlan r = {};
    int s = t, e = t + 1, a = t;
    if (p.b.q_start) {
        s = last_at_most(p.b.S, t, [&](int i) { return (int64_t)p.b.q_start[i]; });
        a = p.b.q_start[s];
        e = p.b.q_start[s + 1];
    }
    const int len = p.b.kv_lens[s] > 0 ? p.b.kv_lens[s] : 0, reach = p.b.width << p.b.page_shift;
    r.row = s;
    r.a = t;
    r.n = a >= 0 && a <= t && t < e && e <= p.b.T;
    r.causal = 1;
    r.pos0 = len - (e - t);
    r.all = len;
    r.len = len < reach ? len : reach;
    return r;
}

// What a plan of attn_shared goes over; and whether a sequence's units of `pieces`
// pieces leave partial outputs to be joined.
template <class F>
__device__ __forceinline__ int planned(const SharedAttnParams &p) { return F::FORM == 2 ? p.groups : p.b.S + (F::FORM == 1 ? p.groups : 0); }
__device__ __forceinline__ bool joined(const CacheAttnParams &, const SeqPlan &, int pieces) { return pieces > 1; }
__device__ __forceinline__ bool joined(const PagesAttnParams &, const SeqPlan &, int pieces) { return pieces > 1; }
__device__ __forceinline__ bool joined(const SharedAttnParams &, const SeqPlan &r, int pieces)
{
    return pieces > 1 || r.lo > 0 || !r.causal;
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

constexpr float SOON = 1.02f, NEVER = 2.0f;   // (of Split.two)

// How row tiles are cut: those of kt key tiles in kt / each pieces, rounded down,
// but in two where that is above `two`, and no shorter than `tiles`.
struct Split {
    float each, two;
    int tiles;
};

template <class F, class P>
__device__ __forceinline__ Share share_of(const P &p, const SeqPlan &r, Split split)
{
    const float x = (float)r.kt * (1.0f / split.each) + 0.01f;   // (an even share stays one under the sums' rounding)
    const float two = std::is_same_v<P, SharedAttnParams> && F::FORM == 1 && r.causal ? SOON : split.two;
    const int c = x > two && x < 2.0f ? 2 : (int)x, most = r.kt / split.tiles, fit = c < most ? c : most;
    const int pieces = fit < 1 ? 1 : fit, units = r.tiles * p.b.Hkv * pieces;
    return {r.tiles, pieces, units, joined(p, r, pieces) ? units : 0};
}

// Sums over a form's row tiles (of one head): their number, the key tiles they
// visit at most and on average (of attn_shared, instead: the number of its groups'
// row tiles); and the most that one visits.
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
    const int tiles = F::FORM == 1 && p.units[0] && !p.apart ? 8 : F::MIN_TILES;
    const float each = fmaxf(w.most * (float)p.b.Hkv * (1.0f / F::TARGET), (float)tiles);
    return {each, F::FORM && w.mean < EVEN * w.tiles * w.longest ? SOON : NEVER, tiles};
}

// Of attn_shared: two of the workgroups of the form for prefixes share a CU, and are
// cut as soon as they can.  The row tiles of prefixes in the form for many are cut in
// two where all halves start at once or not even all whole ones do (questions of 100 to
// 300 tokens about documents: 128 row tiles of 1.98 shares 339 us, uncut 477; 264 of 0.7
// and 1.1: 227, uncut 289; but 232 of 1.0 and 1.1: 190, uncut 163; 168 of 1.45: 195 and
// 166); those of sequences, which are fewer and shorter, always.
template <class F>
__device__ __forceinline__ Split split_of(const SharedAttnParams &p, const Work &w)
{
    const float each = fmaxf(w.most * (float)p.b.Hkv * (1.0f / F::TARGET), (float)F::MIN_TILES);
    const float whole = w.mean * (float)p.b.Hkv * (1.0f / F::TARGET);
    return {each, F::FORM == 2 || (F::FORM == 1 && (whole <= 0.5f || whole > 1.0f)) ? SOON : NEVER, F::MIN_TILES};
}

// Unit `local` of sequence s, whose partial outputs start at `slots`.  (Tables
// that break their rules may count past the bounds: such units are left out.)
template <class F, class P>
__device__ __forceinline__ Unit unit_of(const P &p, int s, int tiles, int c, int local, int slots)
{
    constexpr bool ANY = !std::is_same_v<P, CacheAttnParams>;   // (one piece may have a partial output too)
    const int pair = local / c, slot = slots + local;
    if (local < 0 || pair >= tiles * p.b.Hkv || ((ANY || c > 1) && (slot < 0 || slot >= p.slots[F::FORM]))) return {-1, 0, 0, 0, 0, 0};
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

template <class F>
__device__ __forceinline__ Unit find_unit(const PagesAttnParams &p, int G, int x)
{
    const int tiles = (G + F::ROWS - 1) / F::ROWS, piece = x % p.pieces, y = x / p.pieces, z = y / tiles;
    return {z / p.b.Hkv, y - z * tiles, z % p.b.Hkv, piece, p.pieces, 0};
}

// Unit x and its sequence's plan.
template <class F, class P>
__device__ __forceinline__ void locate(const P &p, int G, int x, Unit &u, SeqPlan &sq)
{
    u = find_unit<F>(p, G, x);
    if (u.s >= 0) sq = seq_plan<F>(p, u.s, G);
}

// What attn_shared's plan of more than SHARED_ALONE groups and sequences leaves for
// each of them and form (workspace): where its units and partial outputs begin, its
// row tiles and pieces of each, and what a unit needs to know of it.
struct SeqInfo {
    int units, slots, tiles, c;
    int row, a, n, all, len, pos0, lo, causal;
};
constexpr int SHARED_ALONE = 128;   // (the launch takes 5.8 us: 250 tokens behind 8192 keys, without others of their own, 74 us with it, 83 without; 160 the same)

// Unit x and its sequence's plan, by a wave that plans for itself: lane l has the EACH
// groups and sequences from EACH l, and the plan comes from the lane that has it.
template <class F, int EACH>
__device__ __forceinline__ void locate_alone(const SharedAttnParams &p, int G, int x, int many, Unit &u, SeqPlan &sq)
{
    const int lane = threadIdx.x & 63;
    SeqPlan r[EACH];
    Work w = {};
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        const int v = EACH * lane + i;
        r[i] = seq_plan<F>(p, v < many ? v : many - 1, G);
        if (v >= many) r[i].tiles = 0;
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
    const uint64_t hit = __ballot(x >= ui - units && x < ui);
    if (!hit) return;
    // in each lane as if it were the one
    int local = x - (ui - units), before = si - slots, k = 0;
#pragma unroll
    for (int i = 1; i < EACH; ++i) {
        if (k == i - 1 && local >= h[i - 1].units) {
            local -= h[i - 1].units;
            before += h[i - 1].slots;
            h[0] = h[i];
            r[0] = r[i];
            k = i;
        }
    }
    const int l = __builtin_ctzll(hit);
    auto of = [&](int v) { return lane_value(v, l); };
    u = unit_of<F>(p, of(EACH * lane + k), of(h[0].tiles), of(h[0].c), of(local), of(before));
    sq = {of(r[0].a), of(r[0].n), of(r[0].all), of(r[0].len), of(r[0].pos0), 0, 0, 0.0f, of(r[0].row), of(r[0].lo), of(r[0].causal)};
}

// Or from the plan of a launch of its own, which has a place for every unit.
template <class F>
__device__ __forceinline__ void locate(const SharedAttnParams &p, int G, int x, Unit &u, SeqPlan &sq)
{
    const int many = planned<F>(p);
    u = {-1, 0, 0, 0, 0, 0};
    if (p.b.S + p.groups > SHARED_ALONE) {
        if (x >= p.counts[F::FORM]) return;
        const int v = __builtin_amdgcn_readfirstlane(static_cast<const int *>(p.unit_seq[F::FORM])[x]);
        const SeqInfo i = static_cast<const SeqInfo *>(p.before[F::FORM])[v];
        u = unit_of<F>(p, v, i.tiles, i.c, x - i.units, i.slots);
        sq = {i.a, i.n, i.all, i.len, i.pos0, 0, 0, 0.0f, i.row, i.lo, i.causal};
    } else if (many <= 64) {
        locate_alone<F, 1>(p, G, x, many, u, sq);
    } else {
        locate_alone<F, SHARED_ALONE / 64>(p, G, x, many, u, sq);
    }
}

template <class F>
__device__ __forceinline__ void write_info(const PagesAttnParams &, const Unit &, const SeqPlan &, int, int) {}

// What cache_join_kernel needs to know of a partial output; each unit writes its own.
struct PartInfo {
    int token, row0, rows, head;   // first token of the sequence, rows [row0, row0 + rows) of it
    int piece, pieces, unused[2];
};

template <class F>
__device__ __forceinline__ void write_info(const CacheAttnParams &p, const Unit &u, const SeqPlan &sq, int row0, int rows)
{
    if (u.pieces > 1 && threadIdx.x == 0) {
        PartInfo *i = static_cast<PartInfo *>(p.info[F::FORM]) + u.slot;
        *i = {sq.a, row0, rows, u.head, u.piece, u.pieces, {0, 0}};
    }
}

// Where a row's partial outputs of one of its two ranges lie, for the join of
// attn_shared: the first one's row among all, and 4 pieces + form (0: none).
struct RowInfo {
    int at, pieces4;
};

// Of the first piece's unit, for its rows: [0][T][Hq] the prefix, [1][T][Hq] the
// keys behind it.
template <class F>
__device__ __forceinline__ void write_info(const SharedAttnParams &p, const Unit &u, const SeqPlan &sq, int row0, int rows)
{
    if (u.piece != 0) return;
    const int G = p.Hq / p.b.Hkv;
    const int base = u.slot * F::ROWS + (F::FORM > 0 ? p.slots[0] * FewRows::ROWS : 0) + (F::FORM > 1 ? p.slots[1] * ManyRows::ROWS : 0);
    const bool part = joined(p, sq, u.pieces);
    RowInfo *info = static_cast<RowInfo *>(p.rows);
    for (int r = (int)threadIdx.x; r < rows; r += (int)blockDim.x) {
        const int gr = row0 + r, t = gr / G;
        const int64_t row = (int64_t)(sq.a + t) * p.Hq + u.head * G + gr - t * G;
        info[(sq.causal ? (int64_t)p.b.T * p.Hq : 0) + row] = part ? RowInfo{base + r, 4 * u.pieces + F::FORM} : RowInfo{0, 0};
        if (sq.causal && sq.lo == 0) info[row] = RowInfo{0, 0};
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

// Over all lanes of the wave, in all of them.
template <class OP>
__device__ __forceinline__ float wave_all(float v, OP op)
{
    auto step = [&](auto ctrl) {
        const int x = __builtin_bit_cast(int, v);
        v = op(v, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(x, x, decltype(ctrl)::value, 0xf, 0xf, false)));
    };
    step(std::integral_constant<int, 0xB1>{});    // quad_perm 1,0,3,2
    step(std::integral_constant<int, 0x4E>{});    // quad_perm 2,3,0,1
    step(std::integral_constant<int, 0x141>{});   // row_half_mirror
    step(std::integral_constant<int, 0x140>{});   // row_mirror
    const auto a = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, v), __builtin_bit_cast(uint32_t, v), false, false);
    v = op(__builtin_bit_cast(float, (uint32_t)a[0]), __builtin_bit_cast(float, (uint32_t)a[1]));
    const auto b = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, v), __builtin_bit_cast(uint32_t, v), false, false);
    return op(__builtin_bit_cast(float, (uint32_t)b[0]), __builtin_bit_cast(float, (uint32_t)b[1]));
}

// A row's partial outputs joined by a wave and written (attn_shared, attn_pages):
// n0 of them from row at0 of `part` on, step0 rows apart, then n1 from at1.  A lane
// holds D/64 channels, and for each 64 partial outputs the maximum and sum of one.
// Bound by latency: 16 rows are requested at once, the first before the maxima are
// waited for (16 partial outputs of 32 rows 3.6 us; with the loads one after another
// 7.2).  Not written where not `live`.
template <int D>
__device__ __forceinline__ void join_row(const float *part, const float *ml, int at0, int step0, int n0, int at1, int step1, int n1, bool live,
                                         uint16_t *o, float *lse)
{
    constexpr int C = D / 64, AT = 16;
    const int lane = threadIdx.x & 63, n = n0 + n1;
    auto row_of = [&](int k) { return k < n0 ? at0 + k * step0 : at1 + (k - n0) * step1; };
    float m = NEG_INF, sum = 0.0f, v[C] = {}, x[AT][C];
    auto request = [&](int k0) {
#pragma unroll
        for (int j = 0; j < AT; ++j) {   // (beyond the last: read again, not added)
            const float *r = part + (int64_t)row_of(k0 + j < n ? k0 + j : k0) * D + C * lane;
#pragma unroll
            for (int e = 0; e < C; ++e) x[j][e] = r[e];
        }
    };
    request(0);
    for (int c0 = 0; c0 < n; c0 += 64) {
        const int mine = c0 + lane;
        const int64_t at = (int64_t)row_of(mine < n ? mine : c0) * 2;
        const float m_at = ml[at], l_at = ml[at + 1], mc = mine < n ? m_at : NEG_INF;
        const float mn = fmaxf(wave_all(mc, [](float a, float b) { return fmaxf(a, b); }), m);
        const float ms = mn == NEG_INF ? 0.0f : mn, f0 = __builtin_amdgcn_exp2f(m - ms);
        const float f = __builtin_amdgcn_exp2f(mc - ms);
        m = mn;
        sum = sum * f0 + wave_all(mine < n ? l_at * f : 0.0f, [](float a, float b) { return a + b; });
#pragma unroll
        for (int e = 0; e < C; ++e) v[e] *= f0;
        const int end = n - c0 < 64 ? n : c0 + 64;
        for (int k0 = c0; k0 < end; k0 += AT) {
#pragma unroll
            for (int j = 0; j < AT; ++j) {
                const bool is = k0 + j < end;   // (no branch: loads would wait in it, one after another)
                const float fj = __builtin_bit_cast(float, lane_value(__builtin_bit_cast(int, f), k0 + j - c0));
#pragma unroll
                for (int e = 0; e < C; ++e) v[e] += is ? x[j][e] * fj : 0.0f;
            }
            if (k0 + AT < n) request(k0 + AT);
        }
    }
    if (!live) return;
    const float inv = finish(m, sum);
    if constexpr (C == 1) {
        o[lane] = (uint16_t)pack2(v[0] * inv, 0.0f);
    } else {
#pragma unroll
        for (int e = 0; e < C; e += 2) *reinterpret_cast<uint32_t *>(o + C * lane + e) = pack2(v[e] * inv, v[e + 1] * inv);
    }
    if (lane == 0) *lse = finish_lse(m, sum);
}

// The same by 16 lanes, for rows of few partial outputs (their weights in each lane).
template <int D>
__device__ __forceinline__ void join_row16(const float *part, const float *ml, int at0, int step0, int n0, int at1, int step1, int n1,
                                           uint16_t *o, float *lse)
{
    constexpr int C = D / 16, AT = 2;
    const int lane = threadIdx.x & 15, n = n0 + n1;
    auto row_of = [&](int k) { return k < n0 ? at0 + k * step0 : at1 + (k - n0) * step1; };
    float m = NEG_INF, sum = 0.0f, v[C] = {};
    for (int c0 = 0; c0 < n; c0 += AT) {
        float mc[AT], lc[AT];
        f32x4 x[AT][C / 4];
#pragma unroll
        for (int k = 0; k < AT; ++k) {   // (beyond the last: read again, not added)
            const int64_t at = row_of(c0 + k < n ? c0 + k : c0);   // (below 2^31 partial outputs)
            mc[k] = ml[at * 2];
            lc[k] = ml[at * 2 + 1];
#pragma unroll
            for (int e = 0; e < C / 4; ++e) x[k][e] = *reinterpret_cast<const f32x4 *>(part + at * D + 4 * (16 * e + lane));
        }
        float mn = m;
#pragma unroll
        for (int k = 0; k < AT; ++k) mn = fmaxf(mn, mc[k]);
        const float ms = mn == NEG_INF ? 0.0f : mn, f0 = __builtin_amdgcn_exp2f(m - ms);
        m = mn;
        sum *= f0;
#pragma unroll
        for (int e = 0; e < C; ++e) v[e] *= f0;
#pragma unroll
        for (int k = 0; k < AT; ++k) {
            const bool is = c0 + k < n;
            const float f = __builtin_amdgcn_exp2f(mc[k] - ms);
            sum += is ? lc[k] * f : 0.0f;
#pragma unroll
            for (int e = 0; e < C; ++e) v[e] += is ? x[k][e / 4][e % 4] * f : 0.0f;
        }
    }
    const float inv = finish(m, sum);
#pragma unroll
    for (int e = 0; e < C; e += 4)
        *reinterpret_cast<u32x2 *>(o + 4 * (16 * (e / 4) + lane)) = u32x2{pack2(v[e] * inv, v[e + 1] * inv), pack2(v[e + 2] * inv, v[e + 3] * inv)};
    if (lane == 0) *lse = finish_lse(m, sum);
}

} // namespace
} // namespace lamp
