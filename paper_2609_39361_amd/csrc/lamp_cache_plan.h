// lamp_cache_plan.h -- the cache attention's division of work and the pieces its
// kernels share (library-internal, device code).
#pragma once
#include <hip/hip_runtime.h>

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
constexpr int TILE = 64;       // keys of the plan's tiles

// The two forms of the attention kernel.  ROWS: query rows of a workgroup (row
// = token * G + head of the group); TARGET: workgroups that fill the 256 CUs;
// MIN_TILES: least key tiles of a piece.
struct FewRows {       // single tokens and short chunks (lamp_cache_attn.hip)
    static constexpr int ROWS = 16, TARGET = 512, MIN_TILES = 4;
};
struct ManyRows {      // prompts (lamp_cache_prompt.hip)
    static constexpr int ROWS = 256, TARGET = 256, MIN_TILES = 8;
};

// The key range of one sequence is cut in pieces when its row tiles alone do
// not fill the device: with `total` the key tiles of all (sequence, row tile,
// kv head) triples, pieces hold about total / target tiles.  Every workgroup
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

template <class F>
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
    const int64_t rows = (int64_t)r.n * G;
    r.tiles = rows > p.rows_above && rows <= p.rows_upto ? (int)((rows + F::ROWS - 1) / F::ROWS) : 0;
    r.kt = (r.len + TILE - 1) / TILE;
    if (p.window > 0) {
        const int64_t span = ((int64_t)p.window + F::ROWS - 1 + TILE - 1) / TILE + 1;
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
template <class F>
__device__ int piece_tiles(const CacheAttnParams &p, int G)
{
    int64_t total = 0;
    for (int s = threadIdx.x & 63; s < p.b.S; s += 64) {
        const SeqPlan r = seq_plan<F>(p, s, G);
        total += (int64_t)r.tiles * r.kt;
    }
    total = wave_sum(total) * p.b.Hkv;
    const int64_t c = (total + F::TARGET - 1) / F::TARGET;
    return (int)(c < F::MIN_TILES ? F::MIN_TILES : (c < 1 << 24 ? c : 1 << 24));
}

// Unit x of the plan; with `joined`, unit x among the (row tile, kv head) pairs
// of split sequences instead (piece 0, slot of the first piece).
template <class F>
__device__ Unit find_unit(const CacheAttnParams &p, int G, int64_t x, bool joined)
{
    const int lane = threadIdx.x & 63;
    const int chunk = piece_tiles<F>(p, G);
    int64_t units = 0, slots = 0;   // of the sequences before this round of 64
    for (int s0 = 0; s0 < p.b.S; s0 += 64) {
        const int s = s0 + lane;
        int64_t pairs = 0;
        int c = 1, tiles = 0;
        if (s < p.b.S) {
            const SeqPlan r = seq_plan<F>(p, s, G);
            tiles = r.tiles;
            pairs = (int64_t)tiles * p.b.Hkv;
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
            r.tile = __shfl(tiles, l, 64) - 1 - (int)(pair / p.b.Hkv);   // (causal: the last row tiles see most keys, and start first)
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

// Row tiles times kv heads that the batch can have at most.
template <class F>
int64_t max_pairs(const CacheAttnParams &p)
{
    const int G = p.Hq / p.b.Hkv;
    return ((int64_t)p.b.T * G / F::ROWS + p.b.S) * p.b.Hkv;
}

// A sequence of kt key tiles and `pairs` row tiles times heads is cut in
// c = ceil(kt / chunk) < 1 + kt / chunk pieces, and sum(pairs kt) / chunk <=
// TARGET: below max_pairs + TARGET units in all.  Where c >= 2, c < 2 kt / chunk:
// below 2 TARGET partial outputs, of below TARGET row tiles times heads.
// Sequences no longer than one piece need none.
template <class F>
int max_units(const CacheAttnParams &p)
{
    return (int)(max_pairs<F>(p) + (p.slots ? F::TARGET : 0));
}

} // namespace
} // namespace lamp
