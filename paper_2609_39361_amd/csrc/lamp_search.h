// lamp_search.h -- a workgroup's place in a ragged batch (library-internal, device
// code).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "lamp_serve.h"

namespace lamp {
namespace {

// Sequence whose range of the non-decreasing starts f(0..S-1) holds x: the
// last s with f(s) <= x, by the whole wave, 64 places at once (each round is
// one load's latency).
template <class F>
__device__ __forceinline__ int last_at_most(int S, int64_t x, F f)
{
    const int lane = threadIdx.x & 63;
    int lo = 0, n = S;
    for (;;) {
        const int step = (n + 63) / 64;
        const int at = lo + lane * step;
        const uint64_t below = __ballot(lane == 0 || (lane * step < n && f(at) <= x));
        lo += (63 - __builtin_clzll(below)) * step;
        if (step == 1) return lo;
        n = S - lo < step ? S - lo : step;
    }
}

// The new tokens of one page: `count` slots from `first`, tokens from `tok`,
// positions from `pos` (count 0: nothing to do).
struct PageWork {
    int64_t page;
    int first, count, tok, pos;
};

// Work of workgroup x.  By token: token x's page, if x is the first new token
// in it.  By slot: sequence s owns the slots from floor(start_s / page) + 2 s,
// which leaves it n/page + 2 of them at least, as many as n tokens can touch.
// Whatever the tables hold, nothing outside the caller's arrays is read.
__device__ PageWork page_work(const PagedBatch &b, int by_token, int x)
{
    const PageWork none = {0, 0, 0, 0, 0};
    auto start = [&](int s) { return b.q_start ? b.q_start[s] : s; };
    const int ps = b.page_shift, page = 1 << ps;
    auto first = [&](int a, int i) { return by_token ? (int64_t)a : (int64_t)(a >> ps) + 2 * (int64_t)i; };
    int s, a, e, keys;
    if (b.S > 1 && b.S <= 64) {   // (a lane for each sequence: one load's latency)
        const int i = (int)(threadIdx.x & 63) < b.S ? (int)(threadIdx.x & 63) : b.S - 1;
        const int ai = start(i), ei = start(i + 1), ki = b.kv_lens[i];
        s = 63 - __builtin_clzll(__ballot(i == 0 || first(ai, i) <= x));
        s = s < b.S ? s : b.S - 1;   // (the lanes behind the last sequence repeat it)
        a = __builtin_amdgcn_readlane(ai, s);
        e = __builtin_amdgcn_readlane(ei, s);
        keys = __builtin_amdgcn_readlane(ki, s);
    } else {
        s = b.S == 1 ? 0 : last_at_most(b.S, x, [&](int i) { return first(start(i), i); });
        a = start(s);
        e = start(s + 1);
        keys = b.kv_lens[s];
    }
    if (a < 0 || e > b.T || e <= a) return none;
    const int64_t len = keys, p0 = len - (e - a);           // position of the first new token
    const int64_t q0 = p0 > 0 ? p0 : 0;                       // first position that exists
    int64_t idx;
    if (by_token) {
        if (x < a || x >= e) return none;
        const int64_t p = p0 + (x - a);
        if (p < q0 || (p != q0 && (p & (page - 1)) != 0)) return none;
        idx = p >> ps;
    } else {
        idx = (q0 >> ps) + (x - ((int64_t)(a >> ps) + 2 * (int64_t)s));
    }
    const int64_t lo = idx << ps, f = q0 > lo ? q0 : lo, end = len < lo + page ? len : lo + page;
    if (f >= end || idx >= b.width) return none;
    const int64_t pg = b.table[s * b.table_stride + idx];
    if (pg < 0 || pg >= b.pages) return none;
    return {pg, (int)(f - lo), (int)(end - f), (int)(a + (f - p0)), (int)f};
}

} // namespace
} // namespace lamp
