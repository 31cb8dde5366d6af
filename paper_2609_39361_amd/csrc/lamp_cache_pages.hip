// lamp_cache_pages.hip -- attention of each new token over the pages of a list: the
// row (token t at position p, head h) sees the keys j <= p of the places that
// places[t][h / G] names, and the mathematics are those of lamp_cache_attn.hip.
//
// A unit is the group of heads of one token and kv head against a part of its
// list, in the form for few rows (lamp_cache_few.h), whose keys are looked up in
// the list.  The lists are cut where tokens times kv heads do not fill the device:
// by their sizes, which the host knows, so that nothing is planned on the device.
// Bound by HBM (32 tokens over 64 pages of 64 keys, 8 heads, d = 128: 267 MB in 54 us, 5.0
// TB/s), for one token by latencies (7.7 us, and 3.6 for the join).
#include <hip/hip_runtime.h>

#include "lamp_cache_few.h"

namespace lamp {
namespace {

template <int D, int KT>
__global__ __launch_bounds__(256, 2) void cache_pages_kernel(PagesAttnParams p)
{
    __shared__ PagesShared<D, 4> sh;
    cache_few<D, KT, 4>(p, (int)blockIdx.x, sh);
}

template <int D>
__global__ __launch_bounds__(256) void pages_join_kernel(PagesAttnParams p)
{
    const int64_t row = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), rows = (int64_t)p.b.T * p.Hq;
    if (row >= rows) return;
    const int t = (int)row / p.Hq, last = p.b.q_start ? p.b.q_start[p.b.S] : p.b.S, first = p.b.q_start ? p.b.q_start[0] : 0;
    join_row<D>(p.part[0], p.part_ml[0], (int)row, (int)rows, p.pieces, 0, 0, 0, t < last && t >= first, p.o + row * D, p.lse + row);
}

struct Cut {
    int pieces, per;
};

// Parts of a list: as many as fill the device, of a tile for each wave at least and
// PAGES_LISTED entries at most, which fit the LDS beside another workgroup's.
Cut cut(int64_t T, int G, int Hkv, int64_t page, int64_t budget)
{
    const int64_t units = T * Hkv * ((G + FewRows::ROWS - 1) / FewRows::ROWS);
    const int64_t tile = page < TILE ? TILE / page : 1;   // entries of whole tiles
    const int64_t least = (FewRows::MIN_TILES * TILE + page - 1) / page;
    int64_t want = units < FewRows::TARGET ? FewRows::TARGET / units : 1;
    int64_t per = (budget + want - 1) / want;
    per = per < least ? least : per;
    per = per < PAGES_LISTED ? (per + tile - 1) / tile * tile : PAGES_LISTED;
    return {(int)((budget + per - 1) / per), (int)per};
}

struct Layout2 {
    size_t ml, part, total;
};

Layout2 pages_layout(int D, const Cut &c, int64_t rows)
{
    if (c.pieces <= 1) return {0, 0, 0};
    const size_t n = (size_t)rows * c.pieces, ml = (n * 2 * sizeof(float) + 255) & ~(size_t)255;
    return {0, ml, ml + n * D * sizeof(float)};
}

template <int D, int KT>
hipError_t launch_pages(const PagesAttnParams &p, hipStream_t s)
{
    const int G = p.Hq / p.b.Hkv;
    const int64_t units = (int64_t)p.b.T * p.b.Hkv * ((G + FewRows::ROWS - 1) / FewRows::ROWS) * p.pieces;
    cache_pages_kernel<D, KT><<<dim3((unsigned)units), 256, 0, s>>>(p);
    if (p.pieces > 1) pages_join_kernel<D><<<dim3((unsigned)(((int64_t)p.b.T * p.Hq + 3) / 4)), 256, 0, s>>>(p);
    return hipGetLastError();
}

} // namespace

size_t pages_attn_workspace(int D, int64_t T, int G, int Hkv, int64_t page, int64_t budget)
{
    return pages_layout(D, cut(T, G, Hkv, page, budget), T * G * Hkv).total;
}

hipError_t launch_pages_attn(int D, PagesAttnParams &p, void *ws, hipStream_t s)
{
    const Cut c = cut(p.b.T, p.Hq / p.b.Hkv, p.b.Hkv, (int64_t)1 << p.b.page_shift, p.budget);
    const Layout2 l = pages_layout(D, c, (int64_t)p.b.T * p.Hq);
    p.pieces = c.pieces;
    p.per = c.per;
    p.part_ml[0] = reinterpret_cast<float *>(static_cast<char *>(ws) + l.ml);
    p.part[0] = reinterpret_cast<float *>(static_cast<char *>(ws) + l.part);
    switch (D) {
    case 64: return launch_pages<64, 64>(p, s);
    case 128: return launch_pages<128, 64>(p, s);
    default: return launch_pages<256, 32>(p, s);
    }
}

} // namespace lamp
