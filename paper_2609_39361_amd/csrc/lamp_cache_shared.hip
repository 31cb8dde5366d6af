// lamp_cache_shared.hip -- causal attention of a ragged batch over the 8-bit paged
// cache where the sequences of a group hold the same first keys (the mathematics as
// in lamp_cache_attn.hip).
//
// A row's softmax over its keys [0, len) is joined from that over the group's prefix
// [0, P) and that over its own keys [P, len): with m_i, l_i, o_i the maximum, sum and
// unfinished output of a part, m = max m_i, l = sum l_i 2^(m_i - m), and likewise o.
// Every row sees the whole prefix, so that the new tokens of all sequences of a group
// are the rows of one product without a mask, and the prefix's codes are read once
// for all.  Both kinds of part, cut further where they do not fill the device, are
// units of one launch (lamp_cache_plan.h: what is planned is the groups, then the
// sequences), in the form for few rows or that for many; a second launch joins each
// row's partial outputs, whose places the first pieces leave (RowInfo).
#include <hip/hip_runtime.h>

#include "lamp_cache_many.h"

namespace lamp {
namespace {

template <int D, int KT>
__global__ __launch_bounds__(256, 2) void shared_few_kernel(SharedAttnParams p)
{
    __shared__ FewShared<D, 4> sh;
    cache_few<D, KT, 4>(p, (int)blockIdx.x, sh);
}

template <int D, int KT, int KF, bool WIDE>
__global__ __launch_bounds__(THREADS, 2) void shared_mixed_kernel(SharedAttnParams p)
{
    constexpr size_t A = sizeof(PromptShared<D, KT>), B = sizeof(FewShared<D, WAVES>);
    __shared__ __attribute__((aligned(16))) char sh[A > B ? A : B];
    const int x = (int)blockIdx.x;
    if (x < p.units[1]) cache_prompt<D, KT, WIDE>(p, x, *reinterpret_cast<PromptShared<D, KT> *>(sh));
    else cache_few<D, KF, WAVES>(p, x - p.units[1], *reinterpret_cast<FewShared<D, WAVES> *>(sh));
}

__global__ __launch_bounds__(1024) void shared_plan_kernel(SharedAttnParams p)
{
    if (p.units[blockIdx.x] == 0) return;
    if (blockIdx.x == 1) plan_form<ManyRows>(p);
    else if (p.units[1]) plan_form<FewRowsOf<8>>(p);
    else plan_form<FewRowsOf<4>>(p);
}

template <int D>
__global__ __launch_bounds__(256) void shared_join_kernel(SharedAttnParams p)
{
    const int64_t row = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), rows = (int64_t)p.b.T * p.Hq;
    if (row >= rows) return;
    const int t = (int)(row / p.Hq), last = p.b.q_start ? p.b.q_start[p.b.S] : p.b.S, first = p.b.q_start ? p.b.q_start[0] : 0;
    if (t >= last || t < first) return;
    const RowInfo *info = static_cast<const RowInfo *>(p.rows);
    const RowInfo a = info[row], b = info[rows + row];
    const int64_t held = (int64_t)p.slots[0] * FewRows::ROWS + (int64_t)p.slots[1] * ManyRows::ROWS;
    auto step = [](const RowInfo &i) { return i.pieces2 & 1 ? ManyRows::ROWS : FewRows::ROWS; };
    // (whatever tables that break their rules leave here, nothing outside the arrays is read)
    auto pieces = [&](const RowInfo &i) {
        const int n = i.pieces2 >> 1;
        return n > 0 && i.at >= 0 && i.at + (int64_t)(n - 1) * step(i) < held ? n : 0;
    };
    const int n0 = pieces(a), n1 = pieces(b);
    if (n0 + n1 == 0) return;   // (written already)
    join_row<D>(p.part[0], p.part_ml[0], a.at, step(a), n0, b.at, step(b), n1, p.o + row * D, p.lse + row);
}

// Groups and sequences of at most FEW rows take the form for few rows.
constexpr int SHARED_FEW = 64;

struct SharedBounds {
    int above[2], upto[2], units[2], slots[2];
};

// The new tokens are rows twice, of their groups and of their sequences, `planned`
// in all.  Units as in lamp_cache_attn.hip; each may have a partial output.
template <class F>
void bound_shared(SharedBounds &b, int64_t pairs, int64_t keys)
{
    const int64_t most = (keys + TILE - 1) / TILE / F::MIN_TILES;
    const int64_t a = pairs + F::TARGET, c = pairs * (most > 1 ? most : 1);
    b.units[F::FORM] = b.slots[F::FORM] = (int)(a < c ? a : c);
}

SharedBounds shared_bounds(int64_t T, int64_t S, int64_t groups, int G, int Hkv, int64_t keys)
{
    SharedBounds b = {};
    const int64_t rows = T * G, planned = S + groups;
    const bool few = rows <= SHARED_FEW;
    const int64_t limit = few ? rows : SHARED_FEW;
    const int64_t most = 2 * rows / FewRows::ROWS + planned, each = planned * ((limit + FewRows::ROWS - 1) / FewRows::ROWS);
    b.upto[0] = (int)limit;
    bound_shared<FewRows>(b, (most < each ? most : each) * Hkv, keys);
    if (!few) {
        const int64_t longer = 2 * rows / (limit + 1);
        b.above[1] = (int)limit;
        b.upto[1] = (int)rows;
        bound_shared<ManyRows>(b, (2 * rows / ManyRows::ROWS + (longer < planned ? longer : planned)) * Hkv, keys);
    }
    return b;
}

struct SharedLayout {
    size_t before[2], rows, ml, part, total;
};

SharedLayout shared_layout(const SharedBounds &b, int D, int64_t T, int Hq, int64_t planned)
{
    SharedLayout l = {};
    size_t at = 256;
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at += (bytes + 255) & ~(size_t)255;
        return here;
    };
    const size_t rows = (size_t)b.slots[0] * FewRows::ROWS + (size_t)b.slots[1] * ManyRows::ROWS;
    for (int f = 0; f < 2; ++f) l.before[f] = take(planned > PLAN_ALONE && b.units[f] ? planned * sizeof(Before) : 0);
    l.rows = take(2 * (size_t)T * Hq * sizeof(RowInfo));
    l.ml = take(rows * 2 * sizeof(float));
    l.part = take(rows * D * sizeof(float));
    l.total = at;
    return l;
}

template <int D, int KT, int KF>
hipError_t launch_shared(const SharedAttnParams &p, hipStream_t s)
{
    if (p.b.S + p.groups > PLAN_ALONE) shared_plan_kernel<<<dim3(2), 1024, 0, s>>>(p);
    const dim3 grid((unsigned)(p.units[0] + p.units[1]));
    if (!p.units[1]) shared_few_kernel<D, KF><<<grid, 256, 0, s>>>(p);
    else if (1 << p.b.page_shift >= KT) shared_mixed_kernel<D, KT, KF, true><<<grid, THREADS, 0, s>>>(p);
    else shared_mixed_kernel<D, KT, KF, false><<<grid, THREADS, 0, s>>>(p);
    shared_join_kernel<D><<<dim3((unsigned)(((int64_t)p.b.T * p.Hq + 3) / 4)), 256, 0, s>>>(p);
    return hipGetLastError();
}

} // namespace

size_t shared_attn_workspace(int D, int64_t T, int64_t S, int64_t groups, int G, int Hkv, int64_t keys)
{
    return shared_layout(shared_bounds(T, S, groups, G, Hkv, keys), D, T, G * Hkv, S + groups).total;
}

hipError_t launch_shared_attn(int D, SharedAttnParams &p, void *ws, hipStream_t s)
{
    const SharedBounds b = shared_bounds(p.b.T, p.b.S, p.groups, p.Hq / p.b.Hkv, p.b.Hkv, (int64_t)p.b.width << p.b.page_shift);
    const SharedLayout l = shared_layout(b, D, p.b.T, p.Hq, (int64_t)p.b.S + p.groups);
    char *base = static_cast<char *>(ws);
    p.apart = 0;
    p.counts = reinterpret_cast<int *>(base);
    p.split = base + 16;
    p.rows = base + l.rows;
    for (int f = 0; f < 2; ++f) {
        p.rows_above[f] = b.above[f];
        p.rows_upto[f] = b.upto[f];
        p.units[f] = b.units[f];
        p.slots[f] = b.slots[f];
        p.before[f] = base + l.before[f];
        const size_t first = f ? (size_t)b.slots[0] * FewRows::ROWS : 0;   // (one array of rows for both forms)
        p.part_ml[f] = reinterpret_cast<float *>(base + l.ml) + first * 2;
        p.part[f] = reinterpret_cast<float *>(base + l.part) + first * D;
    }
    switch (D) {
    case 64: return launch_shared<64, 64, 64>(p, s);
    case 128: return launch_shared<128, 64, 64>(p, s);
    default: return launch_shared<256, 32, 32>(p, s);
    }
}

} // namespace lamp
