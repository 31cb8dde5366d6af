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
// units (lamp_cache_plan.h: what is planned is the groups, then the sequences): of one
// launch the groups' in the form of lamp_cache_prefix.h and the sequences' in that for
// few rows, and, where the batch may hold so many rows, of a second in the form for
// many.  The last launch joins each row's partial outputs, whose places the first
// pieces leave (RowInfo).  (Units of groups and of sequences in turn instead of one
// after the other: slower.)  Four samples of one prompt (1000 keys, 8/8 heads, d = 64): 7.6 us
// and 4.1 for the join; questions of 100 to 300 tokens about two documents of some 4000 keys
// (121 GFLOP): 147 us, 14 for the join of 61 MB.
#include <hip/hip_runtime.h>

#include "lamp_cache_many.h"
#include "lamp_cache_prefix.h"

namespace lamp {
namespace {

// Groups over their prefixes (x < units[2]) beside the form for few rows.
template <int D, int KT, int NPG>
__global__ __launch_bounds__(256, 2) void shared_few_kernel(SharedAttnParams p)
{
    constexpr size_t A = sizeof(PrefixShared<D, KT>), B = sizeof(FewShared<D, 4>);
    __shared__ __attribute__((aligned(16))) char sh[A > B ? A : B];
    const int x = (int)blockIdx.x;
    if (x < p.units[2]) cache_prefix<D, KT, NPG>(p, x, *reinterpret_cast<PrefixShared<D, KT> *>(sh));
    else cache_few<D, KT, 4>(p, x - p.units[2], *reinterpret_cast<FewShared<D, 4> *>(sh));
}

template <int D, int KT, bool WIDE>
__global__ __launch_bounds__(THREADS, 2) void shared_many_kernel(SharedAttnParams p)
{
    __shared__ PromptShared<D, KT> sh;
    cache_prompt<D, KT, WIDE>(p, (int)blockIdx.x, sh);
}

// The plan of many groups and sequences, a workgroup for each form: key tiles of a
// piece from the sum over all, then each one's place and, for each unit, whose it is
// (units of many are written by the whole wave).  A thread takes a group or sequence
// of each 1024.  Bound by the latencies of the loads and the scans; the units'
// workgroups then have two loads to wait for, where planning alone costs each of
// them about 600 instructions a wave.
template <class F>
__device__ void shared_plan(const SharedAttnParams &p)
{
    constexpr int BY = 1024, BW = BY / 64, SMALL = 32;
    __shared__ Work works[BW];
    __shared__ Before sums[BW];
    const int tid = (int)threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), G = p.Hq / p.b.Hkv;
    const int many = planned<F>(p), rounds = (many + BY - 1) / BY;
    SeqPlan r;
    auto plan_of = [&](int k) {
        const int v = k * BY + tid;
        r = seq_plan<F>(p, v < many ? v : many - 1, G);
        if (v >= many) r.tiles = 0;
    };
    Work work = {};
    for (int k = 0; k < rounds; ++k) {
        plan_of(k);
        add(work, r);
    }
    work = wave_work(work);
    if (lane == 0) works[wave] = work;
    __syncthreads();
    work = {};
#pragma unroll
    for (int w = 0; w < BW; ++w) {
        work.tiles += works[w].tiles;
        work.most += works[w].most;
        work.mean += works[w].mean;
        work.longest = fmaxf(work.longest, works[w].longest);
    }
    const Split split = split_of<F>(p, work);
    SeqInfo *info = static_cast<SeqInfo *>(p.before[F::FORM]);
    int *unit_seq = static_cast<int *>(p.unit_seq[F::FORM]);
    Before all = {0, 0};
    for (int k = 0; k < rounds; ++k) {
        if (rounds > 1) plan_of(k);
        const int v = k * BY + tid;
        const Share h = share_of<F>(p, r, split);
        const Before upto = {wave_scan(h.units), wave_scan(h.slots)};
        __syncthreads();   // (the sums before have been read)
        if (lane == 63) sums[wave] = upto;
        __syncthreads();
        Before at = {all.units + upto.units - h.units, all.slots + upto.slots - h.slots};
#pragma unroll
        for (int w = 0; w < BW; ++w) {
            if (w < wave) at.units += sums[w].units, at.slots += sums[w].slots;
            all.units += sums[w].units;
            all.slots += sums[w].slots;
        }
        if (v < many) info[v] = {at.units, at.slots, h.tiles, h.c, r.row, r.a, r.n, r.all, r.len, r.pos0, r.lo, r.causal};
        // (tables that break their rules may count past the bounds: units without a place are left out)
        auto is = [&](int i) { return i >= 0 && i < p.units[F::FORM]; };
        if (h.units <= SMALL)
            for (int i = at.units; i < at.units + h.units; ++i)
                if (is(i)) unit_seq[i] = v;
        for (uint64_t left = __ballot(h.units > SMALL); left; left &= left - 1) {
            const int l = __builtin_ctzll(left), first = lane_value(at.units, l), n = lane_value(h.units, l), who = lane_value(v, l);
            for (int i = lane; i < n; i += 64)
                if (is(first + i)) unit_seq[first + i] = who;
        }
    }
    if (tid == 0) p.counts[F::FORM] = all.units < 0 ? 0 : (all.units < p.units[F::FORM] ? all.units : p.units[F::FORM]);
}

__global__ __launch_bounds__(1024) void shared_plan_kernel(SharedAttnParams p)
{
    if (p.units[blockIdx.x] == 0) return;
    if (blockIdx.x == 0) shared_plan<FewRows>(p);
    else if (blockIdx.x == 1) shared_plan<ManyRows>(p);
    else shared_plan<PrefixRows>(p);
}

// LANES: of a row (64, where there may be many partial outputs of a few rows, or 16).
template <int D, int LANES>
__global__ __launch_bounds__(256) void shared_join_kernel(SharedAttnParams p)
{
    const int64_t row = (int64_t)blockIdx.x * (256 / LANES) + (LANES == 64 ? __builtin_amdgcn_readfirstlane((int)threadIdx.x / LANES) : (int)threadIdx.x / LANES);
    const int64_t rows = (int64_t)p.b.T * p.Hq;
    if (row >= rows) return;
    const RowInfo *info = static_cast<const RowInfo *>(p.rows);
    const RowInfo a = info[row], b = info[rows + row];
    const int t = (int)((int)row / p.Hq), last = p.b.q_start ? p.b.q_start[p.b.S] : p.b.S, first = p.b.q_start ? p.b.q_start[0] : 0;
    if (t >= last || t < first) return;
    const int64_t held = (int64_t)p.slots[0] * FewRows::ROWS + (int64_t)p.slots[1] * ManyRows::ROWS + (int64_t)p.slots[2] * PrefixRows::ROWS;
    auto step = [](const RowInfo &i) { return (i.pieces4 & 3) == 0 ? FewRows::ROWS : ((i.pieces4 & 3) == 1 ? ManyRows::ROWS : PrefixRows::ROWS); };
    // (whatever tables that break their rules leave here, nothing outside the arrays is read)
    auto pieces = [&](const RowInfo &i) {
        const int n = i.pieces4 >> 2;
        return n > 0 && i.at >= 0 && i.at + (int64_t)(n - 1) * step(i) < held ? n : 0;
    };
    const int n0 = pieces(a), n1 = pieces(b);
    if (n0 + n1 == 0) return;   // (written already)
    if constexpr (LANES == 64) join_row<D>(p.part[0], p.part_ml[0], a.at, step(a), n0, b.at, step(b), n1, true, p.o + row * D, p.lse + row);
    else join_row16<D>(p.part[0], p.part_ml[0], a.at, step(a), n0, b.at, step(b), n1, p.o + row * D, p.lse + row);
}

// Groups of up to GROUP_PREFIX rows take the form of lamp_cache_prefix.h, beside the
// sequences, in the form for few rows; where the batch holds more rows than that,
// larger groups, and sequences of more than SHARED_FEW rows, take the form for many
// in a launch of its own.  Single tokens behind 8192 shared keys, without other keys of
// their own (32/8 heads, d = 128): 100 tokens (400 rows) 40 us in the first form and 53 in
// that for many, 250 tokens 73 and 83, 300 tokens 97 and 96, 600 tokens 163 and 160, 1000
// tokens 268 and 247.  One token 14.4, 8 tokens 16.1, where attn_cache, which reads each
// one's keys in the form for few rows, takes 14.1 and 25.2.
constexpr int GROUP_PREFIX = 1024, SHARED_FEW = 64;
constexpr int64_t JOIN_WIDE = 4096;   // rows up to which a wave joins each (a call with 2048 rows 36.6 us, by 16 lanes 37.2; with 8000 rows 107 and 103)

struct SharedBounds {
    int above[3], upto[3], group_above[3], group_upto[3], units[3], slots[3];
};

// Units as in lamp_cache_attn.hip; each may have a partial output.
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
    const int64_t rows = T * G;   // of all sequences, and of all groups
    const bool many = rows > GROUP_PREFIX;
    auto least = [](int64_t x, int64_t y) { return x < y ? x : y; };
    // row tiles of `rows` rows in `n` ranges of `from` rows at least and `upto` at most
    auto tiles = [&](int64_t tile, int64_t n, int64_t from, int64_t upto) {
        const int64_t k = least(n, rows / from);
        return least(rows / tile + k, k * ((upto + tile - 1) / tile));
    };
    b.upto[0] = many ? SHARED_FEW : (int)rows;
    bound_shared<FewRows>(b, tiles(FewRows::ROWS, S, 1, b.upto[0]) * Hkv, keys);
    b.group_upto[2] = GROUP_PREFIX;
    bound_shared<PrefixRows>(b, tiles(PrefixRows::ROWS, groups, 1, GROUP_PREFIX) * Hkv, keys);
    if (many) {
        b.above[1] = SHARED_FEW;
        b.group_above[1] = GROUP_PREFIX;
        b.upto[1] = b.group_upto[1] = (int)rows;
        bound_shared<ManyRows>(b, (tiles(ManyRows::ROWS, S, SHARED_FEW + 1, rows) + tiles(ManyRows::ROWS, groups, GROUP_PREFIX + 1, rows)) * Hkv, keys);
    }
    return b;
}

struct SharedLayout {
    size_t seqs[3], units[3], rows, ml, part, total;
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
    const size_t rows = (size_t)b.slots[0] * FewRows::ROWS + (size_t)b.slots[1] * ManyRows::ROWS + (size_t)b.slots[2] * PrefixRows::ROWS;
    for (int f = 0; f < 3; ++f) {
        const bool plan = planned > SHARED_ALONE && b.units[f];
        l.seqs[f] = take(plan ? planned * sizeof(SeqInfo) : 0);
        l.units[f] = take(plan ? b.units[f] * sizeof(int) : 0);
    }
    l.rows = take(2 * (size_t)T * Hq * sizeof(RowInfo));
    l.ml = take(rows * 2 * sizeof(float));
    l.part = take(rows * D * sizeof(float));
    l.total = at;
    return l;
}

template <int D, int KT>
hipError_t launch_shared(const SharedAttnParams &p, hipStream_t s)
{
    if (p.b.S + p.groups > SHARED_ALONE) shared_plan_kernel<<<dim3(3), 1024, 0, s>>>(p);
    const int page = 1 << p.b.page_shift;
    const dim3 grid((unsigned)(p.units[0] + p.units[2]));
    if (page >= KT) shared_few_kernel<D, KT, 1><<<grid, 256, 0, s>>>(p);
    else if (KT == 32 || page == 32) shared_few_kernel<D, KT, 2><<<grid, 256, 0, s>>>(p);
    else shared_few_kernel<D, KT, KT / 16><<<grid, 256, 0, s>>>(p);
    if (p.units[1]) {
        if (page >= KT) shared_many_kernel<D, KT, true><<<dim3((unsigned)p.units[1]), THREADS, 0, s>>>(p);
        else shared_many_kernel<D, KT, false><<<dim3((unsigned)p.units[1]), THREADS, 0, s>>>(p);
    }
    const int64_t rows = (int64_t)p.b.T * p.Hq;
    if (rows <= JOIN_WIDE) shared_join_kernel<D, 64><<<dim3((unsigned)((rows + 3) / 4)), 256, 0, s>>>(p);
    else shared_join_kernel<D, 16><<<dim3((unsigned)((rows + 15) / 16)), 256, 0, s>>>(p);
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
    p.counts = reinterpret_cast<int *>(base);
    p.rows = base + l.rows;
    for (int f = 0; f < 3; ++f) {
        p.group_above[f] = b.group_above[f];
        p.group_upto[f] = b.group_upto[f];
        p.rows_above[f] = b.above[f];
        p.rows_upto[f] = b.upto[f];
        p.units[f] = b.units[f];
        p.slots[f] = b.slots[f];
        p.before[f] = base + l.seqs[f];
        p.unit_seq[f] = base + l.units[f];
        // (one array of rows for all forms)
        const size_t first = (f > 0 ? (size_t)b.slots[0] * FewRows::ROWS : 0) + (f > 1 ? (size_t)b.slots[1] * ManyRows::ROWS : 0);
        p.part_ml[f] = reinterpret_cast<float *>(base + l.ml) + first * 2;
        p.part[f] = reinterpret_cast<float *>(base + l.part) + first * D;
    }
    switch (D) {
    case 64: return launch_shared<64, 64>(p, s);
    case 128: return launch_shared<128, 64>(p, s);
    default: return launch_shared<256, 32>(p, s);
    }
}

} // namespace lamp
