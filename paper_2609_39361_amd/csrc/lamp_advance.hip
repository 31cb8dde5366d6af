// lamp_advance.hip -- a step of a batch over the paged cache: how many tokens each
// sequence adds become its new length, its first new token in the batch, the
// tokens' positions, and table entries for the pages that it needs, taken from a
// ring of free pages; the pages of sequences that leave go back to its end.
//
// With h_s = ceil(len_s / page) the places that sequence s holds and n_s the tokens
// it adds, it needs ceil((len_s + n_s) / page) - h_s pages; sums over the sequences
// before say which of the ring's, in order.  A workgroup goes over the sequences,
// EACH consecutive ones a thread: sums over all, by which the step is admitted or not,
// and places, sums over those before (saturating in 32 bits, beyond everything that
// is admitted).  The entries and positions of all of them are then spread over the
// threads, each of which searches the places in LDS for its sequence (one may have
// thousands, most have none).  Where there may be many, several workgroups do all of
// this and share the entries and positions.  The lengths, starts and state are the
// first one's to write; in place they are a second launch's, as the others still read
// what they replace.  Bound by the latencies of the loads, the sums, the searches and
// the ring's entries, one after another: 32 sequences 5.1 us, of which a launch is 3.7;
// 4096 whose step takes 3554 pages, gives 3208 back and has 26832 tokens, by 35
// workgroups 8.8 (by 7 13.4; by one, and a launch for the positions, 14.4).
#include <hip/hip_runtime.h>

#include "lamp_cache_plan.h"

namespace lamp {
namespace {

constexpr int ADVANCE_BY = 1024, ADVANCE_WAVES = ADVANCE_BY / 64;
constexpr int SHARE = 1024;    // entries and positions for which a workgroup more is taken

// Why a step is not admitted.
enum { SHORT_OF_PAGES = 1, BEYOND_TABLE = 2, BEYOND_TOKENS = 4 };
// More pages would go back than the ring lacks: none does (tables that break their rules).
constexpr int TOO_MANY_BACK = 8;

struct Step {
    int said, len;       // keys now: as said, and with table entries
    int add;             // new tokens
    int held, need;      // places held, pages needed
    int kept, back;      // places that stay and pages that go back behind them
    bool gone, beyond;   // the sequence leaves; it would not fit the table
};

__device__ __forceinline__ Step step_of(const AdvanceParams &p, int s, bool is)
{
    Step r;
    const int page = 1 << p.page_shift, reach = p.width << p.page_shift;   // (at most 2^30)
    const int len = p.lens[s], add = p.add[s], prefix = p.prefix_lens ? p.prefix_lens[s] : 0;
    r.said = len;
    r.len = len < 0 ? 0 : (len < reach ? len : reach);
    r.gone = is && add < 0;
    r.add = is && add > 0 ? add : 0;
    r.beyond = is && add >= 0 && (int64_t)len + r.add > reach;
    r.held = (r.len + page - 1) >> p.page_shift;
    const int room = reach - r.len, take = r.add < room ? r.add : room;    // (more is not admitted)
    r.need = ((r.len + take + page - 1) >> p.page_shift) - r.held;
    const int kept = prefix > 0 ? prefix >> p.page_shift : 0;
    r.kept = kept < r.held ? kept : r.held;
    r.back = r.gone ? r.held - r.kept : 0;
    return r;
}

__device__ __forceinline__ uint32_t sum(uint32_t a, uint32_t b) { return __builtin_elementwise_add_sat(a, b); }

// Inclusive sum over the wave's lanes.
__device__ __forceinline__ uint32_t wave_sums(uint32_t v)
{
    return wave_scan_by(v, [](uint32_t a, uint32_t b) { return sum(a, b); });
}

// What a launch writes: entries and positions, and the rest.
enum { ENTRIES = 1, OUTPUTS = 2 };

// Where the sequences' taken entries, those that go back and their positions begin
// among all, and where in their rows and from which position on.
template <int N>
struct SeqPlaces {
    int at[3 * N], from[3 * N];
};

// Last i with at[which N + i] <= x for each x (those of the first are, those behind the
// last sequence are not; non-decreasing): without branches, as the reads of one search
// wait for each other.
template <int N, int AT>
__device__ __forceinline__ void owners(const int *at, const int (&which)[AT], const int (&x)[AT], int (&i)[AT])
{
#pragma unroll
    for (int k = 0; k < AT; ++k) i[k] = 0;
#pragma unroll
    for (int half = N / 2; half; half >>= 1) {
        int y[AT];
#pragma unroll
        for (int k = 0; k < AT; ++k) y[k] = at[which[k] * N + i[k] + half];
        __builtin_amdgcn_sched_barrier(0);   // (the compiler would take one search after another)
#pragma unroll
        for (int k = 0; k < AT; ++k) i[k] += y[k] <= x[k] ? half : 0;
    }
}

template <int EACH>
__global__ __launch_bounds__(ADVANCE_BY) void advance_kernel(AdvanceParams p, int what)
{
    __shared__ uint32_t sums[3][ADVANCE_WAVES];
    __shared__ int beyond_any[ADVANCE_WAVES];
    constexpr int N = EACH * ADVANCE_BY;
    __shared__ SeqPlaces<N> places;   // of a round's sequences
    const int tid = (int)threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int pages = p.pages, last = p.S - 1;
    const int part = (int)blockIdx.x * ADVANCE_BY + tid, stride = (int)gridDim.x * ADVANCE_BY;   // of entries and positions
    const bool outputs = (what & OUTPUTS) != 0 && blockIdx.x == 0;
    const int first = p.state[0], free = p.state[1];
    const int rounds = (p.S + EACH * ADVANCE_BY - 1) / (EACH * ADVANCE_BY);
    auto sequence = [&](int round, int i) { return (round * ADVANCE_BY + tid) * EACH + i; };
    // the ring, whatever its state says
    const int head = first >= 0 ? first % pages : 0;
    const int count = free < 0 ? 0 : (free < pages ? free : pages);
    auto in_ring = [&](int64_t i) { return (int)(head + i < pages ? head + i : head + i - pages); };   // (i up to pages)

    Step r[EACH];
    uint32_t mine[3], upto[3], all[3] = {0, 0, 0};   // needed, going back, added: this thread's, with the lanes before, of all
    bool beyond = false;
    auto load = [&](int round) {
        mine[0] = mine[1] = mine[2] = 0;
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const int s = sequence(round, i);
            r[i] = step_of(p, s < last ? s : last, s <= last);
            mine[0] = sum(mine[0], (uint32_t)r[i].need);
            mine[1] = sum(mine[1], (uint32_t)r[i].back);
            mine[2] = sum(mine[2], (uint32_t)r[i].add);
            beyond = beyond || r[i].beyond;
        }
    };
    // this thread's sums among the waves', which LDS holds after the next barrier
    auto place = [&]() {
#pragma unroll
        for (int k = 0; k < 3; ++k) {
            upto[k] = wave_sums(mine[k]);
            if (lane == 63) sums[k][wave] = upto[k];
        }
    };
    for (int round = 0; round < rounds; ++round) {
        load(round);
        if (round) __syncthreads();   // (the sums of the round before have been read)
        place();
        const bool any = __ballot(beyond) != 0;
        if (lane == 0) beyond_any[wave] = any;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < ADVANCE_WAVES; ++w)
#pragma unroll
            for (int k = 0; k < 3; ++k) all[k] = sum(all[k], sums[k][w]);
    }
    beyond = false;
#pragma unroll
    for (int w = 0; rounds && w < ADVANCE_WAVES; ++w) beyond = beyond || beyond_any[w];
    const int no = (all[0] > (uint32_t)count ? SHORT_OF_PAGES : 0) | (beyond ? BEYOND_TABLE : 0) | (all[2] > (uint32_t)p.T ? BEYOND_TOKENS : 0);
    const bool ok = no == 0, returns = all[1] <= (uint32_t)(pages - count);

    int need0 = 0, back0 = 0, add0 = 0;   // of the rounds before
    for (int round = 0; round < rounds; ++round) {
        if (rounds > 1) {
            load(round);
            __syncthreads();   // (what the round before left in LDS has been read)
            place();
            __syncthreads();
        }
        const int from[3] = {need0, back0, add0};
        // (what is not admitted, or does not go back, counts as none)
        int at[3] = {from[0], from[1], from[2]}, end[3] = {from[0], from[1], from[2]};
#pragma unroll
        for (int k = 0; k < 3; ++k) {
            if (k == 1 ? !returns : !ok) continue;
            at[k] += (int)(upto[k] - mine[k]);
#pragma unroll
            for (int w = 0; w < ADVANCE_WAVES; ++w) {
                at[k] += w < wave ? (int)sums[k][w] : 0;
                end[k] += (int)sums[k][w];
            }
        }
        need0 = end[0];
        back0 = end[1];
        add0 = end[2];
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const int s = sequence(round, i);
            const int place = tid * EACH + i, begin[3] = {r[i].held, r[i].kept, r[i].len};
#pragma unroll
            for (int k = 0; k < 3; ++k) places.at[k * N + place] = at[k], places.from[k * N + place] = begin[k];
            if (outputs && s <= last) {
                p.kv_lens[s] = r[i].gone ? 0 : r[i].said + (ok ? r[i].add : 0);
                p.q_start[s] = at[2];
                if (s == last) p.q_start[p.S] = at[2] + (ok ? r[i].add : 0);
            }
            at[0] += ok ? r[i].need : 0;
            at[1] += returns ? r[i].back : 0;
            at[2] += ok ? r[i].add : 0;
        }
        if (!(what & ENTRIES)) continue;
        __syncthreads();
        // entries to take, those that go back and positions as one list, AT of a thread at once, whose
        // searches and loads do not wait for each other (a call of up to 1024 sequences 5.1 to 5.9 us, of one
        // at once 5.8 to 6.3; the step of 4096 8.8, of two 9.6, of four 11.2)
        constexpr int AT = EACH == 1 ? 2 : 1;
        const int64_t taken = need0 - from[0], moved = taken + back0 - from[1], total = moved + add0 - from[2];
        for (int64_t i0 = part; i0 < total; i0 += (int64_t)AT * stride) {
            int which[AT], x[AT], of[AT], value[AT];
            const int *source[AT];
            int *target[AT];
#pragma unroll
            for (int k = 0; k < AT; ++k) {   // (beyond the last: the first again, with the same outcome)
                const int64_t at = i0 + (int64_t)k * stride, i = at < total ? at : i0;
                which[k] = i < taken ? 0 : (i < moved ? 1 : 2);
                x[k] = (int)(i < taken ? from[0] + i : (i < moved ? from[1] + i - taken : from[2] + i - moved));
            }
            owners<N>(places.at, which, x, of);
#pragma unroll
            for (int k = 0; k < AT; ++k) {
                const int l = of[k], begin = places.from[which[k] * N + l] + (x[k] - places.at[which[k] * N + l]);
                int *entry = p.table + (int64_t)(round * N + l) * p.table_stride + begin;
                int *ring = p.ring + (which[k] == 2 ? 0 : in_ring(which[k] == 1 ? (int64_t)count + x[k] : x[k]));
                source[k] = which[k] == 1 ? entry : ring;   // (of positions: whatever the ring's first entry is)
                target[k] = which[k] == 0 ? entry : (which[k] == 1 ? ring : p.positions + x[k]);
                value[k] = begin;
            }
#pragma unroll
            for (int k = 0; k < AT; ++k) {
                const int page = *source[k];
                value[k] = which[k] == 2 ? value[k] : page;
            }
#pragma unroll
            for (int k = 0; k < AT; ++k) *target[k] = value[k];
        }
    }
    if (what & ENTRIES)
        for (int i = add0 + part; i < p.T; i += stride) p.positions[i] = 0;   // (T up to 2^23)
    if (outputs && tid == 0) {
        if (p.S == 0) p.q_start[0] = 0;
        p.state_out[0] = in_ring(need0);
        p.state_out[1] = count - need0 + back0;
        p.state_out[2] = (int)(all[0] < 0x7FFFFFFFu ? all[0] : 0x7FFFFFFFu);
        p.state_out[3] = no | (returns ? 0 : TOO_MANY_BACK);
    }
}

void launch_part(const AdvanceParams &p, int parts, int what, hipStream_t s)
{
    if (p.S <= ADVANCE_BY) advance_kernel<1><<<parts, ADVANCE_BY, 0, s>>>(p, what);
    else advance_kernel<4><<<parts, ADVANCE_BY, 0, s>>>(p, what);
}

} // namespace

hipError_t launch_advance(const AdvanceParams &p, hipStream_t s)
{
    // as many entries as a 64th of the tables
    const int64_t entries = (int64_t)p.S * p.width / 64, most = (p.T + entries) / SHARE;
    const int parts = 1 + (int)(most < 63 ? most : 63);
    const bool in_place = p.kv_lens == p.lens || p.state_out == p.state;
    if (parts == 1 || !in_place) {
        launch_part(p, parts, ENTRIES | OUTPUTS, s);
    } else {
        launch_part(p, parts, ENTRIES, s);
        launch_part(p, 1, OUTPUTS, s);
    }
    return hipGetLastError();
}

} // namespace lamp
