// lamp_advance.hip -- a step of a batch over the paged cache: how many tokens each
// sequence adds become its new length, its first new token in the batch, the
// tokens' positions, and table entries for the pages that it needs, taken from a
// ring of free pages; the pages of sequences that leave go back to its end.
//
// With h_s = ceil(len_s / page) the places that sequence s holds and n_s the tokens
// it adds, it needs ceil((len_s + n_s) / page) - h_s pages; sums over the sequences
// before say which of the ring's, in order.  One workgroup goes over the sequences
// twice, THREADS at a time: once for the sums, by which the step is admitted or not,
// and once to write.  The entries of a round's sequences are spread over all
// threads, by a search in the round's sums (one sequence may need thousands).
// Positions of many tokens are written by a second launch.  Bound by the latencies
// of the loads, scans and barriers of a round.
#include <hip/hip_runtime.h>

#include "lamp_serve.h"

namespace lamp {
namespace {

constexpr int THREADS_ADV = 1024, WAVES_ADV = THREADS_ADV / 64;
constexpr int WITHIN = 8192;   // positions that the first launch writes itself

// Why a step is not admitted.
enum { SHORT_OF_PAGES = 1, BEYOND_TABLE = 2, BEYOND_TOKENS = 4 };
// More pages would go back than the ring lacks: none does (tables that break their rules).
constexpr int TOO_MANY_BACK = 8;

struct Step {
    int64_t len, add;    // keys now, and new
    int64_t held, need, back, kept;   // places held, pages needed, places that go back and those before them
};

__device__ __forceinline__ Step step_of(const AdvanceParams &p, int s)
{
    Step r;
    const int64_t page = 1 << p.page_shift, reach = (int64_t)p.width << p.page_shift;
    const int64_t len = p.lens[s], add = p.add[s], prefix = p.prefix_lens ? p.prefix_lens[s] : 0;
    r.len = len < 0 ? 0 : (len < reach ? len : reach);   // (a longer one has no entries: not admitted below)
    r.add = add > 0 ? add : 0;
    r.held = (r.len + page - 1) >> p.page_shift;
    r.need = (((len + r.add < reach ? r.len + r.add : reach) + page - 1) >> p.page_shift) - r.held;
    r.kept = prefix > 0 ? prefix >> p.page_shift : 0;
    r.kept = r.kept < r.held ? r.kept : r.held;
    r.back = add < 0 ? r.held - r.kept : 0;
    return r;
}

__device__ __forceinline__ int64_t wave_sum_upto(int64_t v, int lane)
{
#pragma unroll
    for (int k = 1; k < 64; k <<= 1) {
        const int64_t y = __shfl_up(v, k, 64);
        v += lane >= k ? y : 0;
    }
    return v;
}

// Last i < n with at[i] <= x (at[0] <= x; non-decreasing).
__device__ __forceinline__ int last_of(const int *at, int n, int x)
{
    int lo = 0;
    for (int half = THREADS_ADV / 2; half; half >>= 1)
        if (lo + half < n && at[lo + half] <= x) lo += half;
    return lo;
}

__global__ __launch_bounds__(THREADS_ADV) void advance_kernel(AdvanceParams p)
{
    __shared__ int64_t sums[3][WAVES_ADV];
    __shared__ int why;
    __shared__ int need_at[THREADS_ADV], back_at[THREADS_ADV], tok_at[THREADS_ADV];   // of a round's sequences, within the round
    __shared__ int held_at[THREADS_ADV], kept_at[THREADS_ADV], len_at[THREADS_ADV];
    const int tid = (int)threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t pages = p.pages;
    int64_t head = p.state[0] % pages, count = p.state[1];
    head = head < 0 ? head + pages : head;
    count = count < 0 ? 0 : (count < pages ? count : pages);
    if (tid == 0) why = 0;
    // the sums of all
    int64_t need = 0, back = 0, add = 0;
    bool beyond = false;
    for (int s = tid; s < p.S; s += THREADS_ADV) {
        const Step r = step_of(p, s);
        need += r.need;
        back += r.back;
        add += r.add;
        beyond = beyond || (p.add[s] >= 0 && (int64_t)p.lens[s] + r.add > (int64_t)p.width << p.page_shift);
    }
    need = wave_sum_upto(need, lane);
    back = wave_sum_upto(back, lane);
    add = wave_sum_upto(add, lane);
    if (lane == 63) sums[0][wave] = need, sums[1][wave] = back, sums[2][wave] = add;
    __syncthreads();
    if (beyond) why = BEYOND_TABLE;
    need = back = add = 0;
    for (int w = 0; w < WAVES_ADV; ++w) need += sums[0][w], back += sums[1][w], add += sums[2][w];
    __syncthreads();
    const int no = why | (need > count ? SHORT_OF_PAGES : 0) | (add > p.T ? BEYOND_TOKENS : 0);
    const bool ok = no == 0, returns = back <= pages - count;
    // a round's sequences
    int64_t need0 = 0, back0 = 0, add0 = 0;
    for (int s0 = 0; s0 < p.S; s0 += THREADS_ADV) {
        const int s = s0 + tid, n = p.S - s0 < THREADS_ADV ? p.S - s0 : THREADS_ADV;
        Step r = {};
        bool gone = false;
        if (s < p.S) {
            r = step_of(p, s);
            gone = p.add[s] < 0;
            if (!ok) r.need = r.add = 0;
            if (!returns) r.back = 0;
        }
        const int64_t needs = wave_sum_upto(r.need, lane), backs = wave_sum_upto(r.back, lane), adds = wave_sum_upto(r.add, lane);
        __syncthreads();   // (the round before is done)
        if (lane == 63) sums[0][wave] = needs, sums[1][wave] = backs, sums[2][wave] = adds;
        __syncthreads();
        int64_t before[3] = {0, 0, 0}, all[3] = {0, 0, 0};
        for (int w = 0; w < WAVES_ADV; ++w)
            for (int k = 0; k < 3; ++k) {
                before[k] += w < wave ? sums[k][w] : 0;
                all[k] += sums[k][w];
            }
        const int64_t tok = add0 + before[2] + adds - r.add;
        need_at[tid] = (int)(before[0] + needs - r.need);
        back_at[tid] = (int)(before[1] + backs - r.back);
        tok_at[tid] = (int)(before[2] + adds - r.add);
        held_at[tid] = (int)r.held;
        kept_at[tid] = (int)r.kept;
        len_at[tid] = (int)r.len;
        if (s < p.S) {
            const int len = p.lens[s];
            p.kv_lens[s] = gone ? 0 : len + (int)r.add;
            p.q_start[s] = (int)tok;
            if (s == p.S - 1) p.q_start[p.S] = (int)(tok + r.add);
        }
        __syncthreads();
        for (int64_t i = tid; i < all[0]; i += THREADS_ADV) {
            const int l = last_of(need_at, n, (int)i);
            p.table[(s0 + l) * p.table_stride + held_at[l] + (i - need_at[l])] = p.ring[(head + need0 + i) % pages];
        }
        for (int64_t i = tid; i < all[1]; i += THREADS_ADV) {
            const int l = last_of(back_at, n, (int)i);
            p.ring[(head + count + back0 + i) % pages] = p.table[(s0 + l) * p.table_stride + kept_at[l] + (i - back_at[l])];
        }
        if (p.T <= WITHIN)
            for (int64_t i = tid; i < all[2]; i += THREADS_ADV) {
                const int l = last_of(tok_at, n, (int)i);
                p.positions[add0 + i] = len_at[l] + (int)(i - tok_at[l]);
            }
        need0 += all[0];
        back0 += all[1];
        add0 += all[2];
    }
    if (p.T <= WITHIN)
        for (int64_t i = add0 + tid; i < p.T; i += THREADS_ADV) p.positions[i] = 0;
    if (tid == 0) {
        if (p.S == 0) p.q_start[0] = 0;
        p.state_out[0] = (int)((head + need0) % pages);
        p.state_out[1] = (int)(count - need0 + back0);
        p.state_out[2] = (int)(need < 0x7FFFFFFF ? need : 0x7FFFFFFF);
        p.state_out[3] = no | (returns ? 0 : TOO_MANY_BACK);
    }
}

// Positions of the tokens of sequence x / parts, a part of them a wave (sequence S:
// the tokens behind the last).
__global__ __launch_bounds__(256) void positions_kernel(AdvanceParams p, int parts)
{
    const int64_t x = (int64_t)blockIdx.x * 4 + ((int)threadIdx.x >> 6);
    const int s = (int)(x / parts), part = (int)(x - (int64_t)s * parts), lane = (int)threadIdx.x & 63;
    if (s > p.S) return;
    const int a = p.q_start[s], e = s < p.S ? p.q_start[s + 1] : p.T, n = e - a;
    const int pos0 = s < p.S ? p.kv_lens[s] - n : 0;
    const int64_t lo = (int64_t)n * part / parts, hi = (int64_t)n * (part + 1) / parts;
    for (int64_t i = lo + lane; i < hi; i += 64) p.positions[a + i] = s < p.S ? pos0 + (int)i : 0;
}

} // namespace

hipError_t launch_advance(const AdvanceParams &p, hipStream_t s)
{
    advance_kernel<<<1, THREADS_ADV, 0, s>>>(p);
    if (p.T > WITHIN) {
        // about 256 tokens a wave
        const int64_t want = (p.T + 256 * ((int64_t)p.S + 1) - 1) / (256 * ((int64_t)p.S + 1)), waves = ((int64_t)p.S + 1) * want;
        positions_kernel<<<dim3((unsigned)((waves + 3) / 4)), 256, 0, s>>>(p, (int)want);
    }
    return hipGetLastError();
}

} // namespace lamp
