// lamp_cache_attn.hip -- attention of a ragged batch of new tokens over the
// 8-bit paged cache.
//
// Row (token i of sequence s, head h) sees keys j < kv_lens[s] with, causal,
// j <= p and, windowed, j > p - window, p the token's position:
//   l_j = scale ks_j (q . kcode_j),  P = softmax(l),  o = sum_j P_j vs_j vcode_j,
// ks_j, vs_j the scales of the key's page.  e4m3 codes are exact in bf16, so
// q.k and P.v run on the bf16 matrix cores with fp32 accumulation and the
// scales apply to the fp32 logits and probabilities.  One pass with the running
// maximum m and sum l of the softmax in fp32 (base-2 exponentials of logits
// pre-multiplied by log2 e).  P_j vs_j is rounded to bf16 for the matrix cores
// (at most 2^-8 of each term, what the bf16 output is rounded by anyway; fp32
// products would run at a sixteenth of the rate); l sums the unrounded ones.
//
// Two forms, for sequences of few rows (lamp_cache_few.h; bound by HBM: 32
// single tokens over 8K keys, 32/8 heads, d = 128: 537 MB in 97 us, 5.5 TB/s) and
// of many (lamp_cache_many.h; bound by the matrix cores and the vector unit:
// an 8K prompt 520 us, 1.06 PFLOP/s), in one launch where a batch holds both, or
// in two where sequences are short on average (CHUNK); then, where a sequence may
// have been cut in pieces, a launch that joins them.
#include <hip/hip_runtime.h>

#include "lamp_cache_few.h"

namespace lamp {
namespace {

template <int D, int KT>
__global__ __launch_bounds__(256, 2) void cache_few_kernel(CacheAttnParams p)
{
    __shared__ FewShared<D, 4> sh;
    cache_few<D, KT, 4>(p, (int)blockIdx.x, sh);
}

// The plan of many sequences, a workgroup for each form: key tiles of a piece
// from the sum over all sequences, then what lies before each.  A thread takes
// consecutive sequences, in three passes over their lengths (bound by these
// loads' latency).
template <class F>
__device__ void plan_form(const CacheAttnParams &p)
{
    constexpr int THREADS = 1024, WAVES = THREADS / 64;
    __shared__ Work works[WAVES];
    __shared__ Before sums[WAVES];
    const int tid = (int)threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), G = p.Hq / p.b.Hkv;
    const int each = (p.b.S + THREADS - 1) / THREADS;
    const int s0 = tid * each < p.b.S ? tid * each : p.b.S, s1 = p.b.S - s0 < each ? p.b.S : s0 + each;
    Work work = {};
#pragma unroll 4
    for (int s = s0; s < s1; ++s) add(work, seq_plan<F>(p, s, G));
    work = wave_work(work);
    if (lane == 0) works[wave] = work;
    __syncthreads();
    work = {};
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        work.tiles += works[w].tiles;
        work.most += works[w].most;
        work.mean += works[w].mean;
        work.longest = fmaxf(work.longest, works[w].longest);
    }
    const Split split = split_of<F>(p, work);
    Before at = {0, 0};
#pragma unroll 4
    for (int s = s0; s < s1; ++s) {
        const Share h = share_of<F>(p, seq_plan<F>(p, s, G), split);
        at.units += h.units;
        at.slots += h.slots;
    }
    const Before own = at;
    at = {wave_scan(at.units), wave_scan(at.slots)};
    if (lane == 63) sums[wave] = at;
    __syncthreads();
    at = {at.units - own.units, at.slots - own.slots};
    int slots = 0;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
        if (w < wave) at.units += sums[w].units, at.slots += sums[w].slots;
        slots += sums[w].slots;
    }
    if (tid == 0) {
        p.counts[F::FORM] = slots;
        static_cast<Split *>(p.split)[F::FORM] = split;
    }
    Before *before = static_cast<Before *>(p.before[F::FORM]);
#pragma unroll 4
    for (int s = s0; s < s1; ++s) {
        const Share h = share_of<F>(p, seq_plan<F>(p, s, G), split);
        before[s] = at;
        at.units += h.units;
        at.slots += h.slots;
    }
}

__global__ __launch_bounds__(1024) void cache_plan_kernel(CacheAttnParams p)
{
    if (p.units[blockIdx.x] == 0) return;
    if (blockIdx.x == 1) plan_form<ManyRows>(p);
    else if (p.units[1] && !p.apart) plan_form<FewRowsOf<8>>(p);   // (of the kernel with both forms)
    else plan_form<FewRowsOf<4>>(p);
}

// The pieces of the rows of split row tiles joined.  The workgroups of a row
// tile's c partial outputs share its rows, the k-th those with row % c = k.
// Few rows (many pieces): a workgroup's waves take the pieces in turn, 16 at
// once each, a row after another; a lane holds D/64 channels.  Many rows (few
// pieces): MANY_BY workgroups for each partial output, 16 lanes a row.  Bound
// by latency: the loads of a step do not wait for each other.
constexpr int MANY_BY = 8;

template <int D>
__device__ __forceinline__ void join_many(const CacheAttnParams &p, const PartInfo &i, int slot0, int by, int G)
{
    constexpr int C = D / 16, AT = 4;   // pieces at once
    const int lane = threadIdx.x & 15;
    const float *part = p.part[1], *ml = p.part_ml[1];
    for (int r = i.piece + i.pieces * (by * 16 + ((int)threadIdx.x >> 4)); r < i.rows; r += i.pieces * 16 * MANY_BY) {
        const int64_t base = (int64_t)slot0 * ManyRows::ROWS + r;
        float m = NEG_INF, sum = 0.0f, v[C] = {};
        for (int c0 = 0; c0 < i.pieces; c0 += AT) {
            float mc[AT], lc[AT];
            f32x4 o[AT][C / 4];
#pragma unroll
            for (int k = 0; k < AT; ++k) {   // (beyond the last: read again, weight 0)
                const int64_t at = base + (int64_t)(c0 + k < i.pieces ? c0 + k : c0) * ManyRows::ROWS;
                mc[k] = ml[at * 2];
                lc[k] = ml[at * 2 + 1];
#pragma unroll
                for (int e = 0; e < C / 4; ++e) o[k][e] = *reinterpret_cast<const f32x4 *>(part + at * D + C * lane + 4 * e);
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
                if (c0 + k < i.pieces) {
                    const float f = __builtin_amdgcn_exp2f(mc[k] - ms);
                    sum += lc[k] * f;
#pragma unroll
                    for (int e = 0; e < C; ++e) v[e] += o[k][e / 4][e % 4] * f;
                }
            }
        }
        const int gr = i.row0 + r, t = gr / G;
        const int64_t orow = (int64_t)(i.token + t) * p.Hq + i.head * G + gr - t * G;
        const float inv = finish(m, sum);
#pragma unroll
        for (int e = 0; e < C; e += 4)
            *reinterpret_cast<u32x2 *>(p.o + orow * D + C * lane + e) =
                u32x2{pack2(v[e] * inv, v[e + 1] * inv), pack2(v[e + 2] * inv, v[e + 3] * inv)};
        if (lane == 0) p.lse[orow] = finish_lse(m, sum);
    }
}

template <int D>
__device__ __forceinline__ void join_few(const CacheAttnParams &p, const PartInfo &i, int slot0, int G)
{
    constexpr int C = D / 64;
    __shared__ float obuf[4 * D], mbuf[4], lbuf[4];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const float *part = p.part[0], *ml = p.part_ml[0];
    for (int r = i.piece; r < i.rows; r += i.pieces) {
        const int64_t base = (int64_t)slot0 * FewRows::ROWS + r;
        float m = NEG_INF, sum = 0.0f, v[C] = {};
        for (int c0 = wave; c0 < i.pieces; c0 += 64) {
            // lane k % 16 has the maximum and sum of the round's piece k (beyond the last: none)
            const int c = c0 + (lane & 15) * 4;
            const int64_t at = (base + (int64_t)(c < i.pieces ? c : c0) * FewRows::ROWS) * 2;
            const float mc = c < i.pieces ? ml[at] : NEG_INF, lc = ml[at + 1];
            float o[16][C];
#pragma unroll
            for (int j = 0; j < 16; ++j)
#pragma unroll
                for (int e = 0; e < C; ++e)
                    o[j][e] = part[(base + (int64_t)(c0 + 4 * j < i.pieces ? c0 + 4 * j : c0) * FewRows::ROWS) * D + C * lane + e];
            float mn = mc;
#pragma unroll
            for (int k = 1; k < 16; k <<= 1) mn = fmaxf(mn, __shfl_xor(mn, k, 64));
            mn = fmaxf(mn, m);
            const float ms = mn == NEG_INF ? 0.0f : mn, f0 = __builtin_amdgcn_exp2f(m - ms);
            const float f = __builtin_amdgcn_exp2f(mc - ms), fl = c < i.pieces ? lc * f : 0.0f;
            m = mn;
            sum *= f0;
#pragma unroll
            for (int e = 0; e < C; ++e) v[e] *= f0;
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                if (c0 + 4 * j < i.pieces) {
                    const float fj = __builtin_bit_cast(float, lane_value(__builtin_bit_cast(int, f), j));
                    sum += __builtin_bit_cast(float, lane_value(__builtin_bit_cast(int, fl), j));
#pragma unroll
                    for (int e = 0; e < C; ++e) v[e] += o[j][e] * fj;
                }
            }
        }
        __syncthreads();   // (the row before has been read)
#pragma unroll
        for (int e = 0; e < C; ++e) obuf[wave * D + C * lane + e] = v[e];
        if (lane == 0) mbuf[wave] = m, lbuf[wave] = sum;
        __syncthreads();
        if (wave != 0) continue;
        m = fmaxf(fmaxf(mbuf[0], mbuf[1]), fmaxf(mbuf[2], mbuf[3]));
        const float ms = m == NEG_INF ? 0.0f : m;
        float f[4];
        sum = 0.0f;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            f[w] = __builtin_amdgcn_exp2f(mbuf[w] - ms);
            sum += lbuf[w] * f[w];
        }
        const int gr = i.row0 + r, t = gr / G;
        const int64_t orow = (int64_t)(i.token + t) * p.Hq + i.head * G + gr - t * G;
        const float inv = finish(m, sum);
        uint16_t *o = p.o + orow * D + C * lane;
#pragma unroll
        for (int e = 0; e < C; ++e) {
            v[e] = 0.0f;
#pragma unroll
            for (int w = 0; w < 4; ++w) v[e] += obuf[w * D + C * lane + e] * f[w];
            v[e] *= inv;
        }
        if constexpr (C == 1) {
            *o = (uint16_t)pack2(v[0], 0.0f);
        } else {
#pragma unroll
            for (int e = 0; e < C; e += 2) *reinterpret_cast<uint32_t *>(o + e) = pack2(v[e], v[e + 1]);
        }
        if (lane == 0) p.lse[orow] = finish_lse(m, sum);
    }
}

template <int D>
__global__ __launch_bounds__(256) void cache_join_kernel(CacheAttnParams p)
{
    const int G = p.Hq / p.b.Hkv, b = (int)blockIdx.x - p.slots[0];
    const bool many = b >= 0;
    // (a row tile's workgroups lie slots apart: neighbours are on different XCDs)
    const int form = many ? 1 : 0, x = many ? b % p.slots[1] : (int)blockIdx.x;
    const int count = p.counts[form];
    const PartInfo i = static_cast<const PartInfo *>(p.info[form])[x];   // (of this call where x < count)
    // (whatever tables that break their rules leave here, nothing outside the arrays is touched)
    const int slot0 = x - i.piece;
    if (x >= count || i.piece < 0 || i.pieces <= i.piece || slot0 < 0 || i.pieces > p.slots[form] - slot0 || i.head < 0 || i.head >= p.b.Hkv
        || i.token < 0 || i.row0 < 0 || i.rows < 0 || i.rows > (many ? ManyRows::ROWS : FewRows::ROWS)
        || i.token + (i.row0 + (int64_t)i.rows - 1) / G >= p.b.T)
        return;
    if (many) join_many<D>(p, i, slot0, b / p.slots[1], G);
    else join_few<D>(p, i, slot0, G);
}

template <int D, int KT>
hipError_t launch_forms(const CacheAttnParams &p, hipStream_t s)
{
    if (p.b.S > PLAN_ALONE) cache_plan_kernel<<<dim3(2), 1024, 0, s>>>(p);
    if (!p.units[1] || p.apart) cache_few_kernel<D, KT><<<dim3((unsigned)p.units[0]), 256, 0, s>>>(p);
    if (p.units[1]) {
        const hipError_t e = launch_cache_prompt(D, p, s);
        if (e != hipSuccess) return e;
    }
    const int joins = p.slots[0] + MANY_BY * p.slots[1];
    if (joins) cache_join_kernel<D><<<dim3((unsigned)joins), 256, 0, s>>>(p);
    return hipGetLastError();
}

size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }

// Sequences of at most this many rows take the form for few rows, where a batch
// holds both (32 sequences of 8K keys, d = 128, 8 kv heads: 32 rows each 143 us
// in it and 243 in the other, 64 rows 227 and 240, 128 rows 428 and 258).
constexpr int FEW = 64;

// Batches of 16 rows a sequence or fewer on average (single tokens, a few drafted
// ones, a chunk beside many of them) take the form for few rows: in the kernel of
// both forms short sequences leave half of its 8 waves idle (200 sequences of up
// to 8 tokens and 500 keys: 23 us, 51 in it).  But an average bounds no sequence,
// and a long chunk among them costs up to 2.5 times what it does in the other
// form.  So that follows in a launch of its own where the longest sequence there
// can be, if every other has a token, could cost far more than a launch: its rows
// times the table's keys, the kv heads and d are CHUNK at least.  Beside 127
// single tokens over 20 to 30000 keys (32/8 heads, d = 128) a chunk of 385 tokens:
// 436 us instead of 728, of 100 314 instead of 396, of 50 (1.4 CHUNK) 295 instead
// of 311.  Where no sequence is long after all, that launch ends at once (128
// sequences of 4 tokens over 8000 keys: 377 us instead of 368; 1000 of 4 over 1000
// 442 instead of 423; 32 of 4 over 300, in a table of 32768, 16 instead of 14).
// Below CHUNK it rather loses (97 tokens beside 31 single ones, all over 8000 keys,
// 0.8 CHUNK: 137 us instead of 116; 512 of one head beside 63, 1.05 CHUNK: 234 and
// 232).
constexpr int64_t CHUNK = (int64_t)1 << 32;

// Bounds of a call from what the host knows: no sequence has more than T G
// rows, and they have T G / S on average.  Either form is right for any
// sequence: which takes which is a matter of time only.
struct Bounds {
    int above[2], upto[2], units[2], slots[2];
    bool apart;   // both forms, in launches of their own
};

// A sequence of kt key tiles and `pairs` row tiles times heads is cut in at most
// kt / each + 0.01 pieces, or two where kt / each > 1.01, and sum(pairs kt) / each
// <= TARGET: below sum(pairs) + TARGET units, and at most kt / MIN_TILES a pair
// (or one).  Where there are two or more they are below 2 kt / each: below
// 2 TARGET partial outputs.  Where no pair can have two there are none.
template <class F>
void bound(Bounds &b, int64_t pairs, int64_t keys)
{
    const int64_t most = (keys + TILE - 1) / TILE / F::MIN_TILES;   // pieces of a pair
    const int64_t a = pairs + F::TARGET, c = pairs * (most > 1 ? most : 1), units = a < c ? a : c;
    const int64_t parts = 2 * F::TARGET;
    b.units[F::FORM] = (int)units;
    b.slots[F::FORM] = most <= 1 ? 0 : (int)(units < parts ? units : parts);
}

Bounds bounds(int D, int64_t T, int64_t S, int G, int Hkv, int64_t keys)
{
    Bounds b = {};
    const int64_t rows = T * G;
    const int64_t longest = (T - S + 1) * G;                     // (rows of one sequence, if every other has a token)
    const bool brief = rows <= FewRows::ROWS * S;
    const bool few = rows <= FEW || (brief && (longest <= FEW || longest * keys * Hkv * D < CHUNK));
    const bool both = !few && S > 1;
    b.apart = both && brief;
    const int64_t limit = few ? rows : (both ? FEW : 0);         // rows up to which a sequence is among the few
    if (few || both) {
        const int64_t most = rows / FewRows::ROWS + S, each = S * ((limit + FewRows::ROWS - 1) / FewRows::ROWS);
        b.upto[0] = (int)limit;
        bound<FewRows>(b, (most < each ? most : each) * Hkv, keys);
    }
    if (!few) {
        b.above[1] = (int)limit;
        b.upto[1] = (int)rows;
        const int64_t longer = rows / (limit + 1);   // sequences of more than `limit` rows at most
        bound<ManyRows>(b, (rows / ManyRows::ROWS + (longer < S ? longer : S)) * Hkv, keys);
    }
    return b;
}

// The workspace: counts, the plan, infos, running maxima and sums, partial outputs.
struct Layout {
    size_t before[2], info[2], ml[2], part[2], total;
};

Layout layout(const Bounds &b, int D, int64_t S)
{
    Layout l = {};
    size_t at = 256;
    const size_t rows[2] = {(size_t)b.slots[0] * FewRows::ROWS, (size_t)b.slots[1] * ManyRows::ROWS};
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at += align256(bytes);
        return here;
    };
    const bool plan = S > PLAN_ALONE;
    for (int f = 0; f < 2; ++f) l.before[f] = take(plan && b.units[f] ? S * sizeof(Before) : 0);
    for (int f = 0; f < 2; ++f) l.info[f] = take(b.slots[f] * sizeof(PartInfo));
    for (int f = 0; f < 2; ++f) l.ml[f] = take(rows[f] * 2 * sizeof(float));
    for (int f = 0; f < 2; ++f) l.part[f] = take(rows[f] * D * sizeof(float));
    l.total = plan || b.slots[0] + b.slots[1] ? at : 0;
    return l;
}

} // namespace

size_t cache_attn_workspace(int D, int64_t T, int64_t S, int G, int Hkv, int64_t keys)
{
    return layout(bounds(D, T, S, G, Hkv, keys), D, S).total;
}

hipError_t launch_cache_attn(int D, CacheAttnParams &p, void *ws, hipStream_t s)
{
    const Bounds b = bounds(D, p.b.T, p.b.S, p.Hq / p.b.Hkv, p.b.Hkv, (int64_t)p.b.width << p.b.page_shift);
    const Layout l = layout(b, D, p.b.S);
    char *base = static_cast<char *>(ws);
    p.apart = b.apart;
    p.counts = reinterpret_cast<int *>(base);
    p.split = base + 16;
    for (int f = 0; f < 2; ++f) {
        p.rows_above[f] = b.above[f];
        p.rows_upto[f] = b.upto[f];
        p.units[f] = b.units[f];
        p.slots[f] = b.slots[f];
        p.before[f] = base + l.before[f];
        p.info[f] = base + l.info[f];
        p.part_ml[f] = reinterpret_cast<float *>(base + l.ml[f]);
        p.part[f] = reinterpret_cast<float *>(base + l.part[f]);
    }
    switch (D) {
    case 64: return launch_forms<64, 64>(p, s);
    case 128: return launch_forms<128, 64>(p, s);
    default: return launch_forms<256, 32>(p, s);
    }
}

} // namespace lamp
