// lamp_pages.hip -- which pages of a long context a token attends: the range of each
// channel over the keys of a page, and the pages with the largest upper bound of a
// logit.
//
// With hi_c and lo_c the largest and smallest code value of channel c over a page's
// keys, no key of the page has a larger product with q than
//   ks sum_c (max(q_c, 0) hi_c + min(q_c, 0) lo_c),
// ks the page's scale.  The ranges are held in int8 in units of 4, rounded outward
// (|hi|, |lo| <= 448 / 4 = 112; a quarter of the codes' bytes would hold them
// exactly, but integers make the score exact), and the queries of a token and kv
// head are rounded to int8 under one power of two (|q'_c| <= 127).  So a score is
// an integer up to d 127 112 < 2^22, exact in whatever order it is summed, times a
// power of two, and the same pages are selected everywhere.
#include <hip/hip_runtime.h>

#include "lamp_cache_plan.h"

namespace lamp {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

constexpr int RANGE_UNIT = 4;      // code values of a step of a range

// The number where the other is a quiet NaN, as conversions make them.  (The compiler
// quiets the operands of its own maximum first: two instructions more for each.  Lane
// exchanges do not read what these write: the compiler does not see their hazards.)
__device__ __forceinline__ f16x2 max2(f16x2 a, f16x2 b)
{
    f16x2 r;
    asm("v_pk_max_f16 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
    return r;
}

__device__ __forceinline__ f16x2 min2(f16x2 a, f16x2 b)
{
    f16x2 r;
    asm("v_pk_min_f16 %0, %1, %2" : "=v"(r) : "v"(a), "v"(b));
    return r;
}

// Max and min over the lanes whose numbers differ in bits of `from` and up, in all of
// them: within rows of 16 lanes by rotation, then over the rows.
template <int FROM, class OP>
__device__ __forceinline__ f16x2 over_lanes(f16x2 v, OP op)
{
    auto bits = [](f16x2 x) { return __builtin_bit_cast(int, x); };
    auto pair = [](int x) { return __builtin_bit_cast(f16x2, x); };
    v = __builtin_elementwise_canonicalize(v);
    if constexpr (FROM <= 4) v = op(v, pair(__builtin_amdgcn_update_dpp(0, bits(v), 0x124, 0xf, 0xf, false)));   // row_ror:4
    if constexpr (FROM <= 8) v = op(v, pair(__builtin_amdgcn_update_dpp(0, bits(v), 0x128, 0xf, 0xf, false)));   // row_ror:8
    const auto a = __builtin_amdgcn_permlane16_swap((uint32_t)bits(v), (uint32_t)bits(v), false, false);
    v = op(pair((int)a[0]), pair((int)a[1]));
    const auto b = __builtin_amdgcn_permlane32_swap((uint32_t)bits(v), (uint32_t)bits(v), false, false);
    return op(pair((int)b[0]), pair((int)b[1]));
}

// A wave ranges over the keys of one page and head that received tokens; a lane
// takes 16 channels of every 64/(D/16)-th key, AT of them at once.  Bound for prompts by
// loads and issue alike (32768 tokens, 8 heads, d = 128: 34.6 MB in 10 us; in fp32
// instead of pairs of fp16, a workgroup for each head: 15.5), for single tokens by the
// latencies of starts, lengths, table and codes (32 tokens: 5.6 us).
template <int D>
__global__ __launch_bounds__(256) void kv_bounds_kernel(BoundsParams p)
{
    constexpr int LPR = D / 16, KEYS = 64 / LPR, AT = 8;   // lanes of a key, keys of a load
    const PageWork w = page_work(p.b, p.by_token, (int)blockIdx.x);
    if (w.count == 0) return;   // (the whole workgroup)
    const int lane = threadIdx.x & 63, page = 1 << p.b.page_shift, keys = w.first + w.count;
    const int head = (int)blockIdx.y * 4 + __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    if (head >= p.b.Hkv) return;
    const uint8_t *codes = p.kc + (w.page * p.b.Hkv + head) * (int64_t)page * D;
    // (e4m3 is exact in fp16: two channels a word)
    const _Float16 inf = (_Float16)__builtin_inff();
    f16x2 hi[8], lo[8];
#pragma unroll
    for (int c = 0; c < 8; ++c) hi[c] = f16x2{-inf, -inf}, lo[c] = f16x2{inf, inf};
    for (int k0 = lane / LPR; k0 - lane / LPR < keys; k0 += AT * KEYS) {
        u32x4 x[AT];
#pragma unroll
        for (int a = 0; a < AT; ++a) {   // (beyond the last key: the last again)
            const int k = k0 + a * KEYS;
            x[a] = *reinterpret_cast<const u32x4 *>(codes + (k < keys ? k : keys - 1) * D + 16 * (lane % LPR));
        }
#pragma unroll
        for (int a = 0; a < AT; ++a)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const f16x2 u = __builtin_bit_cast(f16x2, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(x[a][i], 1.0f, false));
                const f16x2 v = __builtin_bit_cast(f16x2, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(x[a][i], 1.0f, true));
                hi[2 * i] = max2(hi[2 * i], u), lo[2 * i] = min2(lo[2 * i], u);
                hi[2 * i + 1] = max2(hi[2 * i + 1], v), lo[2 * i + 1] = min2(lo[2 * i + 1], v);
            }
    }
    // over the lanes of a channel, then in steps
    uint32_t words[2][4] = {};   // of hi and lo, 4 channels each
#pragma unroll
    for (int c = 0; c < 8; ++c) {
        const f16x2 a = over_lanes<LPR>(hi[c], [](f16x2 u, f16x2 v) { return __builtin_elementwise_max(u, v); });
        const f16x2 b = over_lanes<LPR>(lo[c], [](f16x2 u, f16x2 v) { return __builtin_elementwise_min(u, v); });
#pragma unroll
        for (int e = 0; e < 2; ++e) {   // (a channel with no number: 0)
            const int up = a[e] < -(_Float16)1000 ? 0 : (int)__builtin_ceilf((float)a[e] * (1.0f / RANGE_UNIT));
            const int down = b[e] > (_Float16)1000 ? 0 : (int)__builtin_floorf((float)b[e] * (1.0f / RANGE_UNIT));
            words[0][c / 2] |= (uint32_t)(up & 255) << (16 * (c & 1) + 8 * e);
            words[1][c / 2] |= (uint32_t)(down & 255) << (16 * (c & 1) + 8 * e);
        }
    }
    // lanes 0 .. LPR - 1 hold all channels
    if (lane < LPR) {
        u32x4 *out = reinterpret_cast<u32x4 *>(p.bounds + (w.page * p.b.Hkv + head) * (int64_t)(2 * D));
        out[lane] = u32x4{words[0][0], words[0][1], words[0][2], words[0][3]};
        out[LPR + lane] = u32x4{words[1][0], words[1][1], words[1][2], words[1][3]};
    }
}

// --- selecting ------------------------------------------------------------------

__device__ __forceinline__ bool finite16(uint32_t h)
{
    return (h & 0x7F80u) != 0x7F80u;
}

// The power of two 2^e, e >= -100, under which bf16 magnitudes up to amax (their
// bits) are at most 127, as e: 127/64 is 1.984375, the bf16 mantissa 0x7E.
__device__ __forceinline__ int step_exponent(uint32_t amax)
{
    const int e = (int)(amax >> 7) - 127 - 6 + ((amax & 0x7Fu) == 0x7Fu);
    return e < -100 ? -100 : e;
}

// Order-preserving bits, above MISSING and below FORCED, of x ks: x below 2^22, ks any
// fp32 power of two or 0.  The product passes fp32's range at both ends, so that the
// exponent of ks, from -148 to 128, is added to that of x times its mantissa: 9 bits;
// the last bit of the product's mantissa, 0 for such ks, makes room.
struct Scale {
    float mantissa;
    uint32_t exponent;   // above 0, in place in the bits of an fp32 number
};

__device__ __forceinline__ Scale scale_of(float ks)
{
    return {__builtin_amdgcn_frexp_mantf(ks), (uint32_t)(__builtin_amdgcn_frexp_expf(ks) + 149) << 23};
}

__device__ __forceinline__ uint32_t sortable(int x, const Scale &s)
{
    const float y = (float)x * s.mantissa;
    const uint32_t b = __builtin_bit_cast(uint32_t, y), m = y == 0.0f ? 0u : ((b & 0x7FFFFFFFu) + s.exponent) >> 1;
    return 0x80000000u + (b & 0x80000000u ? 0u - m : m);
}

constexpr uint32_t MISSING = 0, FORCED = ~0u;

// A tile: tokens of one sequence whose groups' heads are the rows of one matrix product.
struct TokenTile {
    int s, tok, n, pos, len;   // sequence (-1: none), first token, tokens, position of the first, keys
};

// Tile x of sequences that have floor(start / per) + s tiles before them (at least
// their number: n tokens have at most n / per + 1).
__device__ __forceinline__ TokenTile token_tile(const PagedBatch &b, int per, int x)
{
    const TokenTile none = {-1, 0, 0, 0, 0};
    auto start = [&](int s) { return b.q_start ? b.q_start[s] : s; };
    auto first = [&](int s) { return (int64_t)(start(s) / per) + (per > 1 ? s : 0); };
    int s, a, e, keys;
    if (b.S <= 64) {   // (a lane for each sequence: one load's latency; those behind the last repeat it)
        const int l = (int)(threadIdx.x & 63) < b.S ? (int)(threadIdx.x & 63) : b.S - 1;
        const int al = start(l), el = start(l + 1), kl = b.kv_lens[l];
        s = 63 - __builtin_clzll(__ballot(l == 0 || (int64_t)(al / per) + (per > 1 ? l : 0) <= x));
        s = s < b.S ? s : b.S - 1;
        a = __builtin_amdgcn_readlane(al, s);
        e = __builtin_amdgcn_readlane(el, s);
        keys = __builtin_amdgcn_readlane(kl, s);
    } else {
        s = last_at_most(b.S, x, first);
        a = start(s);
        e = start(s + 1);
        keys = b.kv_lens[s];
    }
    const int i = (int)(x - ((int64_t)(a / per) + (per > 1 ? s : 0))) * per;
    if (a < 0 || e > b.T || i < 0 || i >= e - a) return none;
    const int len = keys > 0 ? keys : 0;
    return {s, a + i, e - a - i < per ? e - a - i : per, len - (e - a) + i, len};
}

// Places that a position sees (with a table entry).
__device__ __forceinline__ int places_of(const PagedBatch &b, int pos, int len)
{
    const int keys = pos + 1 < len ? pos + 1 : len;
    if (keys <= 0) return 0;
    const int n = ((keys - 1) >> b.page_shift) + 1;
    return n < b.width ? n : b.width;
}

// 8 channels of a tile's queries: chunk i of those of its tokens' groups.
struct Chunk {
    int tk, g, c;
    u32x4 x;
};

template <int D>
__device__ __forceinline__ Chunk load_chunk(const SelectParams &p, const TokenTile &t, int head, int i)
{
    const int G = p.Hq / p.b.Hkv, r = i / (D / 8), tk = r / G;
    Chunk k = {tk, r - tk * G, i - r * (D / 8), {0, 0, 0, 0}};
    const int there = tk < t.n ? tk : 0;   // (tokens behind the last: whatever, loaded without a branch that would wait)
    k.x = *reinterpret_cast<const u32x4 *>(p.q + (int64_t)(t.tok + there) * p.q_st + (int64_t)(head * G + k.g) * p.q_sh + 8 * k.c);
    return k;
}

// Largest bf16 magnitude (its bits) of each token's group among finite ones, into
// amax[16] (LDS, zeroed); `mine` is the thread's first chunk.  RAW (groups of up to 16
// heads): the queries stay in `raw`, by the operand's rows.
template <int D, int THREADS, bool RAW>
__device__ __forceinline__ void group_amax(const SelectParams &p, const TokenTile &t, int head, const Chunk &mine, uint32_t *amax, u32x4 (*raw)[D / 8])
{
    const int G = p.Hq / p.b.Hkv, many = t.n * G * (D / 8);
    auto take = [&](const Chunk &c) {
        uint32_t m = 0;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const uint32_t a = c.x[k] & 0x7FFFu, b = c.x[k] >> 16 & 0x7FFFu;
            m = finite16(a) && a > m ? a : m;
            m = finite16(b) && b > m ? b : m;
        }
        atomicMax(&amax[c.tk], m);
        if (RAW) raw[(c.tk << p.heads_shift) + c.g][c.c] = c.x;
    };
    if ((int)threadIdx.x < many) take(mine);   // (not in the loop, whose loads would be waited for with all that are on the way)
    for (int i = (int)threadIdx.x + THREADS; i < many; i += THREADS) take(load_chunk<D>(p, t, head, i));
}

// The int8 operand [max(q', 0) | min(q', 0)] of 16 rows: of lane l in step k the row
// l % 16 and its bytes (2 D/4) (l / 16) + 16 k.  Row (t << HS) + g is head 16 round + g
// of token t's group (HS = heads_shift; rows without a head repeat the first, those
// without a token are 0).
template <int D, int THREADS, bool RAW>
__device__ __forceinline__ void build_rows(const SelectParams &p, const TokenTile &t, int head, int round, const uint32_t *amax,
                                           const u32x4 (*raw)[D / 8], u32x4 (*rows)[64])
{
    const int G = p.Hq / p.b.Hkv, hs = p.heads_shift;
    for (int i = (int)threadIdx.x; i < 2 * D; i += THREADS) {   // (2 D/64 steps of 64 lanes)
        const int k = i >> 6, l = i & 63, r = l & 15, at = (2 * D / 4) * (l >> 4) + 16 * k;
        const int tk = r >> hs, g = 16 * round + (r & ((1 << hs) - 1));
        u32x4 w = {0, 0, 0, 0};
        if (tk < t.n) {
            const int gg = g < G ? g : 0;
            const uint16_t *src = p.q + (int64_t)(t.tok + tk) * p.q_st + (int64_t)(head * G + gg) * p.q_sh + at % D;
            const u32x4 *from = RAW ? &raw[(tk << hs) + gg][at % D / 8] : reinterpret_cast<const u32x4 *>(src), a = from[0], b = from[1];
            const float inv = __builtin_bit_cast(float, (uint32_t)(127 - step_exponent(amax[tk])) << 23);
            const bool neg = at >= D;
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const uint32_t word = e < 8 ? a[e / 2] : b[e / 2 - 4], bits = e & 1 ? word >> 16 : word & 0xFFFFu;
                const float x = finite16(bits) ? __builtin_bit_cast(float, bits << 16) * inv : 0.0f;
                const int v = (int)__builtin_rintf(x), s = neg ? (v < 0 ? v : 0) : (v > 0 ? v : 0);
                w[e / 4] |= (uint32_t)(s & 255) << (8 * (e % 4));
            }
        }
        rows[k][l] = w;
    }
}

// The ranges of the pages in table entries pg (each of the lane's place, lane % 16),
// and their scales; and their products with the operand: its rows 4 (lane / 16) + e.
template <int D, int AT>
struct Ranges {
    i32x4 x[AT][2 * D / 64];
    float ks[AT];

    __device__ __forceinline__ void load(const SelectParams &p, const int *pg, int head)
    {
        const int lane = threadIdx.x & 63;
#pragma unroll
        for (int j = 0; j < AT; ++j) {
            const bool is = pg[j] >= 0 && pg[j] < p.b.pages;
            const int64_t at = (int64_t)(is ? pg[j] : 0) * p.b.Hkv + head;
            const int8_t *src = p.bounds + at * (2 * D) + (2 * D / 4) * (lane >> 4);
#pragma unroll
            for (int k = 0; k < 2 * D / 64; ++k) x[j][k] = *reinterpret_cast<const i32x4 *>(src + 16 * k);
            ks[j] = p.ks[at];
        }
    }

    __device__ __forceinline__ void multiply(const u32x4 (*rows)[64], i32x4 *acc) const
    {
        const int lane = threadIdx.x & 63;
#pragma unroll
        for (int j = 0; j < AT; ++j) {
            acc[j] = i32x4{0, 0, 0, 0};
#pragma unroll
            for (int k = 0; k < 2 * D / 64; ++k) acc[j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, rows[k][lane]), x[j][k], acc[j], 0, 0, 0);
        }
    }
};

// The largest over each token's rows, in the lanes and elements of their first.
__device__ __forceinline__ void row_max(i32x4 &x, int hs)
{
    if (hs >= 1) x[0] = x[0] > x[1] ? x[0] : x[1], x[2] = x[2] > x[3] ? x[2] : x[3];
    if (hs >= 2) x[0] = x[0] > x[2] ? x[0] : x[2];
    if (hs >= 3) {
        const int y = __shfl_xor(x[0], 16, 64);
        x[0] = x[0] > y ? x[0] : y;
    }
    if (hs >= 4) {
        const int y = __shfl_xor(x[0], 32, 64);
        x[0] = x[0] > y ? x[0] : y;
    }
}

// Token tk's score of the lane's place with page pg, of scale ks, to write(tk, key), by
// the lane that has it.
template <class W>
__device__ __forceinline__ void write_scores(const SelectParams &p, const i32x4 &x, int pg, float ks, int n, W write)
{
    const int lane = threadIdx.x & 63, hs = p.heads_shift;
    const bool is = pg >= 0 && pg < p.b.pages;
    const Scale scale = scale_of(ks);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int r = 4 * (lane >> 4) + e, tk = r >> hs;
        if ((r & ((1 << hs) - 1)) == 0 && tk < n) write(tk, is ? sortable(x[e], scale) : MISSING);
    }
}

// The smallest key of a row that is taken and how many that equal it: 8 bits a step
// from a histogram in LDS.  each(f) goes over the thread's part of the keys.
struct Taken {
    uint32_t key;
    int same;
};

template <int BY, class E>
__device__ __forceinline__ Taken narrow(uint32_t (&hist)[256], int (&found)[2], int budget, E each)
{
    const int tid = (int)threadIdx.x, lane = tid & 63;
    Taken t = {0, budget};
    for (int shift = 24; shift >= 0; shift -= 8) {
        if (tid < 256) hist[tid] = 0;
        __syncthreads();
        const uint32_t mask = shift == 24 ? 0u : ~0u << (shift + 8);
        each([&](uint32_t k) {
            if ((k & mask) == t.key) atomicAdd(&hist[k >> shift & 255], 1u);
        });
        __syncthreads();
        if (tid < 64) {
            // lane l: the 4 digits from 252 - 4 l down in order of size
            uint32_t n[4], sum = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) sum += n[e] = hist[255 - 4 * lane - e];
            uint32_t above = wave_scan(sum) - sum;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (above < (uint32_t)t.same && (uint32_t)t.same <= above + n[e]) found[0] = 255 - 4 * lane - e, found[1] = (int)above;
                above += n[e];
            }
        }
        __syncthreads();
        t.key |= (uint32_t)found[0] << shift;
        t.same -= found[1];
    }
    return t;
}

// Places of the keys above t.key, and of the first t.same that equal it, in order:
// the waves take consecutive parts; key(i) for i < many.
template <int BY, class K>
__device__ __forceinline__ void write_places(const Taken &t, int many, int (&counts)[BY / 64][2], int *out, K key)
{
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int each = ((many + BY / 64 - 1) / (BY / 64) + 63) & ~63, a = wave * each, e = a + each < many ? a + each : many;
    int above = 0, same = 0;
    for (int i = a + lane; i - lane < e; i += 64) {
        const uint32_t k = i < e ? key(i) : 0;
        above += __popcll(__ballot(i < e && k > t.key));
        same += __popcll(__ballot(i < e && k == t.key));
    }
    if (lane == 0) counts[wave][0] = above, counts[wave][1] = same;
    __syncthreads();
    int at = 0, equal = 0;
    for (int w = 0; w < wave; ++w) {
        const int left = t.same - equal > 0 ? t.same - equal : 0, eq = counts[w][1];
        at += counts[w][0] + (eq < left ? eq : left);
        equal += eq;
    }
    const uint64_t below = ((uint64_t)1 << lane) - 1;
    for (int i = a + lane; i - lane < e; i += 64) {
        const uint32_t k = i < e ? key(i) : 0;
        const uint64_t eq = __ballot(i < e && k == t.key);
        const bool take = i < e && (k > t.key || (k == t.key && equal + __popcll(eq & below) < t.same));
        const uint64_t got = __ballot(take);
        if (take) out[at + __popcll(got & below)] = i;
        at += __popcll(got);
        equal += __popcll(eq);
    }
}

// The same by one wave for one row of up to 64 R keys: the largest key that at least
// `budget` reach, bit by bit, their number counted by ballots, until exactly `budget`
// reach one.  Then its places.
template <int R, class K>
__device__ __forceinline__ void select_row(int many, int budget, int *out, K key)
{
    const int lane = threadIdx.x & 63;
    uint32_t k[R], low = 0, high = 0;   // (low: of the complements)
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const bool is = 64 * r + lane < many;
        k[r] = is ? key(64 * r + lane) : 0u;   // (0: below whatever counts)
        high = k[r] > high ? k[r] : high;
        low = is && ~k[r] > low ? ~k[r] : low;
    }
    auto largest = [](uint32_t v) { return (uint32_t)lane_value((int)wave_scan_by(v, [](uint32_t a, uint32_t b) { return a > b ? a : b; }), 63); };
    high = largest(high);
    low = ~largest(low);
    // keys that are at least x (>= 1)
    auto reach = [&](uint32_t x) {
        int n = 0;
#pragma unroll
        for (int r = 0; r < R; ++r) n += __popcll(__ballot(k[r] >= x));
        return n;
    };
    // (the bits that all have in common need no counting)
    const uint32_t differ = low ^ high;
    const int top = differ ? 32 - __builtin_clz(differ) : 0;
    uint32_t least = top == 32 ? 0 : low >> top << top;
    for (int bit = top - 1; bit >= 0; --bit) {
        const uint32_t x = least | 1u << bit;
        const int n = reach(x);
        if (n >= budget) least = x;
        if (n == budget) break;
    }
    const int above = least == ~0u ? 0 : reach(least + 1);
    int same = budget - above, at = 0;   // of those that equal it, the first
    const uint64_t below = ((uint64_t)1 << lane) - 1;
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const bool is = 64 * r + lane < many;
        const uint64_t eq = __ballot(is && k[r] == least);
        const bool take = is && (k[r] > least || (k[r] == least && __popcll(eq & below) < same));
        const uint64_t got = __ballot(take);
        if (take) out[at + __popcll(got & below)] = 64 * r + lane;
        at += __popcll(got);
        same -= __popcll(eq) < same ? __popcll(eq) : same;
    }
}

// A tile's tokens and one kv head, scores in LDS.  Bound by latencies one after another:
// starts and lengths, table, ranges (the queries are made ready meanwhile), products,
// and the counts of the selection (1 token of 313 places, 8 heads: 11 us), with long
// rows by what one CU reads (32 tokens of 188 to 500 places, 22 MB: 17 us).
constexpr int SELECT_BY = 512, WIDEST = 1024;   // threads; places of a row

template <int D, bool RAW>
__global__ __launch_bounds__(SELECT_BY) void select_kernel(SelectParams p)
{
    constexpr int WAVES = SELECT_BY / 64;
    __shared__ u32x4 rows[2 * D / 64][64];
    __shared__ u32x4 raw[16][D / 8];
    __shared__ uint32_t amax[16];
    extern __shared__ uint32_t keys[];             // [tokens][places]
    const int G = p.Hq / p.b.Hkv, hs = p.heads_shift;
    const TokenTile t = token_tile(p.b, p.tokens, (int)blockIdx.x);
    if (t.s < 0) return;
    const int head = (int)blockIdx.y, tid = (int)threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int most = places_of(p.b, t.pos + t.n - 1, t.len);
    auto out_of = [&](int tk) { return p.places + ((int64_t)(t.tok + tk) * p.b.Hkv + head) * p.budget; };
    if (most > p.budget) {
        const int *table = p.b.table + t.s * p.b.table_stride;
        constexpr int AT = D > 128 ? 2 : 4;        // blocks of 16 places of a wave at once
        const Chunk mine = load_chunk<D>(p, t, head, tid);   // (first: loads come back in order)
        int pg[AT];
        auto look_up = [&](int q0) {
#pragma unroll
            for (int j = 0; j < AT; ++j) {
                const int place = q0 + 16 * j + (lane & 15);
                const int entry = table[place < most ? place : most - 1];
                pg[j] = place < most ? entry : -1;
            }
        };
        look_up(wave * 16 * AT);
        Ranges<D, AT> ranges;
        ranges.load(p, pg, head);   // (while the queries are made ready)
        if (tid < 16) amax[tid] = 0;
        __syncthreads();
        group_amax<D, SELECT_BY, RAW>(p, t, head, mine, amax, raw);
        __syncthreads();
        const int rounds = (G + 15) / 16;
        for (int round = 0; round < rounds; ++round) {
            if (round) __syncthreads();
            build_rows<D, SELECT_BY, RAW>(p, t, head, round, amax, raw, rows);
            __syncthreads();
            for (int q0 = wave * 16 * AT; q0 < most; q0 += WAVES * 16 * AT) {
                if (round || q0 >= WAVES * 16 * AT) {
                    look_up(q0);
                    ranges.load(p, pg, head);
                }
                i32x4 x[AT];
                ranges.multiply(rows, x);
#pragma unroll
                for (int j = 0; j < AT; ++j) {
                    const int place = q0 + 16 * j + (lane & 15);
                    row_max(x[j], hs);
                    if (place >= most) continue;
                    if (rounds == 1) {
                        write_scores(p, x[j], pg[j], ranges.ks[j], t.n, [&](int tk, uint32_t k) { keys[tk * p.b.width + place] = k; });
                    } else if (lane < 16) {   // (one token a tile: its products' maximum over the rounds first)
                        const int old = round ? (int)keys[place] : x[j][0], now = x[j][0] > old ? x[j][0] : old;
                        keys[place] = (uint32_t)now;
                        if (round == rounds - 1) write_scores(p, i32x4{now, 0, 0, 0}, pg[j], ranges.ks[j], 1, [&](int, uint32_t k) { keys[place] = k; });
                    }
                }
            }
        }
        __syncthreads();
    }
    // a wave for each token
    for (int tk = wave; tk < t.n; tk += WAVES) {
        const int many = places_of(p.b, t.pos + tk, t.len);
        int *out = out_of(tk);
        auto key = [&](int i) { return i < p.first || i >= many - p.last ? FORCED : keys[tk * p.b.width + i]; };
        if (many <= p.budget) {
            for (int i = lane; i < p.budget; i += 64) out[i] = i < many ? i : -1;
        } else if (many <= 256) {
            select_row<4>(many, p.budget, out, key);
        } else if (many <= 512) {
            select_row<8>(many, p.budget, out, key);
        } else if (many <= 768) {
            select_row<12>(many, p.budget, out, key);
        } else {   // (up to WIDEST)
            select_row<WIDEST / 64>(many, p.budget, out, key);
        }
    }
}

// Where rows are too long for a workgroup each: scores over `chunk` places to memory, ...
template <int D, bool RAW>
__global__ __launch_bounds__(256) void select_score_kernel(SelectParams p)
{
    __shared__ u32x4 rows[2 * D / 64][64], raw[16][D / 8];
    __shared__ uint32_t amax[16];
    const int G = p.Hq / p.b.Hkv, hs = p.heads_shift;
    const TokenTile t = token_tile(p.b, p.tokens, (int)blockIdx.x);
    if (t.s < 0) return;
    const int head = (int)blockIdx.y, tid = (int)threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int many = places_of(p.b, t.pos + t.n - 1, t.len);
    const int p0 = (int)blockIdx.z * p.chunk, p1 = many - p0 < p.chunk ? many : p0 + p.chunk;
    if (p0 >= p1 || many <= p.budget) return;      // (all of them: no scores are looked at)
    const int *table = p.b.table + t.s * p.b.table_stride;
    if (tid < 16) amax[tid] = 0;
    __syncthreads();
    group_amax<D, 256, RAW>(p, t, head, load_chunk<D>(p, t, head, tid), amax, raw);
    __syncthreads();
    const int rounds = (G + 15) / 16;
    constexpr int AT = D > 128 ? 2 : 4;            // blocks of 16 places of a wave at once
    for (int q0 = p0 + wave * 16 * AT; q0 - wave * 16 * AT < p1; q0 += 64 * AT) {
        int pg[AT];
        i32x4 best[AT];
#pragma unroll
        for (int j = 0; j < AT; ++j) {
            const int place = q0 + 16 * j + (lane & 15);
            const int entry = table[place < p1 ? place : p1 - 1];
            pg[j] = place < p1 ? entry : -1;
        }
        Ranges<D, AT> ranges;
        ranges.load(p, pg, head);
        for (int round = 0; round < rounds; ++round) {
            if (q0 < p0 + 64 * AT || rounds > 1) {
                __syncthreads();
                build_rows<D, 256, RAW>(p, t, head, round, amax, raw, rows);
                __syncthreads();
            }
            i32x4 x[AT];
            ranges.multiply(rows, x);
#pragma unroll
            for (int j = 0; j < AT; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) best[j][e] = round == 0 || x[j][e] > best[j][e] ? x[j][e] : best[j][e];
        }
#pragma unroll
        for (int j = 0; j < AT; ++j) {
            const int place = q0 + 16 * j + (lane & 15);
            row_max(best[j], hs);
            if (place >= p1) continue;
            write_scores(p, best[j], pg[j], ranges.ks[j], t.n, [&](int tk, uint32_t k) {
                p.scores[((int64_t)(t.tok + tk) * p.b.Hkv + head) * p.b.width + place] = k;
            });
        }
    }
}

// ... and the places of a token and kv head from those, by a workgroup.
template <int BY>
__global__ __launch_bounds__(BY) void select_top_kernel(SelectParams p)
{
    __shared__ uint32_t hist[256];
    __shared__ int found[2], counts[BY / 64][2];
    const int head = (int)blockIdx.y, tid = (int)threadIdx.x;
    const TokenTile t = token_tile(p.b, 1, (int)blockIdx.x);
    if (t.s < 0) return;
    const int many = places_of(p.b, t.pos, t.len);
    const int64_t row = (int64_t)t.tok * p.b.Hkv + head;
    int *out = p.places + row * p.budget;
    if (many <= p.budget) {
        for (int i = tid; i < p.budget; i += BY) out[i] = i < many ? i : -1;
        return;
    }
    const uint32_t *scores = p.scores + row * p.b.width;
    auto key = [&](int i) { return i < p.first || i >= many - p.last ? FORCED : scores[i]; };
    const Taken taken = narrow<BY>(hist, found, p.budget, [&](auto f) {
        for (int i = tid; i < many; i += BY) f(key(i));
    });
    write_places<BY>(taken, many, counts, out, key);
}

} // namespace

hipError_t launch_kv_bounds(int D, const BoundsParams &params, hipStream_t s)
{
    BoundsParams p = params;
    const int64_t slots = (int64_t)(p.b.T >> p.b.page_shift) + 2 * (int64_t)p.b.S;   // (as for kv_append)
    p.by_token = p.b.T <= slots;
    const dim3 grid((unsigned)(p.by_token ? p.b.T : slots), (unsigned)((p.b.Hkv + 3) / 4));
    switch (D) {
    case 64: kv_bounds_kernel<64><<<grid, 256, 0, s>>>(p); break;
    case 128: kv_bounds_kernel<128><<<grid, 256, 0, s>>>(p); break;
    default: kv_bounds_kernel<256><<<grid, 256, 0, s>>>(p); break;
    }
    return hipGetLastError();
}

// The tokens of a tile; whether one launch does it all.
struct SelectShape {
    int heads_shift, tokens;
    int64_t tiles;
    bool one;
};

// In one launch where a workgroup for each tile is no worse than more of them and a
// second launch: with one token a sequence where it reads up to ALONE bytes of ranges
// (8 heads, d = 128, GPU time one / two: 1 token of 313 places 11.1 / 12.2 us; 32 tokens of
// 500 places 17.7 / 17.6, of 625 26.8 / 23.7, of 1250 42.6 / 32.3; but a call of two
// launches costs 4 us more on the host); with chunks of several, whose tokens share what
// is read and are selected from side by side, up to WIDEST places where the tiles fill the
// device (32 times 8 tokens of 781 places 42.8 / 44.7; 4 times 500 of 625 157 / 186, but 2000
// of 1250 608 / 449).  The scores of a tile fit half of a CU's LDS, KEYS of them.
constexpr int64_t KEYS = 12288, ALONE = (int64_t)1 << 17, CHUNK_TOKENS = 4;
// Places in the table from which a row's workgroup in the second launch is of 1024
// threads (6250 places of 32 tokens and 8 heads: 14 us; of one token and 8 heads 15, of 256
// threads 28).
constexpr int TOP_WIDE = 1024;

static SelectShape select_shape(int D, int64_t T, int64_t S, int G, int Hkv, int64_t width)
{
    SelectShape x = {};
    while (1 << x.heads_shift < G && x.heads_shift < 4) ++x.heads_shift;
    x.tokens = 16 >> x.heads_shift;
    auto tiles = [&](int per) { return per > 1 ? T / per + S : T; };
    x.tiles = tiles(x.tokens);
    // (fewer tokens a tile: the operand's other rows are 0)
    int per = x.tokens;
    while (per > 1 && (per * width > KEYS || tiles(per) * Hkv < 256)) per /= 2;
    x.one = width * per <= KEYS && width <= WIDEST && (width * 2 * D <= ALONE || (T >= CHUNK_TOKENS * S && tiles(per) * Hkv >= 256));
    if (x.one) x.tokens = per, x.tiles = tiles(per);
    return x;
}

size_t select_workspace(int D, int64_t T, int64_t S, int G, int Hkv, int64_t width, int64_t budget)
{
    return width <= budget || select_shape(D, T, S, G, Hkv, width).one ? 0 : (size_t)T * Hkv * width * sizeof(uint32_t);
}

template <int D, bool RAW>
static hipError_t launch_select_of(const SelectParams &p, const SelectShape &x, hipStream_t s)
{
    if (x.one || p.b.width <= p.budget) {
        const size_t keys = p.b.width <= p.budget ? 0 : (size_t)x.tokens * p.b.width * sizeof(uint32_t);
        select_kernel<D, RAW><<<dim3((unsigned)x.tiles, (unsigned)p.b.Hkv), SELECT_BY, keys, s>>>(p);
        return hipGetLastError();
    }
    select_score_kernel<D, RAW><<<dim3((unsigned)x.tiles, (unsigned)p.b.Hkv, (unsigned)((p.b.width + p.chunk - 1) / p.chunk)), 256, 0, s>>>(p);
    const dim3 rows((unsigned)p.b.T, (unsigned)p.b.Hkv);
    if (p.b.width > TOP_WIDE) select_top_kernel<1024><<<rows, 1024, 0, s>>>(p);
    else select_top_kernel<256><<<rows, 256, 0, s>>>(p);
    return hipGetLastError();
}

hipError_t launch_select(int D, SelectParams &p, void *ws, hipStream_t s)
{
    const SelectShape x = select_shape(D, p.b.T, p.b.S, p.Hq / p.b.Hkv, p.b.Hkv, p.b.width);
    p.scores = static_cast<uint32_t *>(ws);
    p.heads_shift = x.heads_shift;
    p.tokens = x.tokens;
    // chunks of 64 places at least, and enough of them to fill the device
    const int64_t most = (p.b.width + 63) / 64, want = (2048 + x.tiles * p.b.Hkv - 1) / (x.tiles * p.b.Hkv), n = want < most ? want : most;
    p.chunk = n > 0 ? (int)(((p.b.width + n - 1) / n + 63) / 64 * 64) : 64;
    const bool raw = p.Hq / p.b.Hkv <= 16;   // (queries in LDS: with a branch in the kernel every wait would be for all loads)
    switch (D) {
    case 64: return raw ? launch_select_of<64, true>(p, x, s) : launch_select_of<64, false>(p, x, s);
    case 128: return raw ? launch_select_of<128, true>(p, x, s) : launch_select_of<128, false>(p, x, s);
    default: return raw ? launch_select_of<256, true>(p, x, s) : launch_select_of<256, false>(p, x, s);
    }
}

} // namespace lamp
