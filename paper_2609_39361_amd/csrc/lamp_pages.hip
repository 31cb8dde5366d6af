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
// an integer below 2 d 127 112 < 2^23 times a power of two: exact in fp32 in
// whatever order it is summed, and the same pages are selected everywhere.
#include <hip/hip_runtime.h>

#include "lamp_search.h"
#include "lamp_serve.h"

namespace lamp {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef short i16x2 __attribute__((ext_vector_type(2)));

constexpr int RANGE_UNIT = 4;      // code values of a step of a range
constexpr int NONE = 1000;         // beyond every range: no key yet

__device__ __forceinline__ i16x2 max2(i16x2 a, i16x2 b) { return __builtin_elementwise_max(a, b); }
__device__ __forceinline__ i16x2 min2(i16x2 a, i16x2 b) { return __builtin_elementwise_min(a, b); }

// One workgroup ranges over the keys of one page and head that received tokens;
// a thread takes 16 channels of every 256/(D/16)-th key.
template <int D>
__global__ __launch_bounds__(256) void kv_bounds_kernel(BoundsParams p)
{
    constexpr int LPR = D / 16, RPB = 256 / LPR;   // threads of a key, keys of a pass
    __shared__ i16x2 red[2][4][D / 2];
    const PageWork w = page_work(p.b, p.by_token, (int)blockIdx.x);
    if (w.count == 0) return;   // (the whole workgroup)
    const int tid = (int)threadIdx.x, head = (int)blockIdx.y, page = 1 << p.b.page_shift, keys = w.first + w.count;
    const uint8_t *codes = p.kc + (w.page * p.b.Hkv + head) * (int64_t)page * D + 16 * (tid % LPR);
    float hi[16], lo[16];
#pragma unroll
    for (int c = 0; c < 16; ++c) hi[c] = -(float)(NONE * RANGE_UNIT), lo[c] = (float)(NONE * RANGE_UNIT);
    for (int k = tid / LPR; k < keys; k += RPB) {
        const u32x4 x = *reinterpret_cast<const u32x4 *>(codes + (int64_t)k * D);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)x[i], false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)x[i], true);
            const float v[4] = {a[0], a[1], b[0], b[1]};
#pragma unroll
            for (int e = 0; e < 4; ++e) hi[4 * i + e] = fmaxf(hi[4 * i + e], v[e]), lo[4 * i + e] = fminf(lo[4 * i + e], v[e]);   // (NaN: left out)
        }
    }
    // in steps, two channels a word, over the lanes of a channel, then over the waves
    i16x2 h2[8], l2[8];
#pragma unroll
    for (int c = 0; c < 8; ++c) {
        h2[c] = i16x2{(short)(int)__builtin_ceilf(hi[2 * c] * (1.0f / RANGE_UNIT)), (short)(int)__builtin_ceilf(hi[2 * c + 1] * (1.0f / RANGE_UNIT))};
        l2[c] = i16x2{(short)(int)__builtin_floorf(lo[2 * c] * (1.0f / RANGE_UNIT)), (short)(int)__builtin_floorf(lo[2 * c + 1] * (1.0f / RANGE_UNIT))};
    }
#pragma unroll
    for (int m = LPR; m < 64; m <<= 1)
#pragma unroll
        for (int c = 0; c < 8; ++c) {
            h2[c] = max2(h2[c], __builtin_bit_cast(i16x2, __shfl_xor(__builtin_bit_cast(int, h2[c]), m, 64)));
            l2[c] = min2(l2[c], __builtin_bit_cast(i16x2, __shfl_xor(__builtin_bit_cast(int, l2[c]), m, 64)));
        }
    if ((tid & 63) < LPR) {
#pragma unroll
        for (int c = 0; c < 8; ++c) red[0][tid >> 6][8 * (tid % LPR) + c] = h2[c], red[1][tid >> 6][8 * (tid % LPR) + c] = l2[c];
    }
    __syncthreads();
    // 4 channels a thread: D/4 words of hi, then of lo
    if (tid < D / 2) {
        const bool is_lo = tid >= D / 4;
        const int c2 = 2 * (tid % (D / 4));
        uint32_t word = 0;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            i16x2 v = red[is_lo][0][c2 + k];
#pragma unroll
            for (int wv = 1; wv < 4; ++wv) v = is_lo ? min2(v, red[1][wv][c2 + k]) : max2(v, red[0][wv][c2 + k]);
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int x = v[e] <= -NONE || v[e] >= NONE ? 0 : v[e];   // (a channel with no number)
                word |= (uint32_t)(x & 255) << (16 * k + 8 * e);
            }
        }
        reinterpret_cast<uint32_t *>(p.bounds + (w.page * p.b.Hkv + head) * (int64_t)(2 * D))[tid] = word;
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

// Order-preserving bits of a finite fp32 number, above 1 and below ~0u - 1.
__device__ __forceinline__ uint32_t sortable(float x)
{
    const uint32_t b = __builtin_bit_cast(uint32_t, x + 0.0f);   // (-0 as 0)
    return b & 0x80000000u ? ~b : b | 0x80000000u;
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
    const int s = last_at_most(b.S, x, first);
    const int a = start(s), e = start(s + 1), i = (int)(x - first(s)) * per;
    if (a < 0 || e > b.T || i < 0 || i >= e - a) return none;
    const int len = b.kv_lens[s] > 0 ? b.kv_lens[s] : 0;
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

// Scores of a tile's tokens and one kv head over `chunk` places: the products of
// int8 rows [max(q', 0) | min(q', 0)] with the ranges, 16 places a wave at a time.
// Rows of the operand: row of token t and head g of the group is (t << HS) + g,
// HS = heads_shift; groups of more than 16 heads go over their heads in rounds.
template <int D>
__global__ __launch_bounds__(256) void select_score_kernel(SelectParams p)
{
    constexpr int KS = 2 * D / 64;                 // 64-channel steps of the product
    __shared__ u32x4 rows[KS][64];                 // the operand: of lane l in step k
    __shared__ uint32_t amax[16];
    const int G = p.Hq / p.b.Hkv, hs = p.heads_shift, per = 16 >> hs;
    const TokenTile t = token_tile(p.b, per, (int)blockIdx.x);
    if (t.s < 0) return;
    const int head = (int)blockIdx.y, tid = (int)threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int many = places_of(p.b, t.pos + t.n - 1, t.len);
    const int p0 = (int)blockIdx.z * p.chunk, p1 = many - p0 < p.chunk ? many : p0 + p.chunk;
    if (p0 >= p1 || many <= p.budget) return;      // (all of them: no scores are looked at)
    const int *table = p.b.table + t.s * p.b.table_stride;
    // largest magnitude of each token's group
    if (tid < 16) amax[tid] = 0;
    __syncthreads();
    for (int i = tid; i < t.n * G * (D / 8); i += 256) {
        const int r = i / (D / 8), c = i - r * (D / 8), tk = r / G, h = head * G + r - tk * G;
        const u32x4 x = *reinterpret_cast<const u32x4 *>(p.q + (int64_t)(t.tok + tk) * p.q_st + (int64_t)h * p.q_sh + 8 * c);
        uint32_t m = 0;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const uint32_t a = x[k] & 0x7FFFu, b = x[k] >> 16 & 0x7FFFu;
            m = finite16(a) && a > m ? a : m;
            m = finite16(b) && b > m ? b : m;
        }
        atomicMax(&amax[tk], m);
    }
    i32x4 best[4];                                 // of 4 blocks of 16 places, until the rounds are over
    for (int q0 = p0; q0 < p1; q0 += 256) {
        for (int round = 0; round << 4 < G; ++round) {
            __syncthreads();
            // lane l's bytes of step k: row l % 16, bytes 2 D / 4 (l / 16) + 16 k of [max | min]
            for (int i = tid; i < KS * 64; i += 256) {
                const int k = i >> 6, l = i & 63, r = l & 15, at = (2 * D / 4) * (l >> 4) + 16 * k;
                const int tk = r >> hs, g = 16 * round + (r & ((1 << hs) - 1));
                u32x4 w = {0, 0, 0, 0};
                if (tk < t.n) {
                    const int h = head * G + (g < G ? g : 0);   // (missing rows repeat the first)
                    const uint16_t *src = p.q + (int64_t)(t.tok + tk) * p.q_st + (int64_t)h * p.q_sh + at % D;
                    const u32x4 a = *reinterpret_cast<const u32x4 *>(src), b = *reinterpret_cast<const u32x4 *>(src + 8);
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
            __syncthreads();
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int place = q0 + 64 * j + 16 * wave + (lane & 15);
                const int pg = place < p1 ? table[place] : -1;
                const bool is = pg >= 0 && pg < p.b.pages;
                const int8_t *src = p.bounds + ((int64_t)(is ? pg : 0) * p.b.Hkv + head) * (2 * D) + (2 * D / 4) * (lane >> 4);
                i32x4 acc = {0, 0, 0, 0};
#pragma unroll
                for (int k = 0; k < KS; ++k)
                    acc = __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, rows[k][lane]),
                                                                *reinterpret_cast<const i32x4 *>(src + 16 * k), acc, 0, 0, 0);
                if (round == 0) best[j] = acc;
                else
#pragma unroll
                    for (int e = 0; e < 4; ++e) best[j][e] = acc[e] > best[j][e] ? acc[e] : best[j][e];
            }
        }
        // lane: place lane % 16, rows 4 (lane / 16) + e
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int place = q0 + 64 * j + 16 * wave + (lane & 15);
            i32x4 x = best[j];
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
            if (place >= p1) continue;
            const int pg = table[place];
            const bool is = pg >= 0 && pg < p.b.pages;
            const float ks = is ? p.ks[(int64_t)pg * p.b.Hkv + head] : 0.0f;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int r = 4 * (lane >> 4) + e, tk = r >> hs;
                if ((r & ((1 << hs) - 1)) != 0 || tk >= t.n) continue;
                const int64_t row = (int64_t)(t.tok + tk) * p.b.Hkv + head;
                p.scores[row * p.b.width + place] = is ? sortable((float)x[e] * ks) : MISSING;
            }
        }
    }
}

// The `budget` largest of a row's scores, in order of their places.  A workgroup
// narrows down the smallest key that is taken by 8 bits a step (a histogram in LDS),
// then counts and writes, a wave a range of consecutive places.
__global__ __launch_bounds__(256) void select_top_kernel(SelectParams p)
{
    __shared__ uint32_t hist[256];
    __shared__ int found[2], counts[4][2];
    const int t = (int)blockIdx.x, head = (int)blockIdx.y, tid = (int)threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const TokenTile tt = token_tile(p.b, 1, t);
    if (tt.s < 0) return;
    const int many = places_of(p.b, tt.pos, tt.len);
    const int64_t row = (int64_t)tt.tok * p.b.Hkv + head;
    int *out = p.places + row * p.budget;
    if (many <= p.budget) {
        for (int i = tid; i < p.budget; i += 256) out[i] = i < many ? i : -1;
        return;
    }
    const uint32_t *scores = p.scores + row * p.b.width;
    auto key = [&](int i) { return i < p.first || i >= many - p.last ? FORCED : scores[i]; };
    uint32_t prefix = 0;
    int need = p.budget;   // of the keys with this prefix
    for (int shift = 24; shift >= 0; shift -= 8) {
        hist[tid] = 0;
        __syncthreads();
        const uint32_t mask = shift == 24 ? 0u : ~0u << (shift + 8);
        for (int i = tid; i < many; i += 256) {
            const uint32_t k = key(i);
            if ((k & mask) == prefix) atomicAdd(&hist[k >> shift & 255], 1u);
        }
        __syncthreads();
        if (wave == 0) {
            // lane l: the 4 digits from 252 - 4 l down in order of size
            uint32_t n[4], sum = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) sum += n[e] = hist[255 - 4 * lane - e];
            uint32_t upto = sum;
#pragma unroll
            for (int k = 1; k < 64; k <<= 1) {
                const uint32_t y = __shfl_up(upto, k, 64);
                upto += lane >= k ? y : 0;
            }
            uint32_t above = upto - sum;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                if (above < (uint32_t)need && (uint32_t)need <= above + n[e]) found[0] = 255 - 4 * lane - e, found[1] = (int)above;
                above += n[e];
            }
        }
        __syncthreads();
        prefix |= (uint32_t)found[0] << shift;
        need -= found[1];
    }
    // keys above `prefix` are taken, and the first `need` that equal it
    const int each = ((many + 3) / 4 + 63) & ~63, a = wave * each, e = a + each < many ? a + each : many;
    int above = 0, same = 0;
    for (int i = a + lane; i - lane < e; i += 64) {
        const uint32_t k = i < e ? key(i) : 0;
        above += __popcll(__ballot(i < e && k > prefix));
        same += __popcll(__ballot(i < e && k == prefix));
    }
    if (lane == 0) counts[wave][0] = above, counts[wave][1] = same;
    __syncthreads();
    int at = 0, equal = 0;
    for (int w = 0; w < wave; ++w) {
        const int left = need - equal > 0 ? need - equal : 0;
        at += counts[w][0] + (counts[w][1] < left ? counts[w][1] : left);
        equal += counts[w][1];
    }
    const uint64_t below = ((uint64_t)1 << lane) - 1;
    for (int i = a + lane; i - lane < e; i += 64) {
        const uint32_t k = i < e ? key(i) : 0;
        const uint64_t eq = __ballot(i < e && k == prefix);
        const bool take = i < e && (k > prefix || (k == prefix && equal + __popcll(eq & below) < need));
        const uint64_t got = __ballot(take);
        if (take) out[at + __popcll(got & below)] = i;
        at += __popcll(got);
        equal += __popcll(eq);
    }
}

} // namespace

hipError_t launch_kv_bounds(int D, const BoundsParams &params, hipStream_t s)
{
    BoundsParams p = params;
    const int64_t slots = (int64_t)(p.b.T >> p.b.page_shift) + 2 * (int64_t)p.b.S;   // (as for kv_append)
    p.by_token = p.b.T <= slots;
    const dim3 grid((unsigned)(p.by_token ? p.b.T : slots), (unsigned)p.b.Hkv);
    switch (D) {
    case 64: kv_bounds_kernel<64><<<grid, 256, 0, s>>>(p); break;
    case 128: kv_bounds_kernel<128><<<grid, 256, 0, s>>>(p); break;
    default: kv_bounds_kernel<256><<<grid, 256, 0, s>>>(p); break;
    }
    return hipGetLastError();
}

size_t select_workspace(int64_t T, int Hkv, int64_t width)
{
    return (size_t)T * Hkv * width * sizeof(uint32_t);
}

hipError_t launch_select(int D, SelectParams &p, void *ws, hipStream_t s)
{
    const int G = p.Hq / p.b.Hkv;
    p.scores = static_cast<uint32_t *>(ws);
    p.heads_shift = 0;
    while (1 << p.heads_shift < G && p.heads_shift < 4) ++p.heads_shift;
    const int per = 16 >> p.heads_shift;
    const int64_t tiles = per > 1 ? (int64_t)p.b.T / per + p.b.S : p.b.T;
    // chunks of 64 places at least, and enough of them to fill the device
    const int64_t most = (p.b.width + 63) / 64, want = (2048 + tiles * p.b.Hkv - 1) / (tiles * p.b.Hkv);
    const int64_t n = want < most ? want : most;
    if (p.b.width > p.budget) {
        p.chunk = (int)(((p.b.width + n - 1) / n + 63) / 64 * 64);
        const dim3 grid((unsigned)tiles, (unsigned)p.b.Hkv, (unsigned)((p.b.width + p.chunk - 1) / p.chunk));
        switch (D) {
        case 64: select_score_kernel<64><<<grid, 256, 0, s>>>(p); break;
        case 128: select_score_kernel<128><<<grid, 256, 0, s>>>(p); break;
        default: select_score_kernel<256><<<grid, 256, 0, s>>>(p); break;
        }
    }
    select_top_kernel<<<dim3((unsigned)p.b.T, (unsigned)p.b.Hkv), 256, 0, s>>>(p);
    return hipGetLastError();
}

} // namespace lamp
