// lamp_serve.hip -- what a server does to the projections' outputs before the
// attention: the RMS norm of every query and key head with the position
// rotation, and appending keys and values to the 8-bit paged cache.
//
// Norm and rotation of one row x in R^D (one head of one token):
//   y = x r w,  r = (mean x^2 + eps)^(-1/2),
//   y'_c = y_c cos_c - y_{c+h} sin_c,  y'_{c+h} = y_{c+h} cos_c + y_c sin_c,
//   c < h = rot/2, channels from rot on unchanged,
// in fp32 from the input to one final rounding (bf16 here, e4m3 in the cache).
// A row is held by D/16 lanes, each with the 8 channels from 8 j and their
// partners from h + 8 j (16 channels from 16 j behind the rotated ones): the
// rotation needs no other lane, and the loads and stores are 16 bytes.
#include <hip/hip_runtime.h>

#include "lamp_device.h"
#include "lamp_search.h"
#include "lamp_serve.h"

namespace lamp {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ void unpack8(const u32x4 &w, float *x)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = __builtin_bit_cast(float, w[i] << 16);
        x[2 * i + 1] = __builtin_bit_cast(float, w[i] & 0xFFFF0000u);
    }
}

// 8 elements at p (16-byte aligned) as fp32.
template <bool F32>
__device__ __forceinline__ void load8(const void *p, int64_t off, float *x)
{
    if constexpr (F32) {
        const f32x4 *s = reinterpret_cast<const f32x4 *>(static_cast<const float *>(p) + off);
        const f32x4 a = s[0], b = s[1];
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = a[i], x[4 + i] = b[i];
    } else {
        unpack8(*reinterpret_cast<const u32x4 *>(static_cast<const uint16_t *>(p) + off), x);
    }
}

__device__ __forceinline__ void load_gain8(const void *p, int off, int f32, float *x)
{
    if (f32) load8<true>(p, off, x);
    else load8<false>(p, off, x);
}

__device__ __forceinline__ u32x4 pack8(const float *x)
{
    u32x4 w;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        bf16x2 b;
        b[0] = (__bf16)x[2 * i];
        b[1] = (__bf16)x[2 * i + 1];
        w[i] = __builtin_bit_cast(uint32_t, b);
    }
    return w;
}

// Channels of lane j of a row: 8 from c0 and 8 from c1; partners of the
// rotation where rotated.
struct Lane {
    int c0, c1;
    bool rotated;
};

__device__ __forceinline__ Lane lane_of(int j, int rot)
{
    if (16 * j < rot) return {8 * j, rot / 2 + 8 * j, true};
    return {16 * j, 16 * j + 8, false};
}

template <int D>
__device__ __forceinline__ float row_sum(float v)
{
#pragma unroll
    for (int m = 1; m < D / 16; m <<= 1) v += __shfl_xor(v, m, 64);
    return v;
}

// Norm (wa null: none) and rotation of the lane's 16 channels a, b.
template <int D>
__device__ __forceinline__ void norm_rotate(float *a, float *b, bool normed, const float *wa, const float *wb, float eps,
                                            bool rotated, const float *cs, const float *sn)
{
    if (normed) {
        float ss = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) ss = __builtin_fmaf(a[i], a[i], __builtin_fmaf(b[i], b[i], ss));
        const float r = 1.0f / __builtin_sqrtf(row_sum<D>(ss) * (1.0f / D) + eps);
#pragma unroll
        for (int i = 0; i < 8; ++i) a[i] = a[i] * r * wa[i], b[i] = b[i] * r * wb[i];
    }
    if (rotated) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float x = a[i], y = b[i];
            a[i] = x * cs[i] - y * sn[i];
            b[i] = y * cs[i] + x * sn[i];
        }
    }
}

// Bound by HBM (each element read and written once); a wave takes whole rows
// of one token, 1024/D at a time, so the token's cos and sin and the gains are
// loaded once and stay in registers over its heads.  4 x 8192 tokens of 32/8
// heads, d = 128: 809 MB in 189 us in a trace, 4.3 TB/s (180 a call back to back;
// a large copy: 5.1), of fp32 1212 MB in 231, 5.2 TB/s; 1999 tokens 14 us; one
// token 4 us, a launch's latency.
template <int D, bool F32>
__global__ __launch_bounds__(256) void norm_rope_kernel(NormRopeParams p)
{
    constexpr int LPR = D / 16, RPW = 64 / LPR;
    const int lane = threadIdx.x & 63, row = lane / LPR;
    const Lane ch = lane_of(lane % LPR, p.rope ? p.rot : 0);
    const int64_t wave = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int64_t token = wave / p.slices;
    if (token >= (int64_t)p.B * p.N) return;
    const int slice = (int)(wave - token * p.slices);
    const int64_t b = token / p.N, n = token - b * p.N;
    float cs[8], sn[8], w[2][16];
    bool lost = false;   // a position outside the table: NaN rows, nothing read
    if (p.rope && ch.rotated) {
        const int64_t pos = p.positions ? p.positions[token] : n;
        lost = pos < 0 || pos >= p.npos;
        const float *t = p.rope + (lost ? 0 : pos) * p.rot + ch.c0;
        load8<true>(t, 0, cs);
        load8<true>(t, p.rot / 2, sn);
        if (lost) {
#pragma unroll
            for (int i = 0; i < 8; ++i) cs[i] = __builtin_nanf("");
        }
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        if (p.w[i]) {
            load_gain8(p.w[i], ch.c0, p.w_f32[i], w[i]);
            load_gain8(p.w[i], ch.c1, p.w_f32[i], w[i] + 8);
        }
    }
    const int h01 = p.H[0] + p.H[1], heads = h01 + p.H[2];
    for (int h0 = slice * RPW; h0 < heads; h0 += p.slices * RPW) {
        const int hh = h0 + row;
        const bool on = hh < heads;
        const int which = hh < p.H[0] ? 0 : (hh < h01 ? 1 : 2);
        const int h = which == 0 ? hh : (which == 1 ? hh - p.H[0] : hh - h01);
        float x[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i] = 0.0f;
        if (on) {
            const RowsIn &r = p.in[which];
            const int64_t off = b * r.sb + n * r.st + h * r.sh;
            load8<F32>(r.p, off + ch.c0, x);
            load8<F32>(r.p, off + ch.c1, x + 8);
        }
        // (the sum over a row's lanes is taken by whole rows: all lanes of a row share `which`)
        if (which < 2) {
            float g[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) g[i] = which == 0 ? w[0][i] : w[1][i];
            norm_rotate<D>(x, x + 8, (which == 0 ? p.w[0] : p.w[1]) != nullptr, g, g + 8, p.eps, p.rope && ch.rotated, cs, sn);
        }
        if (on) {
            const RowsOut &r = p.out[which];
            const int64_t off = b * r.sb + n * r.st + h * r.sh;
            *reinterpret_cast<u32x4 *>(r.p + off + ch.c0) = pack8(x);
            *reinterpret_cast<u32x4 *>(r.p + off + ch.c1) = pack8(x + 8);
        }
    }
}

// --- the 8-bit paged cache ----------------------------------------------------

// Smallest e with amax <= 448 * 2^e (448 = 1.75 * 2^8), at least -100, as the
// power of two 2^e; amax is finite and >= 0.
__device__ __forceinline__ float scale_for(float amax)
{
    const int e = (int)((__builtin_bit_cast(uint32_t, amax) + 0x1FFFFFu) >> 23) - 127 - 8;
    return __builtin_bit_cast(float, (uint32_t)((e < -100 ? -100 : e) + 127) << 23);
}

// 1/s of a power of two 2^e, -100 <= e <= 120.
__device__ __forceinline__ float inv_pow2(float s)
{
    return __builtin_bit_cast(float, (254u << 23) - __builtin_bit_cast(uint32_t, s));
}

__device__ __forceinline__ bool finite(float x)
{
    return (__builtin_bit_cast(uint32_t, x) & 0x7F800000u) != 0x7F800000u;
}

// 4 values times `inv` as e4m3 codes (to nearest even; |x inv| <= 448), what
// is not finite as the NaN code.
__device__ __forceinline__ uint32_t encode4(const float *x, float inv)
{
    float y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = finite(x[i]) ? x[i] * inv : __builtin_nanf("");
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false), true);
}

// 4 codes under a scale grown by 1/ratio (a power of two): exact but for
// values that become subnormal, which round to nearest even.
__device__ __forceinline__ uint32_t rescale4(uint32_t c, float ratio)
{
    const float x[4] = {__builtin_amdgcn_cvt_f32_fp8((int)c, 0), __builtin_amdgcn_cvt_f32_fp8((int)c, 1),
                        __builtin_amdgcn_cvt_f32_fp8((int)c, 2), __builtin_amdgcn_cvt_f32_fp8((int)c, 3)};
    return encode4(x, ratio);
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

// Byte c of four words (4 codes of consecutive channels of 4 tokens) as the
// words of 4 tokens of each channel.
__device__ __forceinline__ void transpose4(uint32_t *w)
{
    const uint32_t a = __builtin_amdgcn_perm(w[1], w[0], 0x05010400u), b = __builtin_amdgcn_perm(w[1], w[0], 0x07030602u);
    const uint32_t c = __builtin_amdgcn_perm(w[3], w[2], 0x05010400u), d = __builtin_amdgcn_perm(w[3], w[2], 0x07030602u);
    w[0] = __builtin_amdgcn_perm(c, a, 0x05040100u);
    w[1] = __builtin_amdgcn_perm(c, a, 0x07060302u);
    w[2] = __builtin_amdgcn_perm(d, b, 0x05040100u);
    w[3] = __builtin_amdgcn_perm(d, b, 0x07060302u);
}

// One workgroup writes the new keys (blockIdx.z 0) or values (1) of one page
// and head: their largest magnitude, the page's scale (a power of two, so that
// growing it keeps the codes already there), then the codes.  The finished
// numbers stay in registers between the two (those of 64 tokens; longer pages
// read the rest again).  Values go through an LDS tile row by row and come out
// as 16 tokens of 4 channels a thread, transposed by byte permutes.  Bound by
// HBM for prompts (32K tokens of 8 heads, d = 128: 218 MB in 59 us, 3.7 TB/s, with
// the rotation's table read from the L2 once a head; keeping cos and sin over 4
// heads instead doubles the registers and takes 78), by the latencies of starts,
// lengths, table and rows for single tokens (32: 5 us).  Short pages leave lanes
// idle (16 tokens of d = 64 are 64 of the 256 threads' rows) and look up as much a
// page as long ones (13 MB of fp32 tokens into pages of 16: 9.6 us).
constexpr int VT = 64;       // slots of the transposing tile

// LONG: pages of more than 64 tokens.
template <int D, bool F32, bool LONG>
__global__ __launch_bounds__(256) void kv_append_kernel(AppendParams p)
{
    constexpr int LPR = D / 16, RPB = 256 / LPR;   // rows of one pass
    constexpr int KEEP = D / 64;                   // rows of a thread in a page of 64
    constexpr int STRIDE = D + 16;                 // bytes of a row of the tile
    __shared__ float red[4];
    __shared__ u32x4 tile[VT * STRIDE / 16];
    const PageWork w = page_work(p.b, p.by_token, (int)blockIdx.x);
    if (w.count == 0) return;   // (the whole workgroup)
    const int tid = (int)threadIdx.x, head = (int)blockIdx.y, page = 1 << p.b.page_shift;
    const bool is_v = blockIdx.z != 0;
    const Lane ch = lane_of(tid % LPR, !is_v && p.rope ? p.rot : 0);
    float wa[8], wb[8];
    const bool normed = !is_v && p.w;
    if (normed) {
        load_gain8(p.w, ch.c0, p.w_f32, wa);
        load_gain8(p.w, ch.c1, p.w_f32, wb);
    }
    const void *src = is_v ? p.v : p.k;
    const int64_t st = is_v ? p.v_st : p.k_st, base = head * (is_v ? p.v_sh : p.k_sh);
    // row i of the page's new tokens, finished in fp32 (i < count)
    auto row = [&](int i, float *x) {
        const int64_t off = base + (int64_t)(w.tok + i) * st;
        load8<F32>(src, off + ch.c0, x);
        load8<F32>(src, off + ch.c1, x + 8);
        float cs[8], sn[8];
        if (ch.rotated) {
            const int pos = w.pos + i;
            const bool lost = pos >= p.npos;
            const float *t = p.rope + (int64_t)(lost ? 0 : pos) * p.rot + ch.c0;
            load8<true>(t, 0, cs);
            load8<true>(t, p.rot / 2, sn);
            if (lost) {
#pragma unroll
                for (int c = 0; c < 8; ++c) cs[c] = __builtin_nanf("");
            }
        }
        norm_rotate<D>(x, x + 8, normed, wa, wb, p.eps, ch.rotated, cs, sn);
    };
    float m = 0.0f, kept[KEEP][16];
    auto widest = [&](const float *x) {
#pragma unroll
        for (int c = 0; c < 16; ++c) m = finite(x[c]) ? fmaxf(m, fabsf(x[c])) : m;
    };
    const int i0 = tid / LPR;
#pragma unroll
    for (int k = 0; k < KEEP; ++k)
        if (i0 + k * RPB < w.count) row(i0 + k * RPB, kept[k]);
#pragma unroll
    for (int k = 0; k < KEEP; ++k)
        if (i0 + k * RPB < w.count) widest(kept[k]);
    for (int i = i0 + KEEP * RPB; LONG && i < w.count; i += RPB) {
        float x[16];
        row(i, x);
        widest(x);
    }
#pragma unroll
    for (int k = 1; k < 64; k <<= 1) m = fmaxf(m, __shfl_xor(m, k, 64));
    if ((tid & 63) == 0) red[tid >> 6] = m;
    float *scale = (is_v ? p.vs : p.ks) + w.page * p.b.Hkv + head;
    uint8_t *codes = (is_v ? p.vc : p.kc) + (w.page * p.b.Hkv + head) * (int64_t)page * D;
    const float old = w.first > 0 ? *scale : 0.0f;
    __syncthreads();   // (and every thread has the old scale)
    m = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
    const float need = scale_for(m), now = w.first > 0 && old > need ? old : need, inv = inv_pow2(now);
    if (w.first > 0 && old < now) {
        // the codes of the slots before, under the new scale (in 16-byte units)
        const float ratio = old * inv;
        if (!is_v) {
            u32x4 *c = reinterpret_cast<u32x4 *>(codes);
            for (int u = tid; u < w.first * (D / 16); u += 256) {
                u32x4 x = c[u];
#pragma unroll
                for (int k = 0; k < 4; ++k) x[k] = rescale4(x[k], ratio);
                c[u] = x;
            }
        } else {
            const int units = (w.first + 15) / 16;
            for (int u = tid; u < D * units; u += 256) {
                const int d = u / units, s0 = (u - d * units) * 16;
                u32x4 *c = reinterpret_cast<u32x4 *>(codes + d * page + s0);
                u32x4 x = *c;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int n = w.first - (s0 + 4 * k);   // slots of this word before the first new one
                    const uint32_t keep = n >= 4 ? 0u : (n <= 0 ? ~0u : ~0u << (8 * n));
                    x[k] = (x[k] & keep) | (rescale4(x[k], ratio) & ~keep);
                }
                *c = x;
            }
        }
    }
    if (tid == 0) *scale = now;
    // the codes of row i: to the cache (keys) or to the tile of slots from t0 (values)
    auto write = [&](int i, const float *x, int t0) {
        uint8_t *c = is_v ? reinterpret_cast<uint8_t *>(tile) + (w.first + i - t0) * STRIDE : codes + (int64_t)(w.first + i) * D;
        *reinterpret_cast<u32x2 *>(c + ch.c0) = u32x2{encode4(x, inv), encode4(x + 4, inv)};
        *reinterpret_cast<u32x2 *>(c + ch.c1) = u32x2{encode4(x + 8, inv), encode4(x + 12, inv)};
    };
    // rows [a, e)
    auto write_rows = [&](int a, int e, int t0) {
#pragma unroll
        for (int k = 0; k < KEEP; ++k)
            if (i0 + k * RPB >= a && i0 + k * RPB < e) write(i0 + k * RPB, kept[k], t0);
        for (int i = i0 + KEEP * RPB; LONG && i < e; i += RPB) {
            if (i < a) continue;
            float x[16];
            row(i, x);
            write(i, x, t0);
        }
    };
    if (!is_v) {
        write_rows(0, w.count, 0);
        return;
    }
    const int last = w.first + w.count;
    for (int t0 = w.first / VT * VT; t0 < last; t0 += VT) {
        const int a = w.first > t0 ? w.first : t0, e = last - t0 < VT ? last : t0 + VT;   // slots of this tile
        __syncthreads();   // the tile is free (and the rescaled codes are written)
        write_rows(a - w.first, e - w.first, t0);
        __syncthreads();
        const int u0 = (a - t0) / 16, un = (e - t0 + 15) / 16 - u0;   // units of 16 slots
        for (int u = tid; u < D / 4 * un; u += 256) {
            const int c4 = u % (D / 4), s0 = (u0 + u / (D / 4)) * 16;
            if (t0 + s0 >= a && t0 + s0 + 16 <= e) {
                uint32_t x[4][4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) x[i][j] = reinterpret_cast<const uint32_t *>(tile)[(s0 + 4 * i + j) * (STRIDE / 4) + c4];
                    transpose4(x[i]);
                }
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    *reinterpret_cast<u32x4 *>(codes + (int64_t)(4 * c4 + j) * page + t0 + s0) = u32x4{x[0][j], x[1][j], x[2][j], x[3][j]};
            } else {   // a unit that holds other slots too
                for (int s = t0 + s0 > a ? t0 + s0 : a; s < t0 + s0 + 16 && s < e; ++s) {
                    const uint32_t x = reinterpret_cast<const uint32_t *>(tile)[(s - t0) * (STRIDE / 4) + c4];
#pragma unroll
                    for (int j = 0; j < 4; ++j) codes[(int64_t)(4 * c4 + j) * page + s] = (uint8_t)(x >> (8 * j));
                }
            }
        }
    }
}

} // namespace

hipError_t launch_norm_rope(int D, bool f32, const NormRopeParams &params, hipStream_t s)
{
    NormRopeParams p = params;
    // few tokens: their heads are spread over waves until these fill the
    // device (16 a CU); many: one wave a token, whose cos, sin and gains it
    // loads once
    const int64_t tokens = (int64_t)p.B * p.N, steps = ((int64_t)(p.H[0] + p.H[1] + p.H[2]) * D + 1023) / 1024;
    const int64_t want = (4096 + tokens - 1) / tokens;
    p.slices = (int)(want < steps ? want : steps);
    const int64_t waves = tokens * p.slices;
    const dim3 grid((unsigned)((waves + 3) / 4));
    switch (D) {
    case 64: f32 ? norm_rope_kernel<64, true><<<grid, 256, 0, s>>>(p) : norm_rope_kernel<64, false><<<grid, 256, 0, s>>>(p); break;
    case 128: f32 ? norm_rope_kernel<128, true><<<grid, 256, 0, s>>>(p) : norm_rope_kernel<128, false><<<grid, 256, 0, s>>>(p); break;
    default: f32 ? norm_rope_kernel<256, true><<<grid, 256, 0, s>>>(p) : norm_rope_kernel<256, false><<<grid, 256, 0, s>>>(p); break;
    }
    return hipGetLastError();
}

template <int D>
static hipError_t launch_append(bool f32, const AppendParams &p, dim3 grid, hipStream_t s)
{
    if (1 << p.b.page_shift <= 64) {
        f32 ? kv_append_kernel<D, true, false><<<grid, 256, 0, s>>>(p) : kv_append_kernel<D, false, false><<<grid, 256, 0, s>>>(p);
    } else {
        f32 ? kv_append_kernel<D, true, true><<<grid, 256, 0, s>>>(p) : kv_append_kernel<D, false, true><<<grid, 256, 0, s>>>(p);
    }
    return hipGetLastError();
}

hipError_t launch_kv_append(int D, bool f32, const AppendParams &params, hipStream_t s)
{
    AppendParams p = params;
    // the smaller grid of the two
    const int64_t slots = (int64_t)(p.b.T >> p.b.page_shift) + 2 * (int64_t)p.b.S;
    p.by_token = p.b.T <= slots;
    const dim3 grid((unsigned)(p.by_token ? p.b.T : slots), (unsigned)p.b.Hkv, 2);
    switch (D) {
    case 64: return launch_append<64>(f32, p, grid, s);
    case 128: return launch_append<128>(f32, p, grid, s);
    default: return launch_append<256>(f32, p, grid, s);
    }
}

} // namespace lamp
