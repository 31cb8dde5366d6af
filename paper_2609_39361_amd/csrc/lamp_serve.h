// lamp_serve.h -- parameter blocks and launchers of the serving operators
// (library-internal; lamp_serve.hip, lamp_cache_attn.hip, lamp_host.cpp):
// norms with the position rotation, appending to the 8-bit paged cache, and
// the attention over it.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace lamp {

// Rows of D channels addressed by (batch, token, head): element strides.
struct RowsIn {
    const void *p;            // bf16 or fp32 elements, or null
    int64_t sb, st, sh;
};

struct RowsOut {
    uint16_t *p;              // bf16, or null
    int64_t sb, st, sh;
};

struct NormRopeParams {
    RowsIn in[3];             // q, k, v (v copied)
    RowsOut out[3];
    const void *w[2];         // gains of q and k [D], or null (not normed)
    const float *rope;        // [npos][rot] cos | sin, or null (not rotated)
    const int *positions;     // [B][N], or null (the token index)
    int H[3];                 // heads of q, k, v (0: absent)
    int B, N, npos, rot;
    int w_f32[2];             // gains in fp32 (otherwise bf16)
    float eps;
    int slices;               // waves a token's heads are spread over (set by the launcher)
};

// f32: the input elements are fp32 (otherwise bf16).
hipError_t launch_norm_rope(int D, bool f32, const NormRopeParams &p, hipStream_t s);

// A batch of sequences over a paged cache.  kv_lens[s] counts the new tokens
// [q_start[s], q_start[s+1]) (null q_start: token s alone); token i of n is at
// position kv_lens[s] - n + i.
struct PagedBatch {
    const int *table;         // [S][width] page of each `1 << page_shift` tokens
    const int *kv_lens;       // [S]
    const int *q_start;       // [S+1] or null
    int64_t table_stride;     // elements from one sequence's entries to the next's
    int S, T, width, pages, page_shift, Hkv;
};

struct AppendParams {
    PagedBatch b;
    const void *k, *v;        // [T][Hkv][D], bf16 or fp32
    int64_t k_st, k_sh, v_st, v_sh;
    uint8_t *kc, *vc;         // codes [pages][Hkv][page][D] and [pages][Hkv][D][page]
    float *ks, *vs;           // scales [pages][Hkv]
    const void *w;            // gain of the keys [D], or null
    const float *rope;        // [npos][rot], or null
    int npos, rot, w_f32;
    float eps;
    // (set by the launcher) a workgroup for every token (the first new one of its
    // page does the work), not for every page that could receive tokens
    int by_token;
};

hipError_t launch_kv_append(int D, bool f32, const AppendParams &p, hipStream_t s);

struct CacheAttnParams {
    PagedBatch b;
    const uint16_t *q;        // [T][Hq][D] bf16
    int64_t q_st, q_sh;
    const uint8_t *kc, *vc;
    const float *ks, *vs;
    uint16_t *o;              // [T][Hq][D] bf16
    float *lse;               // [T][Hq]
    int Hq, causal, window;
    float scale_log2;         // logit scale times log2(e)
    // By form of the kernel (lamp_cache_plan.h; 0: few rows a sequence, 1: many).
    int rows_above[2], rows_upto[2];   // it takes the sequences with this many rows (new tokens times heads of a group)
    int units[2];             // workgroups: no lengths give more
    int slots[2];             // partial outputs of split row tiles that the workspace holds: likewise
    int apart;                // both forms, in launches of their own
    int *counts;              // those that this call has (workspace)
    void *split;              // the plan of more than PLAN_ALONE sequences: Split of each form (workspace)
    void *before[2];          // and [S] Before (workspace)
    void *info[2];            // [slots] PartInfo (workspace)
    float *part[2];           // [slots][rows of a tile][D] (workspace)
    float *part_ml[2];        // their running maxima and sums [slots][rows of a tile][2] (workspace)
};

// Bytes of workspace a call over sequences of at most `keys` keys needs.
size_t cache_attn_workspace(int D, int64_t T, int64_t S, int G, int Hkv, int64_t keys);
// ws: that workspace (null where it needs none).  Fills in p from units on.
hipError_t launch_cache_attn(int D, CacheAttnParams &p, void *ws, hipStream_t s);
// The kernel with the form for many rows (lamp_cache_prompt.hip), and, where
// p.units[0] > 0 and not p.apart, that for few beside it; of launch_cache_attn.
hipError_t launch_cache_prompt(int D, const CacheAttnParams &p, hipStream_t s);

} // namespace lamp
