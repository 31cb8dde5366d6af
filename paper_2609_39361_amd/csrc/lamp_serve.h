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
    // By form of the kernel (lamp_cache_plan.h; 0: few rows a sequence, 1: many, 2: a
    // group over its prefix, of attn_shared alone).
    int rows_above[3], rows_upto[3];   // it takes the sequences with this many rows (new tokens times heads of a group)
    int units[3];             // workgroups: no lengths give more
    int slots[3];             // partial outputs of split row tiles that the workspace holds: likewise
    int apart;                // both forms, in launches of their own
    int *counts;              // those that this call has (workspace)
    void *split;              // the plan of more than PLAN_ALONE sequences: Split of each form (workspace)
    void *before[3];          // and [S] Before (workspace)
    void *info[2];            // [slots] PartInfo (workspace)
    float *part[3];           // [slots][rows of a tile][D] (workspace)
    float *part_ml[3];        // their running maxima and sums [slots][rows of a tile][2] (workspace)
};

// Groups of sequences with a shared prefix (lamp_cache_shared.hip): causal, no window.
struct SharedAttnParams : CacheAttnParams {
    const int *prefix_lens;   // [S]
    const int *group_start;   // [groups + 1], of sequences
    int groups;
    int group_above[3], group_upto[3];   // as rows_above, rows_upto, of the groups
    void *rows;               // RowInfo [2][T][Hq] (workspace)
    void *unit_seq[3];        // the group or sequence of each unit, of more than SHARED_ALONE (workspace)
};

// Attention over the pages of each token's and kv head's list (lamp_cache_pages.hip):
// causal, no window.
struct PagesAttnParams : CacheAttnParams {
    const int *places;        // [T][Hkv][budget] of the sequence's table row
    int budget;
    int pieces, per;          // a list's parts, of `per` entries (set by the launcher)
};

// Bytes of workspace a call over sequences of at most `keys` keys needs.
size_t cache_attn_workspace(int D, int64_t T, int64_t S, int G, int Hkv, int64_t keys);
// ws: that workspace (null where it needs none).  Fills in p from units on.
hipError_t launch_cache_attn(int D, CacheAttnParams &p, void *ws, hipStream_t s);
size_t shared_attn_workspace(int D, int64_t T, int64_t S, int64_t groups, int G, int Hkv, int64_t keys);
hipError_t launch_shared_attn(int D, SharedAttnParams &p, void *ws, hipStream_t s);
size_t pages_attn_workspace(int D, int64_t T, int G, int Hkv, int64_t page, int64_t budget);
hipError_t launch_pages_attn(int D, PagesAttnParams &p, void *ws, hipStream_t s);
// The kernel with the form for many rows (lamp_cache_prompt.hip), and, where
// p.units[0] > 0 and not p.apart, that for few beside it; of launch_cache_attn.
hipError_t launch_cache_prompt(int D, const CacheAttnParams &p, hipStream_t s);

// The range of each channel over a page's keys (lamp_pages.hip).
struct BoundsParams {
    PagedBatch b;
    const uint8_t *kc;        // codes [pages][Hkv][page][D]
    int8_t *bounds;           // [pages][Hkv][2][D]
    int by_token;             // (set by the launcher)
};

hipError_t launch_kv_bounds(int D, const BoundsParams &p, hipStream_t s);

struct SelectParams {
    PagedBatch b;
    const uint16_t *q;        // [T][Hq][D] bf16
    int64_t q_st, q_sh;
    const int8_t *bounds;     // [pages][Hkv][2][D]
    const float *ks;          // [pages][Hkv]
    int *places;              // [T][Hkv][budget]
    int Hq, budget, first, last;
    uint32_t *scores;         // [T][Hkv][width] (workspace)
    // (set by the launcher) log2 of the heads of a group, rounded up, 16 at most; tokens
    // of a tile; places of a workgroup
    int heads_shift, tokens, chunk;
};

size_t select_workspace(int D, int64_t T, int64_t S, int G, int Hkv, int64_t width, int64_t budget);
hipError_t launch_select(int D, SelectParams &p, void *ws, hipStream_t s);

// A step of a batch (lamp_advance.hip).
struct AdvanceParams {
    const int *lens, *add, *prefix_lens;   // [S]; prefix_lens may be null
    int *table;
    int64_t table_stride;
    int *ring;                             // [pages]
    const int *state;                      // [4]: first free entry, free entries, -, -
    int *kv_lens, *q_start, *positions, *state_out;   // [S], [S + 1], [T], [4]
    int S, T, width, pages, page_shift;
};

hipError_t launch_advance(const AdvanceParams &p, hipStream_t s);

} // namespace lamp
