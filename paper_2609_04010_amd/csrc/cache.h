// The 8-bit cache of keys and values: its layout, the e4m3 conversions and the argument blocks of its
// kernels.
#pragma once

#include "kernels.h"

namespace dd {

struct CacheShape {
    int32_t n_blocks, P, H;   // blocks, tokens per block, key / value heads
    int32_t log2p;
};
inline CacheShape cache_shape(const dd_cache* c) {
    int l = 0;
    while ((1 << l) < c->block) ++l;
    return {c->n_blocks, c->block, c->n_kv_heads, l};
}

constexpr int CACHE_EMIN = -100, CACHE_EMAX = 120;   // scales are 2^e within these

// four fp32 numbers as e4m3 codes, nearest even; |x| <= 464 or not finite (which gives a NaN code)
DD_DEV uint32_t enc_fp8x4(float a, float b, float c, float d) {
    const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, lo, true);
}

// 2^e from its bits, -126 <= e <= 127
DD_DEV float pow2i(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }

// bytes of one block and head, and where the values start in it
DD_DEV int64_t cache_slab(const CacheShape& c, int dh, int64_t block, int h) {
    return (block * c.H + h) * (2 * (int64_t)c.P * dh);
}

struct PlanArgs {
    CacheShape c;
    int32_t S, T, ld_table;
    int32_t *table, *held_out, *kv_len, *row_start, *row_seq, *row_pos, *slots;
    const int32_t *seq_len, *n_new, *held;
    int32_t* free_blocks;
    const int32_t* n_free;
    int32_t* n_free_out;
    int32_t* err;
};
dd_status launch_cache_plan(const PlanArgs& a, hipStream_t s);

struct AppendArgs {
    CacheShape c;
    int32_t dh, S, T;
    uint8_t* codes;
    float* scales;
    const int32_t *kv_len, *row_start, *row_seq, *slots;
    const void *k, *v;
    int64_t ld;
    int32_t* err;
    bool by_row;   // set by launch_cache_append, from its grid
};
// How a call is cut: a unit of work per row or per touched block, and whether its keys or values have a workgroup of their own.
struct AppendGrid {
    bool by_row, wide;
    int64_t wgs;
};
AppendGrid cache_append_grid(int32_t S, int32_t T, int32_t P, int32_t H);
dd_status launch_cache_append(int dtype, const AppendArgs& a, hipStream_t s);

struct CacheAttnArgs {
    CacheShape c;
    int32_t dh, S, T, ld_table;
    const uint8_t* codes;
    const float* scales;
    const int32_t *table, *kv_len, *row_start;
    const void* q;
    int64_t ldq;
    void* out;
    int64_t ldo;
    int32_t Hq, G;        // query heads, query heads per key head
    int32_t causal;
    float scale_log2;     // softmax_scale log2(e)
    int32_t max_new, max_kv;
    int32_t chunk, nsplit;   // tokens per workgroup (a multiple of 32) and how many such pieces max_kv has
    float* part;          // nsplit > 1: [T][Hq][nsplit][dh] sums, then [T][Hq][nsplit][2] (maximum, sum)
    int32_t* err;
};
// How a call is cut: shape of a workgroup (an index into the launcher's table), column tiles of a key head,
// tokens per workgroup and how many such pieces max_kv has, bytes of partial results.
struct CacheAttnPlan {
    int shape, chunk, nsplit;
    int threads;   // of a workgroup
    int64_t tiles;
    size_t ws;
};
CacheAttnPlan cache_attn_plan(int32_t S, int32_t T, int32_t Hkv, int32_t Hq, int dh, int32_t max_new, int32_t max_kv);
dd_status launch_cache_attn(int dtype, const CacheAttnArgs& a, const CacheAttnPlan& p, hipStream_t s);

// Ranges of blocks that a fork or a compaction cuts the pool into (n_blocks is below 2^26), and parts of the sequences: as
// many as give every CU something to do.
constexpr int PAGE_RANGE = 8192, PAGE_RANGES = (1 << 26) / PAGE_RANGE;
inline int page_parts(int ranges) { return ranges >= 256 ? 1 : 256 / ranges < 32 ? 256 / ranges : 32; }

struct ForkArgs {
    CacheShape c;
    int32_t S, S_to, ld_table, ld_to;
    const int32_t *table, *held, *seq_len, *src, *keep;
    int32_t *to_table, *to_held, *to_len;
    int32_t* free_blocks;
    const int32_t* n_free;
    int32_t *n_free_out, *moves, *n_moves;
    // workspace: bits per block and part, held by old sequences and whole by new ones; a bit per block that is freed, their
    // number in each range; whether a sequence takes a fresh block; whether an input of a part is no fork's
    uint32_t *old, *whole, *freed;
    int32_t *counts, *copies, *bad;
    int32_t ranges;
    int32_t* err;
    int32_t parts;       // set by launch_cache_fork
};
dd_status launch_cache_fork(const ForkArgs& a, hipStream_t s);

struct CompactArgs {
    CacheShape c;
    int32_t S, ld_table;
    const int32_t *table, *held;
    int32_t *to_table, *free_blocks, *n_free_out, *moves, *n_moves;
    // workspace: a bit per block in use and part, later in all; those of the range before each word of them; those of each
    // range; whether an input of a part is no table
    uint32_t* used;
    int32_t *before, *counts, *bad;
    int32_t ranges;
    int32_t* err;
    int32_t parts;       // set by launch_cache_compact
};
dd_status launch_cache_compact(const CompactArgs& a, hipStream_t s);

struct CopyArgs {
    int32_t n_blocks, heads, layers, max_moves;
    int64_t slab;        // bytes of a block's codes
    uint8_t* codes;
    float* scales;
    const int32_t *moves, *n_moves;
    int32_t* err;
};
dd_status launch_cache_copy(const CopyArgs& a, hipStream_t s);

struct EditArgs {
    const void* logits;
    void* out;
    int64_t ld;
    int32_t rows, V, per;
    dd_logits_edits e;
    int rows_per_wg;   // set by launch_edit
    int32_t* err;
};
dd_status launch_edit(const EditArgs& a, int dtype, hipStream_t s);

}  // namespace dd
