// Internal declarations of the paged-cache operators (rotary positions,
// append, attention): what the host side hands to the kernels.
#pragma once

#include "upr_internal.h"

namespace upr {

// Users of one launch.  They travel as kernel arguments: the host has
// validated their lengths, and a block finds its user with one load and no
// dependence on another launch.  Calls with more users take several launches.
constexpr int kPagedUsers = 128;

struct PagedUsers {
    int32_t n;
    int32_t user[kPagedUsers];          // row of the page table
    int32_t row0[kPagedUsers];          // first row of q / k / v
    int32_t count[kPagedUsers];         // new rows
    int32_t rows[kPagedUsers];          // cached rows when the call ends
    int32_t item0[kPagedUsers + 1];     // first work item; [n]: all items
};

// One plane of a pool: page p's K block at data + p * page_elems, its V block
// half a page further.
struct PagedPool {
    char* data;
    const int32_t* tables;
    int64_t n_pages;
    int32_t stride, page_rows, page_shift;
};

// Rotation as the kernels take it: quarter turns per position.
struct RopeArgs {
    int32_t rot_dim;        // 0: none
    int32_t layout;
    float magnitude;
    double quarters[UPR_ROPE_MAX_PAIRS];
};

// Rows of one tensor: base, elements between rows.
struct RowsOf {
    const void* p;
    int64_t ld;
};

// Rotation of x's rows at positions[r].
hipError_t launch_rope(int dtype, const RopeArgs& rope, int heads, int D, RowsOf x, const int32_t* positions,
                       int64_t rows, void* out, int64_t out_ld, hipStream_t s);

// Append of one launch's users: k and v (null p: none) into the pool, q (null:
// none) to q_out.  `fixed`: every row of a user stands at position rows[u]
// (ranking candidates) instead of at the end of its cache.
struct AppendArgs {
    int n_heads, n_kv_heads, D;
    int fixed;
    RowsOf k, v, q;
    void* q_out;
    int64_t q_out_ld;
};
// Heads per thread for a call of `rows` rows, and the rows of a work item.
int append_batch(int dtype, const RopeArgs& rope, const AppendArgs& a, int64_t rows);
int append_rows(int dtype, const RopeArgs& rope, const AppendArgs& a, int batch);
hipError_t launch_append(int dtype, const RopeArgs& rope, const AppendArgs& a, int batch, const PagedPool& pool,
                         const PagedUsers& users, hipStream_t s);

// First key that a row at position pos sees, rounded down to a block of keys.
__host__ __device__ __forceinline__ int attn_first_key(int pos, int window) {
    return window > 0 && pos - window + 1 > 0 ? (pos - window + 1) & ~31 : 0;
}

// Parts that a user's keys are cut into (chunk 0: none are).
__host__ __device__ __forceinline__ int attn_splits(int rows, int count, bool own, int window, int chunk) {
    if (chunk == 0) return 1;
    const int keys = rows - attn_first_key(own ? rows : rows - count, window);
    return keys > chunk ? (keys + chunk - 1) / chunk : 1;
}

// Attention of one launch's users.  Scores in log2 units: z2 = c (q.k) with c
// = scale log2(e), or with a cap cap2 tanh(q.k scale / cap), cap2 = cap log2(e)
// and ct2 = 2 log2(e) scale / cap; slopes are multiplied by log2(e) in the
// kernel.
enum AttnOut : int { ATTN_OUT_STORAGE = 0, ATTN_OUT_F16 = 1, ATTN_OUT_F32 = 2 };
struct AttnArgs {
    int n_heads, n_kv_heads, D;
    RowsOf q, k_self, v_self;       // k_self.p null: causal
    void* out;
    int64_t out_ld;
    int out_kind;                   // AttnOut: the cache's type, or what bf16 models' projections take
    float c, ct2, cap2;             // cap2 0: none
    const float* slopes;
    int32_t window;                 // 0: none
    // the plan: rows per tile, keys per part (0: all), and with parts their
    // records, `tile` per work item: [D] sums, and reference and weight sum
    int32_t tile, chunk;
    float* part_o;
    float* part_ml;
};
hipError_t launch_paged_attn(int dtype, const AttnArgs& a, const PagedPool& pool, const PagedUsers& users,
                             hipStream_t s);

// Join of a launch's parts.  users: those of the attention's launch with parts,
// items of kJoinRows rows of one key/value head; part0: their first item there.
constexpr int kJoinRows = 4;
struct JoinUsers {
    PagedUsers users;
    int32_t part0[kPagedUsers];
};
hipError_t launch_paged_join(int dtype, const AttnArgs& a, const PagedPool& pool, const JoinUsers& join, hipStream_t s);

}  // namespace upr
