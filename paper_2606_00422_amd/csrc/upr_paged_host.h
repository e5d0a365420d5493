// Host functions of the paged operators that the model calls share with the
// operators' own entry points.
#pragma once

#include "upr_paged.h"

namespace upr {

// Argument checks (each records its message).  check_paged_users: *total is
// the number of rows of the segments; part_of_cache: the rows are the last of
// each user's cache.
upr_status check_page_rows(int32_t page_rows);
upr_status check_paged_cache(const upr_paged_cache* c, bool pointers);
upr_status check_paged_users(const upr_segments* seg, const char* name, const int32_t* rows_host, int32_t page_rows,
                             int32_t table_stride, int n_heads, bool part_of_cache, int64_t* total);
upr_status check_model_rope(const upr_rope* r, int head_dim);

PagedPool paged_pool(const upr_paged_cache& c, size_t plane_bytes, int plane);
RopeArgs rope_args(const upr_rope* r);      // NULL: none

// The launches of validated arguments (users of `seg`, cached rows rows_host).
hipError_t paged_append(int dtype, const RopeArgs& rope, const AppendArgs& a, const PagedPool& pool,
                        const upr_segments* seg, const int32_t* rows_host, hipStream_t s);
// plan_paged_attn sets a's plan (tile, chunk, part_ml's offset) and returns the
// workspace's bytes; paged_attn takes the planned arguments.
size_t plan_paged_attn(int dtype, AttnArgs* a, const upr_segments* seg, const int32_t* rows_host);
hipError_t paged_attn(int dtype, AttnArgs a, const PagedPool& pool, const upr_segments* seg,
                      const int32_t* rows_host, void* ws, hipStream_t s);

}  // namespace upr
