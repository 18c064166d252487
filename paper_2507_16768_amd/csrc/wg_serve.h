// Launchers of what a decode loop needs around the masks: beam selection, page tables, the 8-bit paged cache.  They return the launch's
// own status; arguments have been checked by the entry points (wg_serve.cpp).
#pragma once
#include <hip/hip_runtime.h>

#include "wg_internal.h"

namespace wg {

constexpr uint32_t kBeamMax = 64;            // most beams of a request
constexpr uint32_t kBeamParts = 32;          // most workgroups of a row
constexpr uint32_t kMostRows = 65535;        // rows of a call: a dimension of the grid
uint32_t beam_parts(uint32_t rows, uint32_t V, uint32_t K);
hipError_t launch_beam_select(const void *logits, int dtype, uint32_t rows, uint32_t V, int64_t row_stride, const uint32_t *bitmask, uint32_t K,
                              const float *scores, const wg_state_t *states, float *scores_out, int32_t *parents, int32_t *tokens,
                              wg_state_t *states_out, void *workspace, hipStream_t s);
hipError_t launch_reorder_rows(const void *src, void *dst, const int32_t *parents, uint32_t outer, uint32_t rows, uint64_t row_bytes,
                               int64_t src_outer, int64_t src_row, int64_t dst_outer, int64_t dst_row, hipStream_t s);
uint64_t page_step_bytes(uint32_t rows, uint32_t K, uint32_t columns);
hipError_t launch_page_step(const int32_t *table, uint32_t rows, uint32_t columns, const int32_t *lens, const int32_t *counts, const int32_t *parents,
                            uint32_t K, uint32_t shift, int32_t *ring, uint32_t pages, const uint64_t *counters, int32_t *table_out, int32_t *lens_out,
                            int32_t *starts, int32_t *slots, int32_t *positions, int32_t *origins, uint32_t tokens, uint64_t *counters_out,
                            void *workspace, hipStream_t s);
hipError_t launch_cache_append(const void *k, const void *v, uint32_t tokens, uint32_t heads, uint32_t dim, int64_t k_token, int64_t k_head, int64_t v_token,
                               int64_t v_head, const int32_t *slots, const int32_t *origins, uint8_t *k_cache, uint8_t *v_cache, float *k_scale,
                               float *v_scale, uint32_t pages, uint32_t shift, hipStream_t s);
// Whether one launch holds the call.
bool attend_fits(uint32_t tokens, uint32_t rows, uint32_t heads, uint32_t group, uint32_t dim);
// Shares that a tile's keys may be cut into; each leaves dim + 2 floats for every token and query head.
uint32_t attend_splits(uint32_t tokens, uint32_t rows, uint32_t heads, uint32_t group, uint32_t dim, uint32_t columns, uint32_t shift);
hipError_t launch_cache_attend(const void *q, uint32_t tokens, uint32_t heads, uint32_t group, uint32_t dim, int64_t q_token, int64_t q_head, const uint8_t *k_cache,
                               const uint8_t *v_cache, const float *k_scale, const float *v_scale, uint32_t pages, uint32_t shift, const int32_t *table,
                               uint32_t rows, uint32_t columns, const int32_t *lens, const int32_t *starts, float scale, void *out, void *workspace, hipStream_t s);

}  // namespace wg
