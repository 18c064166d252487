// Launchers of what a decode loop needs around the masks: beam selection, page tables, the 8-bit paged cache.  They return the launch's
// own status; arguments have been checked by the entry points (wg_serve.cpp).
#pragma once
#include <hip/hip_runtime.h>

#include "wg_internal.h"

namespace wg {

constexpr uint32_t kBeamMax = 64;            // most beams of a request
constexpr uint32_t kBeamParts = 32;          // most workgroups of a row
constexpr uint32_t kMostRows = 65535;        // rows of a call: a dimension of the grid
uint32_t beam_parts(uint32_t rows, uint32_t V);
hipError_t launch_beam_select(const void *logits, int dtype, uint32_t rows, uint32_t V, int64_t row_stride, const uint32_t *bitmask, uint32_t K,
                              const float *scores, const wg_state_t *states, float *scores_out, int32_t *parents, int32_t *tokens,
                              wg_state_t *states_out, void *workspace, hipStream_t s);
hipError_t launch_reorder_rows(const void *src, void *dst, const int32_t *parents, uint32_t outer, uint32_t rows, uint64_t row_bytes,
                               int64_t src_outer, int64_t src_row, int64_t dst_outer, int64_t dst_row, hipStream_t s);

}  // namespace wg
