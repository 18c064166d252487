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

// Rotary positions.  strides: of tokens and heads of q, k, q_out and k_out.
hipError_t launch_rotate(const void *q, const void *k, int dtype, uint32_t tokens, uint32_t q_heads, uint32_t k_heads, uint32_t dim, uint32_t rotated, bool interleaved,
                         const int64_t (&strides)[8], const int32_t *positions, const double *frequencies, float magnitude, void *q_out, void *k_out, hipStream_t s);

constexpr uint32_t kLatentKey = 64;          // numbers of a shared key
// Whether a launch (fewer than 2^32 threads) holds so many tokens.
bool latent_append_fits(uint32_t tokens, bool bytes);
bool latent_read_fits(uint32_t tokens);
hipError_t launch_latent_append(const void *c, const void *r, uint32_t tokens, uint32_t latent, int64_t c_token, int64_t r_token, const int32_t *slots, const int32_t *origins,
                                void *c_cache, void *r_cache, float *scale, uint32_t pages, uint32_t shift, hipStream_t s);
hipError_t launch_latent_read(const void *c_cache, const void *r_cache, const float *scale, uint32_t latent, uint32_t pages, uint32_t shift, const int32_t *table, uint32_t rows,
                              uint32_t columns, const int32_t *starts, uint32_t tokens, void *c_out, int64_t c_token, void *r_out, int64_t r_token, hipStream_t s);
// Keys of a block, blocks of a chunk of work at least, and chunks at most: as many workgroups as the chip holds at a time.
constexpr uint32_t kAttendBlock = 128, kAttendLeast = 1, kTileCost = 1, kAttendSlots = 256, kPromptSlots = 512;
bool latent_attend_fits(uint32_t tokens, uint32_t rows, uint32_t heads);
uint64_t latent_attend_bytes(uint32_t tokens, uint32_t rows, uint32_t heads, uint32_t latent, uint32_t columns, uint32_t shift);
// strides: of tokens and heads of q_c and q_r.
hipError_t launch_latent_attend(const void *q_c, const void *q_r, uint32_t tokens, uint32_t heads, uint32_t latent, const int64_t (&strides)[4], const void *c_cache, const void *r_cache,
                                const float *scale, uint32_t pages, uint32_t shift, const int32_t *table, uint32_t rows, uint32_t columns, const int32_t *lens,
                                const int32_t *starts, float factor, void *out, void *workspace, hipStream_t s);
bool latent_prompt_fits(uint32_t tokens, uint32_t rows, uint32_t heads);
uint64_t latent_prompt_bytes(uint32_t tokens, uint32_t rows, uint32_t heads, uint32_t dim, uint32_t keys);
// strides: of tokens and heads of q_n, q_r and k_n, of tokens of k_r, of tokens and heads of v.
hipError_t launch_latent_prompt(const void *q_n, const void *q_r, const void *k_n, const void *k_r, const void *v, uint32_t tokens, uint32_t keys, uint32_t heads, uint32_t dim,
                                const int64_t (&strides)[9], uint32_t rows, const int32_t *starts, const int32_t *key_starts, float factor, void *out, void *workspace, hipStream_t s);

}  // namespace wg
