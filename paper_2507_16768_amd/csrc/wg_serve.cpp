// C ABI of beam selection, page tables and the 8-bit paged cache: argument checks and launches.
#include <hip/hip_runtime.h>

#include <new>
#include <string>

#include "wg_serve.h"

using namespace wg;

namespace {

// What an entry does, f, with its status; messages are made here, and their allocation must not throw out of the library.
template <typename F> int entry(const char *who, F f) {
    try {
        const char *why = nullptr;
        const hipError_t e = f(&why);
        if (why) { set_last_error(std::string(who) + ": " + why); return WG_ERR_INVALID; }
        if (e == hipSuccess) return WG_OK;
        set_last_error(std::string(who) + ": " + hipGetErrorString(e));
        return e == hipErrorOutOfMemory ? WG_ERR_NOMEM : WG_ERR_HIP;
    } catch (const std::bad_alloc &) {
        try { set_last_error(who); } catch (...) {}
        return WG_ERR_NOMEM;
    }
}
#define WG_WANT(cond, text) do { if (!(cond)) { *why = text; return hipSuccess; } } while (0)

// log2 of a page's tokens: 16, 32 or 64; 0 for anything else
uint32_t shift_of(uint32_t page_tokens) { return page_tokens == 16u ? 4u : page_tokens == 32u ? 5u : page_tokens == 64u ? 6u : 0u; }
bool dim_ok(uint32_t dim) { return dim == 64u || dim == 128u || dim == 256u; }
// Rows of numbers in 16 bits that are read 16 bytes at a time.
bool by_sixteen(const void *p, int64_t token, int64_t head) { return reinterpret_cast<uintptr_t>(p) % 16 == 0 && token % 8 == 0 && head % 8 == 0; }

bool aligned(const void *p, uintptr_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

}  // namespace

extern "C" {

uint64_t wg_beam_select_workspace(uint32_t rows, uint32_t V, uint32_t beams) {
    if (rows == 0 || V == 0 || beams == 0 || beams > kBeamMax) return 0;
    return (uint64_t)rows * beam_parts(rows, V, beams) * (beams + 1ull) * 8ull;
}

int wg_beam_select(const void *d_logits, wg_dtype_t dtype, uint32_t rows, uint32_t V, int64_t row_stride_elems, const uint32_t *d_bitmask,
                   uint32_t beams, const float *d_scores, const wg_state_t *d_states, float *d_scores_out, int32_t *d_parents,
                   int32_t *d_tokens, wg_state_t *d_states_out, void *d_workspace, uint64_t workspace_bytes, void *stream) {
    return entry("wg_beam_select", [&](const char **why) {
        WG_WANT(d_logits && d_scores && d_scores_out && d_parents && d_tokens && d_workspace, "null argument");
        WG_WANT(!d_states == !d_states_out, "states go in and out, or neither");
        WG_WANT(rows && V, "empty batch or vocabulary");
        WG_WANT(dtype == WG_F32 || dtype == WG_BF16, "unknown dtype");
        WG_WANT(row_stride_elems >= (int64_t)V, "row stride smaller than V");
        WG_WANT(rows <= kMostRows, "rows above 65535");
        WG_WANT(V <= 0x7FFFFFFFu / 4u, "V above 536870911");
        WG_WANT(beams && beams <= kBeamMax, "beams must be 1 .. 64");
        WG_WANT(rows % beams == 0, "rows must be a multiple of beams");
        WG_WANT(d_scores != d_scores_out && (!d_states || d_states != d_states_out), "scores and states must not be written in place");
        WG_WANT(workspace_bytes >= wg_beam_select_workspace(rows, V, beams), "the workspace is too small (wg_beam_select_workspace)");
        WG_WANT(aligned(d_workspace, 8), "the workspace must be 8-byte aligned");
        return launch_beam_select(d_logits, dtype, rows, V, row_stride_elems, d_bitmask, beams, d_scores, d_states, d_scores_out, d_parents, d_tokens,
                                  d_states_out, d_workspace, static_cast<hipStream_t>(stream));
    });
}

int wg_reorder_rows(const void *d_src, void *d_dst, const int32_t *d_parents, uint32_t outer, uint32_t rows, uint64_t row_bytes,
                    int64_t src_outer_bytes, int64_t src_row_bytes, int64_t dst_outer_bytes, int64_t dst_row_bytes, void *stream) {
    return entry("wg_reorder_rows", [&](const char **why) {
        WG_WANT(d_src && d_dst && d_parents, "null argument");
        WG_WANT(d_src != d_dst, "rows must not be moved in place");
        WG_WANT(outer && rows && row_bytes, "nothing to move");
        WG_WANT(outer <= 65535u && rows <= kMostRows, "outer or rows above 65535");
        WG_WANT(row_bytes <= 1ull << 33, "rows above 2^33 bytes");
        WG_WANT(src_row_bytes >= (int64_t)row_bytes && dst_row_bytes >= (int64_t)row_bytes, "rows overlap");
        return launch_reorder_rows(d_src, d_dst, d_parents, outer, rows, row_bytes, src_outer_bytes, src_row_bytes, dst_outer_bytes, dst_row_bytes,
                                   static_cast<hipStream_t>(stream));
    });
}

uint64_t wg_page_step_workspace(uint32_t rows, uint32_t beams, uint32_t columns) {
    return beams && columns ? page_step_bytes(rows, beams, columns) : 0u;
}

int wg_page_step(const int32_t *d_table, uint32_t rows, uint32_t columns, const int32_t *d_lens, const int32_t *d_counts, const int32_t *d_parents,
                 uint32_t beams, uint32_t page_tokens, int32_t *d_ring, uint32_t pages, const uint64_t *d_counters, int32_t *d_table_out,
                 int32_t *d_lens_out, int32_t *d_starts, int32_t *d_slots, int32_t *d_positions, int32_t *d_origins, uint32_t tokens,
                 uint64_t *d_counters_out, void *d_workspace, uint64_t workspace_bytes, void *stream) {
    return entry("wg_page_step", [&](const char **why) {
        WG_WANT(d_table && d_lens && d_counts && d_ring && d_counters && d_table_out && d_lens_out && d_starts && d_counters_out, "null argument");
        WG_WANT(!tokens || (d_slots && d_positions && d_origins), "null argument");
        WG_WANT(rows && columns && pages, "no rows, columns or pages");
        WG_WANT(rows <= kMostRows, "rows above 65535");
        WG_WANT(shift_of(page_tokens), "page_tokens must be 16, 32 or 64");
        WG_WANT((uint64_t)columns * page_tokens <= 0x7FFFFFFFull && (uint64_t)pages * page_tokens <= 0x7FFFFFFFull && tokens <= 0x7FFFFFFFu, "tokens above 2^31 - 1");
        WG_WANT(beams && beams <= kBeamMax && rows % beams == 0, "beams must be 1 .. 64 and divide rows");
        WG_WANT(!d_parents || columns <= 65535u * 32u, "columns above 2097120 with parents");
        WG_WANT(d_parents || beams == 1u, "beams without parents");
        WG_WANT(!d_parents || d_table != d_table_out, "rows that follow parents must not be written in place");
        WG_WANT(d_lens != d_lens_out && d_counters != d_counters_out, "lengths and counters must not be written in place");
        const uint64_t need = d_parents ? wg_page_step_workspace(rows, beams, columns) : 0u;
        WG_WANT(!need || (d_workspace && workspace_bytes >= need), "the workspace is too small (wg_page_step_workspace)");
        WG_WANT(aligned(d_workspace, 16), "the workspace must be 16-byte aligned");
        return launch_page_step(d_table, rows, columns, d_lens, d_counts, d_parents, beams, shift_of(page_tokens), d_ring, pages, d_counters, d_table_out,
                                d_lens_out, d_starts, d_slots, d_positions, d_origins, tokens, d_counters_out, d_workspace, static_cast<hipStream_t>(stream));
    });
}

int wg_cache_append(const void *d_k, const void *d_v, uint32_t tokens, uint32_t heads, uint32_t dim, int64_t k_token_stride, int64_t k_head_stride,
                    int64_t v_token_stride, int64_t v_head_stride, const int32_t *d_slots, const int32_t *d_origins, uint8_t *d_k_cache,
                    uint8_t *d_v_cache, float *d_k_scale, float *d_v_scale, uint32_t pages, uint32_t page_tokens, void *stream) {
    return entry("wg_cache_append", [&](const char **why) {
        WG_WANT(d_k && d_v && d_slots && d_k_cache && d_v_cache && d_k_scale && d_v_scale, "null argument");
        WG_WANT(tokens && heads && pages, "no tokens, heads or pages");
        WG_WANT(tokens <= 1u << 29 && heads <= 65535u, "tokens above 2^29 or heads above 65535");
        WG_WANT(dim_ok(dim), "dim must be 64, 128 or 256");
        WG_WANT(shift_of(page_tokens), "page_tokens must be 16, 32 or 64");
        WG_WANT((uint64_t)pages * page_tokens <= 0x7FFFFFFFull, "slots above 2^31 - 1");
        WG_WANT(by_sixteen(d_k, k_token_stride, k_head_stride) && by_sixteen(d_v, v_token_stride, v_head_stride), "keys and values must lie at multiples of 16 bytes");
        WG_WANT(k_token_stride >= 0 && v_token_stride >= 0 && k_token_stride < 1 << 24 && v_token_stride < 1 << 24, "tokens must lie 0 to 2^24 - 1 elements apart");
        WG_WANT(aligned(d_k_cache, 16) && aligned(d_v_cache, 16), "the cache must be 16-byte aligned");
        return launch_cache_append(d_k, d_v, tokens, heads, dim, k_token_stride, k_head_stride, v_token_stride, v_head_stride, d_slots, d_origins, d_k_cache,
                                   d_v_cache, d_k_scale, d_v_scale, pages, shift_of(page_tokens), static_cast<hipStream_t>(stream));
    });
}

uint64_t wg_cache_attend_workspace(uint32_t tokens, uint32_t rows, uint32_t q_heads, uint32_t heads, uint32_t dim, uint32_t columns, uint32_t page_tokens) {
    if (!tokens || !rows || !heads || q_heads < heads || !columns || !shift_of(page_tokens)) return 0;
    const uint64_t splits = attend_splits(tokens, rows, heads, q_heads / heads, dim, columns, shift_of(page_tokens));
    return splits < 2u ? 0u : ((uint64_t)tokens * q_heads * splits * (dim + 2u) + tokens) * 4u;
}

int wg_cache_attend(const void *d_q, uint32_t tokens, uint32_t q_heads, uint32_t heads, uint32_t dim, int64_t q_token_stride, int64_t q_head_stride,
                    const uint8_t *d_k_cache, const uint8_t *d_v_cache, const float *d_k_scale, const float *d_v_scale, uint32_t pages, uint32_t page_tokens,
                    const int32_t *d_table, uint32_t rows, uint32_t columns, const int32_t *d_lens, const int32_t *d_starts, float scale, void *d_out,
                    void *d_workspace, uint64_t workspace_bytes, void *stream) {
    return entry("wg_cache_attend", [&](const char **why) {
        WG_WANT(d_q && d_k_cache && d_v_cache && d_k_scale && d_v_scale && d_table && d_lens && d_starts && d_out, "null argument");
        WG_WANT(tokens && rows && columns && pages && heads, "no tokens, rows, columns, pages or heads");
        WG_WANT(tokens <= 0x7FFFFFFFu && rows <= kMostRows && heads <= 4095u, "too many tokens, rows or heads");
        WG_WANT(q_heads >= heads && q_heads % heads == 0 && q_heads <= 65535u, "q_heads must be a multiple of heads, 65535 at most");
        WG_WANT(dim_ok(dim), "dim must be 64, 128 or 256");
        WG_WANT(shift_of(page_tokens), "page_tokens must be 16, 32 or 64");
        WG_WANT((uint64_t)columns * page_tokens <= 0x7FFFFFFFull && (uint64_t)pages * page_tokens <= 0x7FFFFFFFull, "tokens above 2^31 - 1");
        WG_WANT(attend_fits(tokens, rows, heads, q_heads / heads, dim), "too many tokens for one launch");
        WG_WANT(by_sixteen(d_q, q_token_stride, q_head_stride), "queries must lie at multiples of 16 bytes");
        WG_WANT(aligned(d_k_cache, 16) && aligned(d_v_cache, 16) && aligned(d_out, 16), "the cache and the output must be 16-byte aligned");
        WG_WANT(scale == scale && scale - scale == 0.f, "the scale is no number");
        const uint64_t need = wg_cache_attend_workspace(tokens, rows, q_heads, heads, dim, columns, page_tokens);
        WG_WANT(!need || (d_workspace && workspace_bytes >= need), "the workspace is too small (wg_cache_attend_workspace)");
        WG_WANT(aligned(d_workspace, 16), "the workspace must be 16-byte aligned");
        return launch_cache_attend(d_q, tokens, heads, q_heads / heads, dim, q_token_stride, q_head_stride, d_k_cache, d_v_cache, d_k_scale, d_v_scale, pages,
                                   shift_of(page_tokens), d_table, rows, columns, d_lens, d_starts, scale, d_out, d_workspace, static_cast<hipStream_t>(stream));
    });
}

}  // extern "C"
