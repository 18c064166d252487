// C ABI of beam selection, page tables, rotary positions and the paged caches: argument checks and launches.
#include <hip/hip_runtime.h>

#include <cmath>
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
bool latent_ok(uint32_t latent) { return latent == 256u || latent == 512u; }
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

int wg_rotate(const void *d_q, const void *d_k, wg_dtype_t dtype, uint32_t tokens, uint32_t q_heads, uint32_t k_heads, uint32_t dim, uint32_t rotated, int interleaved,
              int64_t q_token_stride, int64_t q_head_stride, int64_t k_token_stride, int64_t k_head_stride, const int32_t *d_positions, const double *d_frequencies,
              float magnitude, void *d_q_out, int64_t q_out_token_stride, int64_t q_out_head_stride, void *d_k_out, int64_t k_out_token_stride,
              int64_t k_out_head_stride, void *stream) {
    return entry("wg_rotate", [&](const char **why) {
        WG_WANT(d_q && d_positions && d_frequencies && d_q_out && (!k_heads || (d_k && d_k_out)), "null argument");
        WG_WANT(tokens && q_heads, "no tokens or heads");
        WG_WANT(dtype == WG_F32 || dtype == WG_BF16, "unknown dtype");
        WG_WANT(q_heads <= 4096u && k_heads <= 4096u, "heads above 4096");
        WG_WANT(dim <= 1024u && rotated >= 2u && rotated <= dim && rotated % 2u == 0u, "rotated must be even, 2 .. dim, and dim 1024 at most");
        WG_WANT(tokens < 1u << 24, "tokens above 2^24 - 1");
        WG_WANT(magnitude == magnitude && magnitude - magnitude == 0.f, "the magnitude is no number");
        const uintptr_t size = dtype == WG_F32 ? 4u : 2u;
        WG_WANT(aligned(d_q, size) && aligned(d_q_out, size) && (!k_heads || (aligned(d_k, size) && aligned(d_k_out, size))) && aligned(d_frequencies, 8), "numbers must lie at multiples of their size");
        WG_WANT((d_q != d_q_out || (q_token_stride == q_out_token_stride && q_head_stride == q_out_head_stride)) &&
                (!k_heads || d_k != d_k_out || (k_token_stride == k_out_token_stride && k_head_stride == k_out_head_stride)), "in place the strides must agree");
        WG_WANT(!k_heads || (d_q_out != d_k_out && d_q_out != d_k && d_k_out != d_q), "queries and keys must not be one another's output");
        const bool keys = k_heads != 0u;
        const int64_t strides[8] = {q_token_stride, q_head_stride, keys ? k_token_stride : 0, keys ? k_head_stride : 0,
                                    q_out_token_stride, q_out_head_stride, keys ? k_out_token_stride : 0, keys ? k_out_head_stride : 0};
        return launch_rotate(d_q, keys ? d_k : nullptr, dtype, tokens, q_heads, k_heads, dim, rotated, interleaved != 0, strides, d_positions, d_frequencies, magnitude, d_q_out,
                             keys ? d_k_out : nullptr, static_cast<hipStream_t>(stream));
    });
}

int wg_rotary_frequencies(double *host_out, uint32_t rotated, double base, double factor, double original, double low, double high, int log_ramp) {
    return entry("wg_rotary_frequencies", [&](const char **why) {
        WG_WANT(host_out, "null argument");
        WG_WANT(rotated >= 2u && rotated % 2u == 0u && rotated <= 1024u, "rotated must be even, 2 .. 1024");
        WG_WANT(base > 0.0 && base - base == 0.0 && factor >= 1.0 && factor - factor == 0.0, "base must be above 0 and factor 1 at least");
        const bool all = low > 0.0 && std::isinf(low);
        WG_WANT(factor == 1.0 || all || (original > 0.0 && original - original == 0.0 && low >= 0.0 && high > low && high - high == 0.0 && (!log_ramp || low > 0.0)),
                "a ramp wants original above 0 and 0 <= low < high (0 < low over the logarithm)");
        for (uint32_t i = 0; i < rotated / 2u; i++) {
            const double f = std::pow(base, -2.0 * i / rotated);
            double kept = 1.0;
            if (factor != 1.0) {
                const double turns = original * f / 6.28318530717958647693;
                kept = all ? 0.0 : log_ramp ? std::log(turns / low) / std::log(high / low) : (turns - low) / (high - low);
                kept = kept < 0.0 ? 0.0 : kept > 1.0 ? 1.0 : kept;
            }
            host_out[i] = kept * f + (1.0 - kept) * f / factor;
        }
        return hipSuccess;
    });
}

int wg_latent_append(const void *d_c, const void *d_r, uint32_t tokens, uint32_t latent, int64_t c_token_stride, int64_t r_token_stride, const int32_t *d_slots,
                     const int32_t *d_origins, void *d_c_cache, void *d_r_cache, float *d_c_scale, uint32_t pages, uint32_t page_tokens, void *stream) {
    return entry("wg_latent_append", [&](const char **why) {
        WG_WANT(d_c && d_r && d_slots && d_c_cache && d_r_cache, "null argument");
        WG_WANT(tokens && pages, "no tokens or pages");
        WG_WANT(tokens <= 1u << 27 && latent_append_fits(tokens, d_c_scale != nullptr), "tokens above 2^27, or, in 8 bits, 2^26 - 4");
        WG_WANT(latent_ok(latent), "latent must be 256 or 512");
        WG_WANT(shift_of(page_tokens), "page_tokens must be 16, 32 or 64");
        WG_WANT((uint64_t)pages * page_tokens <= 0x7FFFFFFFull, "slots above 2^31 - 1");
        WG_WANT(by_sixteen(d_c, c_token_stride, 0) && by_sixteen(d_r, r_token_stride, 0), "vectors and shared keys must lie at multiples of 16 bytes");
        WG_WANT(aligned(d_c_cache, 16) && aligned(d_r_cache, 16) && aligned(d_c_scale, 4), "the cache must be 16-byte aligned");
        return launch_latent_append(d_c, d_r, tokens, latent, c_token_stride, r_token_stride, d_slots, d_origins, d_c_cache, d_r_cache, d_c_scale, pages, shift_of(page_tokens),
                                    static_cast<hipStream_t>(stream));
    });
}

int wg_latent_read(const void *d_c_cache, const void *d_r_cache, const float *d_c_scale, uint32_t latent, uint32_t pages, uint32_t page_tokens, const int32_t *d_table,
                   uint32_t rows, uint32_t columns, const int32_t *d_starts, uint32_t tokens, void *d_c_out, int64_t c_token_stride, void *d_r_out, int64_t r_token_stride, void *stream) {
    return entry("wg_latent_read", [&](const char **why) {
        WG_WANT(d_c_cache && d_r_cache && d_table && d_starts && d_c_out && d_r_out, "null argument");
        WG_WANT(tokens && rows && columns && pages, "no tokens, rows, columns or pages");
        WG_WANT(latent_read_fits(tokens) && rows <= kMostRows, "tokens above 2^28 - 16 or rows above 65535");
        WG_WANT(latent_ok(latent), "latent must be 256 or 512");
        WG_WANT(shift_of(page_tokens), "page_tokens must be 16, 32 or 64");
        WG_WANT((uint64_t)columns * page_tokens <= 0x7FFFFFFFull && (uint64_t)pages * page_tokens <= 0x7FFFFFFFull, "tokens above 2^31 - 1");
        WG_WANT(by_sixteen(d_c_out, c_token_stride, 0) && by_sixteen(d_r_out, r_token_stride, 0), "vectors and shared keys must lie at multiples of 16 bytes");
        WG_WANT(aligned(d_c_cache, 16) && aligned(d_r_cache, 16) && aligned(d_c_scale, 4), "the cache must be 16-byte aligned");
        return launch_latent_read(d_c_cache, d_r_cache, d_c_scale, latent, pages, shift_of(page_tokens), d_table, rows, columns, d_starts, tokens, d_c_out, c_token_stride, d_r_out,
                                  r_token_stride, static_cast<hipStream_t>(stream));
    });
}

uint64_t wg_latent_attend_workspace(uint32_t tokens, uint32_t rows, uint32_t heads, uint32_t latent, uint32_t columns, uint32_t page_tokens) {
    if (!tokens || !rows || !heads || !columns || !shift_of(page_tokens)) return 0;
    return latent_attend_bytes(tokens, rows, heads, latent, columns, shift_of(page_tokens));
}

int wg_latent_attend(const void *d_q_c, const void *d_q_r, uint32_t tokens, uint32_t heads, uint32_t latent, int64_t c_token_stride, int64_t c_head_stride, int64_t r_token_stride,
                     int64_t r_head_stride, const void *d_c_cache, const void *d_r_cache, const float *d_c_scale, uint32_t pages, uint32_t page_tokens, const int32_t *d_table, uint32_t rows,
                     uint32_t columns, const int32_t *d_lens, const int32_t *d_starts, float scale, void *d_out, void *d_workspace, uint64_t workspace_bytes, void *stream) {
    return entry("wg_latent_attend", [&](const char **why) {
        WG_WANT(d_q_c && d_q_r && d_c_cache && d_r_cache && d_table && d_lens && d_starts && d_out, "null argument");
        WG_WANT(tokens && rows && columns && pages && heads, "no tokens, rows, columns, pages or heads");
        WG_WANT(tokens <= 0x7FFFFFFFu && rows <= kMostRows && heads <= 4096u && (uint64_t)tokens * heads <= 0x7FFFFFFFull, "too many tokens, rows or heads");
        WG_WANT(latent_ok(latent), "latent must be 256 or 512");
        WG_WANT(shift_of(page_tokens), "page_tokens must be 16, 32 or 64");
        WG_WANT((uint64_t)columns * page_tokens <= 0x7FFFFFFFull && (uint64_t)pages * page_tokens <= 0x7FFFFFFFull, "tokens above 2^31 - 1");
        WG_WANT(latent_attend_fits(tokens, rows, heads), "too many tokens for one launch");
        WG_WANT(by_sixteen(d_q_c, c_token_stride, c_head_stride) && by_sixteen(d_q_r, r_token_stride, r_head_stride), "queries must lie at multiples of 16 bytes");
        WG_WANT(aligned(d_c_cache, 16) && aligned(d_r_cache, 16) && aligned(d_c_scale, 4) && aligned(d_out, 16), "the cache and the output must be 16-byte aligned");
        WG_WANT(scale * 1.5f - scale * 1.5f == 0.f, "the scale is no number, or too large");
        const uint64_t need = wg_latent_attend_workspace(tokens, rows, heads, latent, columns, page_tokens);
        WG_WANT(!need || (d_workspace && workspace_bytes >= need), "the workspace is too small (wg_latent_attend_workspace)");
        WG_WANT(aligned(d_workspace, 16), "the workspace must be 16-byte aligned");
        const int64_t strides[4] = {c_token_stride, c_head_stride, r_token_stride, r_head_stride};
        return launch_latent_attend(d_q_c, d_q_r, tokens, heads, latent, strides, d_c_cache, d_r_cache, d_c_scale, pages, shift_of(page_tokens), d_table, rows, columns, d_lens, d_starts,
                                    scale, d_out, d_workspace, static_cast<hipStream_t>(stream));
    });
}

uint64_t wg_latent_prompt_workspace(uint32_t tokens, uint32_t rows, uint32_t heads, uint32_t dim, uint32_t keys) {
    if (!tokens || !rows || !heads || !keys) return 0;
    return latent_prompt_bytes(tokens, rows, heads, dim, keys);
}

int wg_latent_prompt(const void *d_q_n, const void *d_q_r, const void *d_k_n, const void *d_k_r, const void *d_v, uint32_t tokens, uint32_t keys, uint32_t heads, uint32_t dim,
                     int64_t q_n_token_stride, int64_t q_n_head_stride, int64_t q_r_token_stride, int64_t q_r_head_stride, int64_t k_n_token_stride, int64_t k_n_head_stride,
                     int64_t k_r_token_stride, int64_t v_token_stride, int64_t v_head_stride, uint32_t rows, const int32_t *d_starts, const int32_t *d_key_starts, float scale,
                     void *d_out, void *d_workspace, uint64_t workspace_bytes, void *stream) {
    return entry("wg_latent_prompt", [&](const char **why) {
        WG_WANT(d_q_n && d_q_r && d_k_n && d_k_r && d_v && d_starts && d_key_starts && d_out, "null argument");
        WG_WANT(tokens && rows && keys && heads, "no tokens, rows, keys or heads");
        WG_WANT(tokens <= 0x7FFFFFFFu && keys <= 0x7FFFFFFFu && rows <= kMostRows && heads <= 4096u && (uint64_t)tokens * heads <= 0x7FFFFFFFull, "too many tokens, keys, rows or heads");
        WG_WANT(dim == 64u || dim == 128u, "dim must be 64 or 128");
        WG_WANT(latent_prompt_fits(tokens, rows, heads), "too many tokens for one launch");
        WG_WANT(by_sixteen(d_q_n, q_n_token_stride, q_n_head_stride) && by_sixteen(d_q_r, q_r_token_stride, q_r_head_stride) && by_sixteen(d_k_n, k_n_token_stride, k_n_head_stride) &&
                by_sixteen(d_k_r, k_r_token_stride, 0) && by_sixteen(d_v, v_token_stride, v_head_stride), "queries, keys and values must lie at multiples of 16 bytes");
        WG_WANT(k_n_token_stride >= 0 && k_r_token_stride >= 0 && v_token_stride >= 0 && k_n_token_stride < 1 << 24 && k_r_token_stride < 1 << 24 && v_token_stride < 1 << 24,
                "keys and values must lie 0 to 2^24 - 1 elements apart");
        WG_WANT(aligned(d_out, 16), "the output must be 16-byte aligned");
        WG_WANT(scale * 1.5f - scale * 1.5f == 0.f, "the scale is no number, or too large");
        const uint64_t need = wg_latent_prompt_workspace(tokens, rows, heads, dim, keys);
        WG_WANT(!need || (d_workspace && workspace_bytes >= need), "the workspace is too small (wg_latent_prompt_workspace)");
        WG_WANT(aligned(d_workspace, 16), "the workspace must be 16-byte aligned");
        const int64_t strides[9] = {q_n_token_stride, q_n_head_stride, q_r_token_stride, q_r_head_stride, k_n_token_stride, k_n_head_stride, k_r_token_stride, v_token_stride, v_head_stride};
        return launch_latent_prompt(d_q_n, d_q_r, d_k_n, d_k_r, d_v, tokens, keys, heads, dim, strides, rows, d_starts, d_key_starts, scale, d_out, d_workspace,
                                    static_cast<hipStream_t>(stream));
    });
}

}  // extern "C"
