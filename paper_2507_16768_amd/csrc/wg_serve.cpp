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

bool aligned(const void *p, uintptr_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

}  // namespace

extern "C" {

uint64_t wg_beam_select_workspace(uint32_t rows, uint32_t V, uint32_t beams) {
    if (rows == 0 || V == 0) return 0;
    return (uint64_t)rows * beam_parts(rows, V) * (beams + 1ull) * 8ull;
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
        WG_WANT(row_bytes <= 1ull << 36, "rows above 2^36 bytes");
        WG_WANT(src_row_bytes >= (int64_t)row_bytes && dst_row_bytes >= (int64_t)row_bytes, "rows overlap");
        return launch_reorder_rows(d_src, d_dst, d_parents, outer, rows, row_bytes, src_outer_bytes, src_row_bytes, dst_outer_bytes, dst_row_bytes,
                                   static_cast<hipStream_t>(stream));
    });
}

}  // extern "C"
