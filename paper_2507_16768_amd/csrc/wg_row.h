// Rows of logits under their masks (gfx950): a row as 16-byte pieces, its mask staged in LDS, the row streamed past a
// function, and the selection of its best tokens by bounds.  What the kernels that read logits share (HIP translation units only).
#pragma once
#include <hip/hip_runtime.h>

#include "wg_buffer.h"
#include "wg_order.h"

namespace wg {

constexpr uint32_t kThreads = 1024;
constexpr uint32_t kWaves = kThreads / 64u;
constexpr uint32_t kSegWords = 8192;                 // mask words staged at a time (32 KB: 262,144 tokens)
constexpr uint32_t kCand = 1024;                     // candidates ranked in LDS
constexpr uint32_t kNoPiece = 0xFFFFFFFFu;

// One row of logits as 16-byte pieces.  kWhole: elements lie at multiples of their size, and pieces are aligned.  Else pieces are
// cut at the row's beginning, each out of the five aligned words that it lies in.  (Element by element, behind branches, a piece was up
// to eight trips to memory one after the other; a kernel for both spent 1 % of the whole rows' time on the choice.)  us at an odd byte,
// mixed masks, so / now, the greedy choice and k = 50: bf16, V = 151,936, B = 40 15.2 41.0 / 7.4 15.3, 256 39.7 56.4 / 12.3 16.5; fp32, V =
// 128,256, B = 64 12.6 34.9 / 8.1 18.4.
template <typename Elem, bool kWhole>
struct Row {
    static constexpr uint32_t kPer = 16u / sizeof(Elem);          // tokens of a piece: 8 bf16, 4 fp32
    static constexpr uint32_t kAll = (1u << kPer) - 1u;
    const Elem *tokens;
    const char *first;                               // the aligned block, or word, that the row's first byte lies in
    uint32_t skew, pieces, V;                        // piece p holds the tokens p * kPer - skew ...
    uint32_t odd;                                    // not whole: bytes of the first word in front of the row

    __device__ __forceinline__ Row(const Elem *row, uint32_t V_) : tokens(row), V(V_)
    {
        const uintptr_t at = reinterpret_cast<uintptr_t>(row);
        odd = (uint32_t)(at % 4u);
        skew = kWhole ? (uint32_t)(at % 16u / sizeof(Elem)) : 0u;
        first = reinterpret_cast<const char *>(row) - (kWhole ? at % 16u : at % 4u);
        pieces = (V + skew + kPer - 1u) / kPer;
    }
    // n pieces from p on.  An aligned block, or word, that holds a byte of the row lies in the row's own memory page, also
    // where it begins before the row or ends behind it.
    __device__ __forceinline__ Window window(uint32_t p, uint32_t n) const
    {
        if (kWhole) return window_of(first + (size_t)p * 16u, n * 16u);
        const uint64_t left = ((odd + (uint64_t)V * sizeof(Elem) + 3u) & ~3ull) - (uint64_t)p * 16u, most = n * 16u + 4u;
        return window_of(first + (size_t)p * 16u, (uint32_t)(left < most ? left : most));
    }
    // The piece at an offset of a window (kNowhere: one without anything to look at).
    __device__ __forceinline__ uint4 piece(const Window &win, uint32_t at) const
    {
        if (kWhole) return block_at(win, at);
        uint32_t w[5];
#pragma unroll
        for (uint32_t k = 0; k < 5u; k++) w[k] = word_at(win, at + 4u * k);
        return uint4{__builtin_amdgcn_alignbyte(w[1], w[0], odd), __builtin_amdgcn_alignbyte(w[2], w[1], odd),
                     __builtin_amdgcn_alignbyte(w[3], w[2], odd), __builtin_amdgcn_alignbyte(w[4], w[3], odd)};
    }
    __device__ __forceinline__ uint32_t token(uint32_t p, uint32_t i) const { return p * kPer + i - skew; }
};

// Word i of the row's mask moved up by the skew: bit s of the result is the token s - skew.
__device__ __forceinline__ uint32_t mask_word(const uint32_t *mask, uint32_t W, uint32_t V, uint32_t skew, uint32_t i)
{
    auto word = [&](uint32_t w) {
        uint32_t x = w < W ? mask[w] : 0u;
        if (w == W - 1u && (V & 31u)) x &= (1u << (V & 31u)) - 1u;
        return x;
    };
    const uint32_t hi = word(i);
    return skew ? (hi << skew) | ((i ? word(i - 1u) : 0u) >> (32u - skew)) : hi;
}

// The words [w0, w0 + nw) of the same, nw up to kSeg, to LDS, and a zero behind them; all of a thread's in flight together.
// The whole workgroup calls it.
template <uint32_t kT, uint32_t kSeg>
__device__ __forceinline__ void stage_mask(const uint32_t *mask, uint32_t W, uint32_t V, uint32_t skew, uint32_t w0, uint32_t nw, uint32_t *words)
{
    constexpr uint32_t kMost = kSeg / kT;
    const Window win = window_of(mask + w0, (W > w0 ? W - w0 < nw ? W - w0 : nw : 0u) * 4u);
    const uint32_t tid = threadIdx.x, last = W - 1u - w0, tail = V & 31u ? (1u << (V & 31u)) - 1u : 0xFFFFFFFFu;
    uint32_t x[kMost], y[kMost];
#pragma unroll
    for (uint32_t j = 0; j < kMost; j++) {
        x[j] = 0u; y[j] = 0u;
        if (j * kT >= nw) continue;
        x[j] = word_at(win, (tid + j * kT) * 4u);
        if (skew) y[j] = tid + j * kT ? word_at(win, (tid + j * kT - 1u) * 4u) : w0 ? mask[w0 - 1u] : 0u;
    }
#pragma unroll
    for (uint32_t j = 0; j < kMost; j++) {
        const uint32_t i = tid + j * kT;
        if (j * kT >= nw) break;
        if (i == last) x[j] &= tail;
        if (skew) x[j] = x[j] << skew | (i == last + 1u ? y[j] & tail : y[j]) >> (32u - skew);
        if (i < nw) words[i] = x[j];
    }
    if (tid == 0) words[nw] = 0u;
}

// In the place of a mask where every token is allowed.
struct NoMask {};
__device__ __forceinline__ uint32_t mask_word(NoMask, uint32_t W, uint32_t V, uint32_t skew, uint32_t i)
{
    auto word = [&](uint32_t w) { return w >= W ? 0u : w == W - 1u && (V & 31u) ? (1u << (V & 31u)) - 1u : 0xFFFFFFFFu; };
    return skew ? (word(i) << skew) | ((i ? word(i - 1u) : 0u) >> (32u - skew)) : word(i);
}
template <uint32_t kT, uint32_t kSeg>
__device__ __forceinline__ void stage_mask(NoMask none, uint32_t W, uint32_t V, uint32_t skew, uint32_t w0, uint32_t nw, uint32_t *words)
{
    for (uint32_t i = threadIdx.x; i <= nw; i += kT) words[i] = i < nw ? mask_word(none, W, V, skew, w0 + i) : 0u;
}

// The allowed tokens of piece p, from the mask as it lies in memory.
template <typename Elem, bool kWhole, typename Mask>
__device__ __forceinline__ uint32_t piece_mask(const Row<Elem, kWhole> &r, Mask mask, uint32_t W, uint32_t p)
{
    const uint32_t bit = p * r.kPer;
    return (mask_word(mask, W, r.V, r.skew, bit >> 5) >> (bit & 31u)) & r.kAll;
}

// The largest allowed number of a piece (NaN when there is none): a disallowed token's bits are
// forced to all ones, which is a NaN in both formats, and the hardware maximum ignores NaNs, so
// NaN logits drop out the same way.
__device__ __forceinline__ float piece_max(const uint4 &v, uint32_t m, uint16_t)
{
    const uint32_t d[4] = {v.x, v.y, v.z, v.w};
    const uint32_t nm = ~m;
    float a = __builtin_nanf(""), b = a;
#pragma unroll
    for (int k = 0; k < 4; k++) {                     // dword k holds tokens 2k (low half) and 2k+1
        const uint32_t lo = (uint32_t)__builtin_amdgcn_sbfe(nm, 2 * k, 1), hi = (uint32_t)__builtin_amdgcn_sbfe(nm, 2 * k + 1, 1);
        const uint32_t x = d[k] | (lo & 0xFFFFu) | (hi << 16);
        a = __builtin_fmaxf(a, __uint_as_float(x << 16));
        b = __builtin_fmaxf(b, __uint_as_float(x & 0xFFFF0000u));
    }
    return __builtin_fmaxf(a, b);
}
__device__ __forceinline__ float piece_max(const uint4 &v, uint32_t m, uint32_t)
{
    const uint32_t d[4] = {v.x, v.y, v.z, v.w};
    const uint32_t nm = ~m;
    float a = __builtin_nanf("");
#pragma unroll
    for (int k = 0; k < 4; k++) a = __builtin_fmaxf(a, __uint_as_float(d[k] | (uint32_t)__builtin_amdgcn_sbfe(nm, k, 1)));
    return a;
}

// Streams the pieces [lo, hi) of the row, lo a multiple of 32: what(p, piece, allowed tokens) for every
// piece of the thread that has an allowed token, in ascending order.  `words` is kSeg + 1
// words of LDS.  The whole workgroup, of kT threads, calls it.
template <uint32_t kT = kThreads, uint32_t kSeg = kSegWords, typename Elem, bool kWhole, typename Mask, typename F>
__device__ __forceinline__ void stream_row(const Row<Elem, kWhole> &r, Mask mask, uint32_t W, uint32_t *words,
                                           uint32_t lo, uint32_t hi, F what)
{
    constexpr uint32_t kPer = Row<Elem, kWhole>::kPer, kSegPieces = kSeg * 32u / kPer;
    const uint32_t tid = threadIdx.x;
    for (uint32_t s0 = lo; s0 < hi; s0 += kSegPieces) {
        const uint32_t n = hi - s0 < kSegPieces ? hi - s0 : kSegPieces;
        const uint32_t w0 = s0 / (32u / kPer), nw = (n * kPer + 31u) / 32u;
        if (s0 != lo) __syncthreads();                     // the segment before is done with the LDS
        stage_mask<kT, kSeg>(mask, W, r.V, r.skew, w0, nw, words);
        __syncthreads();
        const uint32_t none = nw * (32u / kPer);           // a piece of the zero behind the words
        auto allowed = [&](uint32_t q) {
            if (q > none) q = none;
            if (kPer == 8u) return (uint32_t)reinterpret_cast<const uint8_t *>(words)[q];
            return words[q / (32u / kPer)] >> (q * kPer & 31u) & r.kAll;
        };
        // Up to three pieces of a thread are one round: the loop below takes two more for nothing (the greedy choice, mixed, us, before there was
        // the loop / with it alone / so: V = 8,000, B = 1 3.9 / 4.3 / 3.7, 256 4.5 / 5.1 / 4.3; a row of 151,936 tokens in eight shares 5.6 / 6.3 / 5.8).
        constexpr uint32_t kRound = 3u;
        if (n <= kT * kRound) {
            const Window win = r.window(s0, n);
            uint32_t mm[kRound];
            uint4 vv[kRound];
#pragma unroll
            for (uint32_t j = 0; j < kRound; j++) mm[j] = allowed(tid + j * kT);
#pragma unroll
            for (uint32_t j = 0; j < kRound; j++) vv[j] = r.piece(win, mm[j] ? (tid + j * kT) * 16u : kNowhere);
#pragma unroll
            for (uint32_t j = 0; j < kRound; j++) if (mm[j]) what(s0 + tid + j * kT, vv[j], mm[j]);
            continue;
        }
        constexpr uint32_t kHalf = kWhole ? 3u : 2u;       // (of five words each, three are 3 % slower)
        const Window win = r.window(s0, n);
        uint32_t m[2][kHalf];
        uint4 v[2][kHalf];
        auto request = [&](uint32_t (&mm)[kHalf], uint4 (&vv)[kHalf], uint32_t q0) {
#pragma unroll
            for (uint32_t j = 0; j < kHalf; j++) mm[j] = allowed(q0 + j * kT);
#pragma unroll
            for (uint32_t j = 0; j < kHalf; j++) vv[j] = r.piece(win, mm[j] ? (q0 + j * kT) * 16u : kNowhere);
        };
        auto look = [&](const uint32_t (&mm)[kHalf], const uint4 (&vv)[kHalf], uint32_t q0) {
#pragma unroll
            for (uint32_t j = 0; j < kHalf; j++)
                if (mm[j]) what(s0 + q0 + j * kT, vv[j], mm[j]);
        };
        request(m[0], v[0], tid);
#pragma nounroll
        for (uint32_t q0 = tid; q0 < n; q0 += kT * kHalf * 2u) {
            request(m[1], v[1], q0 + kT * kHalf);
            look(m[0], v[0], q0);
            request(m[0], v[0], q0 + kT * kHalf * 2u);
            look(m[1], v[1], q0 + kT * kHalf);
        }
    }
}

// ---------------------------------------------------------------------------------------------
// The best of a row.  The rank of a token is its order key plus one (0: not allowed, 1: a NaN), then the
// lower id.
template <typename Elem>
__device__ __forceinline__ uint32_t rank_of(Elem e) { return order_key(__float_as_uint(elem_float(e))) + 1u; }

// The n-th largest of the wavefront's 64 values with its low 12 bits cleared (0 when fewer than n are
// above 0), by bisection: a ballot and a count per bit.
__device__ __forceinline__ uint32_t nth_of_wave(uint32_t v, uint32_t n)
{
    uint32_t bound = 0;
#pragma unroll
    for (uint32_t bit = 31u; bit >= 12u; bit--) {
        const uint32_t test = bound | 1u << bit;
        if ((uint32_t)__popcll(__ballot(v >= test)) >= n) bound = test;
    }
    return bound;
}

// A value that at least k of the workgroup's values reach (0 when there are none such): the least of
// the wavefronts' ceil(k / n)-th largest.  `least` is a word of LDS per wavefront.
template <uint32_t kN>
__device__ __forceinline__ uint32_t bound_of(uint32_t own, uint32_t k, uint32_t *least)
{
    const uint32_t mine = nth_of_wave(own, (k + kN - 1u) / kN);
    if ((threadIdx.x & 63u) == 0u) least[threadIdx.x >> 6] = mine;
    __syncthreads();
    uint32_t bound = least[0];
#pragma unroll
    for (uint32_t w = 1; w < kN; w++) bound = least[w] < bound ? least[w] : bound;
    return bound;
}

// The number from which on tokens reach a bound above 0 (ranks are order keys plus one).
__device__ __forceinline__ float bound_value(uint32_t bound)
{
    const uint32_t key = bound - 1u;
    uint32_t u = (key & 0x80000000u) ? (key & 0x7FFFFFFFu) : ~key;
    if ((u & 0x7FFFFFFFu) > 0x7F800000u) u = 0xFF800000u;       // below every number: from -inf on
    return __uint_as_float(u);
}
// Which of the allowed tokens of a piece reach the bound (all of them a bound of 0, NaNs too).
__device__ __forceinline__ uint32_t reaching(const uint4 &v, uint32_t m, uint32_t bound, float value, uint16_t)
{
    const uint32_t d[4] = {v.x, v.y, v.z, v.w};
    uint32_t take = 0;
#pragma unroll
    for (int k = 0; k < 4; k++) {
        take |= (uint32_t)(__uint_as_float(d[k] << 16) >= value) << (2 * k);
        take |= (uint32_t)(__uint_as_float(d[k] & 0xFFFF0000u) >= value) << (2 * k + 1);
    }
    return bound ? take & m : m;
}
__device__ __forceinline__ uint32_t reaching(const uint4 &v, uint32_t m, uint32_t bound, float value, uint32_t)
{
    const uint32_t d[4] = {v.x, v.y, v.z, v.w};
    uint32_t take = 0;
#pragma unroll
    for (int k = 0; k < 4; k++) take |= (uint32_t)(__uint_as_float(d[k]) >= value) << k;
    return bound ? take & m : m;
}

// Element i of a piece, and the key of its token.
__device__ __forceinline__ uint32_t element(const uint4 &v, uint32_t i, uint32_t)
{
    // (values: a choice between members is one between their addresses, which puts the piece into memory)
    const uint32_t x = v.x, y = v.y, z = v.z, w = v.w, odd = 0u - (i & 1u), high = 0u - (i >> 1 & 1u);
    const uint32_t lo = (x & ~odd) | (y & odd), hi = (z & ~odd) | (w & odd);
    return (lo & ~high) | (hi & high);
}
__device__ __forceinline__ uint16_t element(const uint4 &v, uint32_t i, uint16_t)
{
    return (uint16_t)(element(v, i >> 1, 0u) >> (16u * (i & 1u)));
}
template <typename Elem, bool kWhole>
__device__ __forceinline__ unsigned long long key_of(const Row<Elem, kWhole> &r, const uint4 &v, uint32_t p, uint32_t i)
{
    return (unsigned long long)rank_of(element(v, i, Elem(0))) << 32 | (0xFFFFFFFFu - r.token(p, i));
}

// The keys of n candidate tokens, from their logits read again (which register of which thread holds a
// candidate's is not known at compile time; they are in the L2).
template <uint32_t kT, typename Elem, bool kWhole>
__device__ __forceinline__ void make_keys(unsigned long long *cand, const uint32_t *ids, uint32_t n, const Row<Elem, kWhole> &r)
{
    for (uint32_t i = threadIdx.x; i < n; i += kT) {
        const uint32_t id = ids[i];
        cand[i] = (unsigned long long)rank_of(r.tokens[id]) << 32 | (0xFFFFFFFFu - id);
    }
}

// Ranks n keys by counting, eight lanes to a key; calls emit(rank, key) for the best k.
template <uint32_t kT, typename F>
__device__ __forceinline__ void rank_keys(const unsigned long long *cand, uint32_t n, uint32_t k, F emit)
{
    const uint32_t sub = threadIdx.x & 7u;
    for (uint32_t i = threadIdx.x >> 3; i < n; i += kT / 8u) {
        const unsigned long long x = cand[i];
        uint32_t better = 0;
#pragma unroll 4
        for (uint32_t q = sub; q < n; q += 8u) better += cand[q] > x;
        better += __shfl_xor(better, 1); better += __shfl_xor(better, 2); better += __shfl_xor(better, 4);
        if (sub == 0u && better < k) emit(better, x);
    }
}

}  // namespace wg
