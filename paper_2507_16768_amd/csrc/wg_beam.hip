// Beam search under the mask for gfx950 (wave64): the best continuations of every request over its beams and the
// vocabulary, and rows of state that follow them.
//
// With x the allowed logits of a beam (its row), m their maximum and Z = sum exp(x - m), a continuation by token v scores
//     s(beam, v) = score(beam) + ((x_v - m) - log Z),
// and a request keeps its K best by (s, lower beam, larger x, lower token).  Within a row s does not decrease with x, so a row's
// share of them is among the row's K best by (x, lower token): no score is made for any other token.  The logits are read once: a
// thread keeps a running maximum and the sum of its tokens' exp against it, rescaled where the maximum moves.
//
// beam_rows_kernel: a workgroup of 256 threads takes one of `parts` shares of a row, and leaves m, Z and the K best tokens as keys.  beam_merge_kernel: a
// workgroup takes a request, joins the parts' m and Z and ranks the K * parts * K keys by their scores.
//
// What bounds them: 256 masked rows of 151,936 bfloat16 logits, eight beams: 25 us for the rows (74 MB, 3.0 TB/s; the vector unit is busy 85 % of the time with an exp and an
// order for every allowed logit), 5.5 for the merge; 120 rows of 100,003 fp32 logits without a mask: 16.5 us (48 MB, 2.9 TB/s) and 4.5; four rows of 32,000: 5.8 and 3.8, two launches
// and trips to memory one behind the other.
#include <hip/hip_runtime.h>

#include <cfloat>

#include "wg_buffer.h"
#include "wg_launch.h"
#include "wg_order.h"
#include "wg_row.h"
#include "wg_serve.h"

namespace wg {

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * kLog2e); }

// What a part leaves besides its keys: +inf counts as the largest number, so that top and every difference from it are finite.  The sum is in 32 bits.  A thread adds up to V / 2,048 + 16
// terms of at most 1 one after the other (a row has eight parts of 256 threads at the least, or as many as it has 2,048 tokens), rescales their sum for every four or eight of them, and
// some 50 additions join those of threads, wavefronts and parts.  Each is off by 2^-24 of the sum at the most and an exp by 2^-22, all together by (V / 1,600 + 80) * 2^-24: 1e-5 for
// 151,936 tokens, 2e-2 for the most that a row may have, where errors all have one sign.
struct PartSum { float top, sum; };

// (256 threads: the first of these takes 33 us with 512, the third the same)
constexpr uint32_t kRowThreads = 256, kRowWaves = kRowThreads / 64u, kRowSeg = 1024, kRowCand = 512;
struct BeamShared {
    uint32_t words[kRowSeg + 1u];                    // the staged mask
    unsigned long long cand[kRowCand];               // the candidates: rank << 32 | ~id
    uint32_t threads[kRowThreads];                   // threads that hold candidates
    uint32_t least[kRowWaves];
    float top[kRowWaves], sum[kRowWaves];
    uint32_t n, n_threads;
};

// A piece's elements as numbers, what is not allowed or a NaN as -inf, +inf as the largest number.
template <uint32_t kPer>
struct Numbers { float x[kPer]; };
__device__ __forceinline__ float tamed(uint32_t bits) { return __builtin_amdgcn_fmed3f(__builtin_fmaxf(__uint_as_float(bits), -__builtin_inff()), -__builtin_inff(), FLT_MAX); }
__device__ __forceinline__ Numbers<8> numbers(const uint4 &v, uint32_t m, uint16_t)
{
    const uint32_t d[4] = {v.x, v.y, v.z, v.w}, nm = ~m;
    Numbers<8> r;
#pragma unroll
    for (int k = 0; k < 4; k++) {
        r.x[2 * k] = tamed(d[k] << 16 | (uint32_t)__builtin_amdgcn_sbfe(nm, 2 * k, 1));
        r.x[2 * k + 1] = tamed((d[k] & 0xFFFF0000u) | (uint32_t)__builtin_amdgcn_sbfe(nm, 2 * k + 1, 1));
    }
    return r;
}
__device__ __forceinline__ Numbers<4> numbers(const uint4 &v, uint32_t m, uint32_t)
{
    const uint32_t d[4] = {v.x, v.y, v.z, v.w}, nm = ~m;
    Numbers<4> r;
#pragma unroll
    for (int k = 0; k < 4; k++) r.x[k] = tamed(d[k] | (uint32_t)__builtin_amdgcn_sbfe(nm, k, 1));
    return r;
}

// bound_of, where wavefronts may have next to nothing: then the most of what each one's k best reach.  (A row's last part, or a request with dead beams, gave no bound
// at all, and everything was ranked: 55 us instead of 8 for the step after 16 prompts.)
template <uint32_t kN>
__device__ __forceinline__ uint32_t bound_of_some(uint32_t own, uint32_t k, uint32_t *least)
{
    uint32_t bound = bound_of<kN>(own, k, least);
    if (bound) return bound;
    __syncthreads();
    const uint32_t mine = nth_of_wave(own, k);
    if ((threadIdx.x & 63u) == 0u) least[threadIdx.x >> 6] = mine;
    __syncthreads();
#pragma unroll
    for (uint32_t w = 0; w < kN; w++) bound = least[w] > bound ? least[w] : bound;
    return bound;
}

__device__ __forceinline__ const uint32_t *mask_of(const uint32_t *mask, uint32_t row, uint32_t W) { return mask + (size_t)row * W; }
__device__ __forceinline__ NoMask mask_of(NoMask none, uint32_t, uint32_t) { return none; }

template <typename Elem, bool kWhole, typename Mask>
__global__ void __launch_bounds__(kRowThreads) __attribute__((amdgpu_waves_per_eu(8)))
beam_rows_kernel(const Elem *__restrict__ logits, int64_t row_stride, uint32_t V, uint32_t W, Mask bitmask,
                 const float *__restrict__ scores, uint32_t K, unsigned long long *__restrict__ lists, PartSum *__restrict__ sums)
{
    constexpr uint32_t kPer = Row<Elem, kWhole>::kPer;
    __shared__ BeamShared sh;
    const uint32_t b = blockIdx.y, tid = threadIdx.x;
    unsigned long long *out = lists + ((size_t)b * gridDim.x + blockIdx.x) * K;
    if (!(scores[b] > -__builtin_inff())) {          // (NaN too) a beam that is not there
        for (uint32_t i = tid; i < K; i += kRowThreads) out[i] = 0ull;
        if (tid == 0) sums[(size_t)b * gridDim.x + blockIdx.x] = PartSum{-FLT_MAX, 0.f};
        return;
    }
    const Mask mask = mask_of(bitmask, b, W);
    const Row<Elem, kWhole> r(logits + (int64_t)b * row_stride, V);
    const uint32_t share = ((r.pieces + gridDim.x - 1u) / gridDim.x + 31u) & ~31u;
    const uint32_t lo = blockIdx.x * share < r.pieces ? blockIdx.x * share : r.pieces;
    const uint32_t hi = r.pieces - lo < share ? r.pieces : lo + share;
    // the thread's first piece with `best`, the most of its other pieces, and the sum of exp against top
    float best = -__builtin_inff(), second = best, top = -FLT_MAX, sum = 0.f;
    uint32_t where = 0, held_mask = 0;
    uint4 held{0u, 0u, 0u, 0u};
    stream_row<kRowThreads, kRowSeg>(r, mask, W, sh.words, lo, hi, [&](uint32_t p, const uint4 &v, uint32_t m) {
        const auto y = numbers(v, m, Elem(0));
        float x = y.x[0];
#pragma unroll
        for (uint32_t i = 1; i < kPer; i++) x = __builtin_fmaxf(x, y.x[i]);
        const float most = __builtin_fmaxf(best, x), high = __builtin_fmaxf(top, x);
        second = __builtin_fmaxf(second, most == best ? x : best);
        if (!(most == best)) { best = most; where = p; held = v; held_mask = m; }
        sum *= exp_of(top - high);
#pragma unroll
        for (uint32_t i = 0; i < kPer; i++) sum += exp_of(y.x[i] - high);
        top = high;
    });
    // (the order key of +inf stands above that of the largest number, which `best` holds for both: a bound by `own` is one for both)
    const uint32_t own = best > -__builtin_inff() ? order_key(__float_as_uint(best)) + 1u : 0u;
    if (tid == 0) { sh.n = 0u; sh.n_threads = 0u; }
    float wave_top = top;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) wave_top = __builtin_fmaxf(wave_top, __shfl_xor(wave_top, o));
    sum *= exp_of(top - wave_top);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
    if ((tid & 63u) == 0u) { sh.top[tid >> 6] = wave_top; sh.sum[tid >> 6] = sum; }
    const uint32_t bound = bound_of_some<kRowWaves>(own, K, sh.least);
    const float value = __builtin_fmaxf(bound ? bound_value(bound) : -FLT_MAX, -FLT_MAX);
    auto put = [&](const uint4 &v, uint32_t p, uint32_t m) {
        uint32_t take = reaching(v, m, 1u, value, Elem(0));
        while (take) {
            const uint32_t i = (uint32_t)__builtin_ctz(take);
            take &= take - 1u;
            const uint32_t at = atomicAdd(&sh.n, 1u);
            if (at < kRowCand) sh.cand[at] = key_of(r, v, p, i);
        }
    };
    // Candidates: the allowed tokens at or above the bound, most of them in the one piece that their thread holds; the pieces of threads that
    // have more of them are looked at again, by all threads.
    if (own && own >= bound) {
        if (bound == 0u || second >= value) sh.threads[atomicAdd(&sh.n_threads, 1u)] = tid;
        else put(held, where, held_mask);
    }
    __syncthreads();
    if (tid == 0) {
        float t = sh.top[0], z = 0.f;
        for (uint32_t w = 1; w < kRowWaves; w++) t = __builtin_fmaxf(t, sh.top[w]);
        for (uint32_t w = 0; w < kRowWaves; w++) z += sh.sum[w] * exp_of(sh.top[w] - t);
        sums[(size_t)b * gridDim.x + blockIdx.x] = PartSum{t, z};
    }
    const uint32_t n_own = hi - lo, per = (n_own + kRowThreads - 1u) / kRowThreads, items = sh.n_threads * per;
    for (uint32_t i = tid; i < items; i += kRowThreads) {
        const uint32_t of = i / per, p = lo + sh.threads[of] + (i - of * per) * kRowThreads;
        const uint32_t m = p < hi ? piece_mask(r, mask, W, p) : 0u;
        if (m) put(r.piece(r.window(p, 1u), 0u), p, m);
    }
    __syncthreads();
    const uint32_t n = sh.n;
    if (n > kRowCand) {
        // Hundreds of tokens tie.  K rounds, the best key below the last one each time.
        unsigned long long last = ~0ull;
        for (uint32_t q = 0; q < K; q++) {
            unsigned long long most = 0ull;
            for (uint32_t p = lo + tid; p < hi; p += kRowThreads) {
                const uint32_t m = piece_mask(r, mask, W, p);
                if (!m) continue;
                const uint4 v = r.piece(r.window(p, 1u), 0u);
                uint32_t take = reaching(v, m, 1u, value, Elem(0));
                while (take) {
                    const uint32_t i = (uint32_t)__builtin_ctz(take);
                    take &= take - 1u;
                    const unsigned long long key = key_of(r, v, p, i);
                    if (key < last && key > most) most = key;
                }
            }
#pragma unroll
            for (int o = 32; o > 0; o >>= 1) { const unsigned long long other = __shfl_xor(most, o); most = other > most ? other : most; }
            __syncthreads();
            if ((tid & 63u) == 0u) sh.cand[tid >> 6] = most;
            __syncthreads();
            last = sh.cand[0];
            for (uint32_t w = 1; w < kRowWaves; w++) last = sh.cand[w] > last ? sh.cand[w] : last;
            if (tid == 0) out[q] = last;
        }
        return;
    }
    rank_keys<kRowThreads>(sh.cand, n, K, [&](uint32_t at, unsigned long long key) { out[at] = key; });
    for (uint32_t i = n + tid; i < K; i += kRowThreads) out[i] = 0ull;
}

// ---------------------------------------------------------------------------------------------
constexpr uint32_t kMergeThreads = 256, kMergeWaves = kMergeThreads / 64u, kMergeCand = 1024;
constexpr uint32_t kMergeHeld = 8;                   // keys of a thread that stay in registers
constexpr uint32_t kMergeSums = 1024;                // parts of a request's rows whose sums are joined out of LDS

// A request's continuations from its rows' lists.  Its time is trips to memory and between wavefronts, one after the other: all that it reads is asked for at once.
__global__ void __launch_bounds__(kMergeThreads)
beam_merge_kernel(const unsigned long long *__restrict__ lists, const PartSum *__restrict__ sums, uint32_t K, uint32_t parts,
                  const float *__restrict__ scores, const wg_state_t *__restrict__ states, float *__restrict__ scores_out,
                  int32_t *__restrict__ parents, int32_t *__restrict__ tokens, wg_state_t *__restrict__ states_out)
{
    __shared__ unsigned long long cand[kMergeCand], cand_key[kMergeCand];      // order key of the score << 32 | ~beam; the row's key
    __shared__ PartSum part[kMergeSums];
    __shared__ float row_top[kBeamMax], row_log[kBeamMax], row_score[kBeamMax];
    __shared__ wg_state_t row_state[kBeamMax];
    __shared__ unsigned long long pair[2][kMergeWaves];
    __shared__ uint32_t least[kMergeWaves], n_cand;
    const uint32_t tid = threadIdx.x, row0 = blockIdx.x * K, n = K * parts * K, entries = K * parts;
    const unsigned long long *list = lists + (size_t)row0 * (parts * K);
    const PartSum *sum = sums + (size_t)row0 * parts;
    const bool staged = entries <= kMergeSums;
    constexpr uint32_t kRound = kMergeHeld * kMergeThreads;
    // The i-th key: in order of rank, the lists' best first.  The wavefronts take them in turn, so that each has as many good ones as another and few reach the bound.  (List by list, a
    // wavefront had some rows only, and where those were bad all keys were ranked: 27 us for 32 requests of eight beams.)
    const uint32_t place = (tid & 63u) * kMergeWaves + (tid >> 6);
    auto list_at = [&](uint32_t i) { return i % entries * K + i / entries; };
    unsigned long long key[kMergeHeld];
#pragma unroll
    for (uint32_t q = 0; q < kMergeHeld; q++) key[q] = place + q * kMergeThreads < n ? list[list_at(place + q * kMergeThreads)] : 0ull;
    for (uint32_t i = tid; staged && i < entries; i += kMergeThreads) part[i] = sum[i];
    if (tid < K) {
        row_score[tid] = scores[row0 + tid];
        if (states) row_state[tid] = states[row0 + tid];
    }
    if (tid == 0) n_cand = 0u;
    __syncthreads();
    if (tid < K) {
        const PartSum *of = staged ? part + tid * parts : sum + tid * parts;
        float t = -FLT_MAX, z = 0.f;
#pragma unroll 8
        for (uint32_t p = 0; p < parts; p++) t = __builtin_fmaxf(t, of[p].top);
#pragma unroll 8
        for (uint32_t p = 0; p < parts; p++) z += of[p].sum * exp_of(of[p].top - t);
        row_top[tid] = t; row_log[tid] = __builtin_amdgcn_logf(z) * kLn2;
    }
    __syncthreads();
    auto score_of = [&](unsigned long long k, uint32_t beam) {
        const uint32_t order = (uint32_t)(k >> 32) - 1u;
        const float x = __builtin_fminf(__uint_as_float((order & 0x80000000u) ? order & 0x7FFFFFFFu : ~order), FLT_MAX);
        return row_score[beam] + ((x - row_top[beam]) - row_log[beam]);
    };
    // what ranks the continuation i of a key, 0 where there is none
    auto rank_at = [&](uint32_t i, unsigned long long k) {
        if (!k) return 0ull;
        const uint32_t beam = i % entries / parts;
        const float s = score_of(k, beam);
        return s > -__builtin_inff() ? (unsigned long long)order_key(__float_as_uint(s)) << 32 | (0xFFFFFFFFu - beam) : 0ull;
    };
    unsigned long long rank[kMergeHeld];
    uint32_t own = 0;
    auto raise = [&](unsigned long long r) { const uint32_t high = (uint32_t)(r >> 32); own = high > own ? high : own; };
#pragma unroll
    for (uint32_t q = 0; q < kMergeHeld; q++) { rank[q] = rank_at(place + q * kMergeThreads, key[q]); raise(rank[q]); }
    const uint32_t bound = bound_of_some<kMergeWaves>(own, K, least);
    auto put = [&](unsigned long long r, unsigned long long k) {
        if (!r || (uint32_t)(r >> 32) < bound) return false;
        const uint32_t at = atomicAdd(&n_cand, 1u);
        if (at < kMergeCand) { cand[at] = r; cand_key[at] = k; }
        return true;
    };
#pragma unroll
    for (uint32_t q = 0; q < kMergeHeld; q++) put(rank[q], key[q]);
    // The others, of requests with many beams, a round of keys at a time.  A list's keys do not get better, so that a rank that reaches the bound in no list ends the search; a
    // round has a whole rank (the host sees to that).  (With all keys for the bound and all again
    // against it a request of 64 beams on 32,000 tokens took 110 us, for 27.)
    for (uint32_t i0 = kRound; i0 < n; i0 += kRound) {
        bool some = false;
#pragma unroll
        for (uint32_t q = 0; q < kMergeHeld; q++) { const uint32_t i = i0 + place + q * kMergeThreads; key[q] = i < n ? list[list_at(i)] : 0ull; }
#pragma unroll
        for (uint32_t q = 0; q < kMergeHeld; q++) some |= put(rank_at(i0 + place + q * kMergeThreads, key[q]), key[q]);
        if (!__syncthreads_or(some)) break;
    }
    __syncthreads();
    uint32_t c = n_cand;
    if (c > kMergeCand) {
        // more tie than there is room for: K rounds, the best below the last one each time
        unsigned long long last = ~0ull, last_key = ~0ull;
        __syncthreads();
        for (uint32_t q = 0; q < K; q++) {
            unsigned long long best = 0ull, best_key = 0ull;
            auto see = [&](unsigned long long r, unsigned long long k) {
                if (r > best || (r == best && k > best_key)) { best = r; best_key = k; }
            };
            for (uint32_t i = tid; i < n; i += kMergeThreads) {
                const unsigned long long k = list[list_at(i)], r = rank_at(i, k);
                if (r < last || (r == last && k < last_key)) see(r, k);
            }
#pragma unroll
            for (int o = 32; o > 0; o >>= 1) { const unsigned long long r = __shfl_xor(best, o), k = __shfl_xor(best_key, o); see(r, k); }
            if ((tid & 63u) == 0u) { pair[0][tid >> 6] = best; pair[1][tid >> 6] = best_key; }
            __syncthreads();
            for (uint32_t w = 0; w < kMergeWaves; w++) see(pair[0][w], pair[1][w]);
            last = best; last_key = best_key;
            if (tid == 0) { cand[q] = best; cand_key[q] = best_key; }
            __syncthreads();
        }
        c = K;
    }
    // ranked by counting, eight lanes to a continuation
    const uint32_t sub = tid & 7u;
    for (uint32_t i = tid >> 3; i < c; i += kMergeThreads / 8u) {
        const unsigned long long s = cand[i], k = cand_key[i];
        uint32_t better = 0;
#pragma unroll 4
        for (uint32_t q = sub; q < c; q += 8u) better += cand[q] > s || (cand[q] == s && cand_key[q] > k);
        better += __shfl_xor(better, 1); better += __shfl_xor(better, 2); better += __shfl_xor(better, 4);
        if (sub == 0u && better < K) {
            const uint32_t beam = 0xFFFFFFFFu - (uint32_t)s, row = row0 + better;
            scores_out[row] = score_of(k, beam);
            parents[row] = (int32_t)(row0 + beam);
            tokens[row] = (int32_t)(0xFFFFFFFFu - (uint32_t)k);
            if (states) states_out[row] = row_state[beam];
        }
    }
    for (uint32_t i = c + tid; i < K; i += kMergeThreads) {           // fewer continuations than beams
        scores_out[row0 + i] = -__builtin_inff();
        parents[row0 + i] = -1;
        tokens[row0 + i] = -1;
        if (states) states_out[row0 + i] = wg_state_t{WG_SID_ERROR, 0u};
    }
}

// Workgroups of a row: about eight per compute unit in all, with at least 2,048 tokens each (twice as many: 256 rows of 151,936 tokens 32 us for 28 with the merge, 120 of 100,003 25
// for 21; half as many: the same).  A multiple of eight where it can be: workgroups go to the chip's eight XCDs in turn, and
// each then has its share of every row, however the rows' masks differ.  The merge's keys stay within what its threads hold, or 8 parts, which leaves two ranks of a
// request's lists to a round of them.
uint32_t beam_parts(uint32_t rows, uint32_t V, uint32_t K)
{
    static_assert(2u * 8u * kBeamMax <= kMergeHeld * kMergeThreads, "a round of the merge has a whole rank");
    const uint32_t most = (V + 2047u) / 2048u, want = 2048u / rows < 8u ? 8u : 2048u / rows, held = kMergeHeld * kMergeThreads / (K * K), room = held < 8u ? 8u : held;
    uint32_t parts = want < most ? want : most;
    if (parts > room) parts = room;
    if (parts > kBeamParts) parts = kBeamParts;
    return parts >= 8u ? parts / 8u * 8u : parts;
}

template <typename Elem, typename Mask>
static hipError_t beam_rows(const Elem *logits, uint32_t rows, uint32_t V, int64_t row_stride, Mask mask, const float *scores, uint32_t K,
                            unsigned long long *lists, PartSum *sums, hipStream_t s)
{
    const bool whole = reinterpret_cast<uintptr_t>(logits) % sizeof(Elem) == 0u;
    return launch(whole ? beam_rows_kernel<Elem, true, Mask> : beam_rows_kernel<Elem, false, Mask>, dim3(beam_parts(rows, V, K), rows), dim3(kRowThreads), 0, s, nullptr,
                  logits, row_stride, V, (V + 31u) / 32u, mask, scores, K, lists, sums);
}

hipError_t launch_beam_select(const void *logits, int dtype, uint32_t rows, uint32_t V, int64_t row_stride, const uint32_t *bitmask, uint32_t K,
                              const float *scores, const wg_state_t *states, float *scores_out, int32_t *parents, int32_t *tokens,
                              wg_state_t *states_out, void *workspace, hipStream_t s)
{
    const uint32_t parts = beam_parts(rows, V, K);
    unsigned long long *lists = static_cast<unsigned long long *>(workspace);
    PartSum *sums = reinterpret_cast<PartSum *>(lists + (size_t)rows * parts * K);
    auto first = [&](auto *x) {
        return bitmask ? beam_rows(x, rows, V, row_stride, bitmask, scores, K, lists, sums, s) : beam_rows(x, rows, V, row_stride, NoMask{}, scores, K, lists, sums, s);
    };
    const hipError_t e = dtype == WG_F32 ? first(static_cast<const uint32_t *>(logits)) : first(static_cast<const uint16_t *>(logits));
    if (e != hipSuccess) return e;
    return launch(beam_merge_kernel, dim3(rows / K), dim3(kMergeThreads), 0, s, nullptr, lists, sums, K, parts, scores, states, scores_out, parents, tokens, states_out);
}

// ---------------------------------------------------------------------------------------------
// Rows of state after their parents: a copy, at the rate of one (134 MB read and written in 21 us: 8 layers of 256 rows of 32 KB).  Sixteen bytes to a lane at multiples of four bytes (the hardware takes them there), else byte by byte.
struct __attribute__((packed, aligned(4))) Four { uint32_t x, y, z, w; };
constexpr uint32_t kReorderThreads = 256, kReorderPer = 4;

template <bool kWords>
__global__ void __launch_bounds__(kReorderThreads)
reorder_kernel(const uint8_t *__restrict__ src, uint8_t *__restrict__ dst, const int32_t *__restrict__ parents, uint32_t rows, uint64_t row_bytes,
               int64_t src_outer, int64_t src_row, int64_t dst_outer, int64_t dst_row)
{
    constexpr uint32_t kUnit = kWords ? 16u : 1u;
    const uint32_t r = blockIdx.y;
    const int32_t parent = parents[r];
    const bool there = (uint32_t)parent < rows;
    const uint8_t *from = src + (int64_t)blockIdx.z * src_outer + (int64_t)(there ? parent : 0) * src_row;
    uint8_t *to = dst + (int64_t)blockIdx.z * dst_outer + (int64_t)r * dst_row;
    const uint64_t units = row_bytes / kUnit, u0 = (uint64_t)blockIdx.x * (kReorderThreads * kReorderPer) + threadIdx.x;
    if (kWords) {
        Four v[kReorderPer];
#pragma unroll
        for (uint32_t j = 0; j < kReorderPer; j++) {
            const uint64_t u = u0 + j * kReorderThreads;
            v[j] = Four{0u, 0u, 0u, 0u};
            if (there && u < units) v[j] = reinterpret_cast<const Four *>(from)[u];
        }
#pragma unroll
        for (uint32_t j = 0; j < kReorderPer; j++) {
            const uint64_t u = u0 + j * kReorderThreads;
            if (u < units) reinterpret_cast<Four *>(to)[u] = v[j];
        }
        const uint64_t tail = row_bytes / 4u - units * 4u;                  // words behind the last sixteen bytes
        if (blockIdx.x == 0u && threadIdx.x < tail)
            reinterpret_cast<uint32_t *>(to)[units * 4u + threadIdx.x] = there ? reinterpret_cast<const uint32_t *>(from)[units * 4u + threadIdx.x] : 0u;
    } else {
        for (uint32_t j = 0; j < kReorderPer; j++) {
            const uint64_t u = u0 + j * kReorderThreads;
            if (u < units) to[u] = there ? from[u] : (uint8_t)0;
        }
    }
}

hipError_t launch_reorder_rows(const void *src, void *dst, const int32_t *parents, uint32_t outer, uint32_t rows, uint64_t row_bytes,
                               int64_t src_outer, int64_t src_row, int64_t dst_outer, int64_t dst_row, hipStream_t s)
{
    const uint64_t all = reinterpret_cast<uintptr_t>(src) | reinterpret_cast<uintptr_t>(dst) | row_bytes | (uint64_t)src_outer | (uint64_t)src_row | (uint64_t)dst_outer | (uint64_t)dst_row;
    const bool words = all % 4u == 0u;
    const uint64_t units = words ? row_bytes / 16u : row_bytes, per = kReorderThreads * kReorderPer;
    const uint64_t chunks = units ? (units + per - 1u) / per : 1u;
    return launch(words ? reorder_kernel<true> : reorder_kernel<false>, dim3((uint32_t)chunks, rows, outer), dim3(kReorderThreads), 0, s, nullptr,
                  static_cast<const uint8_t *>(src), static_cast<uint8_t *>(dst), parents, rows, row_bytes, src_outer, src_row, dst_outer, dst_row);
}

}  // namespace wg
