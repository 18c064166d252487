// A model's cache of keys and values in 8 bits for gfx950: pages of P tokens, a scale for every page and head, keys as [page][head][token][dim], values as
// [page][head][dim][token].
//
// Values lie transposed so that both products of attention find what a lane multiplies in one piece: with scores as S^T = K Q^T (rows: keys), the lane that
// holds the scores of some keys after the first product is the one that needs their weights in the second, O^T = V^T P^T.  Nothing is exchanged between lanes
// in between.
#include <hip/hip_runtime.h>

#include <cfloat>
#include <type_traits>

#include "wg_buffer.h"
#include "wg_launch.h"
#include "wg_number.h"
#include "wg_serve.h"

namespace wg {

// ---------------------------------------------------------------------------------------------
// append.  Tokens that lie one behind the other in a page are one run, which a wavefront takes for a head, and for keys or values: their largest
// magnitude, the page's scale, then the tokens; the earlier tokens of the page are rewritten where the scale grows or where they come from another page.
//
// A wavefront looks at 64 tokens' slots and at the 64 behind them, a lane each, and finds the runs that begin among the first by ballots: prompts have few of them, rows
// that take a token each have 64.  (A wavefront for every token, head and kind, of which all but those of first tokens left at once, took 99 us for 11,000 tokens
// of prompts, 8 heads of 128.)  Runs are dealt out to as many wavefronts as the chip holds.  A run's numbers are looked at twice, the second time out of LDS, or
// of the caches where a run is longer than 8 KB (60,000 tokens 84 us, all out of the caches 96, where 79 MB were read for 50; held in registers 108, for half of the wavefronts).  Those
// 11,000 tokens take 20.7 us, 75 MB at 3.7 TB/s: each run waits for its loads, its largest magnitude and its stores one after the other; a token for each of
// 256 rows, with forks among them, 6.4, a launch and four trips to memory.  Half or twice as many wavefronts change that by less than 2 us.
struct AppendArgs {
    const uint16_t *x[2];                            // keys, values: [token][head][dim]
    int64_t token_stride[2], head_stride[2];         // elements
    uint8_t *cache[2];
    float *scale[2];
    const int32_t *slots, *origins;
    uint32_t tokens, heads, pages, shift;
};

// The bytes of a word at `at` that lie below `end`, as ones.
__device__ __forceinline__ uint32_t bytes_below(uint32_t end, uint32_t at) { return end <= at ? 0u : end - at >= 4u ? 0xFFFFFFFFu : (1u << (8u * (end - at))) - 1u; }

// Behind every run's rows, which are 64 of less than 2^25 bytes from one to the next; with a lane's place in a row added too.
constexpr uint32_t kFar = 0xF0000000u;

// Where a run's tokens go: tokens o .. o + n of a page, behind `o` earlier ones that lie in page `source`.
struct Run { uint32_t token, page, source, o, n; };

// kStash: a run is 8 KB at the most, and the wavefront keeps them in LDS, each lane its own words, for the second pass.
constexpr uint32_t kStashWords = 2048;
template <uint32_t kD, bool kValues, bool kStash>
__device__ __forceinline__ void append_run(const AppendArgs &a, const Run &run, uint32_t h, uint32_t *stash)
{
    constexpr uint32_t kWhich = kValues ? 1u : 0u;
    constexpr uint32_t kLanes = kD / 8u, kTokens = 64u / kLanes;           // keys: eight dims to a lane, so many tokens to a load
    constexpr uint32_t kOwn = kD / 64u, kWords = (kOwn + 1u) / 2u;         // values: dims of a lane, and the words that they are
    constexpr uint32_t kLoadWords = kValues ? kWords : 4u, kLoadTokens = kValues ? 1u : kTokens;
    const uint32_t lane = threadIdx.x & 63u, P = 1u << a.shift, o = run.o, n = run.n, end = o + n;
    const uint16_t *x = a.x[kWhich] + (int64_t)run.token * a.token_stride[kWhich] + (int64_t)h * a.head_stride[kWhich];
    // the run's rows as a buffer: a token behind its last lies behind the end, and reads as zeros
    const uint32_t step = (uint32_t)a.token_stride[kWhich] * 2u;
    const Window win = window_of(x, (n - 1u) * step + kD * 2u);
    uint8_t *to = a.cache[kWhich] + ((size_t)run.page * a.heads + h) * (P * kD);
    const uint8_t *from = a.cache[kWhich] + ((size_t)run.source * a.heads + h) * (P * kD);
    const uint32_t own_token = kValues ? 0u : lane / kLanes, own_dim = kValues ? lane * kOwn : lane % kLanes * 8u;
    const uint32_t own_at = own_token * step + own_dim * 2u;
    // (token: of the wavefront's first lane)
    auto load = [&](uint32_t token, uint32_t (&w)[kLoadWords]) {
        if (!kValues) {
            const FourWords v = __builtin_amdgcn_raw_buffer_load_b128(win, token + own_token < n ? token * step + own_at : kNowhere, 0, 0);
            w[0] = v.x; w[1 % kLoadWords] = v.y; w[2 % kLoadWords] = v.z; w[3 % kLoadWords] = v.w;
            return;
        }
        const uint32_t at = (token < n ? token * step : kFar) + own_at;
        if (kOwn == 1u) w[0] = (uint32_t)__builtin_amdgcn_raw_buffer_load_b16(win, at, 0, 0) << 16;         // (the lower half is a zero)
        else
            for (uint32_t i = 0; i < kWords; i++) w[i] = __builtin_amdgcn_raw_buffer_load_b32(win, at + 4u * i, 0, 0);
    };
    // what the first pass has put aside, or the same load once more
    auto again_at = [&](uint32_t token, uint32_t (&w)[kLoadWords]) {
        if (!kStash) { load(token, w); return; }
        const bool there = token < n;
        const uint32_t at = ((there ? token / kLoadTokens : 0u) * 64u + lane) * kLoadWords;
#pragma unroll
        for (uint32_t k = 0; k < kLoadWords; k++) w[k] = there ? stash[at + k] : 0u;
    };
    const float was = o ? a.scale[kWhich][(size_t)run.source * a.heads + h] : 0.f;
    constexpr uint32_t kRound = kValues ? 16u : 4u;                        // loads in flight together
    float top = 0.f;
#pragma nounroll
    for (uint32_t i = 0; i < n; i += kRound * kLoadTokens) {
        uint32_t w[kRound][kLoadWords];
#pragma unroll
        for (uint32_t j = 0; j < kRound; j++) load(i + j * kLoadTokens, w[j]);
#pragma unroll
        for (uint32_t j = 0; j < kRound; j++)
#pragma unroll
            for (uint32_t k = 0; k < kLoadWords; k++) { top = top_of(top, low(w[j][k])); top = top_of(top, high(w[j][k])); }
        if (kStash)
#pragma unroll
            for (uint32_t j = 0; j < kRound; j++)
                if (i + j * kLoadTokens < n)
#pragma unroll
                    for (uint32_t k = 0; k < kLoadWords; k++) stash[((i / kLoadTokens + j) * 64u + lane) * kLoadWords + k] = w[j][k];
    }
#pragma unroll
    for (int s = 32; s > 0; s >>= 1) top = __builtin_fmaxf(top, __shfl_xor(top, s));
    const float now = __builtin_fmaxf(scale_for(top), was), inverse = 1.f / now, ratio = was / now;
    const bool again = o && (run.source != run.page || now != was);        // the earlier tokens are written too
    if (lane == 0u) a.scale[kWhich][(size_t)run.page * a.heads + h] = now;
    if (!kValues) {
        if (again)
#pragma nounroll
            for (uint32_t u = lane; u < o * kD / 16u; u += 64u) {
                Word4 v = reinterpret_cast<const Word4 *>(from)[u];
#pragma unroll
                for (uint32_t k = 0; k < 4u; k++) v[k] = rescaled(v[k], ratio);
                reinterpret_cast<Word4 *>(to)[u] = v;
            }
#pragma nounroll
        for (uint32_t i = 0; i < n; i += kRound * kLoadTokens) {
            uint32_t w[kRound][kLoadWords];
#pragma unroll
            for (uint32_t j = 0; j < kRound; j++) again_at(i + j * kLoadTokens, w[j]);
#pragma unroll
            for (uint32_t j = 0; j < kRound; j++) {
                const uint32_t token = i + j * kLoadTokens + own_token;
                Word2 r;
#pragma unroll
                for (uint32_t k = 0; k < 2u; k++)
                    r[k] = to_bytes(low(w[j][2u * k % kLoadWords]) * inverse, high(w[j][2u * k % kLoadWords]) * inverse, low(w[j][(2u * k + 1u) % kLoadWords]) * inverse,
                                    high(w[j][(2u * k + 1u) % kLoadWords]) * inverse);
                if (token < n) *reinterpret_cast<Word2 *>(to + (o + token) * kD + own_dim) = r;
            }
        }
        return;
    }
    // Values: sixteen tokens of a dim at a time.
    const uint32_t begin = again ? 0u : o;
#pragma nounroll
    for (uint32_t c = begin & ~15u; c < end; c += 16u) {
        uint32_t w[16][kLoadWords];
#pragma unroll
        for (uint32_t i = 0; i < 16u; i++) again_at(c + i - o, w[i]);          // (in front of the run's tokens a number of none, as behind them)
#pragma unroll
        for (uint32_t d = 0; d < kOwn; d++) {
            uint8_t *out = to + (size_t)(own_dim + d) * P + c;
            auto at = [&](uint32_t i) { const uint32_t x = w[i][d / 2u % kLoadWords]; return (kOwn > 1u && d % 2u == 0u ? low(x) : high(x)) * inverse; };
            Word4 r;
#pragma unroll
            for (uint32_t k = 0; k < 4u; k++) r[k] = to_bytes(at(4u * k), at(4u * k + 1u), at(4u * k + 2u), at(4u * k + 3u));
            if (begin < o && c < o) {
                const Word4 old = *reinterpret_cast<const Word4 *>(from + (size_t)(own_dim + d) * P + c);
#pragma unroll
                for (uint32_t k = 0; k < 4u; k++) { const uint32_t m = bytes_below(o, c + 4u * k); r[k] = (rescaled(old[k], ratio) & m) | (r[k] & ~m); }
            }
            if (begin > c || end < c + 16u) {                              // what is not written stays
                const Word4 there = *reinterpret_cast<const Word4 *>(out);
#pragma unroll
                for (uint32_t k = 0; k < 4u; k++) {
                    const uint32_t m = bytes_below(end, c + 4u * k) & ~bytes_below(begin, c + 4u * k);
                    r[k] = (r[k] & m) | (there[k] & ~m);
                }
            }
            *reinterpret_cast<Word4 *>(out) = r;
        }
    }
}

// A run of one token, as a step of decoding has them: a byte to every dim.  Where the scale grows or the earlier tokens come from another page they are
// written with it, sixteen bytes of the page to a lane; what comes from another page is asked for together with the token.
template <uint32_t kD, bool kValues>
__device__ __forceinline__ void append_one(const AppendArgs &a, const Run &run, uint32_t h)
{
    constexpr uint32_t kWhich = kValues ? 1u : 0u, kOwn = kD / 64u;        // dims of a lane
    constexpr uint32_t kEarly = 4;                                         // sixteen bytes each of the earlier tokens
    const uint32_t lane = threadIdx.x & 63u, P = 1u << a.shift, o = run.o, dim = lane * kOwn;
    const uint16_t *x = a.x[kWhich] + (int64_t)run.token * a.token_stride[kWhich] + (int64_t)h * a.head_stride[kWhich] + dim;
    uint8_t *to = a.cache[kWhich] + ((size_t)run.page * a.heads + h) * (P * kD);
    const uint8_t *from = a.cache[kWhich] + ((size_t)run.source * a.heads + h) * (P * kD);
    float v[4] = {0.f, 0.f, 0.f, 0.f};
    if (kOwn == 1u) v[0] = __uint_as_float((uint32_t)*x << 16);
    else
#pragma unroll
        for (uint32_t i = 0; i < kOwn / 2u; i++) { const uint32_t w = reinterpret_cast<const uint32_t *>(x)[i]; v[2u * i] = low(w); v[2u * i + 1u] = high(w); }
    const float was = o ? a.scale[kWhich][(size_t)run.source * a.heads + h] : 0.f;
    // Sixteen bytes of the page, by their number.  Of keys the earlier tokens are the first o * kD bytes; of values the first o of every P bytes, with the new one behind them.
    const bool moved = o && run.source != run.page, ahead = moved && P * kD <= kEarly * 1024u;
    const uint32_t units = kValues ? P * kD / 16u : o * kD / 16u;
    auto wanted = [&](uint32_t u) { return u < units && (!kValues || (u * 16u & (P - 1u)) <= o); };
    Word4 early[kEarly] = {}, there[kEarly] = {};
    if (ahead)
#pragma unroll
        for (uint32_t i = 0; i < kEarly; i++)
            if (wanted(i * 64u + lane)) {
                early[i] = reinterpret_cast<const Word4 *>(from)[i * 64u + lane];
                if (kValues) there[i] = reinterpret_cast<const Word4 *>(to)[i * 64u + lane];
            }
    float top = 0.f;
#pragma unroll
    for (uint32_t i = 0; i < kOwn; i++) top = top_of(top, v[i]);
#pragma unroll
    for (int s = 32; s > 0; s >>= 1) top = __builtin_fmaxf(top, __shfl_xor(top, s));
    const float now = __builtin_fmaxf(scale_for(top), was), inverse = 1.f / now, ratio = was / now;
    if (lane == 0u) a.scale[kWhich][(size_t)run.page * a.heads + h] = now;
    const uint32_t bytes = to_bytes(v[0] * inverse, v[1] * inverse, v[2] * inverse, v[3] * inverse);
    const bool again = o && (moved || now != was);
    if (again) {
        auto put = [&](uint32_t u, Word4 w, const Word4 &was_there) {
            const uint32_t of = u * 16u / P, at = u * 16u & (P - 1u);      // of values: the dim, and the first of these tokens
            const uint32_t byte = kValues ? __shfl(bytes, of / kOwn) >> (8u * (of % kOwn)) & 0xFFu : 0u;
#pragma unroll
            for (uint32_t k = 0; k < 4u; k++) {
                w[k] = rescaled(w[k], ratio);
                if (!kValues) continue;
                const uint32_t b0 = at + 4u * k, m = bytes_below(o, b0), mine = o - b0 < 4u ? 0xFFu << (8u * (o - b0)) : 0u;
                w[k] = (w[k] & m) | (byte * 0x01010101u & mine) | (was_there[k] & ~(m | mine));
            }
            if (wanted(u)) reinterpret_cast<Word4 *>(to)[u] = w;
        };
        if (ahead) {
#pragma unroll
            for (uint32_t i = 0; i < kEarly; i++) if (i * 64u < units) put(i * 64u + lane, early[i], there[i]);
        } else
#pragma nounroll
            for (uint32_t u0 = 0; u0 < units; u0 += 64u) {
                const uint32_t u = u0 + lane < units ? u0 + lane : units - 1u;
                const Word4 w = reinterpret_cast<const Word4 *>(from)[u];
                put(u0 + lane, w, moved && kValues ? reinterpret_cast<const Word4 *>(to)[u] : w);
            }
    }
    if (kValues) {
        if (!again)
#pragma unroll
            for (uint32_t i = 0; i < kOwn; i++) to[(dim + i) * P + o] = (uint8_t)(bytes >> (8u * i));
    } else if (kOwn == 1u) to[o * kD + dim] = (uint8_t)bytes;
    else if (kOwn == 2u) *reinterpret_cast<uint16_t *>(to + o * kD + dim) = (uint16_t)bytes;
    else *reinterpret_cast<uint32_t *>(to + o * kD + dim) = bytes;
}

constexpr uint32_t kAppendWaves = 4;
template <uint32_t kD, bool kStash>
__global__ void __launch_bounds__(kAppendWaves * 64u) __attribute__((amdgpu_waves_per_eu(kD == 256u ? 3 : 4)))
append_kernel(const AppendArgs a)
{
    __shared__ __attribute__((aligned(16))) uint32_t stashes[kStash ? kAppendWaves * kStashWords : 1u];
    uint32_t *stash = stashes + (kStash ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * kStashWords : 0u);
    const uint32_t lane = threadIdx.x & 63u, P = 1u << a.shift, first = blockIdx.x * 64u, t = first + lane;
    const uint32_t none = 0xFFFFFFFFu;
    const uint32_t slot = t < a.tokens ? (uint32_t)a.slots[t] : none, later = t + 64u < a.tokens ? (uint32_t)a.slots[t + 64u] : none;
    const uint32_t ahead = first ? (uint32_t)a.slots[first - 1u] : none;
    const uint32_t origin = a.origins && t < a.tokens ? (uint32_t)a.origins[t] : none;
    const uint32_t up = __shfl_up(slot, 1), last = __shfl(slot, 63), up_later = __shfl_up(later, 1);
    const uint32_t before = lane ? up : ahead, before_later = lane ? up_later : last;
    // tokens that go on with the run of the one before them (a slot of none does not, and begins none)
    const bool goes = (slot & (P - 1u)) && slot == before + 1u && slot >> a.shift < a.pages && before != none;
    const bool goes_later = (later & (P - 1u)) && later == before_later + 1u && later >> a.shift < a.pages && before_later != none;
    const unsigned long long begins = __ballot(slot >> a.shift < a.pages && !goes), on = __ballot(goes), on_later = __ballot(goes_later);
    const uint32_t items = (uint32_t)__popcll(begins) * a.heads * 2u;
    const uint32_t rank = (uint32_t)__popcll(begins & ((1ull << lane) - 1ull));
    for (uint32_t i = blockIdx.y * kAppendWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); i < items; i += gridDim.y * kAppendWaves) {
        const uint32_t which = i & 1u, h = (i >> 1) % a.heads, nth = (i >> 1) / a.heads;
        const uint32_t at = (uint32_t)__builtin_ctzll(__ballot((begins >> lane & 1ull) && rank == nth));
        // its length: how many of the next tokens go on
        const unsigned long long rest = at == 63u ? on_later : on >> (at + 1u) | on_later << (63u - at);
        const uint32_t follow = ~rest ? (uint32_t)__builtin_ctzll(~rest) : 64u;
        const uint32_t s = __builtin_amdgcn_readlane(slot, at), from = __builtin_amdgcn_readlane(origin, at), page = s >> a.shift;
        const Run run{first + at, page, from < a.pages ? from : page, s & (P - 1u), follow + 1u};
        if (__builtin_expect(run.n == 1u, 0)) {      // (registers that there is no room for are then put aside in this branch, not in the other: 1.8 us of 21)
            if (which) append_one<kD, true>(a, run, h);
            else append_one<kD, false>(a, run, h);
        } else if (which) append_run<kD, true, kStash>(a, run, h, stash);
        else append_run<kD, false, kStash>(a, run, h, stash);
    }
}

hipError_t launch_cache_append(const void *k, const void *v, uint32_t tokens, uint32_t heads, uint32_t dim, int64_t k_token, int64_t k_head, int64_t v_token,
                               int64_t v_head, const int32_t *slots, const int32_t *origins, uint8_t *k_cache, uint8_t *v_cache, float *k_scale,
                               float *v_scale, uint32_t pages, uint32_t shift, hipStream_t s)
{
    const AppendArgs a{{static_cast<const uint16_t *>(k), static_cast<const uint16_t *>(v)}, {k_token, v_token}, {k_head, v_head}, {k_cache, v_cache},
                       {k_scale, v_scale}, slots, origins, tokens, heads, pages, shift};
    // some 8,192 wavefronts, no more than there can be runs
    const uint32_t blocks = (tokens + 63u) / 64u, want = (2048u + blocks - 1u) / blocks, most = (64u * heads * 2u + kAppendWaves - 1u) / kAppendWaves;
    const dim3 grid(blocks, want < most ? want : most), block(kAppendWaves * 64u);
    // (heads of 64, whose runs are half as long, take 11.4 us for 8,000 tokens by reading again and 12.5 with LDS)
    const bool small = (dim << shift) * 2u <= kStashWords * 4u;
    return launch(dim == 64u ? append_kernel<64, false> : dim == 128u ? (small ? append_kernel<128, true> : append_kernel<128, false>)
                  : small ? append_kernel<256, true> : append_kernel<256, false>, grid, block, 0, s, nullptr, a);
}

// ---------------------------------------------------------------------------------------------
// attention.  A tile is 16 query rows of a request and a cached head: its tokens times the query heads that share the head.  A workgroup takes a share of a
// tile's keys, its wavefronts 64 keys at a time in turn: 16 bytes to a lane and load straight into registers, turned into bfloat16 there (exactly), scores,
// a running maximum and sum, weights, weighted values.  A page's scales multiply scores and weights, not its values.  There are two running maxima for it: `top` of the scores,
// which the softmax's terms e = 2^(score - top) and their sum are relative to, and `most` of score + log2(vs), of what the weights e * vs are with the scale of their page's values.
// Weights go into the second product as float16, the largest at 2^14: 11 bits of precision down to 2^-28 of the largest.  (In bfloat16 they had 8,
// which was as large an error as the output's own rounding.)  One exp makes a weight, of score - top + lift, with lift = log2(vs) + top - most + 14 of the page; the sum is that of the
// fp32 weights times 2^-lift.  Far below the others, as a page of zeros, which has the least scale, a lift is held at -80: such a weight is nothing in float16 and something in the sum.
//
// Bound by memory: a token for each of 128 rows of 2,000 to 8,000 tokens, 28 query heads over 4 of 128, 148 us with the join (677 MB, 4.6 TB/s; a copy reaches 5.0); one of 30,000 tokens, 32 over 8,
// 17 us, of which the join, a launch and the shares' own join are 5.
//
// Lane l of a wavefront holds, of 64 keys: of K, for m = l % 16, key (m / 4) * 16 + u * 8 + t * 4 + m % 4 in tile (u, t), of every 64 dims those of its quarter l / 16;
// after S^T of tile (u, t), the scores of query l % 16 and the keys (l / 16) * 16 + u * 8 + t * 4 + 0 .. 3; of V, for dim l % 16 of 16, the keys
// (l / 16) * 16 + 0 .. 15.  Sixteen neighbouring keys lie in one page.
struct AttendArgs {
    const uint16_t *q;
    int64_t q_token, q_head;                         // strides, elements
    const uint8_t *k_cache, *v_cache;
    const float *k_scale, *v_scale;
    const int32_t *table, *lens, *starts;
    uint16_t *out;                                   // [token][head][dim]
    float *partial;                                  // [token][head][split][dim + 2]: a share's output, what its sum is relative to (log2), its sum
    uint32_t *shares;                                // [token]: shares of its keys
    float scale;                                     // of the scores, times log2(e)
    uint32_t tokens, rows, heads, group, columns, pages, shift, splits, least;
};
constexpr uint32_t kAttendWaves = 4, kBlock = 64, kTile = 16;
constexpr float kHeadroom = 14.f;                    // weights go up to 2^14
constexpr float kLeastLift = -80.f, kMostLift = 1000.f;      // (above: of scales that are infinite, in pages that nothing sees)
constexpr uint32_t kLeastBlocks = 16, kFewRows = 8192;       // blocks of a share: half as many of prompts with few query rows
// Shares in all, about (512, 768, 1,024 and 2,048: 64 rows of 2,000 tokens 55, 51, 51 and 51 us, 200 of 1,000 86, 85, 85 and 86); of the kernel for many rows, as many as the chip
// holds at a time (256, 512 and 1,024: a prompt of 512 tokens behind 7,500 174, 104 and 105 us, 128 query rows of 32 rows of 2,000 tokens 74, 74 and 95).
constexpr uint32_t kShares = 1024, kWideShares = 512;
constexpr __host__ __device__ uint32_t wide_rows(uint32_t dim) { return kAttendWaves * kTile * (dim == 256u ? 1u : 2u); }    // query rows of a workgroup of it

typedef _Float16 Short2 __attribute__((ext_vector_type(2)));
typedef _Float16 Short8 __attribute__((ext_vector_type(8)));
__device__ __forceinline__ uint32_t pk_f16(float a, float b) { return __builtin_bit_cast(uint32_t, __builtin_convertvector(Float2{a, b}, Short2)); }
__device__ __forceinline__ Short8 widened16(uint32_t a, uint32_t b)
{
    const Short2 x = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 1.f, false), y = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 1.f, true);
    const Short2 z = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, 1.f, false), w = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, 1.f, true);
    return Short8{x[0], x[1], y[0], y[1], z[0], z[1], w[0], w[1]};
}
__device__ __forceinline__ Half8 widened(uint32_t a, uint32_t b)
{
    const Half2 x = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.f, false), y = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.f, true);
    const Half2 z = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.f, false), w = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.f, true);
    return Half8{x[0], x[1], y[0], y[1], z[0], z[1], w[0], w[1]};
}

// Sixteen bytes, zero from the n-th on.
__device__ __forceinline__ Word4 first_bytes(Word4 v, uint32_t n)
{
#pragma unroll
    for (uint32_t w = 0; w < 4u; w++) {
        const uint32_t k = n <= 4u * w ? 0u : n - 4u * w;
        v[w] &= k >= 4u ? 0xFFFFFFFFu : (1u << (8u * k)) - 1u;
    }
    return v;
}
// The NaNs among sixteen bytes, a byte of 1 (0x38 in the format) for each: their low seven bits are ones, one more carries into the eighth.
__device__ __forceinline__ Word4 nans_of(Word4 v)
{
#pragma unroll
    for (uint32_t w = 0; w < 4u; w++) v[w] = (((v[w] & 0x7F7F7F7Fu) + 0x01010101u) >> 7 & 0x01010101u) * 0x38u;
    return v;
}
// The same sixteen bytes with zeros in their place.
__device__ __forceinline__ Word4 without_nans(Word4 v)
{
#pragma unroll
    for (uint32_t w = 0; w < 4u; w++) {
        const uint32_t top = ((v[w] & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u;
        v[w] &= ~(top | (top - (top >> 7)));
    }
    return v;
}
__device__ __forceinline__ bool differ(Word4 a, Word4 b) { return ((a[0] ^ b[0]) | (a[1] ^ b[1]) | (a[2] ^ b[2]) | (a[3] ^ b[3])) != 0u; }
// Which of a lane's four outputs (dims of a part, for its query) see a NaN among the values of sixteen keys, as bits: the product of what is NaN and what the query sees.
__device__ __forceinline__ uint32_t nans_seen(Word4 v, uint32_t seen)
{
    const Word4 nans = nans_of(v);
    Float4 n{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (uint32_t u = 0; u < 2u; u++) {
        Word4 ones;
#pragma unroll
        for (uint32_t e = 0; e < 4u; e++) ones[e] = (u * 8u + 2u * e < seen ? 0x3C00u : 0u) | (u * 8u + 2u * e + 1u < seen ? 0x3C000000u : 0u);
        n = __builtin_amdgcn_mfma_f32_16x16x32_f16(widened16(nans[u * 2u], nans[u * 2u + 1u]), __builtin_bit_cast(Short8, ones), n, 0, 0, 0);
    }
    return (n[0] > 0.f ? 1u : 0u) | (n[1] > 0.f ? 2u : 0u) | (n[2] > 0.f ? 4u : 0u) | (n[3] > 0.f ? 8u : 0u);
}

// Eight numbers of a query (bfloat16), infinities as NaN: a score that is infinite makes the softmax none, also where all of them are -inf, which would look like a query that sees
// nothing, and where the numbers are taken in 8 bits, which have no infinity.
__device__ __forceinline__ Word4 query_words(const uint16_t *q)
{
    Word4 v = *reinterpret_cast<const Word4 *>(q);
#pragma unroll
    for (uint32_t w = 0; w < 4u; w++) v[w] |= ((v[w] & 0x7F807F80u) + 0x00800080u & 0x80008000u) >> 9;      // (an exponent of ones carries into the sign's place)
    return v;
}

// Where a tile of kTile rows lies: the request whose tiles it is among, from the places at which the requests' tokens begin.  Request r's tiles begin at
// starts[r] * group / kTile + r, which leaves room for each one's last, begun tile.  A wavefront asks 64 requests at a time.
template <uint32_t kTile>
__device__ __forceinline__ uint32_t request_of(const AttendArgs &a, uint32_t tile)
{
    const uint32_t lane = threadIdx.x & 63u;
    auto begins = [&](uint32_t r) { const uint32_t t = (uint32_t)a.starts[r] < a.tokens ? (uint32_t)a.starts[r] : a.tokens; return (uint32_t)((uint64_t)t * a.group / kTile) + r; };
    uint32_t lo = 0, n = a.rows;                     // the request is in [lo, lo + n)
    while (n > 1u) {
        const uint32_t step = (n + 63u) / 64u, r = lo + lane * step;
        const bool at = lane * step < n && begins(r) <= tile;
        const uint32_t k = 63u - (uint32_t)__builtin_clzll(__ballot(at) | 1ull);
        n = n - k * step < step ? n - k * step : step;
        lo += k * step;
    }
    return __builtin_amdgcn_readfirstlane(lo);
}

// Tokens of a row in the cache, as many as its table has pages for.
__device__ __forceinline__ uint32_t tokens_of_row(const AttendArgs &a, uint32_t r)
{
    const uint32_t most = a.columns << a.shift, l = (uint32_t)(a.lens[r] < 0 ? 0 : a.lens[r]);
    return l < most ? l : most;
}

struct TileOf { uint32_t row, first, last, begin; int32_t before; };      // query rows [first, last) of a request whose tokens are those from `begin` on, behind `before` others

template <uint32_t kTile, bool kLastFirst = false>
__device__ __forceinline__ bool tile_of(const AttendArgs &a, uint32_t tile, uint32_t *len, TileOf *out)
{
    const uint32_t r = request_of<kTile>(a, tile);
    const uint32_t b = (uint32_t)a.starts[r] < a.tokens ? (uint32_t)a.starts[r] : a.tokens, e0 = (uint32_t)a.starts[r + 1u], e = e0 < b ? b : e0 < a.tokens ? e0 : a.tokens;
    const uint32_t at = tile - ((uint32_t)((uint64_t)b * a.group / kTile) + r), all = (e - b) * a.group;
    *len = tokens_of_row(a, r);
    if (tile < (uint32_t)((uint64_t)b * a.group / kTile) + r || (uint64_t)at * kTile >= all) return false;
    out->row = r; out->begin = b;
    out->first = (kLastFirst ? (all - 1u) / kTile - at : at) * kTile;
    out->last = all - out->first < kTile ? all : out->first + kTile;
    out->before = (int32_t)*len - (int32_t)(e0 < b ? 0u : e0 - b);       // (with the row's tokens that the call does not have)
    return true;
}
// Shares that a tile's keys are cut into, and the blocks of each: shares of one size, whatever the rows' lengths, so that the workgroups that the chip holds at a time have as
// much to do as one another (128 rows of 2,000 to 8,000 tokens, 4 heads of 128: a share for each row 167 us, as many shares of every row 154 and a join of
// 16, shares of one size 144 and 4).  The number follows from the row and not from the tile: a token of a group that is no power of two can lie in two tiles.
template <uint32_t kRows, bool kWide>
__device__ __forceinline__ uint32_t shares_of(const AttendArgs &a, uint32_t blocks, uint32_t *per)
{
    constexpr uint32_t kAll = kWide ? kWideShares : kShares;
    *per = blocks;
    if (a.splits == 1u || !blocks) return 1u;
    uint64_t all = 0;                                // blocks of all rows' tiles (1,024 rows at most where keys are cut; few have tokens enough for a second tile, but with many of them)
    for (uint32_t r = threadIdx.x & 63u; r < a.rows; r += 64u) {
        const uint32_t tokens = kWide ? (uint32_t)a.starts[r + 1u] - (uint32_t)a.starts[r] : 1u;
        all += (uint64_t)((tokens_of_row(a, r) + kBlock - 1u) / kBlock) * (uint32_t)(((uint64_t)tokens * a.group + kRows - 1u) / kRows);
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) all += __shfl_xor(all, o);
    const uint64_t work = all * a.heads;
    uint32_t share = __builtin_amdgcn_readfirstlane((uint32_t)((work + kAll - 1u) / kAll < blocks ? (work + kAll - 1u) / kAll : blocks));
    share = share < a.least ? a.least : share;
    const uint32_t want = (blocks + share - 1u) / share, n = want < a.splits ? want : a.splits;
    *per = (blocks + n - 1u) / n;
    return (blocks + *per - 1u) / *per;
}
// Keys that query row i of the tile sees.
__device__ __forceinline__ uint32_t seen_by(const TileOf &t, uint32_t i, uint32_t group) { const int32_t n = t.before + (int32_t)(i / group) + 1; return n < 0 ? 0u : (uint32_t)n; }

template <uint32_t kD>
__global__ void __launch_bounds__(kAttendWaves * 64u)
attend_kernel(const AttendArgs a)
{
    constexpr uint32_t kSteps = kD / 32u, kParts = kD / 16u;
    __shared__ float join_o[kAttendWaves][kTile][kD + 4u];
    __shared__ float join_m[kAttendWaves][kTile], join_w[kAttendWaves][kTile], join_l[kAttendWaves][kTile];
    const uint32_t tid = threadIdx.x, lane = tid & 63u, wave = __builtin_amdgcn_readfirstlane(tid >> 6), m = lane & 15u, g = lane >> 4;
    const uint32_t split = blockIdx.z, h = blockIdx.y, P = 1u << a.shift;
    uint32_t len;
    TileOf t;
    if (!tile_of<kTile>(a, blockIdx.x, &len, &t)) return;
    const uint32_t blocks = (seen_by(t, t.last - 1u, a.group) + kBlock - 1u) / kBlock;
    uint32_t per;
    const uint32_t shares = shares_of<kTile, false>(a, (len + kBlock - 1u) / kBlock, &per);
    if (a.splits > 1u && h == 0u && split == 0u && tid < kTile && t.first + tid < t.last) a.shares[t.begin + (t.first + tid) / a.group] = shares;
    if (split >= shares) return;
    const uint32_t b0 = split * per, b1 = b0 + per < blocks ? b0 + per : blocks;             // (a tile that ends before its row may have none in the last share)
    // the lane's query row (a row behind the last is the last again, and is not stored)
    const uint32_t i = t.first + m < t.last ? t.first + m : t.last - 1u;
    const uint32_t sees = seen_by(t, i, a.group), sees_least = seen_by(t, t.first, a.group);
    const uint16_t *q = a.q + (int64_t)(t.begin + i / a.group) * a.q_token + (int64_t)(h * a.group + i % a.group) * a.q_head;
    Half8 qf[kSteps];
#pragma unroll
    for (uint32_t s = 0; s < kSteps; s++) qf[s] = __builtin_bit_cast(Half8, query_words(q + s / 2u * 64u + g * 16u + s % 2u * 8u));
    const int32_t *table = a.table + (size_t)t.row * a.columns;
    const uint32_t last_column = a.columns - 1u;
    auto page_at = [&](uint32_t key) { const uint32_t c = key >> a.shift; return (uint32_t)table[c < last_column ? c : last_column]; };
    auto page_of = [&](uint32_t id) { return id < a.pages ? id : 0u; };      // (what lies behind a row's pages is masked, and must be somewhere)
    // (asked for a block ahead)
    uint32_t k_next = page_at((b0 + wave) * kBlock + (m >> 2) * 16u), v_next = page_at((b0 + wave) * kBlock + g * 16u);
    Float4 o[kParts];
#pragma unroll
    for (uint32_t p = 0; p < kParts; p++) o[p] = Float4{0.f, 0.f, 0.f, 0.f};
    float top = -__builtin_inff(), most = top, sum = 0.f;    // of the lane's query; the sum of the lane's own keys
    for (uint32_t b = b0 + wave; b < b1; b += kAttendWaves) {
        const uint32_t key0 = b * kBlock, mine = key0 + g * 16u, theirs = key0 + (m >> 2) * 16u;
        const uint32_t k_page = page_of(k_next), v_page = page_of(v_next);
        const uint8_t *kp = a.k_cache + (((size_t)k_page * a.heads + h) * P + (theirs & (P - 1u)) + (m & 3u)) * kD + g * 16u;
        const uint8_t *vp = a.v_cache + (((size_t)v_page * a.heads + h) * kD + m) * P + (mine & (P - 1u));
        const float ks = a.k_scale[(size_t)v_page * a.heads + h] * a.scale;
        // (a page of zeros may have a scale of zero; what lies behind a row's pages may have any)
        const float v_log = __builtin_amdgcn_logf(__builtin_fmaxf(a.v_scale[(size_t)v_page * a.heads + h], 0x1p-64f));
        Word4 kw[4][kD / 64u];
#pragma unroll
        for (uint32_t n = 0; n < 4u; n++)
#pragma unroll
            for (uint32_t j = 0; j < kD / 64u; j++) kw[n][j] = *reinterpret_cast<const Word4 *>(kp + n * 4u * kD + j * 64u);
        Word4 vw[kParts];
#pragma unroll
        for (uint32_t p = 0; p < kParts; p++) vw[p] = *reinterpret_cast<const Word4 *>(vp + (size_t)p * 16u * P);
        k_next = page_at(theirs + kAttendWaves * kBlock); v_next = page_at(mine + kAttendWaves * kBlock);
        Float4 s[4];
#pragma unroll
        for (uint32_t n = 0; n < 4u; n++) {
            s[n] = Float4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (uint32_t k = 0; k < kSteps; k++)
                s[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widened(kw[n][k / 2u][k % 2u * 2u], kw[n][k / 2u][k % 2u * 2u + 1u]), qf[k], s[n], 0, 0, 0);
        }
        const bool edge = key0 + kBlock > sees_least;            // a query of the tile does not see all of the block
        float high = -__builtin_inff();
#pragma unroll
        for (uint32_t n = 0; n < 4u; n++)
#pragma unroll
            for (uint32_t e = 0; e < 4u; e++) {
                s[n][e] *= ks;
                if (edge && mine + n * 4u + e >= sees) s[n][e] = -__builtin_inff();
                high = __builtin_fmaxf(high, s[n][e]);
            }
        float large = high + v_log;
        high = __builtin_fmaxf(high, __shfl_xor(high, 16));
        large = __builtin_fmaxf(large, __shfl_xor(large, 16));
        high = __builtin_fmaxf(high, __shfl_xor(high, 32));
        large = __builtin_fmaxf(large, __shfl_xor(large, 32));
        // (relative to 0 where nothing has been seen: all weights are zero there)
        const float next = __builtin_fmaxf(top, high), base = next > -__builtin_inff() ? next : 0.f, next_most = __builtin_fmaxf(most, large);
        const float lift = __builtin_amdgcn_fmed3f(v_log + (next_most > -__builtin_inff() ? base - next_most : 0.f) + kHeadroom, kLeastLift, kMostLift), from = lift - base;
        if (edge) {
            // values behind the row's end are whatever the pages held: they must not be NaN times a weight of zero
            const uint32_t there = mine >= len ? 0u : len - mine < 16u ? len - mine : 16u;
#pragma unroll
            for (uint32_t p = 0; p < kParts; p++) {
                vw[p] = first_bytes(vw[p], there);
                // a NaN among the values reaches the queries that see it, and as a weight of zero times it no other
                const Word4 clean = without_nans(vw[p]);
                if (__ballot(differ(clean, vw[p]))) {
                    const uint32_t bits = nans_seen(vw[p], mine >= sees ? 0u : sees - mine < 16u ? sees - mine : 16u);
#pragma unroll
                    for (uint32_t e = 0; e < 4u; e++) o[p][e] = bits >> e & 1u ? __builtin_nanf("") : o[p][e];
                }
                vw[p] = clean;
            }
        }
        if (__ballot(next != top || next_most != most)) {
            sum *= __builtin_amdgcn_exp2f(top - base);
            const float shrink = __builtin_amdgcn_exp2f(most - (next_most > -__builtin_inff() ? next_most : 0.f));
#pragma unroll
            for (uint32_t p = 0; p < kParts; p++) o[p] *= shrink;
        }
        top = next; most = next_most;
        float part = 0.f;
        Short8 weights[2];
#pragma unroll
        for (uint32_t u = 0; u < 2u; u++) {
            float w[8];
#pragma unroll
            for (uint32_t e = 0; e < 8u; e++) {
                w[e] = __builtin_amdgcn_exp2f(s[u * 2u + e / 4u][e % 4u] + from);
                part += w[e];
            }
            weights[u] = __builtin_bit_cast(Short8, Word4{pk_f16(w[0], w[1]), pk_f16(w[2], w[3]), pk_f16(w[4], w[5]), pk_f16(w[6], w[7])});
        }
        sum = __builtin_fmaf(part, __builtin_amdgcn_exp2f(-lift), sum);
#pragma unroll
        for (uint32_t u = 0; u < 2u; u++)
#pragma unroll
            for (uint32_t p = 0; p < kParts; p++)
                o[p] = __builtin_amdgcn_mfma_f32_16x16x32_f16(widened16(vw[p][u * 2u], vw[p][u * 2u + 1u]), weights[u], o[p], 0, 0, 0);
    }
    sum += __shfl_xor(sum, 16);
    sum += __shfl_xor(sum, 32);
    // the wavefronts' shares joined
    if (g == 0u) { join_m[wave][m] = top; join_w[wave][m] = most; join_l[wave][m] = sum; }
#pragma unroll
    for (uint32_t p = 0; p < kParts; p++) *reinterpret_cast<Float4 *>(&join_o[wave][m][p * 16u + g * 4u]) = o[p];
    __syncthreads();
    constexpr uint32_t kPer = kTile * kD / (kAttendWaves * 64u);          // neighbouring dims of a thread
    const uint32_t row = tid * kPer / kD, d0 = tid * kPer % kD, r = t.first + row;
    if (r >= t.last) return;
    float all = -__builtin_inff(), all_most = all, total = 0.f, acc[kPer];
#pragma unroll
    for (uint32_t w = 0; w < kAttendWaves; w++) { all = __builtin_fmaxf(all, join_m[w][row]); all_most = __builtin_fmaxf(all_most, join_w[w][row]); }
    const float base = all > -__builtin_inff() ? all : 0.f, most_base = all_most > -__builtin_inff() ? all_most : 0.f;
#pragma unroll
    for (uint32_t d = 0; d < kPer; d++) acc[d] = 0.f;
#pragma unroll
    for (uint32_t w = 0; w < kAttendWaves; w++) {
        total += __builtin_amdgcn_exp2f(join_m[w][row] - base) * join_l[w][row];
        const float by = __builtin_amdgcn_exp2f(join_w[w][row] - most_base);
#pragma unroll
        for (uint32_t d = 0; d < kPer; d++) acc[d] += by * join_o[w][row][d0 + d];
    }
    const size_t at = (size_t)(t.begin + r / a.group) * (a.heads * a.group) + h * a.group + r % a.group;
    const float by = total > 0.f ? 1.f / total : total == total ? 0.f : total, up = __builtin_amdgcn_exp2f((most_base - base - kHeadroom) * 0.5f);     // (a row that sees nothing: zeros; up twice, as its square may be below all numbers)
#pragma unroll
    for (uint32_t d = 0; d < kPer; d++) acc[d] = acc[d] * by * up * up;
    if (shares > 1u) {
        float *to = a.partial + (at * a.splits + split) * (kD + 2u);
#pragma unroll
        for (uint32_t d = 0; d < kPer; d++) to[d0 + d] = acc[d];
        if (d0 == 0u) { to[kD] = all; to[kD + 1u] = total; }
        return;
    }
#pragma unroll
    for (uint32_t d = 0; d < kPer; d += 2u) reinterpret_cast<uint32_t *>(a.out + at * kD + d0)[d / 2u] = pk_bf16(acc[d], acc[d + 1u]);
}

// The shares of a token's keys joined, each an output of its own with its sum: kWaves wavefronts for each query head, all that one reads in flight together.  (A wavefront for a
// head of 64 shares, four at a time, took 8 us, four take 3.5; for two shares of 28 heads of 128 tokens, 16 us by four wavefronts, 4 by one.)
template <uint32_t kD, uint32_t kWaves>
__global__ void __launch_bounds__(256)
attend_join_kernel(const AttendArgs a)
{
    constexpr uint32_t kOwn = kD / 64u, kMost = 16u, kHeads = 4u / kWaves; // dims of a lane; shares of a wavefront; heads of a workgroup
    __shared__ float part[4][kD], ends[4][2];
    const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), Q = a.heads * a.group;
    const uint32_t head = blockIdx.y * kHeads + wave / kWaves, first = wave % kWaves;
    if (blockIdx.x >= (uint32_t)a.starts[a.rows]) return;                  // a token of no row, whose shares nothing has written
    const uint32_t said = a.shares[blockIdx.x], shares = said < a.splits ? said : a.splits;
    if (shares < 2u || (kWaves == 1u && head >= Q)) return;
    const size_t at = (size_t)blockIdx.x * Q + head;
    const float *from = a.partial + at * a.splits * (kD + 2u);
    float v[kMost][kOwn], tops[kMost], sums[kMost];
#pragma unroll
    for (uint32_t k = 0; k < kMost; k++) {
        const uint32_t share = first + kWaves * k;
        tops[k] = -__builtin_inff(); sums[k] = 0.f;
#pragma unroll
        for (uint32_t d = 0; d < kOwn; d++) v[k][d] = 0.f;
        if (share >= shares) continue;
        const float *p = from + (size_t)share * (kD + 2u);
        tops[k] = p[kD]; sums[k] = p[kD + 1u];
#pragma unroll
        for (uint32_t d = 0; d < kOwn; d++) v[k][d] = p[lane * kOwn + d];
    }
    float m = -__builtin_inff(), l = 0.f, acc[kOwn];
#pragma unroll
    for (uint32_t k = 0; k < kMost; k++) m = __builtin_fmaxf(m, tops[k]);
    const float base = m > -__builtin_inff() ? m : 0.f;
#pragma unroll
    for (uint32_t d = 0; d < kOwn; d++) acc[d] = 0.f;
#pragma unroll
    for (uint32_t k = 0; k < kMost; k++) { sums[k] *= __builtin_amdgcn_exp2f(tops[k] - base); l += sums[k]; }
    const float by = l > 0.f ? 1.f / l : l == l ? 0.f : l;
#pragma unroll
    for (uint32_t k = 0; k < kMost; k++)
#pragma unroll
        for (uint32_t d = 0; d < kOwn; d++) acc[d] += sums[k] * by * v[k][d];
    if (kWaves > 1u) {
#pragma unroll
        for (uint32_t d = 0; d < kOwn; d++) part[wave][lane * kOwn + d] = acc[d];
        if (lane == 0u) { ends[wave][0] = m; ends[wave][1] = l; }
        __syncthreads();
        if (wave) return;
        m = __builtin_fmaxf(__builtin_fmaxf(ends[0][0], ends[1][0]), __builtin_fmaxf(ends[2][0], ends[3][0]));
        const float all = m > -__builtin_inff() ? m : 0.f;
        float of[4], joined = 0.f;
#pragma unroll
        for (uint32_t w = 0; w < 4u; w++) { of[w] = ends[w][1] * __builtin_amdgcn_exp2f(ends[w][0] - all); joined += of[w]; }
        const float by_all = joined > 0.f ? 1.f / joined : joined == joined ? 0.f : joined;
#pragma unroll
        for (uint32_t d = 0; d < kOwn; d++) acc[d] = 0.f;
#pragma unroll
        for (uint32_t w = 0; w < 4u; w++)
#pragma unroll
            for (uint32_t d = 0; d < kOwn; d++) acc[d] += of[w] * by_all * part[w][lane * kOwn + d];
    }
    uint16_t *out = a.out + at * kD + lane * kOwn;
    if (kOwn == 1u) out[0] = (uint16_t)pk_bf16(acc[0], 0.f);
    else
#pragma unroll
        for (uint32_t d = 0; d < kOwn; d += 2u) reinterpret_cast<uint32_t *>(out)[d / 2u] = pk_bf16(acc[d], acc[(d + 1u) % kOwn]);
}

// ---------------------------------------------------------------------------------------------
// attention of many rows of a request: prompts.  A wavefront holds kTiles tiles of 16 query rows, four of them share their keys, 64 at a time, through LDS.  Bound
// by the vector unit: exp and what goes with it of every score, and the cache's numbers turned into what the products take.  So the keys are not
// turned into anything: scores come from the product of 8-bit numbers, with the queries as sums of two such numbers.  A bfloat16 number has 8 bits of
// mantissa: four of them, rounded, are one, the rest is another, 2^5 times as large; with each row brought to its largest in [128, 256) that is exact for numbers from 2^-7 on,
// 2^-14 of the row's largest, and what is smaller is off by 2^-15, 2^-22 of that, at the most.  The two products take as long as one in bfloat16 does.
//
// The running maximum is not followed from block to block: the softmax's terms e = 2^(score - base) are relative to a base, and that moves only where they get large, which
// their sum shows.  The weights in the second product are e * vs * 2^up, with vs the scale of the page's values: `up`, of each query, puts the largest of them at 2^8 where the base
// moves.  One exp makes a weight, of score - base + lift, lift = log2(vs) + up; the sum is that of the fp32 weights times 2^-lift, which is that of the terms.  Pages of values far below
// the others (of zeros: they have the least scale) have a lift far below zero; that is held at -80, where a weight of e <= 2^40 is nothing in float16 and a term above 2^-46 is
// something in fp32.  So the terms keep their sum whatever the scales are.  (Summed as float16 holds them, such pages' keys went missing.)
//
// 2,000 tokens each of 4 prompts behind up to 2,048, 32 query heads over 8 of 128: 227 us, 881 TFLOP/s (a large library product in bfloat16: 1,313).  The vector unit is busy for 63 % of the
// cycles and the matrix unit for 39: the two wavefronts of a SIMD hardly get to use both at once.  One tile of rows and three or four wavefronts to a SIMD took 1.1 times as
// long, four tiles and one wavefront 2.3 times.
//
// In LDS keys and values lie as in their pages, but for the places of the sixteen bytes of a row: eight lanes that read together find eight different ones.
typedef int Int8 __attribute__((ext_vector_type(8)));
constexpr float kMostSum = 65504.f, kMostTerms = 0x1p40f;    // sums of a lane's sixteen weights, and of what they are without the values' scale, from which on a base moves
constexpr float kRoom = 11.f, kAim = 8.f;            // log2 of the largest weight that stays where a base moves (sixteen of them are 2^15), and of the largest of the others

// Sixteen bytes c of row `key` of the keys: where they lie in their row.
template <uint32_t kD>
__device__ __forceinline__ uint32_t key_place(uint32_t key, uint32_t c)
{
    return kD == 64u ? c ^ ((key >> 1 & 1u) | (key >> 4 & 1u) << 1) : c ^ ((key & 3u) | (key >> 4 & 1u) << 2);
}
__device__ __forceinline__ uint32_t value_place(uint32_t dim, uint32_t c) { return c ^ (dim >> 1 & 3u); }

// LDS is read here and not earlier: asked for all at once, a block's keys and values do not fit the registers, and what is put into memory for them waits behind the
// next block's loads.
__device__ __forceinline__ void ds_fence() { __builtin_amdgcn_sched_barrier(0x1F); }

struct Yes { static constexpr bool value = true; };
struct No { static constexpr bool value = false; };

template <uint32_t kD, uint32_t kTiles>
__global__ void __launch_bounds__(kAttendWaves * 64u, kD == 64u ? 3 : 2)      // (heads of 64: 64 tokens of each of 32 rows of 2,000 60 us, with the registers for two only 81)
attend_wide_kernel(const AttendArgs a)
{
    constexpr uint32_t kSteps = kD / 32u, kParts = kD / 16u, kRows = kAttendWaves * kTile * kTiles, kThreads = kAttendWaves * 64u;
    static_assert(kRows == wide_rows(kD) && kRows <= kThreads, "as the host counts them");
    static_assert(kAttendWaves == kBlock / 16u, "a wavefront for sixteen keys");
    constexpr uint32_t kAhead = kD == 256u ? 1u : 2u, kValuesAhead = kD == 64u ? 2u : 4u;         // tiles of keys and parts of values that are asked for in LDS before they are needed (heads
    // of 64 with four parts: 64 tokens of each of 32 rows of 2,000 77 us for 60, as what waits in registers is put into memory)
    typedef std::conditional_t<kD == 256u, uint64_t, uint32_t> Bits;
    constexpr bool kBytes = kD >= 128u;              // scores from 8-bit numbers: products of 128 of them
    constexpr uint32_t kLoads = kD * kBlock / (16u * kThreads);            // sixteen bytes of a thread, of keys and of values each
    __shared__ Word4 keys[2][kD * kBlock / 16u], values[2][kD * kBlock / 16u];
    __shared__ Float2 scales[2][kBlock / 16u];
    const uint32_t tid = threadIdx.x, lane = tid & 63u, wave = __builtin_amdgcn_readfirstlane(tid >> 6), m = lane & 15u, g = lane >> 4;
    // (heads first: workgroups go to the XCDs in turn, and those of a head find its keys in their L2)
    const uint32_t h = blockIdx.x % a.heads, P = 1u << a.shift;
    uint32_t len;
    TileOf t;
    if (!tile_of<kRows, true>(a, blockIdx.x / a.heads, &len, &t)) return;
    const uint32_t split = blockIdx.y;
    uint32_t per;
    const uint32_t shares = shares_of<kRows, true>(a, (len + kBlock - 1u) / kBlock, &per);
    if (a.splits > 1u && h == 0u && split == 0u && tid < kRows && t.first + tid < t.last) a.shares[t.begin + (t.first + tid) / a.group] = shares;
    if (split >= shares) return;
    const uint32_t seen = (seen_by(t, t.last - 1u, a.group) + kBlock - 1u) / kBlock, b0 = split * per, blocks = b0 + per < seen ? b0 + per : seen;     // (blocks: where they end)
    const int32_t *table = a.table + (size_t)t.row * a.columns;
    const uint32_t last_column = a.columns - 1u;
    // the wavefront's rows
    const uint32_t w0 = t.first + wave * (kTile * kTiles);
    const bool working = w0 < t.last;
    uint32_t sees[kTiles];
    float q_scale[kTiles];
    Int8 q_high[kTiles][kBytes ? kD / 128u : 1u], q_low[kTiles][kBytes ? kD / 128u : 1u];
    Half8 q_half[kTiles][kBytes ? 1u : kSteps];
#pragma unroll
    for (uint32_t n = 0; n < kTiles; n++) {
        const uint32_t i = w0 + n * kTile + m < t.last ? w0 + n * kTile + m : t.last - 1u;
        sees[n] = seen_by(t, i, a.group);
        const uint16_t *q = a.q + (int64_t)(t.begin + i / a.group) * a.q_token + (int64_t)(h * a.group + i % a.group) * a.q_head + g * (kD / 4u);
        q_scale[n] = a.scale;
        if (!kBytes) {
#pragma unroll
            for (uint32_t k = 0; k < (kBytes ? 1u : kSteps); k++) q_half[n][k] = __builtin_bit_cast(Half8, query_words(q + k * 8u));
            continue;
        }
        Word4 raw[kD / 32u];
        float top = 0.f;
#pragma unroll
        for (uint32_t k = 0; k < kD / 32u; k++) {
            raw[k] = query_words(q + k * 8u);
#pragma unroll
            for (uint32_t e = 0; e < 4u; e++) { top = top_of(top, low(raw[k][e])); top = top_of(top, high(raw[k][e])); }
        }
        top = __builtin_fmaxf(top, __shfl_xor(top, 16));
        top = __builtin_fmaxf(top, __shfl_xor(top, 32));
        const int e = 134 - (int)(__float_as_uint(top) >> 23), exponent = top > 0.f ? (e > 126 ? 126 : e) : 0;
        const float up = __uint_as_float((uint32_t)(exponent + 127) << 23);
        q_scale[n] = a.scale * __uint_as_float((uint32_t)(127 - exponent) << 23);
#pragma unroll
        for (uint32_t k = 0; k < kD / 32u; k++)
#pragma unroll
            for (uint32_t e2 = 0; e2 < 2u; e2++) {
                const uint32_t x = raw[k][2u * e2], y = raw[k][2u * e2 + 1u];
                const float v[4] = {low(x) * up, high(x) * up, low(y) * up, high(y) * up};
                const uint32_t first = to_bytes(v[0], v[1], v[2], v[3]);
                const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)first, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)first, true);
                q_high[n][k / 4u][k % 4u * 2u + e2] = (int)first;
                q_low[n][k / 4u][k % 4u * 2u + e2] = (int)to_bytes((v[0] - lo[0]) * 32.f, (v[1] - lo[1]) * 32.f, (v[2] - hi[0]) * 32.f, (v[3] - hi[1]) * 32.f);
            }
    }
    const uint32_t sees_least = working ? seen_by(t, w0, a.group) : 0u, sees_most = working ? seen_by(t, w0 + kTile * kTiles < t.last ? w0 + kTile * kTiles - 1u : t.last - 1u, a.group) : 0u;
    Float4 o[kTiles][kParts];
    float base[kTiles], sum[kTiles], up[kTiles];
    bool begun[kTiles];                              // the lane's query has a base
    Bits nans[kTiles];                               // its outputs that have seen a NaN
#pragma unroll
    for (uint32_t n = 0; n < kTiles; n++) {
        base[n] = 0.f; sum[n] = 0.f; up[n] = 0.f; begun[n] = false; nans[n] = 0u;
#pragma unroll
        for (uint32_t p = 0; p < kParts; p++) o[n][p] = Float4{0.f, 0.f, 0.f, 0.f};
    }
    // What a thread brings of a block, sixteen bytes at a time.  A wavefront's keys are among sixteen neighbours, its values those of sixteen, so that it has one page of
    // each, and an address is a page's, in scalar registers, and a place that stays (by lanes, addresses were a third of a block's vector instructions).  A block
    // begins with a page.
    const uint64_t page_bytes = (uint64_t)a.heads * P * kD;
    const uint8_t *k_head = a.k_cache + (size_t)h * P * kD, *v_head = a.v_cache + (size_t)h * P * kD;
    const uint32_t column_step = kBlock >> a.shift;
    uint32_t k_at[kLoads], v_at[kLoads], v_to[kLoads];
#pragma unroll
    for (uint32_t j = 0; j < kLoads; j++) {
        const uint32_t key = (j * kThreads + tid) * 16u / kD, dim = j * 64u + lane;
        k_at[j] = (key & (P - 1u)) * kD + key_place<kD>(key, (j * kThreads + tid) % (kD / 16u)) * 16u;
        v_at[j] = dim * P + (wave * 16u & (P - 1u));
        v_to[j] = dim * 4u + value_place(dim, wave);
    }
    Word4 next_k[kLoads], next_v[kLoads];
    float next_ks = 0.f, next_vs = 0.f;
    uint32_t page_k[kLoads], page_v = 0;
    auto page_at = [&](uint32_t c) { return (uint32_t)table[c < last_column ? c : last_column]; };
    // (what lies behind a row's pages is masked, and must be somewhere.  Looked at where it is used, a block later: where it is asked for that is a wait for all that was asked for
    // before, and took a fifth of the time)
    auto page_of = [&](uint32_t asked) { const uint32_t id = (uint32_t)__builtin_amdgcn_readfirstlane((int)asked); return id < a.pages ? id : 0u; };
    auto ask_pages = [&](uint32_t b) {
        const uint32_t first = b * column_step;
#pragma unroll
        for (uint32_t j = 0; j < kLoads; j++) page_k[j] = page_at(first + ((j * kThreads + wave * 64u) * 16u / kD >> a.shift));
        page_v = page_at(first + (wave * 16u >> a.shift));
    };
    auto ask = [&]() {
#pragma unroll
        for (uint32_t j = 0; j < kLoads; j++) {
            const uint8_t *k_page = k_head + page_of(page_k[j]) * page_bytes;
            next_k[j] = *reinterpret_cast<const Word4 *>(k_page + k_at[j]);
        }
        const uint32_t page = page_of(page_v);
        const uint8_t *v_page = v_head + page * page_bytes;
#pragma unroll
        for (uint32_t j = 0; j < kLoads; j++) next_v[j] = *reinterpret_cast<const Word4 *>(v_page + v_at[j]);
        next_ks = a.k_scale[(size_t)page * a.heads + h];
        next_vs = a.v_scale[(size_t)page * a.heads + h];
    };
    auto put = [&](uint32_t to) {
#pragma unroll
        for (uint32_t j = 0; j < kLoads; j++) {
            keys[to][j * kThreads + tid] = next_k[j];
            values[to][v_to[j]] = next_v[j];
        }
        if (lane == 0u) scales[to][wave] = Float2{next_ks, next_vs};
    };
    // where the lane's keys and values lie in LDS
    const uint32_t key_row = ((m >> 2) * 16u + (m & 3u)) * (kD / 16u), value_row = m * 4u + value_place(m, g);
    // A block of keys; kEdge: some query of the wavefront does not see all of it.
    auto look = [&](uint32_t b, auto edge) {
        constexpr bool kEdge = decltype(edge)::value;
        const uint32_t at = b & 1u, mine = b * kBlock + g * 16u;
        // (a page of zeros may have a scale of zero; what lies behind a row's pages may have any)
        const Float2 scale = scales[at][g];
        const float ks = scale[0];
        auto log_of = [](float vs) { return __builtin_amdgcn_logf(__builtin_fmaxf(vs, 0x1p-64f)); };
        Float4 s[kTiles][4];
        Word4 weights[kTiles][2];
        float part[kTiles], by[kTiles], add[kTiles];
        auto lift_of = [&](uint32_t i, float v_log) { return __builtin_amdgcn_fmed3f(v_log + up[i], kLeastLift, kMostLift); };
#pragma unroll
        for (uint32_t i = 0; i < kTiles; i++) { by[i] = ks * q_scale[i]; add[i] = lift_of(i, log_of(scale[1])) - base[i]; part[i] = 0.f; }
        // The weights of four keys, and their sum.
        auto weigh = [&](uint32_t i, uint32_t n) {
#pragma unroll
            for (uint32_t e = 0; e < 2u; e++) {
                const float x = __builtin_amdgcn_exp2f(s[i][n][2u * e]), y = __builtin_amdgcn_exp2f(s[i][n][2u * e + 1u]);
                part[i] += x;
                part[i] += y;
                weights[i][n / 2u][n % 2u * 2u + e] = pk_f16(x, y);
            }
        };
        // (weights of four keys while the products of the next four are under way)
        Word4 kw[4][kD / 64u];
        auto key_words = [&](uint32_t n, Word4 (&w)[kD / 64u]) {
#pragma unroll
            for (uint32_t j = 0; j < kD / 64u; j++) w[j] = keys[at][key_row + n * 4u * (kD / 16u) + key_place<kD>((m >> 2) * 16u + (m & 3u), g * (kD / 64u) + j)];
        };
#pragma unroll
        for (uint32_t n = 0; n < kAhead; n++) key_words(n, kw[n]);
#pragma unroll
        for (uint32_t n = 0; n < 5u; n++) {
            if (n < 4u) {
                if (n + kAhead < 4u) key_words(n + kAhead, kw[n + kAhead]);
                ds_fence();
#pragma unroll
                for (uint32_t i = 0; i < kTiles; i++) s[i][n] = Float4{0.f, 0.f, 0.f, 0.f};
                if (kBytes) {
#pragma unroll
                    for (uint32_t k = 0; k < kD / 128u; k++) {
                        const Word4 x = kw[n][(2u * k) % (kD / 64u)], y = kw[n][(2u * k + 1u) % (kD / 64u)];
                        const Int8 bytes{(int)x[0], (int)x[1], (int)x[2], (int)x[3], (int)y[0], (int)y[1], (int)y[2], (int)y[3]};
#pragma unroll
                        for (uint32_t i = 0; i < kTiles; i++)        // (scales of 1 and, for the smaller summands, 2^-5)
                            s[i][n] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(bytes, q_low[i][k], s[i][n], 0, 0, 0, 127, 0, 122);
#pragma unroll
                        for (uint32_t i = 0; i < kTiles; i++)
                            s[i][n] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(bytes, q_high[i][k], s[i][n], 0, 0, 0, 127, 0, 127);
                    }
                } else
#pragma unroll
                    for (uint32_t k = 0; k < kSteps; k++) {
                        const Half8 x = widened(kw[n][k / 2u % (kD / 64u)][k % 2u * 2u], kw[n][k / 2u % (kD / 64u)][k % 2u * 2u + 1u]);
#pragma unroll
                        for (uint32_t i = 0; i < kTiles; i++) s[i][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, q_half[i][k % (kBytes ? 1u : kSteps)], s[i][n], 0, 0, 0);
                    }
            }
            if (n)
#pragma unroll
                for (uint32_t i = 0; i < kTiles; i++) {
#pragma unroll
                    for (uint32_t e = 0; e < 4u; e++) {
                        const float x = __builtin_fmaf(s[i][n - 1u][e], by[i], add[i]);
                        s[i][n - 1u][e] = !kEdge || mine + (n - 1u) * 4u + e < sees[i] ? x : -__builtin_inff();
                    }
                    weigh(i, n - 1u);
                }
        }
        // values are asked for some parts ahead
        Word4 words[kParts];
#pragma unroll
        for (uint32_t p = 0; p < kValuesAhead; p++) words[p] = values[at][p * 64u + value_row];
        float terms[kTiles];                         // sums without the scale
        bool moves = false;                          // (a NaN says so too)
#pragma unroll
        for (uint32_t i = 0; i < kTiles; i++) {
            terms[i] = part[i] * __builtin_amdgcn_exp2f(-(add[i] + base[i]));
            moves |= !begun[i] || !(part[i] <= kMostSum) || !(terms[i] <= kMostTerms);
        }
        if (__ballot(moves)) {
            // (Read again but for heads of 128, where registers have room for it until here: a prompt of 512 tokens behind 7,500, heads of 64, 128 and 256, 86, 103 and 125 us
            // with it held, 81, 106 and 118 without.)
            const float v_log = log_of(kD == 128u ? scale[1] : *const_cast<const volatile float *>(reinterpret_cast<const float *>(&scales[at][g]) + 1));
#pragma unroll
            for (uint32_t i = 0; i < kTiles; i++) {
                // log2 of the largest term, and of the largest weight (where the lift is held, of what it were without)
                float term = -__builtin_inff();
#pragma unroll
                for (uint32_t n = 0; n < 4u; n++)
#pragma unroll
                    for (uint32_t e = 0; e < 4u; e++) term = __builtin_fmaxf(term, s[i][n][e]);
                const float was = add[i] + base[i];
                term -= was;
                float weight = term + (v_log + up[i]);
                term = __builtin_fmaxf(term, __shfl_xor(term, 16));
                weight = __builtin_fmaxf(weight, __shfl_xor(weight, 16));
                term = __builtin_fmaxf(term, __shfl_xor(term, 32));
                weight = __builtin_fmaxf(weight, __shfl_xor(weight, 32));
                // the base goes to the largest term, so that none is above 1; weights follow that, but for those that have to come down
                const bool some = term > -__builtin_inff();
                const float by_base = begun[i] ? __builtin_fmaxf(term, 0.f) : some ? term : 0.f;
                const float by_weight = weight > (begun[i] ? kRoom : -__builtin_inff()) ? weight - kAim : 0.f;
                sum[i] *= begun[i] ? __builtin_amdgcn_exp2f(-by_base) : 1.f;
                const float shrink = begun[i] ? __builtin_amdgcn_exp2f(-by_weight) : 1.f;
#pragma unroll
                for (uint32_t p = 0; p < kParts; p++) o[i][p] *= shrink;
                base[i] += by_base;
                up[i] += by_base - by_weight;
                begun[i] = begun[i] || some;
                const float lift = lift_of(i, v_log), change = lift - was - by_base;
                part[i] = 0.f;
#pragma unroll
                for (uint32_t n = 0; n < 4u; n++) { s[i][n] += change; weigh(i, n); }
                terms[i] = part[i] * __builtin_amdgcn_exp2f(-lift);
            }
        }
#pragma unroll
        for (uint32_t i = 0; i < kTiles; i++) sum[i] += terms[i];
        const uint32_t there = !kEdge ? 16u : mine >= len ? 0u : len - mine < 16u ? len - mine : 16u;
        bool nan = false;
#pragma unroll
        for (uint32_t p = 0; p < kParts; p++) {
            Word4 v = words[p];
            if (p + kValuesAhead < kParts) words[p + kValuesAhead] = values[at][(p + kValuesAhead) * 64u + value_row];
            ds_fence();
            if (kEdge) {
                v = first_bytes(v, there);           // what lies behind the row's end must not be NaN times a weight of zero
                const Word4 clean = without_nans(v);
                nan |= differ(clean, v);
                v = clean;
            }
#pragma unroll
            for (uint32_t u = 0; u < 2u; u++) {
                const Short8 x = widened16(v[u * 2u], v[u * 2u + 1u]);
#pragma unroll
                for (uint32_t i = 0; i < kTiles; i++) o[i][p] = __builtin_amdgcn_mfma_f32_16x16x32_f16(x, __builtin_bit_cast(Short8, weights[i][u]), o[i][p], 0, 0, 0);
            }
        }
        // a NaN among the values reaches the queries that see it, and as a weight of zero times it no other
        if (kEdge && __ballot(nan))
#pragma nounroll
            for (uint32_t p = 0; p < kParts; p++) {
                const Word4 v = first_bytes(values[at][p * 64u + value_row], there);
#pragma unroll
                for (uint32_t i = 0; i < kTiles; i++) nans[i] |= (Bits)nans_seen(v, mine >= sees[i] ? 0u : sees[i] - mine < 16u ? sees[i] - mine : 16u) << (4u * p);
            }
    };
    if (b0 < blocks) {
        ask_pages(b0);
        ask();
        if (b0 + 1u < blocks) ask_pages(b0 + 1u);
        put(b0 & 1u);
    }
    // Blocks that all queries of the wavefront see, then the others, in loops of their own: registers that the second has no room for must not be waited for in the first.
    // (The wavefronts meet at a barrier for every block, in whichever loop each is.)
    const uint32_t whole = sees_least / kBlock < blocks ? sees_least / kBlock : blocks;
    auto step = [&](uint32_t b, auto edge) {
        __syncthreads();
        if (b + 1u < blocks) {
            ask();
            if (b + 2u < blocks) ask_pages(b + 2u);
        }
        if (!decltype(edge)::value || b * kBlock < sees_most) look(b, edge);
        if (b + 1u < blocks) put(b & 1u ^ 1u);       // (its last reader is behind this round's barrier)
    };
    uint32_t b = b0;
#pragma nounroll
    for (; b < whole; b++) step(b, No{});
#pragma nounroll
    for (; b < blocks; b++) step(b, Yes{});
#pragma unroll
    for (uint32_t i = 0; i < kTiles; i++) {
        float total = sum[i];
        total += __shfl_xor(total, 16);
        total += __shfl_xor(total, 32);
        const uint32_t r = w0 + i * kTile + m;
        if (r >= t.last) continue;
        const size_t row = (size_t)(t.begin + r / a.group) * (a.heads * a.group) + h * a.group + r % a.group;
        const float by = total > 0.f ? 1.f / total : total == total ? 0.f : total, down = __builtin_amdgcn_exp2f(up[i] * -0.5f);      // (a row that sees nothing: zeros; down twice, as its square may be below all numbers)
        auto out_at = [&](uint32_t p, uint32_t e) { return nans[i] >> (4u * p + e) & 1u ? __builtin_nanf("") : o[i][p][e] * by * down * down; };
        if (shares > 1u) {
            float *to = a.partial + (row * a.splits + split) * (kD + 2u);
#pragma unroll
            for (uint32_t p = 0; p < kParts; p++)
#pragma unroll
                for (uint32_t e = 0; e < 4u; e += 2u) *reinterpret_cast<Float2 *>(to + p * 16u + g * 4u + e) = Float2{out_at(p, e), out_at(p, e + 1u)};
            if (g == 0u) *reinterpret_cast<Float2 *>(to + kD) = Float2{begun[i] ? base[i] : -__builtin_inff(), total};
            continue;
        }
        uint16_t *out = a.out + row * kD + g * 4u;
#pragma unroll
        for (uint32_t p = 0; p < kParts; p++) *reinterpret_cast<Word2 *>(out + p * 16u) = Word2{pk_bf16(out_at(p, 0u), out_at(p, 1u)), pk_bf16(out_at(p, 2u), out_at(p, 3u))};
    }
}

static uint32_t tiles_of(uint32_t tokens, uint32_t rows, uint32_t group) { return (uint32_t)((uint64_t)tokens * group / kTile) + rows; }

// Whether requests have query rows enough, on average, for the kernel that holds many of them, which costs a request with few as much as one with its tile full.  With 8
// heads of 128 and 4 query heads each, 32 rows of 2,000 tokens took 40 us in the other one and 51 in this for 16 query rows each, 55 and 52 for 32, 92 and 70 for
// 64, 188 and 115 for 256; 4 such rows 16 and 23 for 32, 24 and 24 for 64, 42 and 38 for 256.  Heads of 64, whose scores come from bfloat16 in both: 33 and 38 for 32, 54 and 54 for 64.
static bool attend_is_wide(uint32_t tokens, uint32_t rows, uint32_t group, uint32_t dim) { return (uint64_t)tokens * group >= (dim == 64u ? 64ull : 32ull) * rows; }

// Whether a launch holds the call: below 2^32 threads to a dimension of the grid.
bool attend_fits(uint32_t tokens, uint32_t rows, uint32_t heads, uint32_t group, uint32_t dim)
{
    const uint64_t most = 0xFFFFFFu, all = (uint64_t)tokens * group;
    return attend_is_wide(tokens, rows, group, dim) ? (all / (kTile * kAttendWaves) + rows) * heads <= most : all / kTile + rows <= most;
}

// Blocks that a share has at least: a share more is partial results of all query rows to write and read, and a second kernel.  With 4 blocks, one for each wavefront, 256 rows of 300 tokens
// took 48 us for 38 with 16, and 4 rows of 2,000 11.7 for 14.3.  Prompts, whose shares take longer for as many blocks: a prompt of 1,000 tokens, 32 query heads over 8, took 31 us
// in one share and 45 in two of 8 blocks; 16 new tokens of each of 4 rows of 2,000 33 us in shares of 16 blocks and 24 of 8.
static uint32_t least_blocks(uint32_t tokens, uint32_t rows, uint32_t heads, uint32_t group, uint32_t dim)
{
    return attend_is_wide(tokens, rows, group, dim) && (uint64_t)tokens * group * heads <= kFewRows ? kLeastBlocks / 2u : kLeastBlocks;
}

// The most shares of a tile's keys.  Where each row's keys in one share make four times as many workgroups as there are to be shares, the chip evens them out by itself; else a row may
// have four times its part of them, 64 at most.  Prompts are cut where they leave half of the chip or more idle, to fill it: 64 query rows of each of 8 heads behind 20,000 tokens took 407 us in one share, 31 in 39; a prompt of
// 512 tokens behind 7,500, 175 and 104 in three.
uint32_t attend_splits(uint32_t tokens, uint32_t rows, uint32_t heads, uint32_t group, uint32_t dim, uint32_t columns, uint32_t shift)
{
    if (rows > 1024u) return 1u;
    const uint64_t blocks = (((uint64_t)columns << shift) + kBlock - 1u) / kBlock, requests = tokens < rows ? tokens : rows;
    const bool many = attend_is_wide(tokens, rows, group, dim);
    const uint64_t least = least_blocks(tokens, rows, heads, group, dim), most = (blocks + least - 1u) / least;
    uint64_t want;
    if (many) want = kWideShares / (((uint64_t)tokens * group / wide_rows(dim) + requests) * heads);
    else {
        const uint64_t tiles = requests * ((group + kTile - 1u) / kTile) * heads;
        const uint64_t all = tokens > rows ? (uint64_t)tokens * group / kTile * heads : tiles, n = all > tiles ? all : tiles;
        want = n >= 4u * kShares ? 1u : 4u * ((kShares + n - 1u) / n);
    }
    const uint64_t splits = want < most ? want : most;
    return splits < 1u ? 1u : splits > 64u ? 64u : (uint32_t)splits;
}

hipError_t launch_cache_attend(const void *q, uint32_t tokens, uint32_t heads, uint32_t group, uint32_t dim, int64_t q_token, int64_t q_head, const uint8_t *k_cache,
                               const uint8_t *v_cache, const float *k_scale, const float *v_scale, uint32_t pages, uint32_t shift, const int32_t *table,
                               uint32_t rows, uint32_t columns, const int32_t *lens, const int32_t *starts, float scale, void *out, void *workspace, hipStream_t s)
{
    const uint32_t splits = attend_splits(tokens, rows, heads, group, dim, columns, shift);
    const AttendArgs a{static_cast<const uint16_t *>(q), q_token, q_head, k_cache, v_cache, k_scale, v_scale, table, lens, starts, static_cast<uint16_t *>(out),
                       static_cast<float *>(workspace), splits > 1u ? static_cast<uint32_t *>(workspace) + (size_t)tokens * heads * group * splits * (dim + 2u) : nullptr,
                       scale * 1.44269504088896340736f, tokens, rows, heads, group, columns, pages, shift, splits,
                       least_blocks(tokens, rows, heads, group, dim)};
    const dim3 block(kAttendWaves * 64u);
    hipError_t e;
    if (attend_is_wide(tokens, rows, group, dim)) {
        const dim3 wide(((uint32_t)((uint64_t)tokens * group / wide_rows(dim)) + rows) * heads, splits);
        e = launch(dim == 64u ? attend_wide_kernel<64, 2> : dim == 128u ? attend_wide_kernel<128, 2> : attend_wide_kernel<256, 1>, wide, block, 0, s, nullptr, a);
    } else e = launch(dim == 64u ? attend_kernel<64> : dim == 128u ? attend_kernel<128> : attend_kernel<256>, dim3(tiles_of(tokens, rows, group), heads, splits), block, 0, s, nullptr, a);
    if (e != hipSuccess || splits == 1u) return e;
    const bool many = splits > 16u;                  // more than a wavefront takes
    const dim3 joins(tokens, many ? heads * group : (heads * group + 3u) / 4u);
    return launch(dim == 64u ? (many ? attend_join_kernel<64, 4> : attend_join_kernel<64, 1>) : dim == 128u ? (many ? attend_join_kernel<128, 4> : attend_join_kernel<128, 1>)
                  : many ? attend_join_kernel<256, 4> : attend_join_kernel<256, 1>, joins, dim3(256), 0, s, nullptr, a);
}

}  // namespace wg
