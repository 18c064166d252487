// A cache of latent vectors for gfx950: of every token one vector of C numbers that all heads share, and a shared key of 64 numbers that carries the position.  Pages of P
// tokens: latent vectors [page][token][C] in bfloat16, or in 8 bits with a scale for each token, [page][token]; shared keys [page][token][64] in bfloat16.
#include <hip/hip_runtime.h>

#include "wg_launch.h"
#include "wg_number.h"
#include "wg_serve.h"

namespace wg {

constexpr uint32_t kLatentThreads = 256, kLatentWaves = 4, kNoToken = 0xFFFFFFFFu;

// ---------------------------------------------------------------------------------------------
// append.  A wavefront for each token, or, of many in 16 bits, for four, all asked for at once (20,000 of 512 numbers 9.2 us for 10.6; in 8 bits 11.1 for 10.3).  A token has a scale of its own, so nothing that is in the
// cache is rounded again; what comes along from another page is copied as it is, by all wavefronts of the workgroup (63 tokens at the most, of 644 bytes in 8 bits and 1,152 in 16, with 512 numbers).  Up to 1,024 tokens a workgroup has
// one, so that such copies go side by side (pages of 64, four beams to a request, 8 and 16 bits: 256 rows 4.8 us and 7.7, with four tokens to a workgroup 8.2 and 10.2; 1,024 rows 9.0 and 12.8, with four 11.2 and 15.0; 2,048 rows in 8 bits 14.6, with four 12.8).
// Bound by memory: 16 prompts, 21,000 tokens in 8 bits, 9.8 us, 4.4 TB/s; a token for each of 256 rows 4.8 us, of which 3 are a launch's.
struct LatentAppendArgs {
    const uint16_t *c, *r;
    int64_t c_token, r_token;                        // strides, elements
    const int32_t *slots, *origins;
    uint8_t *c_cache;
    uint16_t *r_cache;
    float *scale;
    uint32_t tokens, pages, shift, per;              // per: tokens of a workgroup
};

__device__ __forceinline__ void copy_words(void *to, const void *from, uint32_t words, uint32_t tid)
{
#pragma unroll 4
    for (uint32_t i = tid; i < words; i += kLatentThreads) static_cast<Word4 *>(to)[i] = static_cast<const Word4 *>(from)[i];
}

template <uint32_t kC, bool kBytes, uint32_t kTokens>
__global__ void __launch_bounds__(kLatentThreads)
latent_append_kernel(const LatentAppendArgs a)
{
    constexpr uint32_t kOwn = kC / 64u, kWords = kOwn / 2u, kRow = kC * (kBytes ? 1u : 2u);               // dims of a lane; words; bytes of a token
    const uint32_t tid = threadIdx.x, lane = tid & 63u, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const uint32_t first = blockIdx.x * a.per;
    uint32_t slot[kTokens], w[kTokens][kWords], r[kTokens];
#pragma unroll
    for (uint32_t k = 0; k < kTokens; k++) {
        const uint32_t t = first + wave * kTokens + k;
        const bool there = wave * kTokens + k < a.per && t < a.tokens;
        const uint32_t at = there ? t : first;
        slot[k] = there ? (uint32_t)a.slots[at] : kNoToken;
        const uint32_t *x = reinterpret_cast<const uint32_t *>(a.c + (int64_t)at * a.c_token) + lane * kWords;
#pragma unroll
        for (uint32_t i = 0; i < kWords; i++) w[k][i] = x[i];
        r[k] = reinterpret_cast<const uint32_t *>(a.r + (int64_t)at * a.r_token)[lane & 31u];
    }
#pragma unroll
    for (uint32_t k = 0; k < kTokens; k++) {
        if (slot[k] >> a.shift >= a.pages) continue;
        uint32_t *to = reinterpret_cast<uint32_t *>(a.c_cache + (size_t)slot[k] * kRow) + lane * (kRow / 256u);
        if (kBytes) {
            float top = 0.f;
#pragma unroll
            for (uint32_t i = 0; i < kWords; i++) { top = top_of(top, low(w[k][i])); top = top_of(top, high(w[k][i])); }
#pragma unroll
            for (int s = 32; s > 0; s >>= 1) top = __builtin_fmaxf(top, __shfl_xor(top, s));
            const float scale = scale_for(top), inverse = 1.f / scale;
            if (lane == 0u) a.scale[slot[k]] = scale;
#pragma unroll
            for (uint32_t i = 0; i < kOwn / 4u; i++)
                to[i] = to_bytes(low(w[k][2u * i]) * inverse, high(w[k][2u * i]) * inverse, low(w[k][2u * i + 1u]) * inverse, high(w[k][2u * i + 1u]) * inverse);
        } else
#pragma unroll
            for (uint32_t i = 0; i < kWords; i++) to[i] = w[k][i];
        if (lane < 32u) reinterpret_cast<uint32_t *>(a.r_cache + (size_t)slot[k] * kLatentKey)[lane] = r[k];
    }
    if (!a.origins) return;
    // tokens whose page has begun in another one: a lane looks at each
    const uint32_t own = lane < a.per && first + lane < a.tokens ? first + lane : kNoToken;
    const uint32_t own_origin = own != kNoToken ? (uint32_t)a.origins[own] : kNoToken, own_slot = own != kNoToken ? (uint32_t)a.slots[own] : kNoToken;
    const bool taken = own_origin < a.pages && own_slot >> a.shift < a.pages && (own_slot & ((1u << a.shift) - 1u)) && own_origin != own_slot >> a.shift;
    for (unsigned long long left = __ballot(taken); left; left &= left - 1ull) {
        const uint32_t i = (uint32_t)__builtin_ctzll(left), origin = __builtin_amdgcn_readlane(own_origin, i), at = __builtin_amdgcn_readlane(own_slot, i), o = at & ((1u << a.shift) - 1u);
        const size_t from = (size_t)origin << a.shift, to = (size_t)(at >> a.shift) << a.shift;
        copy_words(a.c_cache + to * kRow, a.c_cache + from * kRow, o * (kRow / 16u), tid);
        copy_words(a.r_cache + to * kLatentKey, a.r_cache + from * kLatentKey, o * (kLatentKey / 8u), tid);
        if (kBytes && tid < o) a.scale[to + tid] = a.scale[from + tid];
    }
}

constexpr uint32_t kMostGroups = 0xFFFFFFFFu / kLatentThreads;              // workgroups of a launch
static uint32_t groups_of(uint32_t tokens, uint32_t per) { return (uint32_t)(((uint64_t)tokens + per - 1u) / per); }
static bool many_tokens(uint32_t tokens, bool bytes) { return !bytes && tokens > 16384u; }
static uint32_t tokens_of_workgroup(uint32_t tokens, bool bytes) { return tokens <= 1024u ? 1u : kLatentWaves * (many_tokens(tokens, bytes) ? 4u : 1u); }
bool latent_append_fits(uint32_t tokens, bool bytes) { return groups_of(tokens, tokens_of_workgroup(tokens, bytes)) <= kMostGroups; }

hipError_t launch_latent_append(const void *c, const void *r, uint32_t tokens, uint32_t latent, int64_t c_token, int64_t r_token, const int32_t *slots, const int32_t *origins,
                                void *c_cache, void *r_cache, float *scale, uint32_t pages, uint32_t shift, hipStream_t s)
{
    const bool many = many_tokens(tokens, scale != nullptr);
    const uint32_t per = tokens_of_workgroup(tokens, scale != nullptr);
    const LatentAppendArgs a{static_cast<const uint16_t *>(c), static_cast<const uint16_t *>(r), c_token, r_token, slots, origins, static_cast<uint8_t *>(c_cache),
                             static_cast<uint16_t *>(r_cache), scale, tokens, pages, shift, per};
    const dim3 grid(groups_of(tokens, per)), block(kLatentThreads);
    if (many) return launch(latent == 512u ? latent_append_kernel<512, false, 4> : latent_append_kernel<256, false, 4>, grid, block, 0, s, nullptr, a);
    return launch(latent == 512u ? (scale ? latent_append_kernel<512, true, 1> : latent_append_kernel<512, false, 1>) : scale ? latent_append_kernel<256, true, 1> : latent_append_kernel<256, false, 1>,
                  grid, block, 0, s, nullptr, a);
}

// ---------------------------------------------------------------------------------------------
// read.  A wavefront takes four tokens behind one another, all asked for at once; a lane of it finds a token's row and slot.  Bound by memory: 160,000 tokens in 8 bits, 512 numbers, 58.5 us, 5.0 TB/s, as fast as
// a copy (with 16 tokens to a wavefront 62, and one row of 500 7.8 for 3.4; with 8 a row of 500 4.4).
constexpr uint32_t kReadTokens = 4;
struct LatentReadArgs {
    const uint8_t *c_cache;
    const uint16_t *r_cache;
    const float *scale;
    const int32_t *table, *starts;
    uint16_t *c_out, *r_out;
    int64_t c_token, r_token;
    uint32_t rows, columns, tokens, pages, shift;
};
// 8 or 16 bytes of a lane, past the caches' own.
template <uint32_t kN>
__device__ __forceinline__ void stream_words(uint32_t *to, const uint32_t (&w)[kN])
{
    if (kN == 4u) __builtin_nontemporal_store(Word4{w[0], w[1], w[2 % kN], w[3 % kN]}, reinterpret_cast<Word4 *>(to));
    else __builtin_nontemporal_store(Word2{w[0], w[1]}, reinterpret_cast<Word2 *>(to));
}

template <uint32_t kC, bool kBytes>
__global__ void __launch_bounds__(kLatentThreads)
latent_read_kernel(const LatentReadArgs a)
{
    constexpr uint32_t kOwn = kC / 64u, kRow = kC * (kBytes ? 1u : 2u), kWords = kRow / 256u;
    const uint32_t tid = threadIdx.x, lane = tid & 63u, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const uint32_t base = (blockIdx.x * kLatentWaves + wave) * kReadTokens, t = base + lane;
    // the last row that begins at the token or before
    uint32_t slot = 0xFFFFFFFFu;
    bool there = lane < kReadTokens && t < a.tokens && t < (uint32_t)a.starts[a.rows] && t >= (uint32_t)a.starts[0];
    if (there) {
        uint32_t lo = 0, n = a.rows;
        while (n > 1u) { const uint32_t half = n / 2u; if ((uint32_t)a.starts[lo + half] <= t) { lo += half; n -= half; } else n = half; }
        const uint32_t i = t - (uint32_t)a.starts[lo], column = i >> a.shift;
        if (column < a.columns) {
            const uint32_t page = (uint32_t)a.table[(size_t)lo * a.columns + column];
            if (page < a.pages) slot = page << a.shift | (i & ((1u << a.shift) - 1u));
        }
    }
    const uint32_t known = (uint32_t)__ballot(there);
    const float own_scale = kBytes && slot != 0xFFFFFFFFu ? a.scale[slot] : 0.f;
    uint32_t w[kReadTokens][kWords], r[kReadTokens];
#pragma unroll
    for (uint32_t i = 0; i < kReadTokens; i++) {
        const uint32_t at = __builtin_amdgcn_readlane(slot, i);
        const bool real = at != 0xFFFFFFFFu;
        const uint32_t *from = reinterpret_cast<const uint32_t *>(a.c_cache + (size_t)(real ? at : 0u) * kRow) + lane * kWords;
#pragma unroll
        for (uint32_t k = 0; k < kWords; k++) w[i][k] = real ? from[k] : 0u;
        r[i] = real && lane < 32u ? reinterpret_cast<const uint32_t *>(a.r_cache + (size_t)at * kLatentKey)[lane] : 0u;
    }
#pragma unroll
    for (uint32_t i = 0; i < kReadTokens; i++) {
        if (!(known >> i & 1u)) continue;
        uint32_t *to = reinterpret_cast<uint32_t *>(a.c_out + (int64_t)(base + i) * a.c_token) + lane * (kOwn / 2u), out[kOwn / 2u];
        if (kBytes) {
            const float scale = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(own_scale), i));
#pragma unroll
            for (uint32_t k = 0; k < kWords; k++) {
                const auto x = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[i][k], false), y = __builtin_amdgcn_cvt_pk_f32_fp8((int)w[i][k], true);
                out[2u * k] = pk_bf16(x[0] * scale, x[1] * scale);
                out[2u * k + 1u] = pk_bf16(y[0] * scale, y[1] * scale);
            }
        } else
#pragma unroll
            for (uint32_t k = 0; k < kWords; k++) out[k % (kOwn / 2u)] = w[i][k];
        stream_words<kOwn / 2u>(to, out);
        if (lane < 32u) reinterpret_cast<uint32_t *>(a.r_out + (int64_t)(base + i) * a.r_token)[lane] = r[i];
    }
}

bool latent_read_fits(uint32_t tokens) { return groups_of(tokens, kLatentWaves * kReadTokens) <= kMostGroups; }

hipError_t launch_latent_read(const void *c_cache, const void *r_cache, const float *scale, uint32_t latent, uint32_t pages, uint32_t shift, const int32_t *table, uint32_t rows,
                              uint32_t columns, const int32_t *starts, uint32_t tokens, void *c_out, int64_t c_token, void *r_out, int64_t r_token, hipStream_t s)
{
    const LatentReadArgs a{static_cast<const uint8_t *>(c_cache), static_cast<const uint16_t *>(r_cache), scale, table, starts, static_cast<uint16_t *>(c_out),
                           static_cast<uint16_t *>(r_out), c_token, r_token, rows, columns, tokens, pages, shift};
    const dim3 grid(groups_of(tokens, kLatentWaves * kReadTokens)), block(kLatentThreads);
    return launch(latent == 512u ? (scale ? latent_read_kernel<512, true> : latent_read_kernel<512, false>) : scale ? latent_read_kernel<256, true> : latent_read_kernel<256, false>,
                  grid, block, 0, s, nullptr, a);
}

}  // namespace wg
