// Attention with keys and values from one latent vector a token, for gfx950: over the paged cache of the vectors themselves (latent_attend_kernel), and over the
// keys and values of every head made from them beforehand (latent_prompt_kernel).
//
// Both take their products as attention over the 8-bit cache does: scores as S^T = K Q^T (rows: keys), so that the lane that holds the scores of eight keys of a query after the first product is
// the one that needs their weights in the second, O^T = V^T P^T.  The keys that a row of the first product's tiles stands for are numbered for that: lane l of 64, with
// m = l % 16 and g = l / 16, holds for query m the scores of keys 8 g .. 8 g + 7 of 32.  Keys lie in LDS as rows, and the second product's operand, eight keys of one dim, is read from there
// by the transposing read: sixteen lanes that ask for four rows of sixteen numbers get a column of four each.
//
// The softmax is taken in one pass: weights e = 2^(score - base) relative to a base that moves only where a score is 8 above it, by their wavefront as a whole; so it
// costs no exchange between lanes but where it moves.  Weights are rounded to bfloat16, as the values are that they multiply (values go as far as 2^127, which float16 would not hold), and
// their sum, in fp32, is that of the rounded ones: weights off by 2^-8 at the most, by as much as the output's own rounding.
#include <hip/hip_runtime.h>

#include "wg_launch.h"
#include "wg_number.h"
#include "wg_serve.h"

namespace wg {

typedef short Short4 __attribute__((ext_vector_type(4)));
typedef uint32_t Word __attribute__((may_alias));

constexpr uint32_t kThreads = 256, kWaves = 4, kTop = 64;
constexpr float kLift = 8.f;                         // how far above the base a score may be, log2
constexpr uint32_t kNone = 0xFFFFFFFFu;

// Requests and their tokens: query rows [starts[r], starts[r + 1]) of request r are its last ones.
struct Requests {
    const int32_t *starts;
    uint32_t rows, tokens, heads, splits, least;     // splits: the most shares of a row's keys; least: blocks of a share
};

// Where a tile of kRows query rows lies (`heads` rows to a token): request r's tiles begin at starts[r] * heads / kRows + r, which leaves room for each one's last, begun tile.  A
// wavefront asks 64 requests at a time.
struct Tile { uint32_t row, first, last, begin; int32_t before; };         // query rows [first, last) of request `row`, its tokens those from `begin` on, behind `before` others

template <uint32_t kRows>
__device__ __forceinline__ bool tile_of(const Requests &a, uint32_t heads, uint32_t tile, Tile *out, uint32_t *count)
{
    const uint32_t lane = threadIdx.x & 63u;
    auto start = [&](uint32_t r) { const uint32_t t = (uint32_t)a.starts[r]; return t < a.tokens ? t : a.tokens; };
    auto begins = [&](uint32_t r) { return (uint32_t)((uint64_t)start(r) * heads / kRows) + r; };
    uint32_t lo = 0, n = a.rows;
    while (n > 1u) {
        const uint32_t step = (n + 63u) / 64u, r = lo + lane * step;
        const bool at = lane * step < n && begins(r) <= tile;
        const uint32_t k = 63u - (uint32_t)__builtin_clzll(__ballot(at) | 1ull);
        n = n - k * step < step ? n - k * step : step;
        lo += k * step;
    }
    lo = __builtin_amdgcn_readfirstlane(lo);
    const uint32_t b = start(lo), e0 = (uint32_t)a.starts[lo + 1u], e = e0 < b ? b : e0 < a.tokens ? e0 : a.tokens, first_tile = begins(lo), all = (e - b) * heads;
    if (tile < first_tile || (uint64_t)(tile - first_tile) * kRows >= all) return false;
    out->row = lo; out->begin = b;
    out->first = (tile - first_tile) * kRows;
    out->last = all - out->first < kRows ? all : out->first + kRows;
    *count = e0 < b ? 0u : e0 - b;                   // (with the request's tokens that the call does not have)
    return true;
}

// Blocks of keys to a share: shares of one size, whatever the rows' lengths, so that the workgroups have as much to do as one another.  The number follows from the row and not from the tile,
// as a token's rows may lie in two tiles.  tiles(r): query tiles of row r; blocks(r): blocks of its keys.
template <typename F>
__device__ __forceinline__ uint32_t shares_of(const Requests &a, uint32_t blocks, uint32_t *per, F work_of)
{
    *per = blocks;
    if (a.splits == 1u || !blocks) return 1u;
    uint64_t all = 0;
    for (uint32_t r = threadIdx.x & 63u; r < a.rows; r += 64u) all += work_of(r);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) all += __shfl_xor(all, o);
    uint64_t share64 = (all + kAttendShares - 1u) / kAttendShares;
    uint32_t share = __builtin_amdgcn_readfirstlane((uint32_t)(share64 < blocks ? share64 : blocks));
    share = share < a.least ? a.least : share;
    const uint32_t want = (blocks + share - 1u) / share, n = want < a.splits ? want : a.splits;
    *per = (blocks + n - 1u) / n;
    return (blocks + *per - 1u) / *per;
}

// Four rows' sixteen numbers, a column of four to each lane: `at` is the lane's four of a row.
__device__ __forceinline__ Short4 column_of(const uint16_t *at)
{
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) Short4 *)at);
}
__device__ __forceinline__ Half8 both(Short4 a, Short4 b)
{
    typedef short Short8s __attribute__((ext_vector_type(8)));
    return __builtin_bit_cast(Half8, Short8s{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]});
}
// Eight numbers in 8 bits, times a power of two: exactly.
__device__ __forceinline__ Word2 wider(uint32_t four, float scale)
{
    return Word2{__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(four, scale, false)),
                 __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(four, scale, true))};
}
// Numbers that are none or infinite, as bits: an exponent of ones carries into the sign's place.
__device__ __forceinline__ uint32_t odd_bits(uint32_t two) { return ((two & 0x7F807F80u) + 0x00800080u) & 0x80008000u; }
__device__ __forceinline__ bool any_odd(Word4 v) { return (odd_bits(v[0]) | odd_bits(v[1]) | odd_bits(v[2]) | odd_bits(v[3])) != 0u; }
// Eight numbers of key `key` with zeros in the place of those; `from` keeps the first key that has one.
__device__ __forceinline__ Word4 without_odd(Word4 v, uint32_t key, uint32_t *from)
{
    if (any_odd(v)) atomicMin(from, key);
#pragma unroll
    for (uint32_t w = 0; w < 4u; w++) { const uint32_t b = odd_bits(v[w]); v[w] &= ~(b | (b - (b >> 15))); }
    return v;
}
// The same for each dim by itself, from dim d on.
__device__ __forceinline__ Word4 without_odd_dims(Word4 v, uint32_t key, uint32_t d, uint32_t *from)
{
    if (!any_odd(v)) return v;
#pragma unroll
    for (uint32_t w = 0; w < 4u; w++) {
        const uint32_t b = odd_bits(v[w]);
        if (b & 0x8000u) atomicMin(from + d + 2u * w, key);
        if (b >> 31) atomicMin(from + d + 2u * w + 1u, key);
        v[w] &= ~(b | (b - (b >> 15)));
    }
    return v;
}

// What is read in the place of a key that there is none of.
__device__ __attribute__((aligned(16))) const uint8_t kZeros[1024] = {};

// What a wavefront holds of its kM tiles of 16 queries: of query m of each, the base and its own part of the sum, and outputs, dims 4 g .. 4 g + 3 of each of kParts.
template <uint32_t kM, uint32_t kParts>
struct Sums {
    Float4 acc[kParts][kM];
    float base[kM], sum[kM];
    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (uint32_t t = 0; t < kM; t++) {
            base[t] = -__builtin_inff(); sum[t] = 0.f;
#pragma unroll
            for (uint32_t d = 0; d < kParts; d++) acc[d][t] = Float4{0.f, 0.f, 0.f, 0.f};
        }
    }
    // Scores (log2, -inf where nothing is seen) of kGroups times 32 keys into weights.
    template <uint32_t kGroups>
    __device__ __forceinline__ void weigh(const float (&s)[kGroups][kM][8], Half8 (&p)[kGroups][kM])
    {
        float top[kM];
        bool grows = false;
#pragma unroll
        for (uint32_t t = 0; t < kM; t++) {
            top[t] = -__builtin_inff();
#pragma unroll
            for (uint32_t k = 0; k < kGroups; k++)
#pragma unroll
                for (uint32_t j = 0; j < 8u; j++) top[t] = __builtin_fmaxf(top[t], s[k][t][j]);
            grows = grows || top[t] > base[t] + kLift;
        }
        if (__ballot(grows)) {
#pragma unroll
            for (uint32_t t = 0; t < kM; t++) {
                float n = __builtin_fmaxf(top[t], __shfl_xor(top[t], 16));
                n = __builtin_fmaxf(base[t], __builtin_fmaxf(n, __shfl_xor(n, 32)));
                const float by = base[t] > -__builtin_inff() ? __builtin_amdgcn_exp2f(base[t] - n) : 0.f;
                base[t] = n; sum[t] *= by;
#pragma unroll
                for (uint32_t d = 0; d < kParts; d++) acc[d][t] *= by;
            }
        }
#pragma unroll
        for (uint32_t t = 0; t < kM; t++) {
            const float from = base[t] > -__builtin_inff() ? base[t] : 0.f;
#pragma unroll
            for (uint32_t k = 0; k < kGroups; k++) {
                Word4 w;
#pragma unroll
                for (uint32_t j = 0; j < 4u; j++) {
                    w[j] = pk_bf16(__builtin_amdgcn_exp2f(s[k][t][2u * j] - from), __builtin_amdgcn_exp2f(s[k][t][2u * j + 1u] - from));
                    sum[t] += low(w[j]) + high(w[j]);
                }
                p[k][t] = __builtin_bit_cast(Half8, w);
            }
        }
    }
    // The queries' sums over all lanes.
    __device__ __forceinline__ float whole_sum(uint32_t t) const
    {
        const float l = sum[t] + __shfl_xor(sum[t], 16);
        return l + __shfl_xor(l, 32);
    }
};

// What a sum makes of an output: 1 / sum; zeros for a query that sees no key, and none for one whose scores are all -inf.
__device__ __forceinline__ float share_of_sum(float sum, bool sees) { return sum > 0.f ? 1.f / sum : sum == 0.f && !sees ? 0.f : __builtin_nanf(""); }
constexpr float kEmpty = -1.f;                       // the sum of a share in which a query sees keys whose scores are all -inf

// ---------------------------------------------------------------------------------------------
// Attention over the cached vectors.  A workgroup takes 16 * kM * kGroups query rows (tokens times heads) of a request and a share of its keys; its wavefronts are kGroups groups of rows
// times 4 / kGroups groups of keys.  All keys of a block, 32 for each group, go through LDS: from memory into registers, while the block before is worked on, and turned into bfloat16 (exactly) on the way.
struct LatentAttendArgs {
    Requests of;
    const uint16_t *q_c, *q_r;
    int64_t c_token, c_head, r_token, r_head;        // strides of queries, elements
    const uint8_t *c_cache;
    const uint16_t *r_cache;
    const float *scale;                              // of each token; null: the vectors are bfloat16
    const int32_t *table, *lens;
    uint16_t *out;                                   // [token][head][C]
    float *partial, *ends;                           // [token][head][split][C]; [token][head][split][2]: base and sum
    uint32_t *shares;                                // [token]: shares of its keys
    float factor;                                    // of the scores, times log2(e)
    uint32_t columns, pages, shift;
};

__device__ __forceinline__ uint32_t cached_tokens(const LatentAttendArgs &a, uint32_t r)
{
    const uint32_t most = a.columns << a.shift, l = (uint32_t)(a.lens[r] < 0 ? 0 : a.lens[r]);
    return l < most ? l : most;
}

template <uint32_t kC, bool kBytes, uint32_t kM, uint32_t kGroups, uint32_t kW>
__global__ void __launch_bounds__(kW * 64u) __attribute__((amdgpu_waves_per_eu(kW / 4u, kW / 4u)))
latent_attend_kernel(const LatentAttendArgs a)
{
    constexpr uint32_t kKeyGroups = kW / kGroups, kKeys = 32u * kKeyGroups, kRows = 16u * kM * kGroups;
    constexpr uint32_t kSteps = (kC + kTop) / 32u, kParts = kC / 16u, kPitch = kC + kTop + 8u;
    constexpr uint32_t kRow = kC * (kBytes ? 1u : 2u), kPer = 1024u / kRow, kStage = kKeys / kW;          // bytes of a vector; keys of a wavefront's load; keys that it brings
    constexpr uint32_t kLoads = kStage / kPer, kTops = (kStage + 7u) / 8u;
    constexpr uint32_t kJoinPitch = kC + 4u, kTileBytes = kKeys * kPitch * 2u, kJoinBytes = kKeyGroups > 1u ? kW * 16u * kJoinPitch * 4u : 0u;
    __shared__ __attribute__((aligned(16))) uint8_t room[kTileBytes > kJoinBytes ? kTileBytes : kJoinBytes];
    __shared__ uint32_t odd_from;                                          // the first key with a number that is none, of those that some rows do not see
    __shared__ float join_base[kW][16], join_sum[kW][16];
    uint16_t *keys = reinterpret_cast<uint16_t *>(room);
    const uint32_t tid = threadIdx.x, lane = tid & 63u, wave = __builtin_amdgcn_readfirstlane(tid >> 6), m = lane & 15u, g = lane >> 4;
    const uint32_t split = blockIdx.y, P = 1u << a.shift, heads = a.of.heads;
    Tile t;
    uint32_t count;
    if (!tile_of<kRows>(a.of, heads, blockIdx.x, &t, &count)) return;
    const uint32_t len = cached_tokens(a, t.row);
    t.before = (int32_t)len - (int32_t)count;
    uint32_t per;
    const uint32_t shares = shares_of(a.of, (len + kAttendBlock - 1u) / kAttendBlock, &per, [&](uint32_t r) {
        const uint32_t n = (uint32_t)a.of.starts[r + 1u] - (uint32_t)a.of.starts[r];
        return (uint64_t)((cached_tokens(a, r) + kAttendBlock - 1u) / kAttendBlock) * (((uint64_t)n * heads + kRows - 1u) / kRows);
    });
    if (a.of.splits > 1u && split == 0u && tid < kRows && t.first + tid < t.last) a.shares[t.begin + (t.first + tid) / heads] = shares;
    if (split >= shares) return;
    auto seen_by = [&](uint32_t i) { const int32_t n = t.before + (int32_t)(i / heads) + 1; return n < 0 ? 0u : (uint32_t)n; };
    const uint32_t seen_least = seen_by(t.first), seen_most = seen_by(t.last - 1u);
    const uint32_t from = split * per * kAttendBlock, to0 = shares > 1u ? from + per * kAttendBlock : seen_most, to = to0 < seen_most ? to0 : seen_most;

    // The wavefront's keys of a block: lane i knows the slot of the i-th.
    auto slot_of = [&](uint32_t block) {
        const uint32_t at = block + wave * kStage + lane;
        if (lane >= kStage || at >= to) return kNone;
        const uint32_t page = (uint32_t)a.table[(size_t)t.row * a.columns + (at >> a.shift)];
        return page < a.pages ? page << a.shift | (at & (P - 1u)) : kNone;
    };
    Word4 raw[kLoads], tops[kTops];
    float scales[kBytes ? kLoads : 1u];
    auto fetch = [&](uint32_t slots) {
#pragma unroll
        for (uint32_t i = 0; i < kLoads; i++) {
            const uint32_t slot = kPer == 1u ? __builtin_amdgcn_readlane(slots, i) : __shfl(slots, i * kPer + lane / (64u / kPer));
            const uint8_t *row = slot != kNone ? a.c_cache + (size_t)slot * kRow : kZeros;
            raw[i] = *reinterpret_cast<const Word4 *>(row + lane % (64u / kPer) * 16u);
            if (kBytes) scales[i % (kBytes ? kLoads : 1u)] = *(slot != kNone ? a.scale + slot : reinterpret_cast<const float *>(kZeros));
        }
#pragma unroll
        for (uint32_t i = 0; i < kTops; i++) {
            const uint32_t slot = __shfl(slots, i * 8u + lane / 8u);
            tops[i] = *reinterpret_cast<const Word4 *>((slot != kNone ? a.r_cache + (size_t)slot * kTop : reinterpret_cast<const uint16_t *>(kZeros)) + lane % 8u * 8u);
        }
    };
    uint32_t ahead = 0;
    if (from < to) {
        fetch(slot_of(from));
        ahead = slot_of(from + kKeys);
    }

    // queries: a row behind the last is the last again, and is not stored
    const uint32_t group = wave % kGroups, key_group = wave / kGroups;
    Half8 q[kM][kSteps];
    uint32_t sees[kM];
#pragma unroll
    for (uint32_t n = 0; n < kM; n++) {
        const uint32_t i0 = t.first + (group * kM + n) * 16u + m, i = i0 < t.last ? i0 : t.last - 1u, token = t.begin + i / heads, head = i % heads;
        const uint16_t *c = a.q_c + (int64_t)token * a.c_token + (int64_t)head * a.c_head + g * 8u, *r = a.q_r + (int64_t)token * a.r_token + (int64_t)head * a.r_head + g * 8u;
#pragma unroll
        for (uint32_t s = 0; s < kSteps; s++) q[n][s] = *reinterpret_cast<const Half8 *>(s < kC / 32u ? c + s * 32u : r + (s - kC / 32u) * 32u);
        const uint32_t all = seen_by(i);
        sees[n] = all < to ? all : to;
    }
    Sums<kM, kParts> sums;
    sums.clear();
    if (tid == 0u) odd_from = kNone;
    __syncthreads();
    for (uint32_t block = from; block < to; block += kKeys) {
        const bool partly = block + kKeys > seen_least;                    // some of the tile's rows do not see all of the block's keys
#pragma unroll
        for (uint32_t i = 0; i < kLoads; i++) {
            const uint32_t key = wave * kStage + i * kPer + lane / (64u / kPer), at = lane % (64u / kPer);
            if (kBytes) {
                const float scale = scales[i % (kBytes ? kLoads : 1u)];
                const Word2 w0 = wider(raw[i][0], scale), w1 = wider(raw[i][1], scale), w2 = wider(raw[i][2], scale), w3 = wider(raw[i][3], scale);
                Word4 x{w0[0], w0[1], w1[0], w1[1]}, y{w2[0], w2[1], w3[0], w3[1]};
                if (partly) { x = without_odd(x, block + key, &odd_from); y = without_odd(y, block + key, &odd_from); }
                Word4 *put = reinterpret_cast<Word4 *>(keys + key * kPitch + at * 16u);
                put[0] = x; put[1] = y;
            } else {
                if (partly) raw[i] = without_odd(raw[i], block + key, &odd_from);
                *reinterpret_cast<Word4 *>(keys + key * kPitch + at * 8u) = raw[i];
            }
        }
        if (kStage >= 8u || lane < kStage * 8u)
#pragma unroll
            for (uint32_t i = 0; i < kTops; i++) *reinterpret_cast<Word4 *>(keys + (wave * kStage + i * 8u + lane / 8u) * kPitch + kC + lane % 8u * 8u) = tops[i];
        __syncthreads();
        if (block + kKeys < to) {
            fetch(ahead);
            ahead = slot_of(block + 2u * kKeys);
        }
        if (block + key_group * 32u < to) {
            const uint16_t *mine = keys + key_group * 32u * kPitch;
            Float4 score[2][kM];
#pragma unroll
            for (uint32_t u = 0; u < 2u; u++)
#pragma unroll
                for (uint32_t n = 0; n < kM; n++) score[u][n] = Float4{0.f, 0.f, 0.f, 0.f};
            const uint16_t *row = mine + (m / 4u * 8u + m % 4u) * kPitch + g * 8u;
#pragma unroll
            for (uint32_t s = 0; s < kSteps; s++)
#pragma unroll
                for (uint32_t u = 0; u < 2u; u++) {
                    const Half8 k = *reinterpret_cast<const Half8 *>(row + u * 4u * kPitch + s * 32u);
#pragma unroll
                    for (uint32_t n = 0; n < kM; n++) score[u][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, q[n][s], score[u][n], 0, 0, 0);
                }
            float s[1][kM][8];
            const uint32_t at = block + key_group * 32u + g * 8u;
#pragma unroll
            for (uint32_t n = 0; n < kM; n++)
#pragma unroll
                for (uint32_t j = 0; j < 8u; j++) s[0][n][j] = score[j / 4u][n][j % 4u] * a.factor;
            if (partly || block + kKeys > to)
#pragma unroll
                for (uint32_t n = 0; n < kM; n++)
#pragma unroll
                    for (uint32_t j = 0; j < 8u; j++) s[0][n][j] = at + j < sees[n] ? s[0][n][j] : -__builtin_inff();
            Half8 p[1][kM];
            sums.template weigh<1>(s, p);
            const uint16_t *column = mine + (g * 8u + m / 4u) * kPitch + m % 4u * 4u;
#pragma unroll
            for (uint32_t d = 0; d < kParts; d++) {
                const Half8 v = both(column_of(column + d * 16u), column_of(column + 4u * kPitch + d * 16u));
#pragma unroll
                for (uint32_t n = 0; n < kM; n++) sums.acc[d][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, p[0][n], sums.acc[d][n], 0, 0, 0);
            }
        }
        __syncthreads();
    }

    // out: this share's output by itself, or the whole.  (Numbers that are none have been left out of the sums of rows that see only some of a block's keys: what a row that sees them makes of them
    // is none.)
    const uint32_t odd = odd_from;
    auto put = [&](uint32_t i, uint32_t d, Float4 v) {                     // dims d .. d + 3 of query row i
        const size_t at = (size_t)t.begin * heads + i;
        if (shares > 1u) *reinterpret_cast<Float4 *>(a.partial + (at * a.of.splits + split) * kC + d) = v;
        else *reinterpret_cast<Word2 *>(a.out + at * kC + d) = Word2{pk_bf16(v[0], v[1]), pk_bf16(v[2], v[3])};
    };
    auto end = [&](uint32_t i, float base, float sum, bool any) {
        float *to_ends = a.ends + (((size_t)t.begin * heads + i) * a.of.splits + split) * 2u;
        to_ends[0] = base; to_ends[1] = any && sum == 0.f ? kEmpty : sum;
    };
#pragma unroll
    for (uint32_t n = 0; n < kM; n++) {
        float sum = sums.whole_sum(n);
        if (odd < sees[n]) sum = __builtin_nanf("");
        const uint32_t own = t.first + (group * kM + n) * 16u + m;
        if (kKeyGroups == 1u) {
            const bool any = sees[n] > from;
            const float by = share_of_sum(sum, any && shares == 1u);
            if (own < t.last) {
#pragma unroll
                for (uint32_t d = 0; d < kParts; d++) put(own, d * 16u + g * 4u, sums.acc[d][n] * by);
                if (shares > 1u && g == 0u) end(own, sums.base[n], sum, any);
            }
            continue;
        }
        float *join = reinterpret_cast<float *>(room);
        if (n) __syncthreads();
#pragma unroll
        for (uint32_t d = 0; d < kParts; d++) *reinterpret_cast<Float4 *>(join + (wave * 16u + m) * kJoinPitch + d * 16u + g * 4u) = sums.acc[d][n];
        if (g == 0u) { join_base[wave][m] = sums.base[n]; join_sum[wave][m] = sum; }
        __syncthreads();
        // rows of all groups, four dims to a thread
        for (uint32_t u = tid; u < kGroups * 16u * (kC / 4u); u += kW * 64u) {
            const uint32_t d = u % (kC / 4u) * 4u, row = u / (kC / 4u) % 16u, of = u / (kC / 4u) / 16u, i = t.first + (of * kM + n) * 16u + row;
            if (i >= t.last) continue;
            float base = -__builtin_inff(), total = 0.f;
#pragma unroll
            for (uint32_t w = 0; w < kKeyGroups; w++) base = __builtin_fmaxf(base, join_base[w * kGroups + of][row]);
            const float rel = base > -__builtin_inff() ? base : 0.f;
            Float4 v{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (uint32_t w = 0; w < kKeyGroups; w++) {
                const float by = __builtin_amdgcn_exp2f(join_base[w * kGroups + of][row] - rel);
                total += by * join_sum[w * kGroups + of][row];
                v += by * *reinterpret_cast<const Float4 *>(join + ((w * kGroups + of) * 16u + row) * kJoinPitch + d);
            }
            const uint32_t all = seen_by(i);
            const bool any = (all < to ? all : to) > from;
            put(i, d, v * share_of_sum(total, any && shares == 1u));
            if (shares > 1u && d == 0u) end(i, base, total, any);
        }
    }
}

// The shares of a query row joined, each an output of its own with its sum: kJoinWaves wavefronts for each.
struct JoinArgs {
    const float *partial, *ends;
    const uint32_t *shares;
    const int32_t *total;                            // starts[rows]: tokens that belong to a row
    uint16_t *out;
    uint32_t heads, splits;
};
template <uint32_t kD, uint32_t kJoinWaves>
__global__ void __launch_bounds__(kThreads)
latent_join_kernel(const JoinArgs a)
{
    constexpr uint32_t kOwn = kD / 64u, kHeads = kWaves / kJoinWaves, kRound = 8u;
    __shared__ float part[kJoinWaves > 1u ? kWaves : 1u][kD];
    const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t token = blockIdx.x, head = blockIdx.y * kHeads + wave / kJoinWaves, first = wave % kJoinWaves;
    if (token >= (uint32_t)*a.total) return;         // a token of no row, whose shares nothing has written
    const uint32_t said = a.shares[token], shares = said < a.splits ? said : a.splits;
    if (shares < 2u || (kJoinWaves == 1u && head >= a.heads)) return;
    const size_t at = (size_t)token * a.heads + head;
    const float *ends = a.ends + at * a.splits * 2u;
    float base = -__builtin_inff(), total = 0.f;
    bool any = false;
    for (uint32_t i = lane; i < shares; i += 64u) base = __builtin_fmaxf(base, ends[2u * i]);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) base = __builtin_fmaxf(base, __shfl_xor(base, o));
    const float rel = base > -__builtin_inff() ? base : 0.f;
    for (uint32_t i = lane; i < shares; i += 64u) {
        const float sum = ends[2u * i + 1u];
        any = any || sum == kEmpty;
        if (sum != kEmpty) total += sum * __builtin_amdgcn_exp2f(ends[2u * i] - rel);
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) total += __shfl_xor(total, o);
    const float by = share_of_sum(total, __ballot(any) != 0ull);
    const float *from = a.partial + at * a.splits * kD + lane * kOwn;
    float acc[kOwn];
#pragma unroll
    for (uint32_t d = 0; d < kOwn; d++) acc[d] = 0.f;
    for (uint32_t i0 = first; i0 < shares; i0 += kRound * kJoinWaves) {
        float v[kRound][kOwn], w[kRound];
#pragma unroll
        for (uint32_t k = 0; k < kRound; k++) {
            const uint32_t i = i0 + k * kJoinWaves;
            w[k] = 0.f;
#pragma unroll
            for (uint32_t d = 0; d < kOwn; d++) v[k][d] = 0.f;
            if (i >= shares) continue;
            const float sum = ends[2u * i + 1u];
            w[k] = sum == 0.f || sum == kEmpty ? 0.f : sum * __builtin_amdgcn_exp2f(ends[2u * i] - rel) * by;
            if (sum == 0.f || sum == kEmpty) continue;
#pragma unroll
            for (uint32_t d = 0; d < kOwn; d++) v[k][d] = from[(size_t)i * kD + d];
        }
#pragma unroll
        for (uint32_t k = 0; k < kRound; k++)
#pragma unroll
            for (uint32_t d = 0; d < kOwn; d++) acc[d] += w[k] * v[k][d];
    }
    if (kJoinWaves > 1u) {
#pragma unroll
        for (uint32_t d = 0; d < kOwn; d++) part[wave % (kJoinWaves > 1u ? kWaves : 1u)][lane * kOwn + d] = acc[d];
        __syncthreads();
        if (wave) return;
#pragma unroll
        for (uint32_t d = 0; d < kOwn; d++) {
            acc[d] = 0.f;
#pragma unroll
            for (uint32_t w = 0; w < kWaves; w++) acc[d] += part[w % (kJoinWaves > 1u ? kWaves : 1u)][lane * kOwn + d];
        }
    }
    if (total == 0.f && by != by)
#pragma unroll
        for (uint32_t d = 0; d < kOwn; d++) acc[d] = by;
    uint16_t *out = a.out + at * kD + lane * kOwn;
    if (kOwn == 1u) out[0] = (uint16_t)pk_bf16(acc[0], 0.f);
    else
#pragma unroll
        for (uint32_t d = 0; d < kOwn; d += 2u) reinterpret_cast<Word *>(out)[d / 2u] = pk_bf16(acc[d], acc[(d + 1u) % kOwn]);
}

template <uint32_t kD>
static hipError_t launch_join(const JoinArgs &j, uint32_t tokens, hipStream_t s)
{
    if (j.splits > 8u) return launch(latent_join_kernel<kD, 4>, dim3(tokens, j.heads), dim3(kThreads), 0, s, nullptr, j);
    return launch(latent_join_kernel<kD, 1>, dim3(tokens, (j.heads + kWaves - 1u) / kWaves), dim3(kThreads), 0, s, nullptr, j);
}

static uint32_t wide_of(uint32_t tokens, uint32_t rows, uint32_t heads) { return (uint64_t)tokens * heads >= 64ull * rows ? 1u : 0u; }
static uint32_t attend_rows(uint32_t tokens, uint32_t rows, uint32_t heads) { return wide_of(tokens, rows, heads) ? 128u : 16u; }

bool latent_attend_fits(uint32_t tokens, uint32_t rows, uint32_t heads)
{
    return (uint64_t)tokens * heads / attend_rows(tokens, rows, heads) + rows <= 0xFFFFFFu;
}

uint32_t latent_attend_splits(uint32_t tokens, uint32_t rows, uint32_t heads, uint32_t columns, uint32_t shift)
{
    if (rows > 1024u) return 1u;
    const uint64_t blocks = (((uint64_t)columns << shift) + kAttendBlock - 1u) / kAttendBlock, requests = tokens < rows ? tokens : rows;
    const uint64_t n0 = (uint64_t)tokens * heads / attend_rows(tokens, rows, heads), n = n0 > requests ? n0 : requests;
    const uint64_t want = n >= 4u * kAttendShares ? 1u : 4u * ((kAttendShares + n - 1u) / n), most = (blocks + kAttendLeast - 1u) / kAttendLeast;
    const uint64_t splits = want < most ? want : most;
    return splits < 1u ? 1u : splits > 128u ? 128u : (uint32_t)splits;
}

template <uint32_t kC, bool kBytes>
static hipError_t launch_latent(const LatentAttendArgs &a, hipStream_t s)
{
    const uint32_t rows = attend_rows(a.of.tokens, a.of.rows, a.of.heads);
    const dim3 grid((uint32_t)((uint64_t)a.of.tokens * a.of.heads / rows) + a.of.rows, a.of.splits);
    const hipError_t e = launch(rows == 128u ? latent_attend_kernel<kC, kBytes, 1, 8, 8> : latent_attend_kernel<kC, kBytes, 1, 1, 4>, grid, dim3(rows == 128u ? 512u : 256u), 0, s, nullptr, a);
    if (e != hipSuccess || a.of.splits == 1u) return e;
    return launch_join<kC>(JoinArgs{a.partial, a.ends, a.shares, a.of.starts + a.of.rows, a.out, a.of.heads, a.of.splits}, a.of.tokens, s);
}

hipError_t launch_latent_attend(const void *q_c, const void *q_r, uint32_t tokens, uint32_t heads, uint32_t latent, const int64_t (&strides)[4], const void *c_cache, const void *r_cache,
                                const float *scale, uint32_t pages, uint32_t shift, const int32_t *table, uint32_t rows, uint32_t columns, const int32_t *lens,
                                const int32_t *starts, float factor, void *out, void *workspace, hipStream_t s)
{
    const uint32_t splits = latent_attend_splits(tokens, rows, heads, columns, shift);
    float *partial = static_cast<float *>(workspace), *ends = partial + (splits > 1u ? (size_t)tokens * heads * splits * latent : 0u);
    const LatentAttendArgs a{{starts, rows, tokens, heads, splits, kAttendLeast}, static_cast<const uint16_t *>(q_c), static_cast<const uint16_t *>(q_r),
                             strides[0], strides[1], strides[2], strides[3], static_cast<const uint8_t *>(c_cache), static_cast<const uint16_t *>(r_cache), scale, table, lens,
                             static_cast<uint16_t *>(out), partial, ends, reinterpret_cast<uint32_t *>(ends + (splits > 1u ? (size_t)tokens * heads * splits * 2u : 0u)),
                             factor * 1.44269504088896340736f, columns, pages, shift};
    if (latent == 512u) return scale ? launch_latent<512, true>(a, s) : launch_latent<512, false>(a, s);
    return scale ? launch_latent<256, true>(a, s) : launch_latent<256, false>(a, s);
}

// ---------------------------------------------------------------------------------------------
// Attention of prompts over keys and values of every head.  A workgroup takes 128 tokens of a request, a head and a share of the keys, 32 tokens to a wavefront; keys and values go
// through LDS 64 at a time.
struct LatentPromptArgs {
    Requests of;
    const uint16_t *q_n, *q_r, *k_n, *k_r, *v;
    int64_t qn_token, qn_head, qr_token, qr_head, kn_token, kn_head, kr_token, v_token, v_head;
    const int32_t *key_starts;
    uint16_t *out;                                   // [token][head][D]
    float *partial, *ends;
    uint32_t *shares;
    float factor;
    uint32_t keys;
};
constexpr uint32_t kPromptRows = 128, kPromptKeys = 64;

__device__ __forceinline__ uint32_t keys_of(const LatentPromptArgs &a, uint32_t r, uint32_t *begin)
{
    const uint32_t b0 = (uint32_t)a.key_starts[r], e0 = (uint32_t)a.key_starts[r + 1u], b = b0 < a.keys ? b0 : a.keys, e = e0 < a.keys ? e0 : a.keys;
    *begin = b;
    return e < b ? 0u : e - b;
}

template <uint32_t kD>
__global__ void __launch_bounds__(kThreads) __attribute__((amdgpu_waves_per_eu(2, 2)))
latent_prompt_kernel(const LatentPromptArgs a)
{
    constexpr uint32_t kM = 2u, kSteps = (kD + kTop) / 32u, kParts = kD / 16u, kPitch = kD + kTop + 8u, kValuePitch = kD + 8u, kStage = kPromptKeys / kWaves;
    constexpr uint32_t kPer = 512u / kD, kLoads = kStage / kPer, kTops = kStage / 8u;
    __shared__ __attribute__((aligned(16))) uint16_t keys[kPromptKeys * kPitch], values[kPromptKeys * kValuePitch];
    __shared__ uint32_t odd_from[kD], any_from;       // of each dim, the first key whose value is none, of those that some rows do not see; the first of all
    const uint32_t tid = threadIdx.x, lane = tid & 63u, wave = __builtin_amdgcn_readfirstlane(tid >> 6), m = lane & 15u, g = lane >> 4;
    const uint32_t head = blockIdx.y, split = blockIdx.z;
    Tile t;
    uint32_t count, begin;
    if (!tile_of<kPromptRows>(a.of, 1u, blockIdx.x, &t, &count)) return;
    const uint32_t len = keys_of(a, t.row, &begin);
    t.before = (int32_t)len - (int32_t)count;
    uint32_t per;
    const uint32_t shares = shares_of(a.of, (len + kAttendBlock - 1u) / kAttendBlock, &per, [&](uint32_t r) {
        const uint32_t n = (uint32_t)a.of.starts[r + 1u] - (uint32_t)a.of.starts[r];
        uint32_t none;
        return (uint64_t)((keys_of(a, r, &none) + kAttendBlock - 1u) / kAttendBlock) * ((n + kPromptRows - 1u) / kPromptRows) * a.of.heads;
    });
    if (a.of.splits > 1u && split == 0u && head == 0u && tid < kPromptRows && t.first + tid < t.last) a.shares[t.begin + t.first + tid] = shares;
    if (split >= shares) return;
    auto seen_by = [&](uint32_t i) { const int32_t n = t.before + (int32_t)i + 1; return n < 0 ? 0u : (uint32_t)n; };
    const uint32_t seen_least = seen_by(t.first), seen_most = seen_by(t.last - 1u);
    const uint32_t from = split * per * kAttendBlock, to0 = shares > 1u ? from + per * kAttendBlock : seen_most, to = to0 < seen_most ? to0 : seen_most;
    Half8 q[kM][kSteps];
    uint32_t sees[kM];
#pragma unroll
    for (uint32_t n = 0; n < kM; n++) {
        const uint32_t i0 = t.first + (wave * kM + n) * 16u + m, i = i0 < t.last ? i0 : t.last - 1u, token = t.begin + i;
        const uint16_t *qn = a.q_n + (int64_t)token * a.qn_token + (int64_t)head * a.qn_head + g * 8u, *qr = a.q_r + (int64_t)token * a.qr_token + (int64_t)head * a.qr_head + g * 8u;
#pragma unroll
        for (uint32_t s = 0; s < kSteps; s++) q[n][s] = *reinterpret_cast<const Half8 *>(s < kD / 32u ? qn + s * 32u : qr + (s - kD / 32u) * 32u);
        const uint32_t all = seen_by(i);
        sees[n] = all < to ? all : to;
    }
    Sums<kM, kParts> sums;
    sums.clear();
    Word4 raw[kLoads], tops[kTops], raw_v[kLoads];
    const uint16_t *k_n = a.k_n + (int64_t)begin * a.kn_token + (int64_t)head * a.kn_head, *k_r = a.k_r + (int64_t)begin * a.kr_token,
                   *v_of = a.v + (int64_t)begin * a.v_token + (int64_t)head * a.v_head;
    auto fetch = [&](uint32_t block) {
#pragma unroll
        for (uint32_t i = 0; i < kLoads; i++) {
            const uint32_t key = block + wave * kStage + i * kPer + lane / (64u / kPer), d = lane % (64u / kPer) * 8u;
            raw[i] = Word4{0u, 0u, 0u, 0u}; raw_v[i] = Word4{0u, 0u, 0u, 0u};
            if (key < to) {
                raw[i] = *reinterpret_cast<const Word4 *>(k_n + (int64_t)key * a.kn_token + d);
                raw_v[i] = *reinterpret_cast<const Word4 *>(v_of + (int64_t)key * a.v_token + d);
            }
        }
#pragma unroll
        for (uint32_t i = 0; i < kTops; i++) {
            const uint32_t key = block + wave * kStage + i * 8u + lane / 8u;
            tops[i] = Word4{0u, 0u, 0u, 0u};
            if (key < to) tops[i] = *reinterpret_cast<const Word4 *>(k_r + (int64_t)key * a.kr_token + lane % 8u * 8u);
        }
    };
    if (tid < kD) odd_from[tid] = kNone;
    if (tid == 0u) any_from = kNone;
    __syncthreads();
    if (from < to) fetch(from);
    for (uint32_t block = from; block < to; block += kPromptKeys) {
        const bool partly = block + kPromptKeys > seen_least;
#pragma unroll
        for (uint32_t i = 0; i < kLoads; i++) {
            const uint32_t key = wave * kStage + i * kPer + lane / (64u / kPer), d = lane % (64u / kPer) * 8u;
            if (partly && any_odd(raw_v[i])) {
                atomicMin(&any_from, block + key);
                raw_v[i] = without_odd_dims(raw_v[i], block + key, d, odd_from);
            }
            *reinterpret_cast<Word4 *>(keys + key * kPitch + d) = raw[i];
            *reinterpret_cast<Word4 *>(values + key * kValuePitch + d) = raw_v[i];
        }
#pragma unroll
        for (uint32_t i = 0; i < kTops; i++) *reinterpret_cast<Word4 *>(keys + (wave * kStage + i * 8u + lane / 8u) * kPitch + kD + lane % 8u * 8u) = tops[i];
        __syncthreads();
        if (block + kPromptKeys < to) fetch(block + kPromptKeys);
        Float4 score[2][2][kM];
        const uint16_t *row = keys + (m / 4u * 8u + m % 4u) * kPitch + g * 8u;
#pragma unroll
        for (uint32_t k = 0; k < 2u; k++)
#pragma unroll
            for (uint32_t u = 0; u < 2u; u++) {
#pragma unroll
                for (uint32_t n = 0; n < kM; n++) score[k][u][n] = Float4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (uint32_t s = 0; s < kSteps; s++) {
                    const Half8 x = *reinterpret_cast<const Half8 *>(row + (k * 32u + u * 4u) * kPitch + s * 32u);
#pragma unroll
                    for (uint32_t n = 0; n < kM; n++) score[k][u][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, q[n][s], score[k][u][n], 0, 0, 0);
                }
            }
        float s[2][kM][8];
        const uint32_t at = block + g * 8u;
#pragma unroll
        for (uint32_t k = 0; k < 2u; k++)
#pragma unroll
            for (uint32_t n = 0; n < kM; n++)
#pragma unroll
                for (uint32_t j = 0; j < 8u; j++) s[k][n][j] = score[k][j / 4u][n][j % 4u] * a.factor;
        if (partly || block + kPromptKeys > to)
#pragma unroll
            for (uint32_t k = 0; k < 2u; k++)
#pragma unroll
                for (uint32_t n = 0; n < kM; n++)
#pragma unroll
                    for (uint32_t j = 0; j < 8u; j++) s[k][n][j] = at + k * 32u + j < sees[n] ? s[k][n][j] : -__builtin_inff();
        Half8 p[2][kM];
        sums.template weigh<2>(s, p);
        const uint16_t *column = values + (g * 8u + m / 4u) * kValuePitch + m % 4u * 4u;
#pragma unroll
        for (uint32_t d = 0; d < kParts; d++)
#pragma unroll
            for (uint32_t k = 0; k < 2u; k++) {
                const uint16_t *of = column + k * 32u * kValuePitch + d * 16u;
                const Half8 x = both(column_of(of), column_of(of + 4u * kValuePitch));
#pragma unroll
                for (uint32_t n = 0; n < kM; n++) sums.acc[d][n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, p[k][n], sums.acc[d][n], 0, 0, 0);
            }
        __syncthreads();
    }
#pragma unroll
    for (uint32_t n = 0; n < kM; n++) {
        const float sum = sums.whole_sum(n);
        const uint32_t own = t.first + (wave * kM + n) * 16u + m;
        const bool any = sees[n] > from;
        const float by = share_of_sum(sum, any && shares == 1u);
        if (own >= t.last) continue;
        const size_t at = (size_t)(t.begin + own) * a.of.heads + head;
#pragma unroll
        for (uint32_t d = 0; d < kParts; d++) {
            Float4 v = sums.acc[d][n] * by;
            if (any_from != kNone)
#pragma unroll
                for (uint32_t e = 0; e < 4u; e++) v[e] = odd_from[d * 16u + g * 4u + e] < sees[n] ? __builtin_nanf("") : v[e];
            if (shares > 1u) *reinterpret_cast<Float4 *>(a.partial + (at * a.of.splits + split) * kD + d * 16u + g * 4u) = v;
            else *reinterpret_cast<Word2 *>(a.out + at * kD + d * 16u + g * 4u) = Word2{pk_bf16(v[0], v[1]), pk_bf16(v[2], v[3])};
        }
        if (shares > 1u && g == 0u) {
            float *to_ends = a.ends + (at * a.of.splits + split) * 2u;
            to_ends[0] = sums.base[n]; to_ends[1] = any && sum == 0.f ? kEmpty : sum;
        }
    }
}

bool latent_prompt_fits(uint32_t tokens, uint32_t rows) { return (uint64_t)tokens / kPromptRows + rows <= 0xFFFFFFu; }

uint32_t latent_prompt_splits(uint32_t tokens, uint32_t rows, uint32_t heads, uint32_t keys)
{
    if (rows > 1024u) return 1u;
    const uint64_t blocks = ((uint64_t)keys + kAttendBlock - 1u) / kAttendBlock, requests = tokens < rows ? tokens : rows;
    const uint64_t n = ((uint64_t)tokens / kPromptRows + requests) * heads;
    const uint64_t want = kAttendShares * 2u / n, most = (blocks + kAttendLeast - 1u) / kAttendLeast, splits = want < most ? want : most;
    return splits < 1u ? 1u : splits > 64u ? 64u : (uint32_t)splits;
}

hipError_t launch_latent_prompt(const void *q_n, const void *q_r, const void *k_n, const void *k_r, const void *v, uint32_t tokens, uint32_t keys, uint32_t heads, uint32_t dim,
                                const int64_t (&strides)[9], uint32_t rows, const int32_t *starts, const int32_t *key_starts, float factor, void *out, void *workspace, hipStream_t s)
{
    const uint32_t splits = latent_prompt_splits(tokens, rows, heads, keys);
    float *partial = static_cast<float *>(workspace), *ends = partial + (splits > 1u ? (size_t)tokens * heads * splits * dim : 0u);
    auto halves = [](const void *p) { return static_cast<const uint16_t *>(p); };
    const LatentPromptArgs a{{starts, rows, tokens, heads, splits, kAttendLeast}, halves(q_n), halves(q_r), halves(k_n), halves(k_r), halves(v),
                             strides[0], strides[1], strides[2], strides[3], strides[4], strides[5], strides[6], strides[7], strides[8], key_starts, static_cast<uint16_t *>(out),
                             partial, ends, reinterpret_cast<uint32_t *>(ends + (splits > 1u ? (size_t)tokens * heads * splits * 2u : 0u)), factor * 1.44269504088896340736f, keys};
    const dim3 grid(tokens / kPromptRows + rows, heads, splits);
    const hipError_t e = launch(dim == 128u ? latent_prompt_kernel<128> : latent_prompt_kernel<64>, grid, dim3(kThreads), 0, s, nullptr, a);
    if (e != hipSuccess || splits == 1u) return e;
    const JoinArgs j{a.partial, a.ends, a.shares, starts + rows, a.out, heads, splits};
    return dim == 128u ? launch_join<128>(j, tokens, s) : launch_join<64>(j, tokens, s);
}

}  // namespace wg
