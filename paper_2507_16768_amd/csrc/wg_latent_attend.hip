// Attention with keys and values from one latent vector a token, for gfx950: over the paged cache of the vectors themselves (latent_attend_kernel), and over the
// keys and values of every head made from them beforehand (latent_prompt_kernel).
//
// Both take their products as attention over the 8-bit cache does: scores as S^T = K Q^T (rows: keys), so that the lane that holds the scores of eight keys of a query after the first product is
// the one that needs their weights in the second, O^T = V^T P^T.  The keys that a row of the first product's tiles stands for are numbered for that: lane l of 64, with
// m = l % 16 and g = l / 16, holds for query m the scores of keys 8 g .. 8 g + 7 of 32.  Keys lie in LDS as rows, and the second product's operand, eight keys of one dim, is read from there
// by the transposing read: sixteen lanes that ask for four rows of sixteen numbers get a column of four each.
//
// The softmax is taken in one pass: weights 2^(score - base - 8) relative to a base that moves only where a score is 8 above it, by their wavefront as a whole; so it
// costs no exchange between lanes but where it moves, and the largest weight is 2^-8 to 1: a sum of values that 2^128 holds is not lost.  Weights are rounded to bfloat16, as the values are that they multiply (values go as far as 2^127,
// which float16 would not hold): they are off by 2^-8 at the most, as the output is by its own rounding.  Their sum, in fp32, is that of the weights before.
#include <hip/hip_runtime.h>

#include "wg_buffer.h"
#include "wg_launch.h"
#include "wg_number.h"
#include "wg_serve.h"

namespace wg {

typedef short Short4 __attribute__((ext_vector_type(4)));
typedef float Float16 __attribute__((ext_vector_type(16)));
typedef uint32_t Word __attribute__((may_alias));

constexpr uint32_t kThreads = 256, kWaves = 4, kTop = 64;
constexpr float kLift = 8.f;                         // how far above the base a score may be, log2
constexpr uint32_t kNone = 0xFFFFFFFFu;

// Requests and their query tokens: tokens [starts[r], starts[r + 1]) of the call are request r's last ones.
struct Requests {
    const int32_t *starts;
    uint32_t rows, tokens, heads;
    uint32_t chunks;                                 // workgroups that all work is dealt out to; 0: one for each tile
};
struct Tile { uint32_t row, first, last, begin, count; int32_t before; };  // query rows [first, last) of request `row`, whose tokens of the call begin at `begin`, behind `before` others (count: all of them)

// What is the same for all lanes, though it comes by a load of each.
__device__ __forceinline__ uint32_t uniform(uint32_t x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ uint32_t start_of(const Requests &a, uint32_t r) { const uint32_t t = (uint32_t)a.starts[r]; return t < a.tokens ? t : a.tokens; }
__device__ __forceinline__ uint32_t tokens_of(const Requests &a, uint32_t r) { const uint32_t b = start_of(a, r), e = start_of(a, r + 1u); return e < b ? 0u : e - b; }

// Tile `tile` of request r, of kRows query rows, `per` to a token; false: there is none.
template <uint32_t kRows>
__device__ __forceinline__ bool tile_at(const Requests &a, uint32_t per, uint32_t r, uint32_t tile, Tile *out)
{
    const uint32_t n = uniform(tokens_of(a, r)), all = n * per, e = uniform((uint32_t)a.starts[r + 1u]);
    out->row = r; out->begin = uniform(start_of(a, r));
    if ((uint64_t)tile * kRows >= all) return false;
    out->first = tile * kRows;
    out->last = all - out->first < kRows ? all : out->first + kRows;
    out->count = e - out->begin;                     // (with the request's tokens that the call does not have)
    return true;
}

// The request whose tiles tile `tile` of the call is among: request r's begin at starts[r] * per / kRows + r, which leaves room for each one's last, begun tile.  A wavefront asks 64
// requests at a time.
template <uint32_t kRows>
__device__ __forceinline__ bool tile_of(const Requests &a, uint32_t per, uint32_t tile, Tile *out)
{
    const uint32_t lane = threadIdx.x & 63u;
    auto begins = [&](uint32_t r) { return (uint32_t)((uint64_t)start_of(a, r) * per / kRows) + r; };
    uint32_t lo = 0, n = a.rows;
    while (n > 1u) {
        const uint32_t step = (n + 63u) / 64u, r = lo + lane * step;
        const bool at = lane * step < n && begins(r) <= tile;
        const uint32_t k = 63u - (uint32_t)__builtin_clzll(__ballot(at) | 1ull);
        n = n - k * step < step ? n - k * step : step;
        lo += k * step;
    }
    lo = __builtin_amdgcn_readfirstlane(lo);
    const uint32_t first = uniform(begins(lo));
    return tile >= first && tile_at<kRows>(a, per, lo, tile - first, out);
}

// All work dealt out: blocks of keys of the tiles of the requests, one behind the other, in chunks of one size, a workgroup each, so that all have as much to do whatever the rows' lengths
// are.  A chunk takes the end of a tile, whole ones, and the beginning of another; what is part of a tile only goes to the workspace and is joined by another kernel.  Chunk w's part of a tile
// that has begun before it lies in place 2 w there, one of a tile that begins in it in place 2 w + 1.
struct Chunk { uint32_t at, end, size, row, off; };  // blocks [at, end) of all work; `at` is block `off` of request `row`

template <typename F>
__device__ __forceinline__ bool chunk_of(const Requests &a, uint32_t w, F work_of, Chunk *out)
{
    const uint32_t lane = threadIdx.x & 63u;
    const uint32_t first = lane < a.rows ? work_of(lane) : 0u;             // (most calls have no more rows: asked for once)
    uint32_t all = first;
    for (uint32_t r = lane + 64u; r < a.rows; r += 64u) all += work_of(r);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) all += __shfl_xor(all, o);
    all = __builtin_amdgcn_readfirstlane(all);
    const uint32_t even = (all + a.chunks - 1u) / a.chunks, size = even < kAttendLeast ? kAttendLeast : even;
    out->size = size;
    out->at = w * size;
    if (w >= a.chunks || out->at >= all) return false;
    out->end = all - out->at < size ? all : out->at + size;
    uint32_t ahead = 0;                              // work of the requests in front
    for (uint32_t base = 0; base < a.rows; base += 64u) {
        const uint32_t own = !base ? first : base + lane < a.rows ? work_of(base + lane) : 0u;
        uint32_t sum = own;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) { const uint32_t x = __shfl_up(sum, o); sum += lane >= (uint32_t)o ? x : 0u; }
        const unsigned long long behind = __ballot(ahead + sum > out->at);
        if (behind) {
            const uint32_t k = (uint32_t)__builtin_ctzll(behind);
            out->row = base + k;
            out->off = uniform(out->at - (ahead + __builtin_amdgcn_readlane(sum, k) - __builtin_amdgcn_readlane(own, k)));
            return true;
        }
        ahead += __builtin_amdgcn_readlane(sum, 63);
    }
    return false;
}

// The next part of a tile: blocks [b0, b0 + n) of its `blocks`, and how many chunks it lies in.  A tile counts as kTileCost blocks more, in front of its own: asking for its queries and storing its
// outputs take that long.  false: the chunk ends among these.  (off: the chunk's place in the tile; work: of the request)
__device__ __forceinline__ bool part_of(Chunk *c, uint32_t off, uint32_t blocks, uint32_t work, uint32_t *b0, uint32_t *n, uint32_t *chunks)
{
    const uint32_t whole = blocks + kTileCost, took = whole - off < c->end - c->at ? whole - off : c->end - c->at, end = off + took;
    const uint32_t begins = c->at - off + kTileCost;                       // where the tile's own blocks do, among all
    *b0 = off > kTileCost ? off - kTileCost : 0u;
    *n = (end > kTileCost ? end - kTileCost : 0u) - *b0;
    *chunks = (begins + blocks - 1u) / c->size - begins / c->size + 1u;
    c->at += took;
    c->off += took;
    if (c->off >= work) { c->off = 0; c->row++; }
    return *n != 0u;
}

// Where the parts of a query row lie: its first chunk and its place in the tile, and how many chunks.
struct Parts { uint32_t chunk_and_row, chunks; };

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

// A load from device memory.  (Of an address that is one of two the compiler knows only that it is some address, and a load from there counts as one from LDS too: the waits for operands
// out of LDS would be waits for memory.)
template <typename T> __device__ __forceinline__ T from_memory(const void *p) { return *(const __attribute__((address_space(1))) T *)p; }

// x, which the compiler is not to know anything about.
__device__ __forceinline__ uint32_t anew(uint32_t x) { asm volatile("" : "+v"(x)); return x; }

// x of lane first + which, `which` below kN.  (Without LDS, in which a shuffle waits for the keys that have been written there:
// three rows' 200 tokens behind 1,500 in bfloat16, 24 heads, 43.2 us for 44.7.  Of 8-bit vectors, whose keys come two to a load, shuffles are the faster: 64 rows' 4 drafts, 16 heads, 89 us for 105.)
template <uint32_t kN>
__device__ __forceinline__ uint32_t of_groups(uint32_t x, uint32_t first, uint32_t which)
{
    uint32_t y = __builtin_amdgcn_readlane(x, first);
#pragma unroll
    for (uint32_t i = 1; i < kN; i++) { const uint32_t z = __builtin_amdgcn_readlane(x, first + i); y = which >= i ? z : y; }
    return y;
}

// What is read in the place of a key that there is none of.
__device__ __attribute__((aligned(16))) const uint8_t kZeros[1024] = {};

// kN operands out of LDS, load(i, place), each for products, use(i, place): kAhead of them are asked for before the kAhead in front of them are used.  (Left to itself the compiler asks for one,
// waits, and uses it.)
template <uint32_t kN, uint32_t kAhead, typename L, typename U>
__device__ __forceinline__ void pipelined(L load, U use)
{
    constexpr uint32_t kRounds = (kN + kAhead - 1u) / kAhead;
#pragma unroll
    for (uint32_t i = 0; i < kAhead && i < kN; i++) load(i, i);
#pragma unroll
    for (uint32_t b = 0; b < kRounds; b++) {
#pragma unroll
        for (uint32_t i = 0; i < kAhead; i++)
            if ((b + 1u) * kAhead + i < kN) load((b + 1u) * kAhead + i, (b + 1u) % 2u * kAhead + i);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (uint32_t i = 0; i < kAhead; i++)
            if (b * kAhead + i < kN) use(b * kAhead + i, b % 2u * kAhead + i);
        __builtin_amdgcn_sched_barrier(0);
    }
}

// Queries that give scores of the factor's sign, which then is 1 or above 0: with it 0 all are zeros.
__device__ __forceinline__ Half8 signed_query(Half8 q, float factor)
{
    const uint32_t flip = factor < 0.f ? 0x80008000u : 0u, keep = factor == 0.f ? 0u : 0xFFFFFFFFu;
    Word4 v = __builtin_bit_cast(Word4, q);
#pragma unroll
    for (uint32_t w = 0; w < 4u; w++) v[w] = (v[w] ^ flip) & keep;
    return __builtin_bit_cast(Half8, v);
}
__host__ __device__ __forceinline__ float size_of(float factor) { return factor == 0.f ? 1.f : __builtin_fabsf(factor); }

// The largest over lanes l, l ^ 16, l ^ 32 and l ^ 48.
__device__ __forceinline__ float most_of_rows(float x)
{
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = __builtin_fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __builtin_fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// A score relative to a base, in log2.  Bases are scores themselves, and the difference is taken before the factor: that of the base's own score is 0 whatever its size, where a product less another one that was
// rounded would leave the rounding's error, which from scores of 2^31 on has the largest weight 0 or infinite.  (An operation more a score: 100 rows, 128 heads 123 us for 119, drafts 89.9 for 88, prompts 142.8 for 140.8;
// one of 16,000 tokens 1,301 for 1,289.  Left to a branch that scores below 2^10 do not take, 123, 88.4, 140 and 1,299.)
__device__ __forceinline__ float in_log2(float score, float base, float factor) { return (score - base) * factor; }
// (no score is more than kLift above its base: a weight is 1 at the most)
__device__ __forceinline__ float weight_of(float score, float base, float factor) { return __builtin_amdgcn_exp2f(in_log2(score, base, factor) - kLift); }

// What a wavefront holds of its 16 queries: of query m, the base and its own part of the sum, and outputs, dims 4 g .. 4 g + 3 of each of kParts.
template <uint32_t kParts>
struct Sums {
    Float4 acc[kParts];
    float base, sum;
    __device__ __forceinline__ void clear()
    {
        base = -__builtin_inff(); sum = 0.f;
#pragma unroll
        for (uint32_t d = 0; d < kParts; d++) acc[d] = Float4{0.f, 0.f, 0.f, 0.f};
    }
    // Scores of eight keys (-inf where nothing is seen) into weights; factor, above 0, makes them scores in log2.
    __device__ __forceinline__ Half8 weigh(const float (&s)[8], float factor)
    {
        float n = s[0];
#pragma unroll
        for (uint32_t j = 0; j < 8u; j++) n = __builtin_fmaxf(n, s[j]);
        if (__ballot(in_log2(n, base, factor) > kLift)) {
            n = __builtin_fmaxf(base, most_of_rows(n));
            const float by = __builtin_amdgcn_exp2f(in_log2(base, n > -__builtin_inff() ? n : 0.f, factor));
            base = n; sum *= by;
#pragma unroll
            for (uint32_t d = 0; d < kParts; d++) acc[d] *= by;
        }
        const float from = base > -__builtin_inff() ? base : 0.f;
        Word4 w;
#pragma unroll
        for (uint32_t j = 0; j < 4u; j++) {
            const float x = weight_of(s[2u * j], from, factor), y = weight_of(s[2u * j + 1u], from, factor);
            w[j] = pk_bf16(x, y);
            sum += x; sum += y;
        }
        return __builtin_bit_cast(Half8, w);
    }
    // The queries' sums over all lanes.
    __device__ __forceinline__ float whole_sum() const
    {
        const float l = sum + __shfl_xor(sum, 16);
        return l + __shfl_xor(l, 32);
    }
};

// What a sum makes of an output: 1 / sum; zeros for a query that sees no key, and none for one whose scores are all -inf.
__device__ __forceinline__ float share_of_sum(float sum, bool sees) { return sum > 0.f ? 1.f / sum : sum == 0.f && !sees ? 0.f : __builtin_nanf(""); }
constexpr float kEmpty = -1.f;                       // the sum of a share in which a query sees keys whose scores are all -inf

// ---------------------------------------------------------------------------------------------
// Attention over the cached vectors.  A workgroup's eight wavefronts are kGroups groups of 16 query rows (tokens times heads), times kCols groups of the vectors' columns (which make
// the scores between them), times groups of 32 keys.  A block's keys go through LDS: from memory into registers, while the block before is worked on, and turned into bfloat16 (exactly) on the way.
//
// What bounds it.  100 rows of 1,000 to 4,000 tokens, 128 heads, bfloat16: 119 to 124 us, 580 to 605 TFLOP/s, an eighth of it joining.  Over its keys, 295 MB, it goes at 5.2 TB/s, what a copy reaches, 57 us; the
// rest is that 256 workgroups, one on each compute unit, ask for 147 KB of queries for each of the two tiles or so that they have a part of, and store 256 KB for each part.  64 rows' 4 drafts, 16 heads, 8 bits: 89 to 90 us,
// 6 of it joining (2.4 TB/s, 270 TFLOP/s): a block of 32 keys takes 3,900 cycles, of which the products are 1,100; the others are what comes one after the other in a block, the scores' exchange, the softmax, the keys to LDS.  One
// row of 30,000, 16 heads, 8 bits: 21.4 us, 6 of it joining, a workgroup having one block of 128 keys: latencies, one behind the other, of lengths, page numbers, keys and stores.
// Tried, and no faster: the keys' way to LDS beside the second product (124 us for 121; 172 with branches, whose waits are for everything), all queries asked for before one is used (123 for 123), two blocks of
// keys asked for at first (122 for 122), slots found before the keys go to LDS (no difference), values asked for before the softmax; 32 query rows to a wavefront (its 256 accumulators leave no registers to scale them in).
struct LatentAttendArgs {
    Requests of;
    const uint16_t *q_c, *q_r;
    int64_t c_token, c_head, r_token, r_head;        // strides of queries, elements
    const uint8_t *c_cache;
    const uint16_t *r_cache;
    const float *scale;                              // of each token; null: the vectors are bfloat16
    const int32_t *table, *lens;
    uint16_t *out;                                   // [token][head][C]
    float *partial, *ends;                           // [chunk][2][row of a tile][C]; [chunk][2][row of a tile][2]: base and sum
    Parts *parts;                                    // [token][head]
    float factor;                                    // of the scores, times log2(e)
    uint32_t columns, pages, shift;
};

__device__ __forceinline__ uint32_t cached_tokens(const LatentAttendArgs &a, uint32_t r)
{
    const uint32_t most = a.columns << a.shift, l = (uint32_t)(a.lens[r] < 0 ? 0 : a.lens[r]);
    return l < most ? l : most;
}
__device__ __forceinline__ uint32_t blocks_of(uint32_t keys) { return keys ? (keys + kAttendBlock - 1u) / kAttendBlock : 1u; }

template <uint32_t kC, bool kBytes, uint32_t kGroups, uint32_t kCols>
__global__ void __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(2, 2)))
latent_attend_kernel(const LatentAttendArgs a)
{
    constexpr uint32_t kW = 8u, kKeyGroups = kW / (kGroups * kCols), kKeys = 32u * kKeyGroups, kRows = 16u * kGroups;
    constexpr uint32_t kSteps = (kC + kTop) / 32u, kParts = kC / 16u / kCols, kPitch = kC + kTop + 16u, kGroupPitch = 32u * kPitch + 192u;
    constexpr uint32_t kRow = kC * (kBytes ? 1u : 2u), kPer = 1024u / kRow, kStage = kKeys / kW;          // bytes of a vector; keys of a wavefront's load; keys that it brings
    constexpr uint32_t kLoads = kStage / kPer, kTops = (kStage + 7u) / 8u, kAhead = kC == 512u && kGroups == 8u ? 2u : 4u, kPut = kC == 512u && kGroups == 8u ? 10u : 0u, kKept = kSteps - kPut;
    constexpr uint32_t kJoinPitch = kC + 4u, kTile = kKeyGroups * kGroupPitch, kTileBytes = kTile * 2u, kJoinBytes = kKeyGroups > 1u ? kKeyGroups * kRows * kJoinPitch * 4u : kW * 16u * 132u * 4u;
    constexpr bool kHalves = kCols > 1u;                                   // two wavefronts that take the same rows and keys make half of the scores each
    __shared__ __attribute__((aligned(16))) uint8_t room[2u * kTileBytes > kJoinBytes ? 2u * kTileBytes : kJoinBytes];   // two blocks of keys: one that is worked on, one that comes
    __shared__ uint32_t odd_from;                                          // the first key with a number that is none, of those that some rows do not see
    __shared__ float join_base[kKeyGroups][kRows], join_sum[kKeyGroups][kRows];
    __shared__ Float4 halves[kHalves ? kW * 64u : 1u];                     // each lane's scores of half of the keys
    __shared__ Half8 q_rest[kPut ? kW * kPut * 64u : 1u];                  // the last steps of the queries, each lane its own: there are no registers for them
    uint16_t *keys = reinterpret_cast<uint16_t *>(room);
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t group = wave % kGroups, column_group = wave / kGroups % kCols, key_group = wave / (kGroups * kCols);
    const uint32_t P = 1u << a.shift, heads = a.of.heads;
    auto tiles = [&](uint32_t r) { return (uint32_t)(((uint64_t)tokens_of(a.of, r) * heads + kRows - 1u) / kRows); };
    Tile t;
    Chunk c{0u, 1u, 0u, 0u, 0u};
    if (a.of.chunks ? !chunk_of(a.of, blockIdx.x, [&](uint32_t r) { return tiles(r) * (blocks_of(cached_tokens(a, r)) + kTileCost); }, &c) : !tile_of<kRows>(a.of, heads, blockIdx.x, &t)) return;
    while (c.at < c.end && c.row < a.of.rows) {
        // (What follows from the thread's number is made anew for each part: kept over the parts it would take registers from the loop over keys.)
        const uint32_t tid = anew(threadIdx.x), lane = tid & 63u, m = lane & 15u, g = lane >> 4;
        // the next part of a tile: blocks [b0, b0 + n) of its `blocks`
        uint32_t b0 = 0, n = 1u, blocks = 1u, chunks = 1u;                 // chunks: that the tile lies in
        if (a.of.chunks) {
            blocks = uniform(blocks_of(cached_tokens(a, c.row)));
            const uint32_t tile = c.off / (blocks + kTileCost), work = uniform(tiles(c.row)) * (blocks + kTileCost);
            if (!work) { c.row++; continue; }                              // (off is 0)
            (void)tile_at<kRows>(a.of, heads, c.row, tile, &t);
            if (!part_of(&c, c.off - tile * (blocks + kTileCost), blocks, work, &b0, &n, &chunks)) continue;
        } else c.at++;
        const uint32_t len = uniform(cached_tokens(a, t.row));
        t.before = (int32_t)len - (int32_t)t.count;
        const bool whole = n == blocks;
        const uint32_t place = 2u * blockIdx.x + (b0 ? 0u : 1u), row_first = t.first;
        if (a.of.chunks && b0 == 0u && tid < kRows && t.first + tid < t.last)
            a.parts[(size_t)t.begin * heads + t.first + tid] = Parts{blockIdx.x | tid << 16, chunks};
        auto seen_by = [&](uint32_t i) { const int32_t k = t.before + (int32_t)(i / heads) + 1; return k < 0 ? 0u : (uint32_t)k < len ? (uint32_t)k : len; };
        const uint32_t seen_least = seen_by(t.first), seen_most = seen_by(t.last - 1u);
        const uint32_t from = b0 * kAttendBlock, to0 = whole ? seen_most : from + n * kAttendBlock, to = to0 < seen_most ? to0 : seen_most;

        // The wavefront's keys of a block: lane i knows the slot of the i-th.  A page's number is asked for a block ahead of the keys, and looked at when they are asked for: before that,
        // the wait for it would be one for all that has been asked for earlier.
        const int32_t *pages_of_row = a.table + (size_t)t.row * a.columns;
        auto page_of = [&](uint32_t block) {
            const uint32_t at = block + wave * kStage + lane % kStage;
            return from_memory<uint32_t>(at < to ? static_cast<const void *>(pages_of_row + (at >> a.shift)) : kZeros);
        };
        auto slot_of = [&](uint32_t block, uint32_t page) {
            const uint32_t at = block + wave * kStage + lane;
            return lane < kStage && at < to && page < a.pages ? page << a.shift | (at & (P - 1u)) : kNone;
        };
        Word4 raw[kLoads], tops[kTops];
        float scales = 0.f;                                                // lane i: of the i-th key
        auto fetch = [&](uint32_t slots) {
            if (kBytes) scales = from_memory<float>(slots != kNone ? static_cast<const void *>(a.scale + slots) : kZeros);
#pragma unroll
            for (uint32_t i = 0; i < kLoads; i++) {
                const uint32_t slot = kBytes && kPer > 1u ? (uint32_t)__shfl(slots, i * kPer + lane / (64u / kPer)) : of_groups<kPer>(slots, i * kPer, lane / (64u / kPer));
                const uint8_t *row = slot != kNone ? a.c_cache + (size_t)slot * kRow : kZeros;
                raw[i] = from_memory<Word4>(row + lane % (64u / kPer) * 16u);
            }
#pragma unroll
            for (uint32_t i = 0; i < kTops; i++) {
                const uint32_t slot = kBytes ? (uint32_t)__shfl(slots, i * 8u + lane / 8u) : of_groups<kStage < 8u ? kStage : 8u>(slots, i * 8u, lane / 8u);
                tops[i] = from_memory<Word4>((slot != kNone ? reinterpret_cast<const uint8_t *>(a.r_cache) + (size_t)slot * (kTop * 2u) : kZeros) + lane % 8u * 16u);
            }
        };
        // Keys of a block into LDS, which serves 16 lanes' sixteen bytes in a cycle, lanes 0 .. 3, 12 .. 15 and 20 .. 27 of 32 and the others of these, or 32 lanes' eight, from 64 banks.  So the
        // operands of the first product, sixteen bytes of rows 0 .. 3, 8 .. 11, 16 .. 19 and 24 .. 27, and of the second, 32 bytes each of four rows and of the four that lie eight further, are
        // to lie in different sixteenths of 256 bytes: a row takes 2 or 10 of them more than whole ones, and every eight rows have 8 more behind them.
        auto row_at = [&](uint32_t key) { return key / 32u * kGroupPitch + key % 32u * kPitch + key % 32u / 8u * 64u; };
        auto stage = [&](uint32_t block, uint16_t *to_keys) {
            const bool partly = block + kKeys > seen_least;                // some of the tile's rows do not see all of the block's keys
#pragma unroll
            for (uint32_t i = 0; i < kLoads; i++) {
                const uint32_t key = wave * kStage + i * kPer + lane / (64u / kPer), at = lane % (64u / kPer);
                if (kBytes) {
                    const float scale = __shfl(scales, i * kPer + lane / (64u / kPer));
                    const Word2 w0 = wider(raw[i][0], scale), w1 = wider(raw[i][1], scale), w2 = wider(raw[i][2], scale), w3 = wider(raw[i][3], scale);
                    Word4 x{w0[0], w0[1], w1[0], w1[1]}, y{w2[0], w2[1], w3[0], w3[1]};
                    if (partly) { x = without_odd(x, block + key, &odd_from); y = without_odd(y, block + key, &odd_from); }
                    Word4 *put = reinterpret_cast<Word4 *>(to_keys + row_at(key) + at * 16u);
                    put[0] = x; put[1] = y;
                } else {
                    if (partly) raw[i] = without_odd(raw[i], block + key, &odd_from);
                    *reinterpret_cast<Word4 *>(to_keys + row_at(key) + at * 8u) = raw[i];
                }
            }
            if (kStage >= 8u || lane < kStage * 8u)
#pragma unroll
                for (uint32_t i = 0; i < kTops; i++) *reinterpret_cast<Word4 *>(to_keys + row_at(wave * kStage + i * 8u + lane / 8u) + kC + lane % 8u * 8u) = tops[i];
        };
        uint32_t ahead = 0;
        if (from < to) {
            const uint32_t first = page_of(from);
            ahead = page_of(from + kKeys);
            fetch(slot_of(from, first));
        }
        auto fetch_next = [&](uint32_t block) {
            const uint32_t slots = slot_of(block, ahead);
            ahead = page_of(block + kKeys);
            fetch(slots);
        };

        // queries: a row behind the last is the last again, and is not stored
        Half8 q[kKept];
        uint32_t sees;
        {
            const uint32_t i0 = t.first + group * 16u + m, i = i0 < t.last ? i0 : t.last - 1u, token = t.begin + i / heads, head = i % heads;
            const uint16_t *c = a.q_c + (int64_t)token * a.c_token + (int64_t)head * a.c_head + g * 8u, *r = a.q_r + (int64_t)token * a.r_token + (int64_t)head * a.r_head + g * 8u;
#pragma unroll
            for (uint32_t s = 0; s < kSteps; s++) {
                const Half8 x = signed_query(*reinterpret_cast<const Half8 *>(s < kC / 32u ? c + s * 32u : r + (s - kC / 32u) * 32u), a.factor);
                if (s < kKept) q[s % kKept] = x;
                else q_rest[(wave * kPut + s - kKept) * 64u + lane] = x;
            }
            const uint32_t all = seen_by(i);
            sees = all < to ? all : to;
        }
        Sums<kParts> sums;
        sums.clear();
        if (tid == 0u) odd_from = kNone;
        __syncthreads();
        if (from < to) stage(from, keys);
        // (vmcnt(0): the queries are here before anything else is asked for.  A wait for them in the loop would be one for the keys that come)
        __builtin_amdgcn_s_waitcnt(0x0F70);
        if (from + kKeys < to) fetch_next(from + kKeys);
        uint32_t turn = 0;
        for (uint32_t block = from; block < to; block += kKeys, turn ^= 1u) {
            __syncthreads();
            const uint16_t *mine = keys + turn * kTile + key_group * kGroupPitch, *row = mine + row_at(m / 4u * 8u + m % 4u) + g * 8u;
            Float4 score[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
            Half8 k[2][kAhead], rest[2][(kAhead + 1u) / 2u];
            if (kHalves) {
                const uint32_t half = column_group % 2u;
                const uint16_t *half_row = row + half * 4u * kPitch;
                Float4 own[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};                          // (two sums, so that a product need not wait for the one before)
                pipelined<kSteps, kAhead>([&](uint32_t i, uint32_t at) { k[at / kAhead][at % kAhead] = *reinterpret_cast<const Half8 *>(half_row + i * 32u); },
                                          [&](uint32_t i, uint32_t at) { own[i % 2u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[at / kAhead][at % kAhead], q[i % kKept], own[i % 2u], 0, 0, 0); });
                own[0] += own[1];
                halves[wave * 64u + lane] = own[0];
                __syncthreads();
                const Float4 other = halves[(wave ^ kGroups) * 64u + lane];
#pragma unroll
                for (uint32_t e = 0; e < 4u; e++) { score[0][e] = half ? other[e] : own[0][e]; score[1][e] = half ? own[0][e] : other[e]; }
            } else
                pipelined<2u * kSteps, kAhead>([&](uint32_t i, uint32_t at) {
                                                   k[at / kAhead][at % kAhead] = *reinterpret_cast<const Half8 *>(row + i % 2u * 4u * kPitch + i / 2u * 32u);
                                                   if (i / 2u >= kKept && i % 2u == 0u) rest[at / kAhead][at % kAhead / 2u] = q_rest[(wave * kPut + i / 2u - kKept) * 64u + lane];
                                               },
                                               [&](uint32_t i, uint32_t at) {
                                                   const Half8 x = i / 2u < kKept ? q[i / 2u % kKept] : rest[at / kAhead][at % kAhead / 2u];
                                                   score[i % 2u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[at / kAhead][at % kAhead], x, score[i % 2u], 0, 0, 0);
                                               });
            float s[8];
            const uint32_t at = block + key_group * 32u + g * 8u;
#pragma unroll
            for (uint32_t j = 0; j < 8u; j++) s[j] = score[j / 4u][j % 4u];
            if (block + kKeys > seen_least || block + kKeys > to)
#pragma unroll
                for (uint32_t j = 0; j < 8u; j++) s[j] = at + j < sees ? s[j] : -__builtin_inff();
            const Half8 p = sums.weigh(s, size_of(a.factor));
            if (block + kKeys < to) {
                stage(block + kKeys, keys + (turn ^ 1u) * kTile);
                if (block + 2u * kKeys < to) fetch_next(block + 2u * kKeys);
            }
            const uint16_t *column = mine + row_at(g * 8u + m / 4u) + column_group * (kC / kCols) + m % 4u * 4u;
            pipelined<kParts, kAhead>([&](uint32_t d, uint32_t at) { k[at / kAhead][at % kAhead] = both(column_of(column + d * 16u), column_of(column + 4u * kPitch + d * 16u)); },
                                      [&](uint32_t d, uint32_t at) { sums.acc[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[at / kAhead][at % kAhead], p, sums.acc[d], 0, 0, 0); });
        }
        __syncthreads();

        // Out: this part by itself, or the whole.  (Numbers that are none have been left out of the sums of rows that see only some of a block's keys: what a row that sees them makes of them
        // is none.)
        const uint32_t odd = odd_from;
        const float sum = sums.whole_sum();
        auto put = [&](uint32_t i, uint32_t d, Float4 v) {                 // dims d .. d + 3 of query row i of the tile
            if (whole) *reinterpret_cast<Word2 *>(a.out + ((size_t)t.begin * heads + row_first + i) * kC + d) = Word2{pk_bf16(v[0], v[1]), pk_bf16(v[2], v[3])};
            else *reinterpret_cast<Float4 *>(a.partial + ((size_t)place * kRows + i) * kC + d) = v;
        };
        auto finish = [&](uint32_t i, float base, float sum_of, float *by) {   // what the row's outputs are multiplied by
            const uint32_t all = seen_by(row_first + i), end = all < to ? all : to;
            const float l = odd < end ? __builtin_nanf("") : sum_of;
            *by = share_of_sum(l, end > from && whole);
            return Float2{base, end > from && l == 0.f ? kEmpty : l};
        };
        if (kKeyGroups == 1u) {
            const uint32_t i = group * 16u + m;
            float by;
            const Float2 ends = finish(i, sums.base, sum, &by);
            if (row_first + i < t.last && !whole && g == 0u && column_group == 0u) *reinterpret_cast<Float2 *>(a.ends + ((size_t)place * kRows + i) * 2u) = ends;
            // Through LDS, 128 dims of the wavefront's 16 rows at a time, so that it stores 512 bytes beside each other.
            float *turned = reinterpret_cast<float *>(room) + wave * (16u * 132u);
#pragma unroll
            for (uint32_t d0 = 0; d0 < kC / kCols; d0 += 128u) {
#pragma unroll
                for (uint32_t d = 0; d < 8u; d++) *reinterpret_cast<Float4 *>(turned + m * 132u + d * 16u + g * 4u) = sums.acc[d0 / 16u + d] * by;
                __builtin_amdgcn_wave_barrier();
#pragma unroll
                for (uint32_t k = 0; k < 8u; k++) {
                    const uint32_t row = k * 2u + lane / 32u;
                    const Float4 v = *reinterpret_cast<const Float4 *>(turned + row * 132u + lane % 32u * 4u);
                    if (row_first + group * 16u + row < t.last) put(group * 16u + row, column_group * (kC / kCols) + d0 + lane % 32u * 4u, v);
                }
                __builtin_amdgcn_wave_barrier();
            }
            __syncthreads();
            continue;
        }
        float *join = reinterpret_cast<float *>(room);
        const uint32_t own = key_group * kRows + group * 16u + m;
#pragma unroll
        for (uint32_t d = 0; d < kParts; d++) *reinterpret_cast<Float4 *>(join + own * kJoinPitch + column_group * (kC / kCols) + d * 16u + g * 4u) = sums.acc[d];
        if (g == 0u && column_group == 0u) { join_base[key_group][group * 16u + m] = sums.base; join_sum[key_group][group * 16u + m] = sum; }
        __syncthreads();
        // four dims of a row to a thread
        for (uint32_t u = tid; u < kRows * (kC / 4u); u += kW * 64u) {
            const uint32_t d = u % (kC / 4u) * 4u, i = u / (kC / 4u);
            if (row_first + i >= t.last) continue;
            float base = -__builtin_inff(), total = 0.f;
#pragma unroll
            for (uint32_t w = 0; w < kKeyGroups; w++) base = __builtin_fmaxf(base, join_base[w][i]);
            const float rel = base > -__builtin_inff() ? base : 0.f;
            Float4 v{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (uint32_t w = 0; w < kKeyGroups; w++) {
                const float by = __builtin_amdgcn_exp2f(in_log2(join_base[w][i], rel, size_of(a.factor)));
                total += by * join_sum[w][i];
                v += by * *reinterpret_cast<const Float4 *>(join + (w * kRows + i) * kJoinPitch + d);
            }
            float by;
            const Float2 ends = finish(i, base, total, &by);
            put(i, d, v * by);
            if (!whole && d == 0u) *reinterpret_cast<Float2 *>(a.ends + ((size_t)place * kRows + i) * 2u) = ends;
        }
        __syncthreads();
    }
}

// The parts of a query row joined, each an output of its own with its sum.
struct JoinArgs {
    const float *partial, *ends;
    const Parts *parts;
    const int32_t *starts;
    uint16_t *out;
    uint32_t requests, heads, chunks, rows;          // rows: of a tile
    float factor;                                    // above 0: of the bases, to log2
};
// Few parts of a row are a wavefront's, all dims and all parts asked for together.  Many are dealt out to the four wavefronts of a workgroup, 64 at a time, and the dims, 64 at a time, to workgroups.  16 heads, a token
// a row, attention and this: one row of 30,000, cut into 235 parts, 24 us dealt out and 58 not; four rows of 16,000, 64 parts each, 26 and 31; ten of 8,000, 25 parts, 27.6 and 27.2; 64 of 4,000, 68 and 43.
constexpr uint32_t kManyParts = 16;                  // parts of a tile, as many as can be (it is counted as two where requests fill one)
template <uint32_t kD, bool kMany>
__global__ void __launch_bounds__(256)
latent_join_kernel(const JoinArgs a)
{
    constexpr uint32_t kOwn = kMany ? 1u : kD / 64u, kShare = kMany ? 4u : 1u, kHeads = 4u / kShare, kRound = kMany ? 32u : 4u;
    __shared__ float part[4][64], tops[4], sums[4];
    __shared__ uint32_t empties[4];
    const uint32_t lane = threadIdx.x & 63u, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t token = blockIdx.x, head = blockIdx.y * kHeads + wave / kShare, d0 = (kMany ? blockIdx.z * 64u : 0u) + lane * kOwn;
    if (token < (uint32_t)a.starts[0] || token >= (uint32_t)a.starts[a.requests] || head >= a.heads) return;          // (a token of no row has no parts)
    const size_t at = (size_t)token * a.heads + head;
    const Parts p = a.parts[at];
    const uint32_t chunk = uniform(p.chunk_and_row & 0xFFFFu), row = uniform(p.chunk_and_row >> 16);
    if (p.chunks < 2u || row >= a.rows || chunk >= a.chunks) return;
    const uint32_t n = uniform(p.chunks < a.chunks - chunk ? p.chunks : a.chunks - chunk);
    auto place = [&](uint32_t i) { return (size_t)(i ? 2u * (chunk + i) : 2u * chunk + 1u) * a.rows + row; };
    // a lane for each part, 64 at a time: what it weighs
    float base = -__builtin_inff(), total = 0.f;
    bool any = false;
    float acc[kOwn];
#pragma unroll
    for (uint32_t d = 0; d < kOwn; d++) acc[d] = 0.f;
    for (uint32_t i0 = wave % kShare * 64u; i0 < n; i0 += 64u * kShare) {
        const Float2 e = i0 + lane < n ? *reinterpret_cast<const Float2 *>(a.ends + place(i0 + lane) * 2u) : Float2{-__builtin_inff(), 0.f};
        const uint32_t more = n - i0 < 64u ? n - i0 : 64u;
        float v[kRound][kOwn];
        auto ask = [&](uint32_t k0) {
#pragma unroll
            for (uint32_t k = 0; k < kRound; k++) {
                const float *from = a.partial + place(i0 + (k0 + k < more ? k0 + k : 0u)) * kD + d0;
#pragma unroll
                for (uint32_t d = 0; d < kOwn; d++) v[k][d] = from[d];
            }
        };
        ask(0u);
        float top = __builtin_fmaxf(base, e[0]);
#pragma unroll
        for (int o = 32; o > 0; o >>= 1) top = __builtin_fmaxf(top, __shfl_xor(top, o));
        const float rel = top > -__builtin_inff() ? top : 0.f, by = __builtin_amdgcn_exp2f(in_log2(base, rel, a.factor));
        any = any || e[1] == kEmpty;
        const float w = e[1] == kEmpty || e[1] == 0.f ? 0.f : e[1] * __builtin_amdgcn_exp2f(in_log2(e[0], rel, a.factor));
        total = total * by + w;
        base = top;
#pragma unroll
        for (uint32_t d = 0; d < kOwn; d++) acc[d] *= by;
        for (uint32_t k0 = 0; k0 < more; k0 += kRound) {
            if (k0) ask(k0);
#pragma unroll
            for (uint32_t k = 0; k < kRound; k++) {
                const float wk = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(w), k0 + k < 64u ? k0 + k : 63u));
                if (k0 + k >= more) continue;                              // (one that weighs nothing counts: it is none where a value that is none has been weighed with 0)
#pragma unroll
                for (uint32_t d = 0; d < kOwn; d++) acc[d] += wk * v[k][d];
            }
        }
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) total += __shfl_xor(total, o);
    bool empty = __ballot(any) != 0ull;
    if (kMany) {
        part[wave][lane] = acc[0];
        if (lane == 0u) { tops[wave] = base; sums[wave] = total; empties[wave] = empty; }
        __syncthreads();
        if (wave) return;
        const float top = __builtin_fmaxf(__builtin_fmaxf(tops[0], tops[1]), __builtin_fmaxf(tops[2], tops[3])), rel = top > -__builtin_inff() ? top : 0.f;
        acc[0] = 0.f; total = 0.f;
#pragma unroll
        for (uint32_t w = 0; w < 4u; w++) {
            const float by = __builtin_amdgcn_exp2f(in_log2(tops[w], rel, a.factor));
            acc[0] += by * part[w][lane]; total += by * sums[w];
            empty = empty || empties[w];
        }
    }
    const float by = share_of_sum(total, empty);
#pragma unroll
    for (uint32_t d = 0; d < kOwn; d++) acc[d] *= by;                      // (nothing but -inf: 0 times none)
    uint16_t *out = a.out + at * kD + d0;
    if (kOwn == 1u) out[0] = (uint16_t)pk_bf16(acc[0], 0.f);
    else
#pragma unroll
        for (uint32_t d = 0; d < kOwn; d += 2u) reinterpret_cast<Word *>(out)[d / 2u] = pk_bf16(acc[d], acc[(d + 1u) % kOwn]);
}

// Whether all work is dealt out, over how many workgroups, and the workspace's parts.  (tiles, blocks: the most there can be; of_row: blocks of keys of a row, as far as that is known.)  Tiles of a request's many tokens
// see more keys the later they come, which the chunks do not know: with twice as many as the chip holds at a time they are left to it; where requests have few tokens, as they decode, all work is dealt out however
// many there are (256 rows of 1,000 to 4,000 tokens, 128 heads, a tile each: 541 us left to the chip, 307 dealt out).
//
// A tile of few blocks is a workgroup's, since joining it would cost more than it saves: of one or two (one token of a row of 200, 16 heads: 17.3 us dealt out, 16.2 by one; with three blocks 16.3 and 18.0), and, where
// requests have many tokens or keys of their own for each head, of up to four that would be cut into two or so (100 tokens of a row of 500, 128 heads 51 and 36, of 800 55 and 62; prompts of 400, 32 heads 26 and
// 19, three of 170 24 and 11; 128 tokens behind 500 20 and 26).
struct Plan { uint32_t chunks; uint64_t partial, ends, parts; };
static Plan plan_of(uint64_t tiles, uint64_t blocks, uint64_t of_row, uint32_t rows, bool few, bool cut_late, uint32_t tile_rows, uint32_t dim, uint32_t slots, uint64_t outputs)
{
    Plan p{0u, 0u, 0u, 0u};
    if (rows > 1024u || of_row < 3u || (tiles >= 2u * slots && !few) || tiles * (blocks + kTileCost) > 0x7FFFFFFFull) return p;
    if (cut_late && of_row <= (tiles * (of_row + kTileCost) > slots ? 4u : 3u)) return p;
    const uint64_t most = (tiles * (blocks + kTileCost) + kAttendLeast - 1u) / kAttendLeast;
    p.chunks = (uint32_t)(most < slots ? most : slots);
    p.partial = (uint64_t)p.chunks * 2u * tile_rows * dim;
    p.ends = (uint64_t)p.chunks * 2u * tile_rows * 2u;
    p.parts = outputs * 2u;
    return p;
}
static uint64_t plan_bytes(const Plan &p) { return (p.partial + p.ends + p.parts) * 4u; }

template <uint32_t kD>
static hipError_t launch_join(const JoinArgs &j, uint32_t tokens, bool many, hipStream_t s)
{
    if (many) return launch(latent_join_kernel<kD, true>, dim3(tokens, j.heads, kD / 64u), dim3(256), 0, s, nullptr, j);
    return launch(latent_join_kernel<kD, false>, dim3(tokens, (j.heads + 3u) / 4u), dim3(256), 0, s, nullptr, j);
}

static uint64_t attend_blocks(uint32_t columns, uint32_t shift) { return (((uint64_t)columns << shift) + kAttendBlock - 1u) / kAttendBlock; }
static uint64_t tiles_of(uint32_t tokens, uint32_t rows, uint32_t heads, uint32_t tile) { return (uint64_t)tokens * heads / tile + (rows < tokens ? rows : tokens); }
static uint32_t rows_of_request(uint32_t tokens, uint32_t rows, uint32_t heads)
{
    const uint64_t n = (uint64_t)tokens * heads, r = rows < tokens ? rows : tokens;
    return n <= 16u * r ? 16u : n <= 32u * r ? 32u : n <= 64u * r ? 64u : 128u;
}
// Query rows of a tile: 16, 32, 64 or 128.  As many as a request has read its keys once (in bfloat16, 512 numbers: 100 rows of 4,000 tokens, 128 heads 118 us with 128, 144 with 64, 337 with 16; 64 of 8,000, 32 heads 92
// with 32, 126 with 16, 116 with 128).  But a workgroup has its queries to ask for and its part to store however few keys it has, and where all tiles have only two blocks of keys for each
// workgroup, or four, as far as the table's width tells, smaller ones are faster, whose parts are smaller (128 heads: one row of 2,000 tokens 21.5 us with 16, 27.5 with 128; four of 2,000 26 and 42; one of
// 30,000 37 with 64, 42 with 128, 56 with 16; 50 tokens of a row of 4,000, 24 heads 39 with 64, 68 with 128).
static uint32_t attend_rows(uint32_t tokens, uint32_t rows, uint32_t heads, uint64_t blocks)
{
    const uint32_t most = rows_of_request(tokens, rows, heads);
    const uint64_t n = (uint64_t)tokens * heads;
    for (uint32_t tile = 16u; tile < most; tile *= 2u)
        if (((n + tile - 1u) / tile) * blocks <= (tile == 64u ? 4u : 2u) * kAttendSlots) return tile;
    return most;
}
static uint64_t attend_tiles(uint32_t tokens, uint32_t rows, uint32_t heads, uint64_t blocks) { return tiles_of(tokens, rows, heads, attend_rows(tokens, rows, heads, blocks)); }

bool latent_attend_fits(uint32_t tokens, uint32_t rows, uint32_t heads) { return (uint64_t)tokens * heads / rows_of_request(tokens, rows, heads) + rows <= 0x7FFFFFu; }

static Plan attend_plan(uint32_t tokens, uint32_t rows, uint32_t heads, uint32_t latent, uint32_t columns, uint32_t shift)
{
    const uint64_t blocks = attend_blocks(columns, shift);
    const bool few = tokens <= 16u * rows;
    return plan_of(attend_tiles(tokens, rows, heads, blocks), blocks, blocks, rows, few, !few, attend_rows(tokens, rows, heads, blocks), latent, kAttendSlots, (uint64_t)tokens * heads);
}
uint64_t latent_attend_bytes(uint32_t tokens, uint32_t rows, uint32_t heads, uint32_t latent, uint32_t columns, uint32_t shift)
{
    return plan_bytes(attend_plan(tokens, rows, heads, latent, columns, shift));
}

template <uint32_t kC, bool kBytes>
static hipError_t launch_latent(const LatentAttendArgs &a, hipStream_t s)
{
    const uint64_t blocks = attend_blocks(a.columns, a.shift);
    const uint32_t rows = attend_rows(a.of.tokens, a.of.rows, a.of.heads, blocks);
    const dim3 grid(a.of.chunks ? a.of.chunks : (uint32_t)((uint64_t)a.of.tokens * a.of.heads / rows) + a.of.rows);
    const hipError_t e = launch(rows == 16u ? latent_attend_kernel<kC, kBytes, 1, 4> : rows == 32u ? latent_attend_kernel<kC, kBytes, 2, 2> : rows == 64u ? latent_attend_kernel<kC, kBytes, 4, 2>
                                : latent_attend_kernel<kC, kBytes, 8, 1>, grid, dim3(512), 0, s, nullptr, a);
    if (e != hipSuccess || !a.of.chunks) return e;
    return launch_join<kC>(JoinArgs{a.partial, a.ends, a.parts, a.of.starts, a.out, a.of.rows, a.of.heads, a.of.chunks, rows, size_of(a.factor)}, a.of.tokens,
                           a.of.chunks > kManyParts * attend_tiles(a.of.tokens, a.of.rows, a.of.heads, blocks), s);
}

hipError_t launch_latent_attend(const void *q_c, const void *q_r, uint32_t tokens, uint32_t heads, uint32_t latent, const int64_t (&strides)[4], const void *c_cache, const void *r_cache,
                                const float *scale, uint32_t pages, uint32_t shift, const int32_t *table, uint32_t rows, uint32_t columns, const int32_t *lens,
                                const int32_t *starts, float factor, void *out, void *workspace, hipStream_t s)
{
    const Plan p = attend_plan(tokens, rows, heads, latent, columns, shift);
    float *partial = static_cast<float *>(workspace), *ends = partial + p.partial;
    const LatentAttendArgs a{{starts, rows, tokens, heads, p.chunks}, static_cast<const uint16_t *>(q_c), static_cast<const uint16_t *>(q_r),
                             strides[0], strides[1], strides[2], strides[3], static_cast<const uint8_t *>(c_cache), static_cast<const uint16_t *>(r_cache), scale, table, lens,
                             static_cast<uint16_t *>(out), partial, ends, reinterpret_cast<Parts *>(ends + p.ends), factor * 1.44269504088896340736f, columns, pages, shift};
    if (latent == 512u) return scale ? launch_latent<512, true>(a, s) : launch_latent<512, false>(a, s);
    return scale ? launch_latent<256, true>(a, s) : launch_latent<256, false>(a, s);
}

// ---------------------------------------------------------------------------------------------
// Attention of prompts over keys and values of every head.  A workgroup takes 128 tokens of a request, a head and a share of the keys, 32 tokens to a wavefront, a query to a lane (products of 32 by 32, whose
// operands out of LDS serve twice as many queries as those of 16 by 16: 138 us for 158); keys and values go through LDS 32 at a time, two workgroups on a compute unit (211 us with one).  Tiles of many tokens are
// left to the chip, the last of a row first.
//
// What bounds it.  Four prompts of 800 to 2,000 tokens, 32 heads of 128: 134 to 143 us, 680 to 723 TFLOP/s (one of 16,000, 16 heads: 1,010 to 1,050; a large matrix product reaches 1,222; with heads of 64 numbers 94 us, 620); two of 600 to 1,500 with
// 128 heads 190 us, 679.  Left out, the softmax's arithmetic would save
// 18 us of it, the second product 26, the keys' way from memory 12: no part bounds it alone.  131 queries behind 9,000 keys, 16 heads: 41 us, 1.9 TB/s; its 32 tiles are cut, and what the parts cost adds.
// Tried, and no faster: 256 tokens to a workgroup (143 us for 135; 131 queries behind 9,000 keys 37 for 41), one block's softmax under the next one's products with three blocks in LDS (143 us for 143), tiles in order of their keys over all rows (146 for 146), 16 rows to a wavefront and four of
// them to a SIMD (158).
struct LatentPromptArgs {
    Requests of;
    const uint16_t *q_n, *q_r, *k_n, *k_r, *v;
    int64_t qn_token, qn_head, qr_token, qr_head, kn_token, kn_head, kr_token, v_token, v_head;
    const int32_t *key_starts;
    uint16_t *out;                                   // [token][head][D]
    float *partial, *ends;                           // as in LatentAttendArgs
    Parts *parts;
    float factor;
    uint32_t keys;
};
constexpr uint32_t kPromptRows = 128, kPromptKeys = 32;

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
    constexpr uint32_t kSteps = (kD + kTop) / 16u, kParts = kD / 32u, kPitch = kD + kTop + 8u, kValuePitch = kD + 32u, kStage = kPromptKeys / kWaves;
    constexpr uint32_t kPer = 512u / kD, kLoads = kStage / kPer, kTops = kStage / 8u, kAhead = 4u;
    constexpr uint32_t kBlocks = 2u * 32u * (kPitch + kValuePitch) * 2u, kTurned = 32u * 68u;
    __shared__ __attribute__((aligned(16))) uint8_t room[kBlocks > kWaves * kTurned * 4u ? kBlocks : kWaves * kTurned * 4u];   // two blocks of keys and values: one that is worked on, one that comes
    uint16_t *keys = reinterpret_cast<uint16_t *>(room), *values = keys + 2u * 32u * kPitch;
    __shared__ uint32_t odd_from[kD], any_from;       // of each dim, the first key whose value is none, of those that some rows do not see; the first of all
    const uint32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), heads = a.of.heads;
    auto tiles = [&](uint32_t r) { return (tokens_of(a.of, r) + kPromptRows - 1u) / kPromptRows; };
    auto blocks_at = [&](uint32_t r) { uint32_t none; return blocks_of(keys_of(a, r, &none)); };
    Tile t;
    Chunk c{0u, 1u, 0u, 0u, 0u};
    uint32_t head = uniform(blockIdx.x % heads);
    if (a.of.chunks ? !chunk_of(a.of, blockIdx.x, [&](uint32_t r) { return tiles(r) * heads * (blocks_at(r) + kTileCost); }, &c) : !tile_of<kPromptRows>(a.of, 1u, blockIdx.x / heads, &t)) return;
    if (!a.of.chunks) (void)tile_at<kPromptRows>(a.of, 1u, t.row, uniform(tiles(t.row)) - 1u - t.first / kPromptRows, &t);             // the last, which see the most keys, first
    while (c.at < c.end && c.row < a.of.rows) {
        const uint32_t tid = anew(threadIdx.x), lane = tid & 63u, m = lane & 31u, h = lane >> 5;
        uint32_t b0 = 0, n_blocks = 1u, blocks = 1u, chunks = 1u, begin;
        if (a.of.chunks) {
            blocks = uniform(blocks_at(c.row));
            const uint32_t unit = c.off / (blocks + kTileCost), work = uniform(tiles(c.row)) * heads * (blocks + kTileCost);
            if (!work) { c.row++; continue; }                              // (off is 0)
            head = uniform(unit % heads);
            (void)tile_at<kPromptRows>(a.of, 1u, c.row, unit / heads, &t);
            if (!part_of(&c, c.off - unit * (blocks + kTileCost), blocks, work, &b0, &n_blocks, &chunks)) continue;
        } else c.at++;
        const uint32_t len = uniform(keys_of(a, t.row, &begin));
        begin = uniform(begin);
        t.before = (int32_t)len - (int32_t)t.count;
        const bool whole = n_blocks == blocks;
        const uint32_t place = 2u * blockIdx.x + (b0 ? 0u : 1u);
        if (a.of.chunks && b0 == 0u && tid < kPromptRows && t.first + tid < t.last)
            a.parts[(size_t)(t.begin + t.first + tid) * heads + head] = Parts{blockIdx.x | tid << 16, chunks};
        auto seen_by = [&](uint32_t i) { const int32_t k = t.before + (int32_t)i + 1; return k < 0 ? 0u : (uint32_t)k < len ? (uint32_t)k : len; };
        const uint32_t seen_least = seen_by(t.first), seen_most = seen_by(t.last - 1u);
        const uint32_t from = b0 * kAttendBlock, to0 = whole ? seen_most : from + n_blocks * kAttendBlock, to = to0 < seen_most ? to0 : seen_most;

        Word4 raw[kLoads], tops[kTops], raw_v[kLoads];
        const uint32_t head_now = uniform(head);
        const uint16_t *k_n = a.k_n + (int64_t)begin * a.kn_token + (int64_t)head_now * a.kn_head, *k_r = a.k_r + (int64_t)begin * a.kr_token, *v_of = a.v + (int64_t)begin * a.v_token + (int64_t)head_now * a.v_head;
        // a block's rows as buffers: keys behind the last lie behind their ends, and read as zeros
        auto rows_from = [&](const uint16_t *p, uint32_t block, int64_t token, uint32_t dim) {
            const uint32_t n = to - block < kPromptKeys ? to - block : kPromptKeys;
            return window_of(p + (int64_t)block * token, ((n - 1u) * (uint32_t)token + dim) * 2u);
        };
        auto four = [&](Window w, uint32_t at) { const FourWords x = __builtin_amdgcn_raw_buffer_load_b128(w, at, 0, 0); return Word4{x.x, x.y, x.z, x.w}; };
        const uint32_t own_key = wave * kStage + lane / (64u / kPer), own_dim = lane % (64u / kPer) * 16u, own_top = (wave * kStage + lane / 8u) * (uint32_t)a.kr_token * 2u + lane % 8u * 16u;
        const uint32_t own_k = own_key * (uint32_t)a.kn_token * 2u + own_dim, own_v = own_key * (uint32_t)a.v_token * 2u + own_dim;
        auto fetch = [&](uint32_t block) {
            const Window kw = rows_from(k_n, block, a.kn_token, kD), vw = rows_from(v_of, block, a.v_token, kD), rw = rows_from(k_r, block, a.kr_token, kTop);
#pragma unroll
            for (uint32_t i = 0; i < kLoads; i++) {
                raw[i] = four(kw, own_k + i * kPer * (uint32_t)a.kn_token * 2u);
                raw_v[i] = four(vw, own_v + i * kPer * (uint32_t)a.v_token * 2u);
            }
#pragma unroll
            for (uint32_t i = 0; i < kTops; i++) tops[i] = four(rw, own_top + i * 8u * (uint32_t)a.kr_token * 2u);
        };
        // Rows of keys take a sixteenth of 256 bytes more than whole eighths of that, rows of values four, so that what LDS serves in a cycle lies in different ones: of the first product rows 4 q .. 4 q + 3
        // for q of 0, 3, 5, 6 or 1, 2, 4, 7, of the second 64 bytes each of four neighbouring rows.
        auto row_at = [&](uint32_t key) { return key * kPitch; };
        auto value_at = [&](uint32_t key) { return key * kValuePitch; };
        auto stage = [&](uint32_t block, uint32_t turn) {
            const bool partly = block + kPromptKeys > seen_least;
#pragma unroll
            for (uint32_t i = 0; i < kLoads; i++) {
                const uint32_t key = wave * kStage + i * kPer + lane / (64u / kPer), d = lane % (64u / kPer) * 8u;
                if (partly && any_odd(raw_v[i])) {
                    atomicMin(&any_from, block + key);
                    raw_v[i] = without_odd_dims(raw_v[i], block + key, d, odd_from);
                }
                *reinterpret_cast<Word4 *>(keys + turn * 32u * kPitch + row_at(key) + d) = raw[i];
                *reinterpret_cast<Word4 *>(values + turn * 32u * kValuePitch + value_at(key) + d) = raw_v[i];
            }
#pragma unroll
            for (uint32_t i = 0; i < kTops; i++) *reinterpret_cast<Word4 *>(keys + turn * 32u * kPitch + row_at(wave * kStage + i * 8u + lane / 8u) + kD + lane % 8u * 8u) = tops[i];
        };
        if (from < to) fetch(from);
        const uint32_t own = wave * 32u + m, i0 = t.first + own, i = i0 < t.last ? i0 : t.last - 1u;
        Half8 q[kSteps];
        {
            const uint16_t *qn = a.q_n + (int64_t)(t.begin + i) * a.qn_token + (int64_t)head_now * a.qn_head + h * 8u, *qr = a.q_r + (int64_t)(t.begin + i) * a.qr_token + (int64_t)head_now * a.qr_head + h * 8u;
#pragma unroll
            for (uint32_t s = 0; s < kSteps; s++) q[s] = signed_query(*reinterpret_cast<const Half8 *>(s < kD / 16u ? qn + s * 16u : qr + (s - kD / 16u) * 16u), a.factor);
        }
        const uint32_t all = seen_by(i), sees = all < to ? all : to;
        Float16 acc[kParts];
        float base = -__builtin_inff(), sum = 0.f;
#pragma unroll
        for (uint32_t d = 0; d < kParts; d++)
#pragma unroll
            for (uint32_t e = 0; e < 16u; e++) acc[d][e] = 0.f;
        if (tid < kD) odd_from[tid] = kNone;
        if (tid == 0u) any_from = kNone;
        __syncthreads();
        if (from < to) stage(from, 0u);
        __builtin_amdgcn_s_waitcnt(0x0F70);                                // (as in latent_attend_kernel)
        if (from + kPromptKeys < to) fetch(from + kPromptKeys);
        const float factor = size_of(a.factor);
        const bool some = uniform(t.first + wave * 32u) < t.last;            // a wavefront that has no query only brings keys (131 queries, 16 heads, behind 9,000 keys: 40.8 us for 42.8)
        uint32_t turn = 0;
        for (uint32_t block = from; block < to; block += kPromptKeys, turn ^= 1u) {
            __syncthreads();
            // row r of the first product's tile is key 16 (r / 16) + 8 (r / 4 % 2) + 4 (r / 8 % 2) + r % 4: the lane then has the scores of keys 8 h .. 8 h + 7 of each sixteen
            const uint16_t *row = keys + turn * 32u * kPitch + row_at(m / 16u * 16u + m / 4u % 2u * 8u + m / 8u % 2u * 4u + m % 4u) + h * 8u;
            Float16 score;
#pragma unroll
            for (uint32_t e = 0; e < 16u; e++) score[e] = 0.f;
            Half8 x[2][kAhead], p[2];
            if (some) {
                __builtin_amdgcn_s_setprio(1);                             // scores go before another wavefront's other work (136 us for 138; in latent_attend_kernel no difference)
                pipelined<kSteps, kAhead>([&](uint32_t i, uint32_t at) { x[at / kAhead][at % kAhead] = *reinterpret_cast<const Half8 *>(row + i * 16u); },
                                          [&](uint32_t i, uint32_t at) { score = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x[at / kAhead][at % kAhead], q[i], score, 0, 0, 0); });
                __builtin_amdgcn_s_setprio(0);
                const uint32_t at = block + h * 8u;
                if (block + kPromptKeys > seen_least || block + kPromptKeys > to)
#pragma unroll
                    for (uint32_t e = 0; e < 16u; e++) score[e] = at + e / 8u * 16u + e % 8u < sees ? score[e] : -__builtin_inff();
                float top = score[0];
#pragma unroll
                for (uint32_t e = 1; e < 16u; e++) top = __builtin_fmaxf(top, score[e]);
                if (__ballot(in_log2(top, base, factor) > kLift)) {
                    const auto both_halves = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false);
                    top = __builtin_fmaxf(base, __builtin_fmaxf(__uint_as_float(both_halves[0]), __uint_as_float(both_halves[1])));
                    const float by = __builtin_amdgcn_exp2f(in_log2(base, top > -__builtin_inff() ? top : 0.f, factor));
                    base = top; sum *= by;
#pragma unroll
                    for (uint32_t d = 0; d < kParts; d++) acc[d] *= by;
                }
                const float rel = base > -__builtin_inff() ? base : 0.f;
#pragma unroll
                for (uint32_t k = 0; k < 2u; k++) {
                    Word4 w;
#pragma unroll
                    for (uint32_t j = 0; j < 4u; j++) {
                        const float u = weight_of(score[8u * k + 2u * j], rel, factor), v = weight_of(score[8u * k + 2u * j + 1u], rel, factor);
                        w[j] = pk_bf16(u, v);
                        sum += u; sum += v;
                    }
                    p[k] = __builtin_bit_cast(Half8, w);
                }
            }
            if (block + kPromptKeys < to) {
                stage(block + kPromptKeys, turn ^ 1u);
                if (block + 2u * kPromptKeys < to) fetch(block + 2u * kPromptKeys);
            }
            if (!some) continue;

            const uint16_t *column = values + turn * 32u * kValuePitch + value_at(h * 8u + lane % 16u / 4u) + lane / 16u % 2u * 16u + lane % 4u * 4u;
            pipelined<2u * kParts, kAhead>([&](uint32_t i, uint32_t at) {
                                               const uint16_t *of = column + i / kParts * 16u * kValuePitch + i % kParts * 32u;
                                               x[at / kAhead][at % kAhead] = both(column_of(of), column_of(of + 4u * kValuePitch));
                                           },
                                           [&](uint32_t i, uint32_t at) { acc[i % kParts] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x[at / kAhead][at % kAhead], p[i / kParts], acc[i % kParts], 0, 0, 0); });
        }
        __syncthreads();
        sum += __shfl_xor(sum, 32);
        const bool any = sees > from;
        const float by = share_of_sum(sum, any && whole);
        if (i0 < t.last && !whole && h == 0u) *reinterpret_cast<Float2 *>(a.ends + ((size_t)place * kPromptRows + own) * 2u) = Float2{base, any && sum == 0.f ? kEmpty : sum};
        // through LDS (as in latent_attend_kernel), 64 dims of the wavefront's 32 rows at a time
        float *turned = reinterpret_cast<float *>(room) + wave * kTurned;
#pragma unroll
        for (uint32_t d0 = 0; d0 < kD; d0 += 64u) {
#pragma unroll
            for (uint32_t d = 0; d < 64u; d += 8u) {
                const uint32_t dim = d0 + d + h * 4u, of = (d0 + d) / 32u, e = d / 8u % 4u;
                Float4 v{acc[of][4u * e] * by, acc[of][4u * e + 1u] * by, acc[of][4u * e + 2u] * by, acc[of][4u * e + 3u] * by};
                if (any_from != kNone)
#pragma unroll
                    for (uint32_t j = 0; j < 4u; j++) v[j] = odd_from[dim + j] < sees ? __builtin_nanf("") : v[j];
                *reinterpret_cast<Float4 *>(turned + m * 68u + d + h * 4u) = v;
            }
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (uint32_t k = 0; k < 8u; k++) {
                const uint32_t i = k * 4u + lane / 16u, dim = d0 + lane % 16u * 4u;
                const Float4 v = *reinterpret_cast<const Float4 *>(turned + i * 68u + lane % 16u * 4u);
                if (t.first + wave * 32u + i >= t.last) continue;
                if (whole) *reinterpret_cast<Word2 *>(a.out + ((size_t)(t.begin + t.first + wave * 32u + i) * heads + head_now) * kD + dim) = Word2{pk_bf16(v[0], v[1]), pk_bf16(v[2], v[3])};
                else *reinterpret_cast<Float4 *>(a.partial + ((size_t)place * kPromptRows + wave * 32u + i) * kD + dim) = v;
            }
            __builtin_amdgcn_wave_barrier();
        }
        __syncthreads();
    }
}

bool latent_prompt_fits(uint32_t tokens, uint32_t rows, uint32_t heads) { return ((uint64_t)tokens / kPromptRows + rows) * heads <= 0xFFFFFFu; }

static uint64_t prompt_tiles(uint32_t tokens, uint32_t rows, uint32_t heads) { return ((uint64_t)tokens / kPromptRows + (rows < tokens ? rows : tokens)) * heads; }
static Plan prompt_plan(uint32_t tokens, uint32_t rows, uint32_t heads, uint32_t dim, uint32_t keys)
{
    const uint64_t tiles = prompt_tiles(tokens, rows, heads), blocks = ((uint64_t)keys + kAttendBlock - 1u) / kAttendBlock;
    // Keys are known for all rows together.  Up to 12 blocks of 128 rows are taken to have as many each, and are left whole where that is few; above, one of them may have them all, and what is left whole would be long.  16 heads, us
    // left whole and cut: rows that are alike, 4 of 384 tokens 20 and 29, 5 of 384 23 and 31, 8 of 200 16 and 25; one row with nearly all keys, 128 tokens behind 1,500 51 and 20, behind 2,500 80 and 22, behind 4,000 124 and 26.  So
    // prompts that are alike, and a few too many for the 12 blocks, pay for those that are not.
    return plan_of(tiles, blocks, blocks <= 12u ? (blocks + rows - 1u) / rows : blocks, rows, tokens <= kPromptRows * rows, true, kPromptRows, dim, kPromptSlots, (uint64_t)tokens * heads);
}
uint64_t latent_prompt_bytes(uint32_t tokens, uint32_t rows, uint32_t heads, uint32_t dim, uint32_t keys) { return plan_bytes(prompt_plan(tokens, rows, heads, dim, keys)); }

hipError_t launch_latent_prompt(const void *q_n, const void *q_r, const void *k_n, const void *k_r, const void *v, uint32_t tokens, uint32_t keys, uint32_t heads, uint32_t dim,
                                const int64_t (&strides)[9], uint32_t rows, const int32_t *starts, const int32_t *key_starts, float factor, void *out, void *workspace, hipStream_t s)
{
    const Plan p = prompt_plan(tokens, rows, heads, dim, keys);
    float *partial = static_cast<float *>(workspace), *ends = partial + p.partial;
    auto halves = [](const void *x) { return static_cast<const uint16_t *>(x); };
    const LatentPromptArgs a{{starts, rows, tokens, heads, p.chunks}, halves(q_n), halves(q_r), halves(k_n), halves(k_r), halves(v),
                             strides[0], strides[1], strides[2], strides[3], strides[4], strides[5], strides[6], strides[7], strides[8], key_starts, static_cast<uint16_t *>(out),
                             partial, ends, reinterpret_cast<Parts *>(ends + p.ends), factor * 1.44269504088896340736f, keys};
    const dim3 grid(p.chunks ? p.chunks : (tokens / kPromptRows + rows) * heads);
    const hipError_t e = launch(dim == 128u ? latent_prompt_kernel<128> : latent_prompt_kernel<64>, grid, dim3(kThreads), 0, s, nullptr, a);
    if (e != hipSuccess || !p.chunks) return e;
    const JoinArgs j{a.partial, a.ends, a.parts, starts, a.out, rows, heads, p.chunks, kPromptRows, size_of(a.factor)};
    const bool many = p.chunks > kManyParts * prompt_tiles(tokens, rows, heads);
    return dim == 128u ? launch_join<128>(j, tokens, many, s) : launch_join<64>(j, tokens, many, s);
}

}  // namespace wg
