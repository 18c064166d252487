// The pages of a model's cache for gfx950: tables, slots and positions from the lengths of the rows, with the rows of a beam search following
// their parents (pages shared, a begun page copied, pages that nobody refers to given back).
//
// All of it is whole numbers: prefix sums over rows of pages needed, pages released and tokens.  Bound by launches and trips to memory, not by
// bytes: rows wait for the sums of the rows before them, which every workgroup works out by itself from the lengths (a few KB in the L2) in place of
// waiting for another.  Where rows follow parents, a first kernel counts what each request needs and releases (page_count_kernel); the second
// (page_beam_kernel) sums that up and writes.  A workgroup of either takes up to 256 columns of a request's tables, which it holds in LDS: a thread's loads of eight rows are
// in flight together, and what it looks for among the rows of a column it finds there.
//
// A row's new table is its parent's whole one, so that within a request a page is referred to at one place of the tables only, and an old row with a
// child keeps all of its pages but for a begun one that all of its children copy.  Only what lies in the tables of rows without children is compared.
//
// 256 rows without parents 3.9 us; 64 requests of eight beams with 1,024 columns 6.0 and 11.2 (2.6 MB read and written: 0.5 us of a copy).
#include <hip/hip_runtime.h>

#include "wg_launch.h"
#include "wg_serve.h"

namespace wg {

constexpr uint32_t kPageThreads = 256, kPageWaves = kPageThreads / 64u;

// What a request needs: pages (kTooLong: a table that would not hold them), and its tokens.
struct GroupNeed { uint32_t pages, tokens; };
// Pages that a request gives back from some columns of its tables: whatever becomes of it, and where it is served besides.
struct Back { uint32_t always, served; };
constexpr uint32_t kTooLong = 0xFFFFFFFFu;

// Threads that share a column of a request's tables, and with it the rows whose pages are looked for among the others: each has eight of them at the most.  (A thread
// for a column of any number of rows took 256 us for 8 requests of 64 beams and 512 columns, eight take 75; for 32 requests of 16 beams 50, two take 28.)  A workgroup takes as
// many columns as that leaves it.  kFew: up to eight rows, of kernels that know it (18.4 us without, 17.7 with, for 32 requests of eight beams).
static __host__ __device__ inline uint32_t sharers_of(uint32_t K) { return K <= 8u ? 1u : K <= 16u ? 2u : K <= 32u ? 4u : 8u; }
static __host__ __device__ inline uint32_t columns_of(uint32_t K) { return kPageThreads / sharers_of(K); }

// The rows of a request before the step, after they took over their parents' tables.
struct Rows {
    // of the new row: the row of the request whose table it takes (-1: none), its pages, its pages in all with the step, the place of a begun page that it
    // copies (kNoFork: none)
    int4 rows[kBeamMax];
    uint32_t length[kBeamMax], count[kBeamMax], need[kBeamMax];    // its tokens, tokens to come, pages to be handed out
    // of the old row: its pages; those of them that some child has (all or none); those that a child goes on with (all but a begun one that all children copy)
    uint4 ends[kBeamMax];
};
constexpr uint32_t kNoFork = 0xFFFFFFFFu;

__device__ __forceinline__ uint32_t tokens_of(int32_t n, uint32_t most) { return n < 0 ? 0u : (uint32_t)n < most ? (uint32_t)n : most; }

// The request's columns [j0, j0 + width) to LDS, row by row.
__device__ __forceinline__ void read_columns(int32_t *ids, const int32_t *table, uint32_t row0, uint32_t K, uint32_t M, uint32_t j0, uint32_t width)
{
    const uint32_t tid = threadIdx.x, c = tid & (width - 1u), j = j0 + c, step = kPageThreads / width;
    if (j >= M) return;
    uint32_t k = tid / width;
    for (; k + 7u * step < K; k += 8u * step) {
        int32_t x[8];
#pragma unroll
        for (uint32_t i = 0; i < 8u; i++) x[i] = table[(size_t)(row0 + k + i * step) * M + j];
#pragma unroll
        for (uint32_t i = 0; i < 8u; i++) ids[(k + i * step) * width + c] = x[i];
    }
    for (; k < K; k += step) ids[k * width + c] = table[(size_t)(row0 + k) * M + j];
}

// What a thread k < K asks for of its row, early.
struct RowLoads { int32_t parent, len, count; uint32_t fork; };
__device__ __forceinline__ RowLoads load_row(const int32_t *lens, const int32_t *counts, const int32_t *parents, const uint32_t *forks, uint32_t row0, uint32_t K)
{
    const uint32_t k = threadIdx.x, r = row0 + k;
    return k < K ? RowLoads{parents[r], lens[r], counts[r], forks ? forks[r] : 0u} : RowLoads{0, 0, 0, 0u};
}

// Fills in g.  kFind: and finds the forks (else they came with x): those that begin in the columns [j0, j0 + width), which lie in ids, and with `all` the others
// too.  The first wavefront does it, a lane to a row, with the rows' values out of its registers.  The whole workgroup calls it, behind a barrier after
// read_columns where forks are to be found; it ends behind a barrier.
template <bool kFind>
__device__ __forceinline__ void read_rows(Rows &g, const RowLoads &x, const int32_t *table, const int32_t *ids, uint32_t j0, uint32_t width, bool all, uint32_t row0, uint32_t K,
                                          uint32_t M, uint32_t shift)
{
    const uint32_t k = threadIdx.x, page = 1u << shift;
    if (k < 64u) {
        const bool row = k < K;
        const int32_t p = x.parent - (int32_t)row0;
        const int32_t source = row && (uint32_t)p < K ? p : -1;
        const uint32_t old = row ? tokens_of(x.len, M << shift) : 0u, count = tokens_of(x.count, 0x7FFFFFFFu), parents = (uint32_t)__shfl((int32_t)old, source < 0 ? 0 : source);
        const uint32_t length = source < 0 ? 0u : parents, have = (length + page - 1u) >> shift, col = length >> shift;
        const bool begun = row && count && (length & (page - 1u));
        uint32_t fork = x.fork;
        if (kFind) {
            fork = 0u;
#pragma unroll 4
            for (uint32_t r = 0; r < K; r++) {            // a begun page that another row has too
                const uint32_t c = (uint32_t)__builtin_amdgcn_readlane((int32_t)col, r), mine = (uint32_t)__builtin_amdgcn_readlane(source, r);
                const bool here = c - j0 < width, there = have > c && k != r;
                if (!here && !all) continue;
                int32_t id = 0, of = 0;
                if (there) {
                    id = here ? ids[(uint32_t)source * width + c - j0] : table[(size_t)(row0 + (uint32_t)source) * M + c];
                    of = (int32_t)mine < 0 ? 0 : here ? ids[mine * width + c - j0] : table[(size_t)(row0 + mine) * M + c];
                }
                const bool shared = __ballot(there && id == of) != 0ull;
                if (k == r) fork = begun && shared;
            }
        }
        bool child = false, copied = true;
#pragma unroll 8
        for (uint32_t c = 0; c < K; c++)
            if (__builtin_amdgcn_readlane(source, c) == (int32_t)k) { child = true; copied &= __builtin_amdgcn_readlane((int32_t)fork, c) != 0; }
        if (row) {
            const uint32_t pages = (old + page - 1u) >> shift, want = (uint32_t)(((uint64_t)length + count + page - 1u) >> shift);
            g.ends[k] = uint4{pages, child ? pages : 0u, child ? (copied ? old >> shift : pages) : 0u, 0u};
            g.rows[k] = int4{source, (int32_t)have, (int32_t)want, (int32_t)(fork ? col : kNoFork)};
            g.length[k] = length; g.count[k] = count; g.need[k] = (fork ? 1u : 0u) + want - have;
        }
    }
    __syncthreads();
}

// The old rows whose page at column j goes back, as bits: whatever becomes of the request, and where it is served besides.  ids: the column.  Of several threads of a
// column each one answers for the rows that are `turn` modulo their number.
struct Gone { unsigned long long always, served; };
template <bool kFew>
__device__ __forceinline__ Gone gone_at(const Rows &g, const int32_t *ids, uint32_t width, uint32_t K, uint32_t j, uint32_t turn)
{
    Gone r{0ull, 0ull};
    if (kFew) {
        // eight rows out of registers (by the loop below, trips to LDS one after the other, twice as long: 2.7 us for eight beams)
        int32_t id[8];
        uint32_t in = 0, referred = 0, kept = 0;      // the rows whose tables reach so far; as far as a child has them; as far as one goes on with them
#pragma unroll
        for (uint32_t o = 0; o < 8u; o++) {
            const uint32_t k = o < K ? o : 0u;
            const uint4 e = g.ends[k];
            id[o] = ids[k * width];
            in |= (uint32_t)(o < K && j < e.x) << o;
            referred |= (uint32_t)(o < K && j < e.y) << o;
            kept |= (uint32_t)(o < K && j < e.z) << o;
        }
        uint32_t always = 0, served = 0;
#pragma unroll
        for (uint32_t b = 0; b < 8u; b++) {
            uint32_t same = 0;
#pragma unroll
            for (uint32_t o = 0; o < 8u; o++) same |= (uint32_t)(id[o] == id[b]) << o;
            same &= in;
            const bool gone = (same >> b & 1u) && !(same & ((1u << b) - 1u)) && !(same & kept);
            if (gone) { if (same & referred) served |= 1u << b; else always |= 1u << b; }
        }
        r.always = always; r.served = served;
        return r;
    }
    unsigned long long in = 0, referred = 0, kept = 0;
#pragma unroll 8
    for (uint32_t o = 0; o < K; o++) {
        const uint4 e = g.ends[o];
        in |= (unsigned long long)(j < e.x) << o;
        referred |= (unsigned long long)(j < e.y) << o;
        kept |= (unsigned long long)(j < e.z) << o;
    }
    const uint32_t sharers = kPageThreads / width;
    for (uint32_t b = turn; b < K; b += sharers) {
        if (!((in & ~kept) >> b & 1ull)) continue;    // (a child goes on with the others)
        const int32_t id = ids[b * width];
        unsigned long long same = 0;
        uint32_t o = 0;
        for (; o + 8u <= K; o += 8u) {
            uint32_t eight = 0;
#pragma unroll
            for (uint32_t i = 0; i < 8u; i++) eight |= (uint32_t)(ids[(o + i) * width] == id) << i;
            same |= (unsigned long long)eight << o;
        }
        for (; o < K; o++) same |= (unsigned long long)(ids[o * width] == id) << o;
        same &= in;
        if ((same & ((1ull << b) - 1ull)) || (same & kept)) continue;
        if (same & referred) r.served |= 1ull << b; else r.always |= 1ull << b;
    }
    return r;
}

__device__ __forceinline__ uint32_t wave_sum(uint32_t x)
{
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o);
    return x;
}
// The sums of the workgroup's values up to each thread's, its own with it, and of all; `part` is kPageWaves words of LDS.
__device__ __forceinline__ uint32_t block_scan(uint32_t x, uint32_t *part, uint32_t *all)
{
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6;
#pragma unroll
    for (uint32_t o = 1; o < 64u; o <<= 1) { const uint32_t y = __shfl_up(x, o); if (lane >= o) x += y; }
    __syncthreads();
    if (lane == 63u) part[wave] = x;
    __syncthreads();
    uint32_t before = 0, sum = 0;
#pragma unroll
    for (uint32_t w = 0; w < kPageWaves; w++) { if (w < wave) before += part[w]; sum += part[w]; }
    *all = sum;
    return x + before;
}

template <bool kFew>
__global__ void __launch_bounds__(kPageThreads)
page_count_kernel(const int32_t *__restrict__ table, const int32_t *__restrict__ lens, const int32_t *__restrict__ counts, const int32_t *__restrict__ parents,
                  uint32_t K, uint32_t M, uint32_t shift, GroupNeed *__restrict__ needs, uint32_t *__restrict__ forks, Back *__restrict__ back)
{
    extern __shared__ int32_t ids[];
    __shared__ Rows g;
    __shared__ uint32_t part[2][kPageWaves];
    const uint32_t tid = threadIdx.x, row0 = blockIdx.x * K, width = kFew ? kPageThreads : columns_of(K), sharers = kPageThreads / width, c = tid / sharers, j = blockIdx.y * width + c;
    const RowLoads row = load_row(lens, counts, parents, nullptr, row0, K);
    read_columns(ids, table, row0, K, M, blockIdx.y * width, width);
    __syncthreads();
    read_rows<true>(g, row, table, ids, blockIdx.y * width, width, blockIdx.y == 0u, row0, K, M, shift);
    Gone gone{0ull, 0ull};
    if (j < M) gone = gone_at<kFew>(g, ids + c, width, K, j, tid % sharers);
    const uint32_t always = wave_sum((uint32_t)__popcll(gone.always)), served = wave_sum((uint32_t)__popcll(gone.served));
    if ((tid & 63u) == 0u) { part[0][tid >> 6] = always; part[1][tid >> 6] = served; }
    __syncthreads();
    if (blockIdx.y == 0u && tid < K) forks[row0 + tid] = (uint32_t)g.rows[tid].w != kNoFork;
    if (tid) return;
    Back b{0u, 0u};
    for (uint32_t w = 0; w < kPageWaves; w++) { b.always += part[0][w]; b.served += part[1][w]; }
    back[(size_t)blockIdx.x * gridDim.y + blockIdx.y] = b;
    if (blockIdx.y) return;
    GroupNeed n{0u, 0u};
    bool fits = true;
#pragma unroll 8
    for (uint32_t k = 0; k < K; k++) {
        n.tokens += g.count[k];
        n.pages += g.need[k];
        fits &= (uint32_t)g.rows[k].z <= M;
    }
    if (!fits) n.pages = kTooLong;
    needs[blockIdx.x] = n;
}

struct PageArgs {
    const int32_t *table, *lens, *counts, *parents;
    int32_t *ring;
    const uint64_t *counters;
    int32_t *table_out, *lens_out, *starts, *slots, *positions, *origins;
    uint64_t *counters_out;
    const GroupNeed *needs;
    const uint32_t *forks;
    const Back *back;
    uint32_t rows, K, M, shift, N, tokens, per;      // per: requests of a workgroup
};

__device__ __forceinline__ uint32_t ring_at(uint32_t base, uint32_t off, uint32_t N)
{
    const uint64_t i = (uint64_t)base + off;
    return (uint32_t)(i < N ? i : i - N < N ? i - N : i % N);
}

// Pages asked for: they end above what is free once a request is not served, and then no later one that needs any is either.  (Saturating: the sum may pass 32 bits.)
__device__ __forceinline__ uint32_t add(uint32_t x, uint32_t y) { return x + y < x ? 0xFFFFFFFEu : x + y; }

// Sums over the requests before one: pages asked for, handed out and given back, tokens.
struct Sums { uint32_t pages, used, released, tokens; };
struct Served { uint32_t asks, end; bool yes; };
__device__ __forceinline__ Served served_of(const GroupNeed &n, uint32_t before, uint32_t free, uint32_t N)
{
    const uint32_t asks = n.pages == kTooLong ? 0u : n.pages < N + 1u ? n.pages : N + 1u, end = add(before, asks);
    return Served{asks, end, n.pages != kTooLong && (asks == 0u || end <= free)};
}

// The workgroup's sums of five values of its threads; `part` is 5 * kPageWaves words of LDS.
struct Five { uint32_t x[5]; };
__device__ __forceinline__ Five block_sums(Five v, uint32_t *part)
{
#pragma unroll
    for (uint32_t i = 0; i < 5u; i++) v.x[i] = wave_sum(v.x[i]);
    __syncthreads();
    if ((threadIdx.x & 63u) == 0u)
#pragma unroll
        for (uint32_t i = 0; i < 5u; i++) part[i * kPageWaves + (threadIdx.x >> 6)] = v.x[i];
    __syncthreads();
#pragma unroll
    for (uint32_t i = 0; i < 5u; i++) {
        v.x[i] = 0u;
#pragma unroll
        for (uint32_t w = 0; w < kPageWaves; w++) v.x[i] += part[i * kPageWaves + w];
    }
    return v;
}

// Without parents: requests of one row.
__global__ void __launch_bounds__(kPageThreads)
page_kernel(const PageArgs a)
{
    __shared__ uint32_t part[5u * kPageWaves];
    const uint32_t tid = threadIdx.x, page = 1u << a.shift;
    const uint32_t r0 = blockIdx.x * a.per, r1 = a.rows - r0 < a.per ? a.rows : r0 + a.per;
    const uint64_t taken = a.counters[0], given = a.counters[1];
    const uint32_t free = given <= taken ? 0u : given - taken < a.N ? (uint32_t)(given - taken) : a.N, head = (uint32_t)(taken % a.N);
    auto need_of = [&](uint32_t r) {
        const uint32_t length = tokens_of(a.lens[r], a.M << a.shift), count = tokens_of(a.counts[r], 0x7FFFFFFFu);
        const uint32_t have = (length + page - 1u) >> a.shift, want = (uint32_t)(((uint64_t)length + count + page - 1u) >> a.shift);
        return GroupNeed{want > a.M ? kTooLong : want - have, count};
    };
    Sums s{0u, 0u, 0u, 0u};
    Five own{{0u, 0u, 0u, 0u, 0u}};                   // the thread's share: pages handed out, tokens
    for (uint32_t i0 = 0; i0 < r0; i0 += kPageThreads) {
        const GroupNeed n = i0 + tid < r0 ? need_of(i0 + tid) : GroupNeed{0u, 0u};
        const uint32_t asks = served_of(n, 0u, 0u, a.N).asks;
        uint32_t all;
        const uint32_t end = block_scan(asks, part, &all);
        own.x[0] += served_of(n, add(s.pages, end - asks), free, a.N).yes ? asks : 0u;
        own.x[1] += n.tokens;
        s.pages = add(s.pages, all);
    }
    if (r0) { own = block_sums(own, part); s.used = own.x[0]; s.tokens = own.x[1]; }
    for (uint32_t r = r0; r < r1; r++) {
        const GroupNeed n = need_of(r);
        const Served v = served_of(n, s.pages, free, a.N);
        const uint32_t length = tokens_of(a.lens[r], a.M << a.shift), have = (length + page - 1u) >> a.shift;
        const uint32_t want = v.yes ? (length + n.tokens + page - 1u) >> a.shift : have, first = s.pages;
        const int32_t *from = a.table + (size_t)r * a.M;
        int32_t *to = a.table_out + (size_t)r * a.M;
        auto page_at = [&](uint32_t j) { return j >= have ? a.ring[ring_at(head, first + j - have, a.N)] : from[j]; };
        for (uint32_t j = (from == to ? have : 0u) + tid; j < want; j += kPageThreads) to[j] = page_at(j);
        for (uint32_t t = tid; t < n.tokens; t += kPageThreads) {
            const uint32_t at = s.tokens + t, pos = length + t;
            if (at >= a.tokens || at < s.tokens) break;
            a.positions[at] = (int32_t)pos;
            a.slots[at] = v.yes ? page_at(pos >> a.shift) << a.shift | (int32_t)(pos & (page - 1u)) : -1;
            a.origins[at] = -1;
        }
        if (tid == 0u) { a.lens_out[r] = (int32_t)(v.yes ? length + n.tokens : length); a.starts[r] = (int32_t)s.tokens; }
        s.pages = v.end;
        if (v.yes) s.used += v.asks;
        s.tokens += n.tokens;
    }
    if (r1 == a.rows && tid == 0u) {
        a.starts[a.rows] = (int32_t)s.tokens;
        a.counters_out[0] = taken + s.used;
        a.counters_out[1] = given;
    }
}

// With parents: a workgroup takes some columns of a request's tables; the one of the first columns also the tokens.
template <bool kFew>
__global__ void __launch_bounds__(kPageThreads)
page_beam_kernel(const PageArgs a)
{
    extern __shared__ int32_t ids[];
    __shared__ Rows g;
    __shared__ uint32_t part[5u * kPageWaves], begins[2][kBeamMax], flags[kPageThreads];
    const uint32_t tid = threadIdx.x, page = 1u << a.shift, K = a.K, G = a.rows / K, width = kFew ? kPageThreads : columns_of(K), sharers = kPageThreads / width, j0 = blockIdx.y * width, chunks = gridDim.y;
    const uint32_t g0 = blockIdx.x * a.per, g1 = G - g0 < a.per ? G : g0 + a.per;
    const uint64_t taken = a.counters[0], given = a.counters[1];
    const uint32_t free = given <= taken ? 0u : given - taken < a.N ? (uint32_t)(given - taken) : a.N;
    const uint32_t head = (uint32_t)(taken % a.N), tail = (uint32_t)(given % a.N);
    // Asked for at once: the columns, the rows of the workgroup's first request, and of the requests before it what the first rounds below look at.
    constexpr uint32_t kAhead = 4;
    RowLoads row = load_row(a.lens, a.counts, a.parents, a.forks, g0 * K, K);
    GroupNeed need = a.needs[g0];
    Back mine = tid < chunks ? a.back[(size_t)g0 * chunks + tid] : Back{0u, 0u};
    const GroupNeed first_need = tid < g0 ? a.needs[tid] : GroupNeed{0u, 0u};
    const uint32_t first_entries = (g0 < kPageThreads ? g0 : kPageThreads) * chunks;
    Back first_back[kAhead];
#pragma unroll
    for (uint32_t q = 0; q < kAhead; q++) first_back[q] = tid + q * kPageThreads < first_entries ? a.back[tid + q * kPageThreads] : Back{0u, 0u};
    read_columns(ids, a.table, g0 * K, K, a.M, j0, width);
    Sums s{0u, 0u, 0u, 0u};
    Five own{{0u, 0u, 0u, 0u, 0u}};                   // the thread's share: pages handed out, tokens, pages given back; those of the own request, and before these columns
    for (uint32_t i0 = 0; i0 < g0; i0 += kPageThreads) {
        const uint32_t n_groups = g0 - i0 < kPageThreads ? g0 - i0 : kPageThreads, entries = n_groups * chunks;
        const GroupNeed n = !i0 ? first_need : tid < n_groups ? a.needs[i0 + tid] : GroupNeed{0u, 0u};
        const uint32_t asks = served_of(n, 0u, 0u, a.N).asks;
        uint32_t all;
        const uint32_t end = block_scan(asks, part, &all);
        const bool yes = served_of(n, add(s.pages, end - asks), free, a.N).yes;
        own.x[0] += yes ? asks : 0u;
        own.x[1] += n.tokens;
        s.pages = add(s.pages, all);
        flags[tid] = yes;
        __syncthreads();
        auto back = [&](uint32_t e, const Back &b) { own.x[2] += b.always + (b.served && flags[e / chunks] ? b.served : 0u); };
        if (!i0)
#pragma unroll
            for (uint32_t q = 0; q < kAhead; q++) if (tid + q * kPageThreads < entries) back(tid + q * kPageThreads, first_back[q]);
        for (uint32_t e = tid + (i0 ? 0u : kAhead * kPageThreads); e < entries; e += kPageThreads) back(e, a.back[(size_t)i0 * chunks + e]);
    }
    for (uint32_t i = g0; i < g1; i++) {
        const uint32_t row0 = i * K;
        if (i != g0) {
            __syncthreads();
            row = load_row(a.lens, a.counts, a.parents, a.forks, row0, K);
            need = a.needs[i];
            mine = tid < chunks ? a.back[(size_t)i * chunks + tid] : Back{0u, 0u};
            read_columns(ids, a.table, row0, K, a.M, j0, width);
        }
        const GroupNeed n = need;
        const Served v = served_of(n, s.pages, free, a.N);
        own.x[3] = own.x[4] = 0u;
        for (uint32_t c = tid; c < chunks; c += kPageThreads) {
            const Back b = c == tid ? mine : a.back[(size_t)i * chunks + c];
            const uint32_t x = b.always + (v.yes ? b.served : 0u);
            own.x[3] += x;
            if (c < blockIdx.y) own.x[4] += x;
        }
        const Five sums = block_sums(own, part);
        if (i == g0) { s.used = sums.x[0]; s.tokens = sums.x[1]; s.released = sums.x[2]; }
        const uint32_t back = sums.x[3], before = sums.x[4];
        read_rows<false>(g, row, a.table, ids, j0, width, false, row0, K, a.M, a.shift);
        if (tid < K) {                                // where each row's pages and tokens begin
            uint32_t p = s.pages, t = s.tokens;
#pragma unroll 8
            for (uint32_t k = 0; k < tid; k++) { p += g.need[k]; t += g.count[k]; }
            begins[0][tid] = p; begins[1][tid] = t;
        }
        __syncthreads();
        auto page_of = [&](uint32_t k, uint32_t at) { return a.ring[ring_at(head, begins[0][k] + at, a.N)]; };
        {
            const uint32_t c = tid & (width - 1u), j = j0 + c;
#pragma unroll 4
            for (uint32_t k = tid / width; k < K; k += sharers) {
                const int4 row = g.rows[k];               // source, pages, pages with the step, place of the fork
                const uint32_t have = (uint32_t)row.y, fork = v.yes ? (uint32_t)row.w : kNoFork;
                if (j >= (v.yes ? (uint32_t)row.z : have)) continue;
                int32_t id = ids[(row.x < 0 ? 0u : (uint32_t)row.x) * width + c];
                if (j >= have) id = page_of(k, (fork != kNoFork ? 1u : 0u) + j - have);
                else if (j == fork) id = page_of(k, 0u);
                a.table_out[(size_t)(row0 + k) * a.M + j] = id;
            }
        }
        if (blockIdx.y == 0u) {
            for (uint32_t k = tid >> 6; k < K; k += kPageWaves) {
                const int4 row = g.rows[k];
                const uint32_t length = g.length[k], count = g.count[k], have = (uint32_t)row.y, fork = v.yes ? (uint32_t)row.w : kNoFork, first = begins[1][k], r = row0 + k;
                const int32_t *from = a.table + (size_t)(row0 + (row.x < 0 ? 0u : (uint32_t)row.x)) * a.M;
                auto page_at = [&](uint32_t c) { return c >= have ? page_of(k, (fork != kNoFork ? 1u : 0u) + c - have) : c == fork ? page_of(k, 0u) : from[c]; };
                for (uint32_t t = tid & 63u; t < count; t += 64u) {
                    const uint32_t at = first + t, pos = length + t;
                    if (at >= a.tokens || at < first) break;
                    a.positions[at] = (int32_t)pos;
                    a.slots[at] = v.yes ? page_at(pos >> a.shift) << a.shift | (int32_t)(pos & (page - 1u)) : -1;
                    a.origins[at] = t == 0u && fork != kNoFork ? from[fork] : -1;
                }
                if ((tid & 63u) == 0u) { a.lens_out[r] = (int32_t)(v.yes ? length + count : length); a.starts[r] = (int32_t)first; }
            }
        }
        if (back) {
            // pages go back by place in the tables, then by row
            Gone gone{0ull, 0ull};
            const uint32_t c = tid / sharers, turn = tid % sharers;
            if (j0 + c < a.M) gone = gone_at<kFew>(g, ids + c, width, K, j0 + c, turn);
            unsigned long long rows = gone.always | (v.yes ? gone.served : 0ull);
            for (uint32_t o = 1; o < sharers; o <<= 1) rows |= __shfl_xor(rows, o);
            if (turn) rows = 0ull;                    // (the first one writes them)
            const uint32_t count = (uint32_t)__popcll(rows);
            uint32_t all, at = s.released + before + block_scan(count, part, &all) - count;
            for (; rows; rows &= rows - 1ull) a.ring[ring_at(tail, at++, a.N)] = ids[(uint32_t)__builtin_ctzll(rows) * width + c];
        }
        s.pages = v.end;
        if (v.yes) s.used += v.asks;
        s.released += back;
        s.tokens += n.tokens;
    }
    if (g1 == G && blockIdx.y == 0u && tid == 0u) {
        a.starts[a.rows] = (int32_t)s.tokens;
        a.counters_out[0] = taken + s.used;
        a.counters_out[1] = given + s.released;
    }
}

static uint32_t chunks_of(uint32_t K, uint32_t columns) { return (columns + columns_of(K) - 1u) / columns_of(K); }

uint64_t page_step_bytes(uint32_t rows, uint32_t K, uint32_t columns)
{
    const uint64_t G = rows / K;
    return G * (sizeof(GroupNeed) + chunks_of(K, columns) * sizeof(Back)) + rows * 4ull;
}

hipError_t launch_page_step(const int32_t *table, uint32_t rows, uint32_t columns, const int32_t *lens, const int32_t *counts, const int32_t *parents,
                            uint32_t K, uint32_t shift, int32_t *ring, uint32_t pages, const uint64_t *counters, int32_t *table_out, int32_t *lens_out,
                            int32_t *starts, int32_t *slots, int32_t *positions, int32_t *origins, uint32_t tokens, uint64_t *counters_out,
                            void *workspace, hipStream_t s)
{
    const uint32_t G = rows / K, chunks = chunks_of(K, columns);
    GroupNeed *needs = static_cast<GroupNeed *>(workspace);
    Back *back = reinterpret_cast<Back *>(needs + G);
    uint32_t *forks = reinterpret_cast<uint32_t *>(back + (size_t)G * chunks);
    // every workgroup goes over all requests before its own: at most 2,048 of them for the same columns (of 4,096 requests of
    // four beams: 81 us with 512, 65 with 2,048)
    const uint32_t per = (G + 2047u) / 2048u;
    const PageArgs a{table, lens, counts, parents, ring, counters, table_out, lens_out, starts, slots, positions, origins, counters_out,
                     needs, forks, back, rows, K, columns, shift, pages, tokens, per};
    const dim3 block(kPageThreads);
    if (!parents) return launch(page_kernel, dim3((G + per - 1u) / per), block, 0, s, nullptr, a);
    const bool few = K <= 8u;
    const uint32_t lds = K * columns_of(K) * 4u;
    const hipError_t e = launch(few ? page_count_kernel<true> : page_count_kernel<false>, dim3(G, chunks), block, lds, s, nullptr, table, lens, counts, parents, K, columns, shift, needs, forks, back);
    if (e != hipSuccess) return e;
    return launch(few ? page_beam_kernel<true> : page_beam_kernel<false>, dim3((G + per - 1u) / per, chunks), block, lds, s, nullptr, a);
}

}  // namespace wg
