// The pages of a model's cache for gfx950: tables, slots and positions from the lengths of the rows, with the rows of a beam search following
// their parents (pages shared, a begun page copied, pages that nobody refers to given back).
//
// All of it is whole numbers: prefix sums over rows of pages needed, pages released and tokens.  Bound by launches and trips to memory, not by
// bytes: rows wait for the sums of the rows before them, which every workgroup works out by itself from the lengths (a few KB in the L2) in place of
// waiting for another.  Where rows follow parents, a first kernel counts for each request what it needs and releases (page_count_kernel), a workgroup for
// each; the second (page_kernel) sums that up and writes.
//
// A row's new table is its parent's whole one, so that within a request a page is referred to at one place of the tables only, and an old row with a
// child keeps all of its pages but for a begun one that all of its children copy.  Only what lies in the tables of rows without children is compared.
#include <hip/hip_runtime.h>

#include "wg_launch.h"
#include "wg_serve.h"

namespace wg {

constexpr uint32_t kPageThreads = 256, kPageWaves = kPageThreads / 64u;

// What a request needs: pages (kTooLong: a table that would not hold them), pages given back whatever becomes of it and those given back
// where it is served, tokens.
struct GroupNeed { uint32_t pages, released, released_served, tokens; };
constexpr uint32_t kTooLong = 0xFFFFFFFFu;

// The rows of a request before the step, after they took over their parents' tables.
struct Rows {
    int32_t source[kBeamMax];                        // the row whose table it takes; -1: none
    uint32_t length[kBeamMax], have[kBeamMax], count[kBeamMax];    // of the new row: tokens, pages, tokens to come
    uint32_t old_have[kBeamMax], col[kBeamMax];      // of the old row: pages; the place of the page that its children begin in
    uint32_t child[kBeamMax], all_fork[kBeamMax];    // of the old row: has children; all of them copy their begun page
    uint32_t fork[kBeamMax];                         // the new row copies its begun page
    uint32_t need[kBeamMax];
};

__device__ __forceinline__ uint32_t tokens_of(int32_t n, uint32_t most) { return n < 0 ? 0u : (uint32_t)n < most ? (uint32_t)n : most; }

__device__ __forceinline__ void read_rows(Rows &g, const int32_t *lens, const int32_t *counts, const int32_t *parents, uint32_t row0, uint32_t K, uint32_t M, uint32_t shift)
{
    const uint32_t k = threadIdx.x, page = 1u << shift;
    if (k < K) {
        const int32_t p = parents[row0 + k];
        const bool there = (uint32_t)p - row0 < K;
        g.source[k] = there ? p : -1;
        g.length[k] = there ? tokens_of(lens[p], M << shift) : 0u;
        g.count[k] = tokens_of(counts[row0 + k], 0x7FFFFFFFu);
        g.have[k] = (g.length[k] + page - 1u) >> shift;
        const uint32_t old = tokens_of(lens[row0 + k], M << shift);
        g.old_have[k] = (old + page - 1u) >> shift;
        g.col[k] = old >> shift;
        g.child[k] = 0u;
        g.all_fork[k] = 1u;
    }
}

// (after the forks are known; between two barriers)
__device__ __forceinline__ void follow_rows(Rows &g, uint32_t row0, uint32_t K, uint32_t shift)
{
    const uint32_t k = threadIdx.x, page = 1u << shift;
    if (k >= K) return;
    for (uint32_t c = 0; c < K; c++)
        if (g.source[c] == (int32_t)(row0 + k)) { g.child[k] = 1u; g.all_fork[k] &= g.fork[c]; }
    const uint64_t all = (uint64_t)g.length[k] + g.count[k];
    g.need[k] = g.fork[k] + (uint32_t)((all + page - 1u) >> shift) - g.have[k];
}

// Calls gone(b, id, whatever) for the pages of column j that no new row refers to, in the order of the old rows; whatever: they go whether or not the request
// is served.
template <typename F>
__device__ __forceinline__ void released_at(const Rows &g, const int32_t *table, uint32_t row0, uint32_t K, uint32_t M, uint32_t j, F gone)
{
    for (uint32_t b = 0; b < K; b++) {
        if (j >= g.old_have[b]) continue;
        if (g.child[b] && !(g.all_fork[b] && j == g.col[b])) continue;          // a child goes on with it
        const int32_t id = table[(size_t)(row0 + b) * M + j];
        bool first = true, referred = false, kept = false;
        for (uint32_t o = 0; o < K; o++) {
            if (j >= g.old_have[o] || table[(size_t)(row0 + o) * M + j] != id) continue;
            if (o < b) first = false;
            if (g.child[o]) { referred = true; kept |= !(g.all_fork[o] && j == g.col[o]); }
        }
        if (first && !kept) gone(id, !referred);
    }
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

__global__ void __launch_bounds__(kPageThreads)
page_count_kernel(const int32_t *__restrict__ table, const int32_t *__restrict__ lens, const int32_t *__restrict__ counts, const int32_t *__restrict__ parents,
                  uint32_t K, uint32_t M, uint32_t shift, GroupNeed *__restrict__ needs, uint32_t *__restrict__ forks)
{
    __shared__ Rows g;
    __shared__ uint32_t part[2][kPageWaves];
    const uint32_t tid = threadIdx.x, row0 = blockIdx.x * K, page = 1u << shift;
    read_rows(g, lens, counts, parents, row0, K, M, shift);
    __syncthreads();
    if (tid < K) {
        // a begun page that another row has too
        uint32_t fork = 0;
        if (g.count[tid] && (g.length[tid] & (page - 1u))) {
            const uint32_t c = g.length[tid] >> shift;
            const int32_t mine = table[(size_t)g.source[tid] * M + c];
            for (uint32_t o = 0; o < K; o++)
                if (o != tid && g.have[o] > c) fork |= table[(size_t)g.source[o] * M + c] == mine;
        }
        g.fork[tid] = fork;
        forks[row0 + tid] = fork;
    }
    __syncthreads();
    follow_rows(g, row0, K, shift);
    __syncthreads();
    uint32_t most = 0;
    for (uint32_t b = 0; b < K; b++) most = g.old_have[b] > most ? g.old_have[b] : most;
    uint32_t released = 0, served = 0;
    for (uint32_t j = tid; j < most; j += kPageThreads)
        released_at(g, table, row0, K, M, j, [&](int32_t, bool whatever) { (whatever ? released : served)++; });
    released = wave_sum(released); served = wave_sum(served);
    if ((tid & 63u) == 0u) { part[0][tid >> 6] = released; part[1][tid >> 6] = served; }
    __syncthreads();
    if (tid) return;
    GroupNeed n{0u, 0u, 0u, 0u};
    for (uint32_t w = 0; w < kPageWaves; w++) { n.released += part[0][w]; n.released_served += part[1][w]; }
    bool fits = true;
    for (uint32_t k = 0; k < K; k++) {
        n.tokens += g.count[k];
        n.pages += g.need[k];
        fits &= g.have[k] + g.need[k] - g.fork[k] <= M;
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
    uint32_t rows, K, M, shift, N, tokens, per;      // per: requests of a workgroup
};

__device__ __forceinline__ uint32_t ring_at(uint32_t base, uint32_t off, uint32_t N)
{
    const uint64_t i = (uint64_t)base + off;
    return (uint32_t)(i < N ? i : i - N < N ? i - N : i % N);
}

template <bool kParents>
__global__ void __launch_bounds__(kPageThreads)
page_kernel(const PageArgs a)
{
    __shared__ Rows g;
    __shared__ uint32_t part[kPageWaves];
    const uint32_t tid = threadIdx.x, page = 1u << a.shift, K = kParents ? a.K : 1u, G = a.rows / K;
    const uint32_t g0 = blockIdx.x * a.per, g1 = G - g0 < a.per ? G : g0 + a.per;
    const uint64_t taken = a.counters[0], given = a.counters[1];
    const uint32_t free = given <= taken ? 0u : given - taken < a.N ? (uint32_t)(given - taken) : a.N;
    const uint32_t head = (uint32_t)(taken % a.N), tail = (uint32_t)(given % a.N);
    auto need_of = [&](uint32_t i) {
        if (kParents) return a.needs[i];
        const uint32_t length = tokens_of(a.lens[i], a.M << a.shift), count = tokens_of(a.counts[i], 0x7FFFFFFFu);
        const uint32_t have = (length + page - 1u) >> a.shift, want = (uint32_t)(((uint64_t)length + count + page - 1u) >> a.shift);
        return GroupNeed{want > a.M ? kTooLong : want - have, 0u, 0u, count};
    };
    // The sums over the requests before this workgroup's, then request by request.  The last workgroup also goes over its own for the totals.
    uint32_t pages = 0, used = 0, released = 0, tokens = 0;       // pages asked for, pages handed out, pages given back, tokens
    // (pages asked for end above `free` once a request is not served, and every later one that needs any is not either; saturating: the sum of
    // what is asked for may pass 32 bits)
    auto add = [](uint32_t x, uint32_t y) { return x + y < x ? 0xFFFFFFFEu : x + y; };
    for (uint32_t i0 = 0; i0 < g0; i0 += kPageThreads) {
        const uint32_t i = i0 + tid;
        const GroupNeed n = i < g0 ? need_of(i) : GroupNeed{0u, 0u, 0u, 0u};
        const uint32_t asks = n.pages == kTooLong ? 0u : n.pages < a.N + 1u ? n.pages : a.N + 1u;
        uint32_t all;
        const uint32_t end = add(pages, block_scan(asks, part, &all));
        const bool served = n.pages != kTooLong && (asks == 0u || end <= free);
        pages = add(pages, all);
        (void)block_scan(served ? asks : 0u, part, &all);
        used += all;
        if (kParents) { (void)block_scan(n.released + (served ? n.released_served : 0u), part, &all); released += all; }
        (void)block_scan(n.tokens, part, &all);
        tokens += all;
    }
    for (uint32_t i = g0; i < g1; i++) {
        const GroupNeed n = need_of(i);
        const uint32_t asks = n.pages == kTooLong ? 0u : n.pages < a.N + 1u ? n.pages : a.N + 1u, end = add(pages, asks), row0 = i * K;
        const bool served = n.pages != kTooLong && (asks == 0u || end <= free);
        if (kParents) {
            __syncthreads();
            read_rows(g, a.lens, a.counts, a.parents, row0, K, a.M, a.shift);
            if (tid < K) g.fork[tid] = a.forks[row0 + tid];
            __syncthreads();
            follow_rows(g, row0, K, a.shift);
            __syncthreads();
        }
        uint32_t first_page = pages, first_token = tokens;
        for (uint32_t k = 0; k < K; k++) {
            const uint32_t r = row0 + k;
            const uint32_t length = kParents ? g.length[k] : tokens_of(a.lens[r], a.M << a.shift), have = (length + page - 1u) >> a.shift;
            const uint32_t count = kParents ? g.count[k] : n.tokens, fork = kParents && served ? g.fork[k] : 0u;
            const uint32_t want = served ? (length + count + page - 1u) >> a.shift : have, col = length >> a.shift;
            const int32_t *from = a.table + (size_t)(kParents ? (g.source[k] < 0 ? 0 : g.source[k]) : (int32_t)r) * a.M;
            int32_t *to = a.table_out + (size_t)r * a.M;
            auto fresh = [&](uint32_t at) { return a.ring[ring_at(head, first_page + at, a.N)]; };
            auto page_at = [&](uint32_t j) { return j >= have ? fresh(fork + j - have) : fork && j == col ? fresh(0u) : from[j]; };
            for (uint32_t j = (from == to ? have : 0u) + tid; j < want; j += kPageThreads) to[j] = page_at(j);
            for (uint32_t t = tid; t < count; t += kPageThreads) {
                const uint32_t at = first_token + t, pos = length + t;
                if (at >= a.tokens || at < first_token) break;
                a.positions[at] = (int32_t)pos;
                a.slots[at] = served ? page_at(pos >> a.shift) << a.shift | (int32_t)(pos & (page - 1u)) : -1;
                a.origins[at] = t == 0u && fork ? from[col] : -1;
            }
            if (tid == 0u) { a.lens_out[r] = (int32_t)(served ? length + count : length); a.starts[r] = (int32_t)first_token; }
            if (served) first_page += kParents ? g.need[k] : asks;
            first_token += count;
        }
        if (kParents && (n.released || (served && n.released_served))) {
            // pages go back by place in the tables, then by row
            uint32_t most = 0, base = released;
            for (uint32_t b = 0; b < K; b++) most = g.old_have[b] > most ? g.old_have[b] : most;
            for (uint32_t j0 = 0; j0 < most; j0 += kPageThreads) {
                uint32_t mine = 0, all;
                if (j0 + tid < most) released_at(g, a.table, row0, K, a.M, j0 + tid, [&](int32_t, bool whatever) { mine += whatever || served; });
                uint32_t at = base + block_scan(mine, part, &all) - mine;
                if (mine)
                    released_at(g, a.table, row0, K, a.M, j0 + tid, [&](int32_t id, bool whatever) { if (whatever || served) a.ring[ring_at(tail, at++, a.N)] = id; });
                base += all;
            }
        }
        pages = end;
        if (served) used += asks;
        released += n.released + (served ? n.released_served : 0u);
        tokens += n.tokens;
    }
    if (g1 == G && tid == 0u) {
        a.starts[a.rows] = (int32_t)tokens;
        a.counters_out[0] = taken + used;
        a.counters_out[1] = given + released;
    }
}

hipError_t launch_page_step(const int32_t *table, uint32_t rows, uint32_t columns, const int32_t *lens, const int32_t *counts, const int32_t *parents,
                            uint32_t K, uint32_t shift, int32_t *ring, uint32_t pages, const uint64_t *counters, int32_t *table_out, int32_t *lens_out,
                            int32_t *starts, int32_t *slots, int32_t *positions, int32_t *origins, uint32_t tokens, uint64_t *counters_out,
                            void *workspace, hipStream_t s)
{
    GroupNeed *needs = static_cast<GroupNeed *>(workspace);
    const uint32_t G = rows / K;
    uint32_t *forks = reinterpret_cast<uint32_t *>(needs + G);
    // every workgroup goes over all requests before its own: at most 512 of them
    const uint32_t per = (G + 511u) / 512u;
    const PageArgs a{table, lens, counts, parents, ring, counters, table_out, lens_out, starts, slots, positions, origins, counters_out,
                     needs, forks, rows, K, columns, shift, pages, tokens, per};
    const dim3 grid((G + per - 1u) / per), block(kPageThreads);
    if (!parents) return launch(page_kernel<false>, grid, block, 0, s, nullptr, a);
    const hipError_t e = launch(page_count_kernel, dim3(G), block, 0, s, nullptr, table, lens, counts, parents, K, columns, shift, needs, forks);
    if (e != hipSuccess) return e;
    return launch(page_kernel<true>, grid, block, 0, s, nullptr, a);
}

}  // namespace wg
