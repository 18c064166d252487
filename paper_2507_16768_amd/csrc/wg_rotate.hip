// Rotary positions for gfx950: pairs of a head's numbers turned by the angle position * frequency.
#include <hip/hip_runtime.h>

#include "wg_launch.h"
#include "wg_number.h"
#include "wg_serve.h"

namespace wg {

constexpr uint32_t kRotateThreads = 256, kOnce = 4;

struct RotateArgs {
    const void *x[2];                                // queries, keys: [token][head][dim]
    void *out[2];
    int64_t x_token[2], x_head[2], out_token[2], out_head[2];              // strides, elements
    const int32_t *positions;
    const double *frequencies;
    float magnitude;
    uint32_t tokens, heads[2], dim, pairs, per, units, turned_units;       // per: tokens of a workgroup
};

// Sine and cosine of position * frequency.  The angle is made in 64 bits, in quarters of a turn: at position 2^20 a frequency of 1 in 32 bits would leave an
// angle that is off by 2^-4.  What is left after the whole quarters, at most an eighth of a turn either way, goes into the functions' series (the first terms that are left out are
// below 2^-28 there).
__device__ __forceinline__ float2 cos_sin(int32_t position, double frequency)
{
    const double quarters = (double)position * (frequency * 0.63661977236758134308), whole = __builtin_rint(quarters);
    const float x = (float)((quarters - whole) * 1.57079632679489661923), y = x * x;
    const uint32_t k = (uint32_t)(int32_t)(whole - 4.0 * __builtin_floor(whole * 0.25));
    const float s = x + x * y * (-1.f / 6.f + y * (1.f / 120.f + y * (-1.f / 5040.f + y * (1.f / 362880.f))));
    const float c = 1.f + y * (-0.5f + y * (1.f / 24.f + y * (-1.f / 720.f + y * (1.f / 40320.f + y * (-1.f / 3628800.f)))));
    const float a = k & 1u ? s : c, b = k & 1u ? c : s;
    return make_float2(k == 1u || k == 2u ? -a : a, k & 2u ? -b : b);
}

// kN numbers of a head, 16, 8 or 4 bytes of them or one.
template <typename T, uint32_t kN> struct Numbers;
template <uint32_t kN> struct Numbers<uint16_t, kN> {
    typedef uint32_t Words __attribute__((ext_vector_type(kN / 2u)));
    static __device__ __forceinline__ void load(const uint16_t *p, float (&v)[kN])
    {
        const Words w = *reinterpret_cast<const Words *>(p);
#pragma unroll
        for (uint32_t i = 0; i < kN / 2u; i++) { v[2u * i] = low(w[i]); v[2u * i + 1u] = high(w[i]); }
    }
    static __device__ __forceinline__ void store(uint16_t *p, const float (&v)[kN])
    {
        Words w;
#pragma unroll
        for (uint32_t i = 0; i < kN / 2u; i++) w[i] = pk_bf16(v[2u * i], v[2u * i + 1u]);
        __builtin_nontemporal_store(w, reinterpret_cast<Words *>(p));
    }
};
template <uint32_t kN> struct Numbers<float, kN> {
    typedef float Floats __attribute__((ext_vector_type(kN)));
    static __device__ __forceinline__ void load(const float *p, float (&v)[kN])
    {
        const Floats w = *reinterpret_cast<const Floats *>(p);
#pragma unroll
        for (uint32_t i = 0; i < kN; i++) v[i] = w[i];
    }
    static __device__ __forceinline__ void store(float *p, const float (&v)[kN])
    {
        Floats w;
#pragma unroll
        for (uint32_t i = 0; i < kN; i++) w[i] = v[i];
        __builtin_nontemporal_store(w, reinterpret_cast<Floats *>(p));
    }
};
template <> struct Numbers<uint16_t, 1> {
    static __device__ __forceinline__ void load(const uint16_t *p, float (&v)[1]) { v[0] = __uint_as_float((uint32_t)*p << 16); }
    static __device__ __forceinline__ void store(uint16_t *p, const float (&v)[1]) { *p = (uint16_t)pk_bf16(v[0], 0.f); }
};
template <> struct Numbers<float, 1> {
    static __device__ __forceinline__ void load(const float *p, float (&v)[1]) { v[0] = *p; }
    static __device__ __forceinline__ void store(float *p, const float (&v)[1]) { *p = v[0]; }
};

// A workgroup makes the sines and cosines of a few tokens once, in LDS, and turns the numbers of all heads with them (heads are dealt out to more workgroups where there
// are few tokens).  A unit is what a thread takes at once: two pieces of up to 16 bytes that are turned together (kBeside: one piece of neighbouring pairs), or, behind the pairs, one that is
// copied.  Bound by memory: 7,001 tokens, 48 heads of 128 in bfloat16, half of each turned, 27.5 us, 6.2 TB/s (some of it does not leave the last cache); in fp32 69 us, 5.0 TB/s; a token alone 3 to 4 us, a launch's time.
template <typename T, uint32_t kN, bool kBeside>
__global__ void __launch_bounds__(kRotateThreads)
rotate_kernel(const RotateArgs a)
{
    extern __shared__ float2 turns[];                // [token][pair]
    const uint32_t first = blockIdx.x * a.per, n = a.tokens - first < a.per ? a.tokens - first : a.per;
    for (uint32_t i = threadIdx.x; i < n * a.pairs; i += kRotateThreads) {
        const uint32_t t = i / a.pairs;
        const float2 cs = cos_sin(a.positions[first + t], a.frequencies[i - t * a.pairs]);
        turns[i] = make_float2(cs.x * a.magnitude, cs.y * a.magnitude);
    }
    __syncthreads();
    // A thread has one unit's place of a head; its heads' numbers (rows) are asked for kAsked at a time.
    constexpr uint32_t kAsked = kN > 1u ? kOnce : 1u;
    const uint32_t heads = a.heads[0] + a.heads[1], rows = n * heads, at_once = kRotateThreads / a.units ? kRotateThreads / a.units : 1u, step = gridDim.y * at_once;
    for (uint32_t u = threadIdx.x % (at_once * a.units) % a.units; threadIdx.x < at_once * a.units && u < a.units; u += kRotateThreads) {
        const bool turned = u < a.turned_units;
        const uint32_t d = turned ? (kBeside && kN == 1u ? 2u * u : u * kN) : 2u * a.pairs + (u - a.turned_units) * kN, e = d + (kBeside ? 1u : a.pairs);
        const float2 *turn = turns + (kBeside && kN > 1u ? u * (kN / 2u) : u * kN);
        auto place = [&](uint32_t r, const T **x, T **out) {
            const uint32_t t = r / heads, h0 = r - t * heads, which = h0 >= a.heads[0] ? 1u : 0u, h = which ? h0 - a.heads[0] : h0;
            *x = static_cast<const T *>(a.x[which]) + (int64_t)(first + t) * a.x_token[which] + (int64_t)h * a.x_head[which];
            *out = static_cast<T *>(a.out[which]) + (int64_t)(first + t) * a.out_token[which] + (int64_t)h * a.out_head[which];
            return t;
        };
        for (uint32_t r0 = blockIdx.y * at_once + threadIdx.x / a.units % at_once; r0 < rows; r0 += step * kAsked) {
            float v[kAsked][kN], w[kAsked][kN];
            T *out[kAsked];
            uint32_t t[kAsked];
            bool moved[kAsked];
#pragma unroll
            for (uint32_t j = 0; j < kAsked; j++) {
                const uint32_t r = r0 + j * step;
                const T *x;
                t[j] = place(r < rows ? r : r0, &x, &out[j]);
                moved[j] = r < rows && (turned || x != out[j]);
                Numbers<T, kN>::load(x + d, v[j]);
                if (turned && (!kBeside || kN == 1u)) Numbers<T, kN>::load(x + e, w[j]);
            }
#pragma unroll
            for (uint32_t j = 0; j < kAsked; j++) {
                if (!moved[j]) continue;
                if (!turned) { Numbers<T, kN>::store(out[j] + d, v[j]); continue; }             // behind the pairs
                const float2 *cs = turn + t[j] * a.pairs;
                if (kBeside && kN > 1u) {
#pragma unroll
                    for (uint32_t k = 0; k < kN / 2u; k++) {
                        const float p = v[j][2u * k], q = v[j][(2u * k + 1u) % kN];
                        v[j][2u * k] = p * cs[k].x - q * cs[k].y; v[j][(2u * k + 1u) % kN] = p * cs[k].y + q * cs[k].x;
                    }
                } else {
#pragma unroll
                    for (uint32_t k = 0; k < kN; k++) {
                        const float p = v[j][k], q = w[j][k];
                        v[j][k] = p * cs[k].x - q * cs[k].y; w[j][k] = p * cs[k].y + q * cs[k].x;
                    }
                    Numbers<T, kN>::store(out[j] + e, w[j]);
                }
                Numbers<T, kN>::store(out[j] + d, v[j]);
            }
        }
    }
}

hipError_t launch_rotate(const void *q, const void *k, int dtype, uint32_t tokens, uint32_t q_heads, uint32_t k_heads, uint32_t dim, uint32_t rotated, bool interleaved,
                         const int64_t (&strides)[8], const int32_t *positions, const double *frequencies, float magnitude, void *q_out, void *k_out, hipStream_t s)
{
    RotateArgs a{{q, k}, {q_out, k_out}, {strides[0], strides[2]}, {strides[1], strides[3]}, {strides[4], strides[6]}, {strides[5], strides[7]},
                 positions, frequencies, magnitude, tokens, {q_heads, k_heads}, dim, rotated / 2u, 0, 0, 0};
    const bool f32 = dtype == WG_F32;
    // by 16, 8 or 4 bytes, as all pieces lie at multiples of them (20,000 tokens of 20 heads of 80 numbers, 20 of them turned, by 4 bytes: 45 us, 2.9 TB/s, a thread
    // asking for 16 bytes at once where it asks for 64 by pieces of 16; by single numbers 110)
    auto lies = [&](uint32_t n) {
        bool fits = dim % n == 0 && (interleaved ? rotated % n == 0 : a.pairs % n == 0);
        for (const int64_t stride : strides) fits = fits && stride % n == 0;
        for (const void *p : {q, k, static_cast<const void *>(q_out), static_cast<const void *>(k_out)}) fits = fits && reinterpret_cast<uintptr_t>(p) % (n * (f32 ? 4u : 2u)) == 0;
        return fits;
    };
    uint32_t piece = f32 ? 4u : 8u;
    while (!lies(piece)) piece /= 2u;
    const bool wide = piece > 1u;
    a.turned_units = wide && interleaved ? rotated / piece : a.pairs / piece;
    a.units = a.turned_units + (dim - rotated) / piece;
    const uint32_t fit = kRotateThreads / a.pairs;
    a.per = fit < 1u ? 1u : fit > 16u ? 16u : fit;
    if (a.per > tokens) a.per = tokens;
    // Workgroups for each share of tokens: by more than a number, so many that each thread has kOnce rows, all of which it asks for at once (700 tokens of 48 heads 5.0 us, with half as many to a thread 6.1; 7,001
    // tokens 27.5, with three times as many 29.3); where these are few, or by single numbers, more, as far as there is something for each thread to do.
    const uint32_t blocks = (tokens + a.per - 1u) / a.per, at_once = kRotateThreads / a.units ? kRotateThreads / a.units : 1u, rows = a.per * (q_heads + k_heads);
    const uint32_t full = wide ? (rows + at_once * kOnce - 1u) / (at_once * kOnce) : 1u;
    const uint64_t most = ((uint64_t)rows * a.units + kRotateThreads - 1u) / kRotateThreads, want = ((wide ? 256u : 1024u) + blocks - 1u) / blocks, least = want < most ? want : most;
    const dim3 grid(blocks, full > least ? full : (uint32_t)least), block(kRotateThreads);
    const uint32_t lds = a.per * a.pairs * (uint32_t)sizeof(float2);
    auto go = [&](auto beside, auto straight) { return launch(interleaved ? beside : straight, grid, block, lds, s, nullptr, a); };
    if (f32)
        return piece == 4u ? go(rotate_kernel<float, 4, true>, rotate_kernel<float, 4, false>) : piece == 2u ? go(rotate_kernel<float, 2, true>, rotate_kernel<float, 2, false>)
                                                                                                             : go(rotate_kernel<float, 1, true>, rotate_kernel<float, 1, false>);
    return piece == 8u   ? go(rotate_kernel<uint16_t, 8, true>, rotate_kernel<uint16_t, 8, false>)
           : piece == 4u ? go(rotate_kernel<uint16_t, 4, true>, rotate_kernel<uint16_t, 4, false>)
           : piece == 2u ? go(rotate_kernel<uint16_t, 2, true>, rotate_kernel<uint16_t, 2, false>)
                         : go(rotate_kernel<uint16_t, 1, true>, rotate_kernel<uint16_t, 1, false>);
}

}  // namespace wg
