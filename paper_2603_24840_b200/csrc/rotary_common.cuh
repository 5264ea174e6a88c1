// What turns queries and keys by their positions: shared by the rotary calls and the cache's append.
#pragma once
#include <cuda_bf16.h>
#include <stdint.h>

#include "arrol_internal.h"

namespace {

struct RotaryPairs {
    const double* frequencies;    // [R / 2]
    int R, interleaved;
    float factor, sign;           // sign: -1 for the gradients
};

// Cosine and sine of position * frequency.  The angle is formed as turns in 64 bits, its whole turns leave exactly, and the rest, at most half a turn, keeps fp32's
// relative precision: far positions cost nothing (in fp32 the angle of position 100,000 would be off by 0.004).
__device__ __forceinline__ float2 rotary_cos_sin(const RotaryPairs& r, int pair, int64_t position) {
    double turns = (double)position * r.frequencies[pair] * 0.15915494309189533577;
    turns -= rint(turns);
    float s, c;
    sincospif(2.0f * (float)turns, &s, &c);
    return make_float2(c * r.factor, s * r.factor * r.sign);
}
// One way to round, whichever kernel turns a pair.
__device__ __forceinline__ float rotary_first(float x1, float x2, float2 cs) { return fmaf(x1, cs.x, -(x2 * cs.y)); }
__device__ __forceinline__ float rotary_second(float x1, float x2, float2 cs) { return fmaf(x2, cs.x, x1 * cs.y); }

// A head of D dimensions is D / (2 V) units of two chunks of V: first the units that turn, then those that stay.  The chunks of a unit that turns begin at `a` and `b`;
// with halves as pairs chunk b holds the partners of chunk a, with neighbours as pairs each chunk holds V / 2 whole pairs (V = 1: a and b are one pair).
template <int V>
struct RotaryUnit {
    int a, b;
    bool turns;
    float2 cs[V];
    __device__ __forceinline__ RotaryUnit(const RotaryPairs& r, int unit) {
        const int turning = r.R / (2 * V);
        turns = unit < turning;
        if (!turns) {
            a = r.R + (unit - turning) * 2 * V;
            b = a + V;
        } else if (V == 1 && r.interleaved) {
            a = 2 * unit;
            b = a + 1;
        } else {
            a = unit * V;
            b = r.R / 2 + a;
        }
    }
    __device__ __forceinline__ void at(const RotaryPairs& r, int64_t position) {
        if (!turns) return;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            int pair;
            if (V > 1 && r.interleaved) pair = (i < V / 2 ? a / 2 : b / 2 - V / 2) + i;
            else pair = (V == 1 && r.interleaved ? a / 2 : a) + i;
            cs[i] = rotary_cos_sin(r, pair, position);
        }
    }
    __device__ __forceinline__ void turn(const RotaryPairs& r, float (&x)[V], float (&y)[V]) const {
        if (!turns) return;
        if (V > 1 && r.interleaved) {
#pragma unroll
            for (int i = 0; i < V / 2; ++i) {
                const float x1 = x[2 * i], x2 = x[2 * i + 1], y1 = y[2 * i], y2 = y[2 * i + 1];
                x[2 * i] = rotary_first(x1, x2, cs[i]);
                x[2 * i + 1] = rotary_second(x1, x2, cs[i]);
                y[2 * i] = rotary_first(y1, y2, cs[V / 2 + i]);
                y[2 * i + 1] = rotary_second(y1, y2, cs[V / 2 + i]);
            }
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float x1 = x[i], x2 = y[i];
                x[i] = rotary_first(x1, x2, cs[i]);
                y[i] = rotary_second(x1, x2, cs[i]);
            }
        }
    }
};

// The largest of 8, 4, 2, 1 that divides both the pairs and half of the dimensions that stay: chunks then lie at multiples of their own size.
inline int rotary_vector(int D, int R) {
    const int both = (R / 2) | ((D - R) / 2);
    return both % 8 == 0 ? 8 : both % 4 == 0 ? 4 : both % 2 == 0 ? 2 : 1;
}

template <int V>
struct Bf16Chunk;
template <>
struct Bf16Chunk<8> { typedef uint4 type; };
template <>
struct Bf16Chunk<4> { typedef uint2 type; };
template <>
struct Bf16Chunk<2> { typedef uint32_t type; };
template <>
struct Bf16Chunk<1> { typedef uint16_t type; };

template <int V>
__device__ __forceinline__ void chunk_to_floats(const typename Bf16Chunk<V>::type& c, float (&x)[V]) {
    if constexpr (V == 1) {
        x[0] = __uint_as_float((uint32_t)c << 16);
    } else {
        const uint32_t* w = reinterpret_cast<const uint32_t*>(&c);
#pragma unroll
        for (int i = 0; i < V / 2; ++i) {
            x[2 * i] = __uint_as_float(w[i] << 16);
            x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
        }
    }
}
template <int V>
__device__ __forceinline__ typename Bf16Chunk<V>::type floats_to_chunk(const float (&x)[V]) {
    typename Bf16Chunk<V>::type c;
    if constexpr (V == 1) {
        c = __bfloat16_as_ushort(__float2bfloat16_rn(x[0]));
    } else {
        uint32_t* w = reinterpret_cast<uint32_t*>(&c);
#pragma unroll
        for (int i = 0; i < V / 2; ++i) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w[i]) : "f"(x[2 * i + 1]), "f"(x[2 * i]));
    }
    return c;
}

// The first i in [0, n] for which before(i) is false, for a before() that is true up to some place and false from there on; by a whole block, every thread gets it.
// A round asks as many places as there are threads.
template <typename F>
__device__ __forceinline__ int64_t block_search(int64_t n, F before) {
    int64_t lo = 0, hi = n;
    while (lo < hi) {
        const int64_t step = (hi - lo + blockDim.x - 1) / blockDim.x, i = lo + threadIdx.x * step;
        const int c = __syncthreads_count(i < hi && before(i));
        hi = lo + c * step < hi ? lo + c * step : hi;
        lo = c ? lo + (c - 1) * step + 1 : hi;
    }
    return lo;
}

}  // namespace
