// arrol_cache_append: new tokens' keys and values into the paged 8-bit cache, keys and queries turned by their positions on the way.
//
// Bound by HBM where there are many tokens (bf16 in, 8 bits out, queries in and out), by one launch and a chain of dependent loads (length, page number, scale) where
// there are few.  A page's scale needs the largest entry of all of its new tokens before the first can be rounded, so a page and head belong to one block
// (append_runs_kernel: runs of tokens) or one warp (append_one_kernel: a token per sequence), which keeps what it loaded in shared memory or registers in between (but for
// odd sizes, see append_runs_kernel) and needs no atomics in global memory.
//
// 38,000 prompt tokens of 16 heads of 128 on 8 (600 MB) 137 us, 4.4 TB/s: no unit is full (instructions issued in half of the cycles, DRAM at 0.55); the keys are turned twice.  One
// token each of 512 live rollouts, 32 heads on 8 (12 MB), 12 us from a graph, of 4,096 70: a warp of four heads has its own chain of loads and its own angles.
#include <type_traits>

#include "cache_common.cuh"
#include "rotary_common.cuh"

namespace {

constexpr int ONE_WARPS = 4;
constexpr int64_t APPEND_MAX_ROWS = ((int64_t)1 << 31) - 512;

struct AppendParams {
    arrol_cache_append_args a;
    RotaryPairs pairs;
    int units;                     // of a head (append_runs_kernel)
    int passes;                    // of a block over a page's units
    uint32_t* status;
};

// Page and first new token of a sequence whose new tokens are `fresh`; false where there is nothing to write.
__device__ __forceinline__ bool append_start(const arrol_cache_append_args& a, int i, int64_t fresh, int64_t& start, int& len, bool& bad) {
    len = cache_tokens(a.lengths, i, a.table_pages, a.cache.page, bad);
    start = len - fresh;
    if (start < 0) { bad = true; return false; }
    return fresh > 0;
}
__device__ __forceinline__ bool append_page(const arrol_cache_append_args& a, int i, int64_t ordinal, int& page, bool& bad) {
    page = a.page_table[(int64_t)i * a.table_stride + ordinal];
    if (page < 0 || page >= a.cache.pages) { bad = true; return false; }
    return true;
}
__device__ __forceinline__ int64_t append_offset(const arrol_cache_append_args& a, int i) { return a.prompt_lengths ? a.prompt_lengths[i / a.G] : 0; }

// Numbers of `bytes` bytes (a multiple of 16) times 2^-shift, by threads `at`, `at + step`, ...: exact but for those that become subnormal.
__device__ __forceinline__ void append_rescale(uint8_t* page, int bytes, float by, int at, int step) {
    for (int x = at * 16; x < bytes; x += step * 16) {
        uint4 w = *reinterpret_cast<uint4*>(page + x);
        uint32_t* u = reinterpret_cast<uint32_t*>(&w);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float2 a = e4m3_pair_to_float((uint16_t)u[j]), b = e4m3_pair_to_float((uint16_t)(u[j] >> 16));
            u[j] = e4m3_pair(a.x * by, a.y * by) | (uint32_t)e4m3_pair(b.x * by, b.y * by) << 16;
        }
        *reinterpret_cast<uint4*>(page + x) = w;
    }
}
// Scale of a page and head whose new entries are `amax` at most, `old` before: the exponent, and whether what the page holds moves to it.
__device__ __forceinline__ int append_exponent(float amax, int slot, float old, bool& grows) {
    const int e = cache_exponent(amax);
    grows = false;
    if (slot == 0) return e;
    const int had = (int)(__float_as_uint(old) >> 23 & 255u) - 127;
    if (had >= e) return had > 127 ? 127 : had;              // 127: not a scale that was written here
    grows = true;
    return e;
}

// ---- one token per sequence: a warp per sequence and PER of its heads (keys', then values', then queries'), four dimensions a lane.  Where one a head
// would be more warps than the SMs have places for, four heads share the angles and the chain of loads in front of them (heads of 128, 32 on 8, from a graph: 64 rollouts 4.5 us
// with one and 5.1 with four, 256 9.1 and 6.5, 512 live of 1,024 17.7 and 11.7, 4,096 109 and 70; with two 13.0 and 76, with eight 15.9 and 88, for the last two).
template <int PER>
__global__ void __launch_bounds__(32 * ONE_WARPS) append_one_kernel(const AppendParams p) {
    pdl_launch_dependents();
    pdl_wait();
    const arrol_cache_append_args& a = p.a;
    const int lane = threadIdx.x & 31, Hkv = a.cache.Hkv, tasks = 2 * Hkv + (a.q ? a.Hq : 0), groups = (tasks + PER - 1) / PER, D = a.cache.D, R = p.pairs.R, half = R / 2;
    const int64_t item = (int64_t)blockIdx.x * ONE_WARPS + (threadIdx.x >> 5);
    const int64_t seq = item / groups;
    if (seq >= a.N) return;
    const int i = (int)seq, task0 = (int)(item - seq * groups) * PER;
    if (a.keep && !a.keep[i]) return;
    const int d0 = lane * 4;
    const bool interleaved = p.pairs.interleaved;
    uint2 raw[PER];
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        const int task = task0 + k;
        const bool value = task >= Hkv && task < 2 * Hkv, query = task >= 2 * Hkv;
        const int h = query ? task - 2 * Hkv : value ? task - Hkv : task;
        const __nv_bfloat16* x = static_cast<const __nv_bfloat16*>(query ? a.q : value ? a.v : a.k) + (query ? a.q_stride : value ? a.v_stride : a.k_stride) * i + (int64_t)h * D;
        raw[k] = task < tasks && d0 < D ? *reinterpret_cast<const uint2*>(x + d0) : make_uint2(0u, 0u);
    }
    bool bad = false;
    int64_t start;
    int len, page = 0;
    bool ok = append_start(a, i, 1, start, len, bad);
    const int64_t position = start + append_offset(a, i);
    if (ok) ok = append_page(a, i, start / a.cache.page, page, bad);        // for queries too: a token that has no page has no rows
    if (bad && lane == 0) atomicOr(p.status, ARROL_DEV_BAD_INDEX);
    if (!ok) return;
    const int slot = (int)(start % a.cache.page);
    float* scale[PER];
    float old[PER];
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        const int task = task0 + k;
        scale[k] = task < Hkv ? a.cache.k_scale + page * a.cache.k_scale_stride + task : a.cache.v_scale + page * a.cache.v_scale_stride + (task - Hkv);
        old[k] = task < 2 * Hkv && slot ? *scale[k] : 0.f;
    }
    float2 cs[4];
    const bool all_values = task0 >= Hkv && task0 + PER <= 2 * Hkv;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int d = d0 + j;
        cs[j] = make_float2(1.f, 0.f);
        if (d < R && !all_values) cs[j] = rotary_cos_sin(p.pairs, interleaved ? d >> 1 : d < half ? d : d - half, position);
    }
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        const int task = task0 + k;
        if (task >= tasks) break;
        const bool value = task >= Hkv && task < 2 * Hkv, query = task >= 2 * Hkv;
        const int h = query ? task - 2 * Hkv : value ? task - Hkv : task;
        float y[4];
        chunk_to_floats<4>(raw[k], y);
        if (!value && R > 0) {
            // the partners lie in other lanes, but for pairs of neighbours
            float partner[4];
            if (interleaved) {
#pragma unroll
                for (int j = 0; j < 4; ++j) partner[j] = y[j ^ 1];
            } else if (half % 4 == 0) {
                const int from = d0 < half ? lane + half / 4 : lane - half / 4;
                const uint2 other = make_uint2(__shfl_sync(0xffffffffu, raw[k].x, from & 31), __shfl_sync(0xffffffffu, raw[k].y, from & 31));
                chunk_to_floats<4>(other, partner);
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int d = d0 + j, of = d < half ? d + half : d - half;
                    const uint32_t lo = __shfl_sync(0xffffffffu, raw[k].x, (of >> 2) & 31), hi = __shfl_sync(0xffffffffu, raw[k].y, (of >> 2) & 31), w = of & 2 ? hi : lo;
                    partner[j] = __uint_as_float(of & 1 ? w & 0xFFFF0000u : w << 16);
                }
            }
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (d0 + j < R) {
                    const bool first = interleaved ? (j & 1) == 0 : d0 + j < half;
                    y[j] = first ? rotary_first(y[j], partner[j], cs[j]) : rotary_second(partner[j], y[j], cs[j]);
                }
        }
        if (query || (!value && a.k_out)) {
            __nv_bfloat16* to = query ? static_cast<__nv_bfloat16*>(a.q_out) + a.q_out_stride * i : static_cast<__nv_bfloat16*>(a.k_out) + a.k_out_stride * i;
            if (d0 < D) *reinterpret_cast<uint2*>(to + (int64_t)h * D + d0) = floats_to_chunk<4>(y);
        }
        if (query) continue;
        float amax = 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) amax = finite_max(amax, y[j]);
        amax = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(amax)));
        bool grows;
        const int e = append_exponent(amax, slot, old[k], grows);
        uint8_t* const codes = static_cast<uint8_t*>(value ? a.cache.v_cache : a.cache.k_cache) + page * (value ? a.cache.v_page_stride : a.cache.k_page_stride) +
                               (int64_t)h * a.cache.page * D;
        if (grows) append_rescale(codes, slot * D, old[k] * cache_power(-e), lane, 32);
        const float by = cache_power(-e);
        if (d0 < D)
            *reinterpret_cast<uint32_t*>(codes + slot * D + d0) = e4m3_pair(y[0] * by, y[1] * by) | (uint32_t)e4m3_pair(y[2] * by, y[3] * by) << 16;
        if (lane == 0 && (slot == 0 || grows)) *scale[k] = cache_power(e);
    }
}

// ---- runs of tokens: a block per page that gets some, for keys and queries or for values (and part of the heads); a thread has one unit of one token, its angles in
// registers, and goes through the heads.  Where a page's units are more than 1,024 threads (pages of 128 tokens with narrow chunks) it has several units in turn, reads their rows twice
// and forms their angles anew for every head: 38,000 tokens, 16 heads of 80 on 8, 40 of 80 turned, 322 us with pages of 128, 139 of 64.  Chunks of 8 numbers: 64 registers, 60 bytes spilled.
template <int V>
__device__ __forceinline__ void not_finite_to_nan(float (&x)[V], float (&y)[V]) {
#pragma unroll
    for (int j = 0; j < V; ++j) { x[j] += x[j] - x[j]; y[j] += y[j] - y[j]; }
}
// V numbers times `by`, none of them infinite.
template <int V>
__device__ __forceinline__ void append_codes(uint8_t* to, const float (&x)[V], float by) {
    if constexpr (V == 1) {
        *to = (uint8_t)e4m3_pair_finite(x[0] * by, 0.f);
    } else if constexpr (V == 2) {
        *reinterpret_cast<uint16_t*>(to) = e4m3_pair_finite(x[0] * by, x[1] * by);
    } else {
        uint32_t w[V / 4];
#pragma unroll
        for (int j = 0; j < V / 4; ++j)
            w[j] = e4m3_pair_finite(x[4 * j] * by, x[4 * j + 1] * by) | (uint32_t)e4m3_pair_finite(x[4 * j + 2] * by, x[4 * j + 3] * by) << 16;
        if constexpr (V == 8) *reinterpret_cast<uint2*>(to) = make_uint2(w[0], w[1]);
        else *reinterpret_cast<uint32_t*>(to) = w[0];
    }
}

// Heads on their way.  38,000 prompt tokens: 2 140 us, 3 or 4 137, 6 149 (shared memory is then taken from what the spilled registers lie in); the next head in registers 143.
// Two heads a meeting: 137, four 150.
constexpr int APPEND_DEPTH = 4;

template <int BYTES>
__device__ __forceinline__ void copy_async(uint32_t to, const void* from) {
    if constexpr (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(to), "l"(from), "n"(BYTES) : "memory");
}

// RING: a page's units fit the block.  A thread's own chunks come by asynchronous copies into places of its own, several heads ahead; otherwise they are read where they lie.
template <int V, int THREADS, bool RING>
__global__ void __launch_bounds__(THREADS, 1024 / THREADS) append_runs_kernel(const AppendParams p) {
    typedef typename Bf16Chunk<V>::type Chunk;
    __shared__ uint32_t most[3];                             // largest of a head, as bits: in turn
    extern __shared__ __align__(16) uint8_t ring[];          // [APPEND_DEPTH][2][threads] chunks
    pdl_launch_dependents();
    pdl_wait();
    const arrol_cache_append_args& a = p.a;
    const int page_size = a.cache.page, D = a.cache.D, Hkv = a.cache.Hkv, lane = threadIdx.x & 31;
    const int64_t* cu = pdl_acquire(a.cu_new);
    if (threadIdx.x < 3) most[threadIdx.x] = 0u;             // published by the search's barriers
    // Rows out of order or behind the last may belong to sequences that no block comes to: the grid, more threads than sequences, looks at all of them.
    const int64_t seen = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    if (blockIdx.y == 0 && blockIdx.z == 0 && seen < a.N) {
        const int64_t first = cu[seen], end = cu[seen + 1];
        if (first < 0 || end < first || end > a.rows || (seen == 0 && first != 0)) atomicOr(p.status, ARROL_DEV_BAD_INDEX);
    }
    // Sequence i has the blocks from cu[i] / page + 2 i on: a run of n tokens touches n / page + 2 pages at most, whatever slot it begins in.
    const int64_t u = blockIdx.x;
    const int64_t i64 = block_search(a.N, [&](int64_t i) { return cu[i + 1] / page_size + 2 * (i + 1) <= u; });
    if (i64 >= a.N) return;
    const int i = (int)i64;
    if (a.keep && !a.keep[i]) return;
    const int64_t row0 = cu[i], fresh = cu[i + 1] - row0;
    bool bad = false;
    int64_t start = 0;
    int len = 0, page = 0;
    bool ok = row0 >= 0 && fresh >= 0 && row0 + fresh <= a.rows;
    if (!ok) bad = true;
    ok = ok && append_start(a, i, fresh, start, len, bad);
    const int64_t ordinal = start / page_size + u - (row0 / page_size + 2 * i64);
    const int64_t from = ordinal * page_size > start ? ordinal * page_size : start, to = (ordinal + 1) * page_size < len ? (ordinal + 1) * page_size : len;
    ok = ok && ordinal >= 0 && from < to;
    if (ok) ok = append_page(a, i, ordinal, page, bad);
    if (bad && threadIdx.x == 0) atomicOr(p.status, ARROL_DEV_BAD_INDEX);
    if (!ok) return;
    const int slot0 = (int)(from - ordinal * page_size), tokens = (int)(to - from);
    const int64_t first_row = row0 + (from - start), first_position = from + append_offset(a, i);
    // unit `x` of the page's tokens * units: token x / units
    const int items = tokens * p.units;
    int tok = threadIdx.x / p.units;
    RotaryUnit<V> unit(p.pairs, threadIdx.x - tok * p.units);
    bool mine = (int)threadIdx.x < items;
    const int passes = RING || THREADS == 512 ? 1 : p.passes;
    auto pass_to = [&](int pass) {                           // only where a page's units are more than the block's threads
        const int x = threadIdx.x + pass * blockDim.x;
        tok = x / p.units;
        unit = RotaryUnit<V>(p.pairs, x - tok * p.units);
        mine = x < items;
        if (mine && blockIdx.z == 0) unit.at(p.pairs, first_position + tok);
    };
    const bool values = blockIdx.z != 0;
    const __nv_bfloat16* const rows = static_cast<const __nv_bfloat16*>(values ? a.v : a.k) + first_row * (values ? a.v_stride : a.k_stride);
    const __nv_bfloat16* const queries = static_cast<const __nv_bfloat16*>(a.q) + first_row * a.q_stride;
    const int64_t stride = values ? a.v_stride : a.k_stride;
    float* const scales = values ? a.cache.v_scale + page * a.cache.v_scale_stride : a.cache.k_scale + page * a.cache.k_scale_stride;
    uint8_t* const codes = static_cast<uint8_t*>(values ? a.cache.v_cache : a.cache.k_cache) + page * (values ? a.cache.v_page_stride : a.cache.k_page_stride);
    // The block's heads one behind another: of keys or values, then of queries.
    const int split = gridDim.y, heads = ((int)blockIdx.y < Hkv ? (Hkv - 1 - (int)blockIdx.y) / split + 1 : 0);
    const int all = heads + (!values && a.q && (int)blockIdx.y < a.Hq ? (a.Hq - 1 - (int)blockIdx.y) / split + 1 : 0);
    auto source = [&](int t) {
        return t < heads ? rows + tok * stride + (int64_t)(blockIdx.y + t * split) * D : queries + tok * a.q_stride + (int64_t)(blockIdx.y + (t - heads) * split) * D;
    };
    const uint32_t place = (uint32_t)__cvta_generic_to_shared(ring) + threadIdx.x * (uint32_t)sizeof(Chunk);
    auto place_of = [&](int slot, int second) { return (uint32_t)(slot * 2 + second) * blockDim.x * (uint32_t)sizeof(Chunk); };
    // head t into its place, which nobody but this thread reads, and which it has read
    auto bring = [&](int t, int slot) {
        if constexpr (RING) {
            if (mine && t < all) {
                const __nv_bfloat16* row = source(t);
                copy_async<sizeof(Chunk)>(place + place_of(slot, 0), row + unit.a);
                copy_async<sizeof(Chunk)>(place + place_of(slot, 1), row + unit.b);
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
        }
    };
    auto arrived = [&] {
        if constexpr (RING) asm volatile("cp.async.wait_group %0;" ::"n"(APPEND_DEPTH - 1) : "memory");
    };
    int at = 0;                                              // place of the head that is worked on
    if constexpr (RING)
        for (int t = 0; t < APPEND_DEPTH; ++t) bring(t, t);
    if (mine && blockIdx.z == 0) unit.at(p.pairs, first_position + tok);
    // What was loaded is turned twice, for the largest and for the codes: kept as floats it would need twice the registers, and half of the threads would not fit.
    auto turned = [&](int t, float (&x)[V], float (&y)[V]) {
        Chunk c = {}, d = {};
        if (mine) {
            if constexpr (RING) {
                const Chunk* from = reinterpret_cast<const Chunk*>(ring) + threadIdx.x;
                c = from[(at * 2) * blockDim.x];
                d = from[(at * 2 + 1) * blockDim.x];
            } else {
                const __nv_bfloat16* row = source(t);
                c = *reinterpret_cast<const Chunk*>(row + unit.a);
                d = *reinterpret_cast<const Chunk*>(row + unit.b);
            }
        }
        chunk_to_floats<V>(c, x);
        chunk_to_floats<V>(d, y);
        if (!values) unit.turn(p.pairs, x, y);
    };
    auto done = [&](int t) {
        bring(t + APPEND_DEPTH, at);
        at = at == APPEND_DEPTH - 1 ? 0 : at + 1;
    };
    // The largest of all threads' values; what is not finite is left out only where there is an infinity among them (a NaN the maximum passes over by itself).
    auto largest = [&](float m, int slot) {
        const uint32_t x = __reduce_max_sync(0xffffffffu, __float_as_uint(m));
        if (lane == 0) atomicMax(&most[slot], x);
        __syncthreads();
        return __uint_as_float(most[slot]);
    };
    int slot = 0;
    for (int t = 0; t < heads; ++t) {
        const int h = blockIdx.y + t * split;
        const float old = slot0 ? scales[h] : 0.f;
        arrived();
        auto own_largest = [&](auto finite) {
            float m = 0.f;
            for (int pass = 0; pass < passes; ++pass) {
                if (passes > 1) pass_to(pass);
                float x[V], y[V];
                turned(t, x, y);
#pragma unroll
                for (int j = 0; j < V; ++j) m = decltype(finite)::value ? finite_max(finite_max(m, x[j]), y[j]) : fmaxf(fmaxf(m, fabsf(x[j])), fabsf(y[j]));
            }
            return m;
        };
        float m = largest(own_largest(std::false_type()), slot);
        // A word is cleared two meetings before it is used again: all have read it then, in front of the meeting between.
        auto next_slot = [&] {
            if (threadIdx.x == 0) most[slot == 0 ? 2 : slot - 1] = 0u;
            slot = slot == 2 ? 0 : slot + 1;
        };
        next_slot();
        const bool infinite = isinf(m);
        if (__builtin_expect(infinite, 0)) {
            m = largest(own_largest(std::true_type()), slot);
            next_slot();
        }
        bool grows;
        const int e = append_exponent(m, slot0, old, grows);
        uint8_t* const to_head = codes + (int64_t)h * page_size * D;
        const float by = cache_power(-e);
        if (grows) append_rescale(to_head, slot0 * D, old * by, threadIdx.x, blockDim.x);
        for (int pass = 0; pass < passes; ++pass) {
            if (passes > 1) pass_to(pass);
            if (mine) {
                const int to = (slot0 + tok) * D;
                float x[V], y[V];
                turned(t, x, y);
                if (!values && a.k_out) {
                    __nv_bfloat16* out = static_cast<__nv_bfloat16*>(a.k_out) + (first_row + tok) * a.k_out_stride + h * D;
                    *reinterpret_cast<Chunk*>(out + unit.a) = floats_to_chunk<V>(x);
                    *reinterpret_cast<Chunk*>(out + unit.b) = floats_to_chunk<V>(y);
                }
                if (__builtin_expect(infinite, 0)) not_finite_to_nan<V>(x, y);
                append_codes<V>(to_head + to + unit.a, x, by);
                append_codes<V>(to_head + to + unit.b, y, by);
            }
        }
        if (threadIdx.x == 0 && (slot0 == 0 || grows)) scales[h] = cache_power(e);
        done(t);
    }
    for (int t = heads; t < all; ++t) {
        const int h = blockIdx.y + (t - heads) * split;
        arrived();
        for (int pass = 0; pass < passes; ++pass) {
            if (passes > 1) pass_to(pass);
            if (mine) {
                __nv_bfloat16* const to = static_cast<__nv_bfloat16*>(a.q_out) + (first_row + tok) * a.q_out_stride + (int64_t)h * D;
                float x[V], y[V];
                turned(t, x, y);
                *reinterpret_cast<Chunk*>(to + unit.a) = floats_to_chunk<V>(x);
                *reinterpret_cast<Chunk*>(to + unit.b) = floats_to_chunk<V>(y);
            }
        }
        done(t);
    }
}

template <int V, int THREADS, bool RING>
int launch_append_runs(arrol_ctx* ctx, const AppendParams& p, dim3 grid, int threads, bool& set, cudaStream_t s) {
    const size_t bytes = RING ? (size_t)APPEND_DEPTH * 2 * threads * 2 * V : 0;
    if (RING && !set) {
        ARROL_CUDA_OK(cudaFuncSetAttribute(append_runs_kernel<V, THREADS, RING>, cudaFuncAttributeMaxDynamicSharedMemorySize, APPEND_DEPTH * 2 * THREADS * 2 * V));
        set = true;
    }
    ARROL_CUDA_OK(arrol_launch_pdl(append_runs_kernel<V, THREADS, RING>, grid, dim3(threads), bytes, s, p));
    ctx->launches += 1;
    return ARROL_OK;
}

}  // namespace

extern "C" int arrol_cache_append(arrol_ctx* ctx, const arrol_cache_append_args* a, void* stream) {
    if (!ctx || !a) return ARROL_ERR_INVALID_ARG;
    const int cache = cache_check(a->cache);
    if (cache == ARROL_ERR_INVALID_ARG) return cache;
    if (a->N < 0 || a->P < 0 || a->rows < 0 || a->table_pages < 0 || a->table_stride < a->table_pages || a->R < 0 || a->R % 2 || a->R > a->cache.D || !isfinite(a->factor))
        return ARROL_ERR_INVALID_ARG;
    if ((a->R > 0) != (a->frequencies != nullptr) || !arrol_aligned(a->frequencies, 8)) return ARROL_ERR_INVALID_ARG;
    if (a->P > 0 ? a->G < 1 || (int64_t)a->P * a->G != a->N || !a->prompt_lengths : a->prompt_lengths != nullptr) return ARROL_ERR_INVALID_ARG;
    if (!a->cu_new && a->rows != a->N) return ARROL_ERR_INVALID_ARG;
    if ((a->q != nullptr) != (a->q_out != nullptr) || (a->q && a->Hq < 1)) return ARROL_ERR_INVALID_ARG;
    if (cache != ARROL_OK || a->N > (1 << 24) || a->rows >= APPEND_MAX_ROWS || (a->q && a->Hq > 65536)) return ARROL_ERR_UNSUPPORTED;
    if (a->N == 0 || a->rows == 0) return ARROL_OK;
    const int D = a->cache.D, Hkv = a->cache.Hkv;
    if (a->cache.pages == 0 || !a->page_table || !a->lengths || a->table_pages == 0) return ARROL_ERR_INVALID_ARG;
    if (!cache_rows_ok(a->k, a->k_stride, Hkv, D) || !cache_rows_ok(a->v, a->v_stride, Hkv, D)) return ARROL_ERR_INVALID_ARG;
    if (a->q && (!cache_rows_ok(a->q, a->q_stride, a->Hq, D) || !cache_rows_ok(a->q_out, a->q_out_stride, a->Hq, D))) return ARROL_ERR_INVALID_ARG;
    if (a->k_out && !cache_rows_ok(a->k_out, a->k_out_stride, Hkv, D)) return ARROL_ERR_INVALID_ARG;
    if ((a->q && a->q == a->q_out && a->q_stride != a->q_out_stride) || (a->k_out == a->k && a->k_stride != a->k_out_stride)) return ARROL_ERR_INVALID_ARG;
    AppendParams p = {};
    p.a = *a;
    p.pairs = {a->frequencies, a->R, a->interleaved != 0, a->factor, 1.0f};
    p.status = ctx->d_status;
    ArrolDeviceGuard guard(ctx->device);
    if (!guard.ok) return ARROL_ERR_CUDA;
    if (!a->cu_new) {
        const int tasks = 2 * Hkv + (a->q ? a->Hq : 0);
        const int per = (int64_t)a->N * tasks > (int64_t)ctx->sm_count * 64 ? 4 : 1;
        const int64_t blocks = ((int64_t)a->N * ((tasks + per - 1) / per) + ONE_WARPS - 1) / ONE_WARPS;
        if (blocks >= ((int64_t)1 << 31)) return ARROL_ERR_UNSUPPORTED;
        ARROL_CUDA_OK(arrol_launch_pdl(per == 4 ? append_one_kernel<4> : append_one_kernel<1>, dim3((unsigned)blocks), dim3(32 * ONE_WARPS), 0, (cudaStream_t)stream, p));
    } else {
        // The widest chunks that the sizes allow: 4 numbers and twice the threads took 200 to 247 us where this took 143 for 38,000 prompt tokens.
        const int V = rotary_vector(D, a->R);
        p.units = D / (2 * V);
        const int items = a->cache.page * p.units, threads = items > 1024 ? 1024 : (items + 31) & ~31;
        p.passes = (items + threads - 1) / threads;
        const int64_t pages = a->rows / a->cache.page + 2 * (int64_t)a->N;
        // Enough blocks for two an SM at 512 threads each; as many heads a block as that leaves, for the angles are formed once a block.
        const int most = a->q && a->Hq > Hkv ? a->Hq : Hkv;
        int64_t split = (int64_t)(4 * ctx->sm_count) * 512 / threads / (a->rows / a->cache.page + 1);
        split = split < 1 ? 1 : split > most ? most : split;
        const dim3 grid((unsigned)pages, (unsigned)split, 2);
        const cudaStream_t s = (cudaStream_t)stream;
        const bool small = threads <= 512;
        bool* set = ctx->cache_append_smem_set[small];
        if (p.passes > 1)                                    // chunks of 8 numbers always fit
            return V == 4 ? launch_append_runs<4, 1024, false>(ctx, p, grid, threads, set[0], s) : V == 2 ? launch_append_runs<2, 1024, false>(ctx, p, grid, threads, set[0], s)
                                                                                                 : launch_append_runs<1, 1024, false>(ctx, p, grid, threads, set[0], s);
        if (V == 8) return small ? launch_append_runs<8, 512, true>(ctx, p, grid, threads, set[0], s) : launch_append_runs<8, 1024, true>(ctx, p, grid, threads, set[0], s);
        if (V == 4) return small ? launch_append_runs<4, 512, true>(ctx, p, grid, threads, set[1], s) : launch_append_runs<4, 1024, true>(ctx, p, grid, threads, set[1], s);
        if (V == 2) return small ? launch_append_runs<2, 512, true>(ctx, p, grid, threads, set[2], s) : launch_append_runs<2, 1024, true>(ctx, p, grid, threads, set[2], s);
        return small ? launch_append_runs<1, 512, false>(ctx, p, grid, threads, set[0], s) : launch_append_runs<1, 1024, false>(ctx, p, grid, threads, set[0], s);
    }
    ctx->launches += 1;
    return ARROL_OK;
}
