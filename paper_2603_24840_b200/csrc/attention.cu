// arrol_attention: attention of the packed survivors over their shared prompts and their own tokens.
//
//     z_j = scale q . k_j,   o = sum_j exp(z_j - m) v_j / l,   l = sum_j exp(z_j - m),   lse = m + log l
// over the rows of the sequence's prompt and its own rows up to the query's.  One pass over the keys: per block of 128 of them S = Q K^T into tensor memory,
// a thread takes a row of it, P = exp(S - m) goes back as bf16 (the one rounding beside o's; l is summed before it), O += P V.  m is a reference
// that the running maximum may be 2^8 ahead of: sums and products carry the same factor 2^-m, so a row's O is scaled again only when
// that is passed.  4 D flops a pair against one exponential: with 128 dimensions the tensor cores (512 cycles each for S and P V of a tile and
// block) and the exponentials (1,024 cycles a tile and block at 16 a cycle) are level, with 64 the exponentials are the longer.  By the counters neither unit is
// full: with 128 both are busy about half of the cycles, with 64 0.53 and 0.28.  What fills the rest was not measured; the way between them is what is left.
// One launch finds every token's range of keys, one computes: 148 blocks that take (256 query rows, key head) items from a counter.
// Measured, calls from a graph: 8,192 tokens, 32 heads of 128 on 8 458 to 479 us (1.15 to 1.20 PFLOP/s, 0.68 to 0.71 of the measured burst rate, tensor
// pipe busy 0.55 of the cycles); with heads of 64 379 us; 48 survivors of 40 to 333 tokens over 16,000 prompt tokens, 28 heads on 4 394 to 422 us (0.86 to
// 0.92 PFLOP/s).  Calls from the host one by one: 535 to 554, and 440 to 445 us.  Where few rows leave most blocks without an item, an item's keys are
// split and a third launch joins the parts (attn_key_splits).
#include "attention_common.cuh"

namespace {

constexpr int BOUNDS_THREADS = 256;

// Largest i in [0, n) with table[i] <= x; 0 where there is none.
__device__ __forceinline__ int last_not_above(const int64_t* table, int n, int64_t x) {
    int lo = 0, hi = n;                 // table[lo] <= x (or lo == 0), table[hi] > x
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (table[mid] <= x) lo = mid; else hi = mid;
    }
    return lo;
}
// First sequence s in [0, S) of a prompt not below p.
__device__ __forceinline__ int first_of_prompt(const int32_t* survivor_idx, int S, int G, int p) {
    int lo = 0, hi = S;
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if ((survivor_idx ? survivor_idx[mid] : mid) / G < p) lo = mid + 1; else hi = mid;
    }
    return lo;
}
// What the backward needs of a query row too: lse log2(e) and delta = sum_d d_o[t, h, d] o[t, h, d].
struct RowStats {
    const __nv_bfloat16 *o, *d_o;
    int64_t o_stride, d_o_stride;
    const float* lse;
    float2* stats;           // NULL: not wanted
    int Hq, D;
};

// One thread per packed token and per prompt row.  Everything that the other kernels follow is clamped to the buffers here, so numbers out
// of order give wrong results and a status bit, never an access outside.
__global__ void __launch_bounds__(BOUNDS_THREADS)
attention_bounds_kernel(const int64_t* __restrict__ cu_seqlens, const int64_t* __restrict__ d_num, const int64_t* __restrict__ cu_prompts,
                        const int32_t* __restrict__ survivor_idx, int S_max, int T_max, int P, int G, int prompt_rows,
                        TokenBounds* __restrict__ bounds, int2* __restrict__ prompt_range, uint32_t* __restrict__ counters,
                        uint32_t* __restrict__ status, const RowStats rs) {
    pdl_launch_dependents();
    pdl_wait();
    cu_seqlens = pdl_acquire(cu_seqlens); d_num = pdl_acquire(d_num); cu_prompts = pdl_acquire(cu_prompts); survivor_idx = pdl_acquire(survivor_idx);
    const int S = clamp_row(d_num[0], 0, S_max), T = clamp_row(d_num[1], 0, T_max);
    const int64_t tid = blockIdx.x * (int64_t)BOUNDS_THREADS + threadIdx.x, threads = (int64_t)gridDim.x * BOUNDS_THREADS;
    if (tid < 64) counters[tid] = 0u;
    bool bad = false;
    for (int64_t t = tid; t < T; t += threads) {
        TokenBounds b = {0, 0, (int)t, (int)t + 1};
        if (S > 0) {
            const int s = last_not_above(cu_seqlens, S, t);
            b.own_lo = clamp_row(cu_seqlens[s], 0, (int)t);
            b.own_hi = clamp_row(cu_seqlens[s + 1], (int)t + 1, T);
            const int p = (survivor_idx ? survivor_idx[s] : s) / G;
            if (P > 0 && p >= 0 && p < P) {
                b.pre_lo = clamp_row(cu_prompts[p], 0, prompt_rows);
                b.pre_hi = clamp_row(cu_prompts[p + 1], b.pre_lo, prompt_rows);
            }
        }
        bounds[t] = b;
    }
    // the arrays themselves
    for (int64_t s = tid; s < S; s += threads) {
        const int p = (survivor_idx ? survivor_idx[s] : (int)s) / G;
        bad |= cu_seqlens[s] > cu_seqlens[s + 1] || (s == 0 && cu_seqlens[0] != 0) || (s == S - 1 && cu_seqlens[S] < T);
        if (P > 0) bad |= p < 0 || p >= P || (survivor_idx && survivor_idx[s] < 0) || (s > 0 && (survivor_idx ? survivor_idx[s - 1] : (int)s - 1) / G > p);
    }
    bad |= tid == 0 && S == 0 && T > 0;
    for (int64_t p = tid; p < P; p += threads)
        bad |= cu_prompts[p] > cu_prompts[p + 1] || (p == 0 && cu_prompts[0] != 0) || (p == P - 1 && cu_prompts[P] > prompt_rows);
    if (prompt_range) {
        const int live = P > 0 ? clamp_row(cu_prompts[P], 0, prompt_rows) : 0;
        for (int64_t j = tid; j < live; j += threads) {
            const int p = last_not_above(cu_prompts, P, j);
            const int s0 = first_of_prompt(survivor_idx, S, G, p), s1 = first_of_prompt(survivor_idx, S, G, p + 1);
            int2 r = {0, 0};
            if (s0 < s1) {
                r.x = clamp_row(cu_seqlens[s0], 0, T);
                r.y = clamp_row(cu_seqlens[s1], r.x, T);
            }
            prompt_range[j] = r;
        }
    }
    if (bad) atomicOr(status, ARROL_DEV_BAD_INDEX);
    if (rs.stats) {
        const __nv_bfloat16 *o = pdl_acquire(rs.o), *d_o = pdl_acquire(rs.d_o);
        const float* lse = pdl_acquire(rs.lse);
        // 16 bytes a lane, 8 or 16 lanes a row, four rows of each group of lanes in flight
        constexpr int AT_ONCE = 4;
        const int width = rs.D <= 64 ? 8 : 16, c = (threadIdx.x & (width - 1)) * 8;
        const int64_t rows = (int64_t)T * rs.Hq, groups = threads / width;
        for (int64_t i0 = tid / width; i0 - (threadIdx.x & 31) / width < rows; i0 += AT_ONCE * groups) {
            uint4 x[AT_ONCE], y[AT_ONCE];
            float log_sum[AT_ONCE];
#pragma unroll
            for (int k = 0; k < AT_ONCE; ++k) {
                const int64_t i = i0 + k * groups, t = i / rs.Hq;
                const int h = (int)(i - t * rs.Hq);
                x[k] = y[k] = make_uint4(0u, 0u, 0u, 0u);
                log_sum[k] = 0.f;
                if (i < rows && c < rs.D) {
                    x[k] = *reinterpret_cast<const uint4*>(o + t * rs.o_stride + (int64_t)h * rs.D + c);
                    y[k] = *reinterpret_cast<const uint4*>(d_o + t * rs.d_o_stride + (int64_t)h * rs.D + c);
                    if (c == 0) log_sum[k] = lse[i];
                }
            }
#pragma unroll
            for (int k = 0; k < AT_ONCE; ++k) {
                const int64_t i = i0 + k * groups;
                const uint32_t u[4] = {x[k].x, x[k].y, x[k].z, x[k].w}, v[4] = {y[k].x, y[k].y, y[k].z, y[k].w};
                float sum = 0.f;
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const float2 a = bf16_pair(u[w]), b = bf16_pair(v[w]);
                    sum += a.x * b.x + a.y * b.y;
                }
#pragma unroll
                for (int m = 8; m > 0; m >>= 1)
                    if (m < width) sum += __shfl_xor_sync(0xffffffffu, sum, m);
                if (c == 0 && i < rows) rs.stats[i] = make_float2(log_sum[k] * LOG2E, sum);
            }
        }
    }
}

// ---- the tensor-core kernel ------------------------------------------------------------------------------------------------------
// Work item = (2 TOK consecutive packed tokens, key head).  Its query rows are all of these tokens' heads of the group, token-major, so a group of
// any size fills the 128 rows of a tile (TOK = 128 / ratio tokens, rounded down) and keys are loaded once per group; two tiles share the loads.
// Keys come in blocks of 128: those of the tiles' prompts (consecutive prompts are consecutive rows), then the own ones; a block
// that lies inside every row's range is not masked at all.
constexpr int FWD_BLOCK = 128;
constexpr int FWD_THREADS = 384;             // producer, MMA issuer, scanner, second MMA issuer or a spare warp; two softmax groups of four warps
constexpr int FWD_SLOTS = 2;                 // work items announced ahead
constexpr uint32_t HALF_BYTES = 128 * 128;   // 128 rows x 64 dimensions
constexpr int APART_FROM = 16, APART_CYCLES = 1200;        // blocks of an item, cycles
constexpr float RESCALE_AT = 8.0f;           // the running maximum follows once it is 2^8 behind

struct FwdTile {
    int tokens;                              // live tokens of the tile
    int pad[3];
    int4 need;                               // blocks with keys that any row has: prompt blocks [x, y), own blocks [z, w)
    int4 whole;                              // blocks whose keys every row has, likewise
};
struct alignas(16) FwdItem {
    int t0, g, valid, split;
    int pre0, n_pre, own0, n;                // block b < n_pre: prompt rows pre0 + 128 b .., then own rows own0 + 128 (b - n_pre) ..
    FwdTile tile[2];
};
__device__ __forceinline__ bool in_ranges(const int4& r, int b) { return (b >= r.x && b < r.y) || (b >= r.z && b < r.w); }
// Blocks of 128 keys from `base` on, the first of them number `b0`, that meet [lo, hi); and that lie inside.
__device__ __forceinline__ int2 blocks_meeting(int lo, int hi, int base, int b0) {
    return hi > lo ? make_int2(b0 + (lo - base) / FWD_BLOCK, b0 + (hi - base + FWD_BLOCK - 1) / FWD_BLOCK) : make_int2(0, 0);
}
__device__ __forceinline__ int2 blocks_inside(int lo, int hi, int base, int b0) {
    return hi > lo && hi > base ? make_int2(b0 + (max(lo - base, 0) + FWD_BLOCK - 1) / FWD_BLOCK, b0 + (hi - base) / FWD_BLOCK) : make_int2(0, 0);
}

template <int DP>
struct FwdConf {
    static constexpr int HALVES = DP / 64;
    static constexpr uint32_t TILE_BYTES = HALVES * HALF_BYTES;
    static constexpr int STAGES = DP == 128 ? 4 : 8;
    static constexpr size_t SMEM = 1024 + (2 + STAGES) * (size_t)TILE_BYTES;
    // Tensor memory: S of the two tiles at 0 and 128, O behind them.  With 64 dimensions there is room for P beside S, and the next block's S is
    // computed while this one's exponentials are; with 128 P takes the place of S, whose next block has to wait for P V.
    static constexpr bool AHEAD = DP == 64;
    static constexpr uint32_t O_AT = 256, P_AT = AHEAD ? 384 : 0, P_STEP = AHEAD ? 64 : 128;
};

struct FwdParams {
    AttnShape sh;
    __nv_bfloat16* o;
    int64_t o_stride;
    float* lse;
    uint32_t* counter;
    uint32_t* status;
    int tile_tokens;                         // TOK
    int splits;                              // parts of an item's keys, each an item; with more than one their sums go to
    float* part_o;                           // [splits][T_max][Hq][D] and
    float2* part_ml;                         // [splits][T_max][Hq]: the reference that the sums are taken against, l
};

struct FwdShared {
    uint64_t full[8], empty[8], scanned[8];                                    // per stage
    uint64_t q_full[2], q_empty[2], s_full[2], s_free[2], p_most[2], p_full[2], pv_done[2], drain[2];      // per tile
    uint64_t item_full[FWD_SLOTS], item_empty[FWD_SLOTS], item_scanned[FWD_SLOTS];
    alignas(16) uint32_t bad_keys[8][4];     // per stage with values: keys of an edge block that are not finite
    FwdItem items[FWD_SLOTS];
    uint32_t bad_whole[FWD_SLOTS];           // tiles that have values which are not finite in a block that they do not mask
    uint32_t tmem, abort;
};

template <int DP, bool SPLIT>
__global__ void __launch_bounds__(FWD_THREADS, 1)
attention_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v,
                 const __grid_constant__ CUtensorMap map_pk, const __grid_constant__ CUtensorMap map_pv, const FwdParams p) {
    using C = FwdConf<DP>;
    extern __shared__ uint8_t smem_raw[];
    __shared__ FwdShared sm;
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    uint8_t* const q_tiles = smem;
    uint8_t* const ring = smem + 2 * C::TILE_BYTES;
    volatile uint32_t* abort_flag = &sm.abort;
    const int warp = uniform((int)threadIdx.x >> 5), lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int i = 0; i < C::STAGES; ++i) {
            mbar_init(&sm.full[i], 1);
            mbar_init(&sm.empty[i], C::AHEAD ? 3 : 1 + (i & 1));         // odd stages hold values, which the scanner hands back too (and keys, see there)
            mbar_init(&sm.scanned[i], 1);
        }
        for (int i = 0; i < 2; ++i) {
            for (uint64_t* bar : {&sm.q_full[i], &sm.q_empty[i], &sm.s_full[i], &sm.pv_done[i], &sm.drain[i]}) mbar_init(bar, 1);
            for (uint64_t* bar : {&sm.s_free[i], &sm.p_most[i], &sm.p_full[i]}) mbar_init(bar, 4);
        }
        for (int i = 0; i < FWD_SLOTS; ++i) {
            mbar_init(&sm.item_scanned[i], 1);
            mbar_init(&sm.item_full[i], 1);
            mbar_init(&sm.item_empty[i], C::AHEAD ? 11 : 10);
        }
        sm.abort = 0u;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&map_q) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&map_k) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&map_v) : "memory");
    }
    if (warp == 1) {
        tcgen05_alloc(&sm.tmem, 512);
        tcgen05_relinquish();
    }
    tcgen05_fence_before();
    __syncthreads();
    tcgen05_fence_after();
    const uint32_t tmem = uniform(sm.tmem);  // S of the two tiles (P in its place), then O
    pdl_launch_dependents();
    pdl_wait();
    const int T = clamp_row(*pdl_acquire(p.sh.d_num + 1), 0, p.sh.T_max);
    const int ratio = p.sh.ratio, TOK = p.tile_tokens;
    const int pairs = (T + 2 * TOK - 1) / (2 * TOK);
    const int64_t items = (int64_t)pairs * p.sh.Hkv * (SPLIT ? p.splits : 1);

    if (warp == 0) {
        // ---- producer: fetches work items, announces them, loads queries, keys and values
        const TokenBounds* bounds = pdl_acquire(p.sh.bounds);
        uint32_t pos = 0, q_loads[2] = {0, 0};   // ring positions filled, tiles of queries asked for so far
        bool ok = true;
        for (uint32_t n = 0; ok; ++n) {
            const uint32_t slot = n % FWD_SLOTS, use = n / FWD_SLOTS;
            if (!mbar_wait_warp(&sm.item_empty[slot], (use & 1u) ^ 1u, abort_flag)) { ok = false; break; }
            uint32_t idx = 0;
            if (lane == 0) idx = atomicAdd(p.counter, 1u);
            idx = __shfl_sync(0xffffffffu, idx, 0);
            FwdItem& it = sm.items[slot];
            const bool valid = (int64_t)idx < items;
            if (valid) {
                // last tokens first: theirs are the longest ranges of a long sequence
                const uint32_t head_item = SPLIT ? idx / (uint32_t)p.splits : idx;
                const int split = SPLIT ? (int)(idx - head_item * (uint32_t)p.splits) : 0;
                const int t0 = (pairs - 1 - (int)(head_item / (uint32_t)p.sh.Hkv)) * 2 * TOK;
                TokenBounds a = {0, 0, 0, 0}, z = a;     // of the tile's first and last live token; lane = tile
                int tokens = 0, last = 0;
                const int first = t0 + lane * TOK;
                if (lane < 2 && first < T) {
                    tokens = min(TOK, T - first);
                    last = first + tokens - 1;
                    a = bounds[first];
                    z = bounds[last];
                }
                // what the two tiles need together; the second may have no tokens, a tile no prompt rows
                const bool has_pre = tokens > 0 && z.pre_hi > a.pre_lo;
                const int pl = __reduce_min_sync(0xffffffffu, has_pre ? a.pre_lo : INT_MAX), ph = __reduce_max_sync(0xffffffffu, has_pre ? z.pre_hi : 0);
                const int ol = __reduce_min_sync(0xffffffffu, tokens > 0 ? a.own_lo : INT_MAX), oh = __reduce_max_sync(0xffffffffu, tokens > 0 ? last + 1 : 0);
                const int n_pre = ph > pl ? (ph - pl + FWD_BLOCK - 1) / FWD_BLOCK : 0;
                const int n_own = (oh - ol + FWD_BLOCK - 1) / FWD_BLOCK, n_all = n_pre + n_own;
                // this part's blocks: [from, to) of all of them, numbered from 0
                const int each = SPLIT ? (n_all + p.splits - 1) / p.splits : n_all, from = SPLIT ? min(split * each, n_all) : 0, to = min(from + each, n_all);
                if (lane < 2) {
                    FwdTile tl = {};
                    tl.tokens = tokens;
                    if (tokens > 0) {
                        const int2 np = has_pre ? blocks_meeting(a.pre_lo, z.pre_hi, pl, 0) : make_int2(0, 0);
                        const int2 no = blocks_meeting(a.own_lo, last + 1, ol, n_pre);
                        const int2 wp = blocks_inside(z.pre_lo, a.pre_hi, pl, 0), wo = blocks_inside(z.own_lo, first + 1, ol, n_pre);
                        if constexpr (SPLIT) {
                            auto cut = [&](int2 r) {
                                r = make_int2(max(r.x, from) - from, min(r.y, to) - from);
                                return r.x < r.y ? r : make_int2(0, 0);
                            };
                            const int2 cp = cut(np), co = cut(no), whole_p = cut(make_int2(wp.x, min(wp.y, n_pre))), whole_o = cut(wo);
                            // where there are no own blocks the prompt's take their place: a tile's last block is the one before need.w
                            tl.need = co.y > co.x ? make_int4(cp.x, cp.y, co.x, co.y) : make_int4(0, 0, cp.x, cp.y);
                            tl.whole = make_int4(whole_p.x, whole_p.y, whole_o.x, whole_o.y);
                        } else {
                            tl.need = make_int4(np.x, np.y, no.x, no.y);
                            tl.whole = make_int4(wp.x, min(wp.y, n_pre), wo.x, wo.y);
                        }
                    }
                    it.tile[lane] = tl;
                }
                if (lane == 0) {
                    it.t0 = t0;
                    it.g = (int)(head_item % (uint32_t)p.sh.Hkv);
                    it.split = split;
                    it.n_pre = SPLIT ? max(min(n_pre, to) - from, 0) : n_pre;
                    it.pre0 = pl + from * FWD_BLOCK;
                    it.own0 = SPLIT ? ol + max(from - n_pre, 0) * FWD_BLOCK : ol;
                    it.n = to - from;
                }
            }
            if (lane == 0) it.valid = valid;
            __syncwarp();
            if (lane == 0) mbar_arrive(&sm.item_full[slot]);
            __syncwarp();
            if (!valid) break;
            const int g = it.g, t0 = it.t0, blocks = it.n, n_pre = it.n_pre, pre0 = it.pre0, own0 = it.own0;
            auto load_q = [&](int i) {
                if (!mbar_wait_warp(&sm.q_empty[i], (n & 1u) ^ 1u, abort_flag)) return false;
                if (elect_one()) {
                    mbar_expect_tx(&sm.q_full[i], C::HALVES * (uint32_t)(TOK * ratio) * 128u);
#pragma unroll
                    for (int h = 0; h < C::HALVES; ++h)
                        tma_load_3d(q_tiles + i * C::TILE_BYTES + h * HALF_BYTES, &map_q, h * 64, g * ratio, t0 + i * TOK, &sm.q_full[i]);
                }
                __syncwarp();
                ++q_loads[i];
                return true;
            };
            for (int b = 0; b < blocks && ok; ++b) {
                const bool pre = b < n_pre;
                const int row = pre ? pre0 + b * FWD_BLOCK : own0 + (b - n_pre) * FWD_BLOCK;
#pragma unroll
                for (int kv = 0; kv < 2; ++kv, ++pos) {
                    const uint32_t st = pos % C::STAGES;
                    // queries behind the first keys and values: those stages are free earlier than the last item's queries
                    if (b == 0 && kv == 1 && !(load_q(0) && load_q(1))) { ok = false; break; }
                    if (!mbar_wait_warp(&sm.empty[st], ((pos / C::STAGES) & 1u) ^ 1u, abort_flag)) { ok = false; break; }
                    if (elect_one()) {
                        mbar_expect_tx(&sm.full[st], C::TILE_BYTES);
                        const CUtensorMap* m = kv == 0 ? (pre ? &map_pk : &map_k) : (pre ? &map_pv : &map_v);
#pragma unroll
                        for (int h = 0; h < C::HALVES; ++h) tma_load_3d(ring + st * C::TILE_BYTES + h * HALF_BYTES, m, h * 64, g, row, &sm.full[st]);
                    }
                    __syncwarp();
                }
            }
            // a part without blocks: every item has its queries loaded, the issuers wait for them and hand them back
            if (SPLIT && ok && blocks == 0) ok = load_q(0) && load_q(1);
        }
        if (!ok) {                           // let the copies in flight land before the block's shared memory goes away
            for (uint32_t i = 1; i <= C::STAGES && i <= pos; ++i)
                for (uint32_t spin = 0; spin < SPIN_LIMIT; ++spin)
                    if (mbar_try_wait(&sm.full[(pos - i) % C::STAGES], ((pos - i) / C::STAGES) & 1u)) break;
            for (int i = 0; i < 2; ++i)
                for (uint32_t spin = 0; q_loads[i] > 0 && spin < SPIN_LIMIT; ++spin)
                    if (mbar_try_wait(&sm.q_full[i], (q_loads[i] - 1u) & 1u)) break;
        }
        __syncwarp();
    } else if (!C::AHEAD && warp == 1) {
        // ---- MMA issuer.  Per tile and block: S = Q K^T, and once the softmax group has written P (three quarters are enough to begin), O += P V.
        // One warp for both tiles, in turn, where P V and the next S of a tile follow each other: that keeps their softmax groups half a block apart, so
        // that one's exponentials run while the tensor cores work for the other.  (A warp per tile let them fall in step, both waiting for the same
        // unit: 8,192 tokens of 32 heads of 128 517 -> 700 us.)
        // One thread: the waits need no votes and no converging barriers then (8,192 tokens as above 487 -> 475 us).
        if (elect_one()) {
            constexpr uint32_t idesc_s = make_idesc(128, FWD_BLOCK), idesc_o = make_idesc(128, DP, false, true);
            const uint32_t q_base = smem_u32(q_tiles), ring_base = smem_u32(ring);
            uint32_t pos0 = 0, parity_p[2] = {0, 0};
            bool ok = true;
            auto wait_stage = [&](uint32_t pos) { return mbar_wait(&sm.full[pos % C::STAGES], (pos / C::STAGES) & 1u, abort_flag); };
            for (uint32_t n = 0; ok; ++n) {
                const uint32_t slot = n % FWD_SLOTS;
                if (!mbar_wait(&sm.item_full[slot], (n / FWD_SLOTS) & 1u, abort_flag)) { ok = false; break; }
                const FwdItem& it = sm.items[slot];
                if (!it.valid) break;
                const int blocks = it.n;
                const int4 need0 = it.tile[0].need, need1 = it.tile[1].need;
                bool first[2] = {true, true};
                uint32_t pv_pos[2] = {0, 0};             // ring position of the values whose P V is still to be issued; 0: none
                bool pv_frees[2] = {false, false};       // and whether no other tile uses them after that
                auto issue_s = [&](int i, uint32_t pos, bool frees, bool last) {
                    const uint32_t st = pos % C::STAGES;
                    tcgen05_fence_after();
                    mma_over_dims<C::HALVES>(tmem + i * 128, q_base + i * C::TILE_BYTES, HALF_BYTES, ring_base + st * C::TILE_BYTES, HALF_BYTES, idesc_s);
                    tcgen05_commit(&sm.s_full[i]);
                    if (frees) tcgen05_commit(&sm.empty[st]);
                    if (last) tcgen05_commit(&sm.q_empty[i]);
                };
                auto issue_pv = [&](int i) {
                    const uint32_t st = pv_pos[i] % C::STAGES, o_at = tmem + C::O_AT + i * DP, p_at = tmem + C::P_AT + i * C::P_STEP;
                    if (!wait_stage(pv_pos[i]) || !mbar_wait(&sm.p_most[i], parity_p[i], abort_flag)) return false;
                    tcgen05_fence_after();
                    mma_over_rows<FWD_BLOCK, 0, 6>(o_at, p_at, ring_base + st * C::TILE_BYTES, idesc_o, first[i]);
                    if (!mbar_wait(&sm.p_full[i], parity_p[i], abort_flag)) return false;
                    tcgen05_fence_after();
                    mma_over_rows<FWD_BLOCK, 6, 8>(o_at, p_at, ring_base + st * C::TILE_BYTES, idesc_o, false);
                    if (pv_frees[i]) tcgen05_commit(&sm.empty[st]);
                    tcgen05_commit(&sm.pv_done[i]);
                    parity_p[i] ^= 1u;
                    first[i] = false;
                    pv_pos[i] = 0;
                    return true;
                };
                bool q_here[2] = {false, false};
                for (int b = 0; b < blocks && ok; ++b) {
                    const uint32_t pos = pos0 + 2 * b;
                    const bool use[2] = {in_ranges(need0, b), in_ranges(need1, b)};
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        // a tile's pending P V goes first even where it does not need this block: stages are freed in order, tile 1 last
                        if (ok && pv_pos[i] && !issue_pv(i)) ok = false;
                        if (use[i] && ok) {
                            if (!q_here[i] && !mbar_wait(&sm.q_full[i], n & 1u, abort_flag)) { ok = false; break; }
                            q_here[i] = true;
                            if (!(i == 1 && use[0]) && !wait_stage(pos)) { ok = false; break; }
                            issue_s(i, pos, i == 1 || !use[1], b + 1 == (i ? need1.w : need0.w));
                            pv_pos[i] = pos + 1;
                            pv_frees[i] = i == 1 || !use[1];
                        }
                    }
                    if (!use[0] && !use[1] && ok) {      // keys of prompts between the tiles' that have no survivors, or row numbers out of order
                        if (!wait_stage(pos) || !wait_stage(pos + 1)) { ok = false; break; }
                        mbar_arrive(&sm.empty[pos % C::STAGES]);
                        mbar_arrive(&sm.empty[(pos + 1) % C::STAGES]);
                    }
                }
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    if (ok && pv_pos[i] && !issue_pv(i)) ok = false;
                    if (ok && !q_here[i]) {              // a tile without tokens
                        if (!mbar_wait(&sm.q_full[i], n & 1u, abort_flag)) ok = false;
                        else mbar_arrive(&sm.q_empty[i]);
                    }
                }
                pos0 += 2 * blocks;
                if (ok) mbar_arrive(&sm.item_empty[slot]);
            }
            if (!ok) {
                tcgen05_commit(&sm.drain[0]);
                for (uint32_t spin = 0; spin < SPIN_LIMIT; ++spin)
                    if (mbar_try_wait(&sm.drain[0], 0u)) break;
            }
        }
        __syncwarp();
    } else if (C::AHEAD && (warp == 1 || warp == 3)) {
        // ---- MMA issuer of tile i where S runs ahead: neither tile's P V is in the way of the other's S then
        constexpr uint32_t idesc_s = make_idesc(128, FWD_BLOCK), idesc_o = make_idesc(128, DP, false, true);
        const int i = warp >> 1;
        const uint32_t q_base = smem_u32(q_tiles) + i * C::TILE_BYTES, ring_base = smem_u32(ring);
        const uint32_t s_at = tmem + i * 128, o_at = tmem + C::O_AT + i * DP, p_at = tmem + C::P_AT + i * C::P_STEP;
        uint32_t pos0 = 0, parity_p = 0, parity_s = 0;
        bool ok = true, s_used = false;              // S was written before
        auto wait_stage = [&](uint32_t pos) { return mbar_wait_warp(&sm.full[pos % C::STAGES], (pos / C::STAGES) & 1u, abort_flag); };
        for (uint32_t n = 0; ok; ++n) {
            const uint32_t slot = n % FWD_SLOTS;
            if (!mbar_wait_warp(&sm.item_full[slot], (n / FWD_SLOTS) & 1u, abort_flag)) { ok = false; break; }
            const FwdItem& it = sm.items[slot];
            if (!it.valid) break;
            const int blocks = uniform(it.n);
            const int4 need = uniform(it.tile[i].need);
            bool pending = false, first = true;      // P V of the block before
            if (!mbar_wait_warp(&sm.q_full[i], n & 1u, abort_flag)) { ok = false; break; }
            for (int b = 0; b <= blocks; ++b) {
                const uint32_t pos = pos0 + 2 * b, st = pos % C::STAGES;
                const bool use = b < blocks && in_ranges(need, b);
                if (b < blocks && !wait_stage(pos)) { ok = false; break; }
                if (use) {
                    if (s_used) {
                        if (!mbar_wait_warp(&sm.s_free[i], parity_s, abort_flag)) { ok = false; break; }
                        parity_s ^= 1u;
                    }
                    s_used = true;
                    tcgen05_fence_after();
                    if (elect_one()) {
                        mma_over_dims<C::HALVES>(s_at, q_base, HALF_BYTES, ring_base + st * C::TILE_BYTES, HALF_BYTES, idesc_s);
                        tcgen05_commit(&sm.s_full[i]);
                        tcgen05_commit(&sm.empty[st]);
                        if (b + 1 == need.w) tcgen05_commit(&sm.q_empty[i]);
                    }
                    __syncwarp();
                }
                if (pending) {
                    const uint32_t sv = (pos - 1) % C::STAGES;
                    if (!wait_stage(pos - 1) || !mbar_wait_warp(&sm.p_full[i], parity_p, abort_flag)) { ok = false; break; }
                    parity_p ^= 1u;
                    tcgen05_fence_after();
                    if (elect_one()) {
                        mma_over_rows<FWD_BLOCK, 0, 8>(o_at, p_at, ring_base + sv * C::TILE_BYTES, idesc_o, first);
                        tcgen05_commit(&sm.pv_done[i]);
                        tcgen05_commit(&sm.empty[sv]);
                    }
                    __syncwarp();
                    first = false;
                }
                pending = use;
                if (b < blocks && !use) {            // handed back as it came, but not before: a stage's uses are counted in order
                    if (!wait_stage(pos + 1)) { ok = false; break; }
                    if (elect_one()) { mbar_arrive(&sm.empty[st]); mbar_arrive(&sm.empty[(pos + 1) % C::STAGES]); }
                    __syncwarp();
                }
            }
            pos0 += 2 * blocks;
            if (ok && elect_one()) {
                if (need.w == 0) mbar_arrive(&sm.q_empty[i]);       // a tile without tokens
                mbar_arrive(&sm.item_empty[slot]);
            }
            __syncwarp();
        }
        if (!ok) {
            if (elect_one()) tcgen05_commit(&sm.drain[i]);
            __syncwarp();
            for (uint32_t spin = 0; spin < SPIN_LIMIT; ++spin)
                if (mbar_try_wait(&sm.drain[i], 0u)) break;
        }
        __syncwarp();
    } else if (warp == 2) {
        // ---- scanner.  Where a block lies at the edge of some row's range, 0 times an infinity or a NaN would carry values of keys that the row does not
        // attend to into its sum: such values become zeros here, and the softmax groups give NaN to rows that do attend to them.
        uint32_t pos0 = 0;
        bool ok = true;
        for (uint32_t n = 0; ok; ++n) {
            const uint32_t slot = n % FWD_SLOTS;
            if (!mbar_wait_warp(&sm.item_full[slot], (n / FWD_SLOTS) & 1u, abort_flag)) break;
            const FwdItem& it = sm.items[slot];
            if (!it.valid) break;
            const int blocks = it.n;
            const int4 need0 = it.tile[0].need, need1 = it.tile[1].need, whole0 = it.tile[0].whole, whole1 = it.tile[1].whole;
            uint32_t bad_whole = 0u;             // bit i: a block that all rows of tile i have was cleaned for the other one
            for (int b = 0; b < blocks; ++b) {
                const uint32_t pos = pos0 + 2 * b + 1, st = pos % C::STAGES;
                if (!mbar_wait_warp(&sm.full[st], (pos / C::STAGES) & 1u, abort_flag)) { ok = false; break; }
                if ((in_ranges(need0, b) && !in_ranges(whole0, b)) || (in_ranges(need1, b) && !in_ranges(whole1, b))) {
#pragma unroll 1
                    for (int w = 0; w < 4; ++w) {
                        bool bad = false;
#pragma unroll
                        for (int h = 0; h < C::HALVES; ++h) {
                            uint8_t* at = ring + st * C::TILE_BYTES + h * HALF_BYTES + (w * 32 + lane) * 128;
                            if (row_not_finite(at, lane)) {
                                bad = true;
                                drop_not_finite(at);
                                fence_proxy_async_smem();
                            }
                        }
                        const uint32_t all = __ballot_sync(0xffffffffu, bad);
                        if (lane == 0) sm.bad_keys[st][w] = all;
                        if (all) bad_whole |= (in_ranges(whole0, b) ? 1u : 0u) | (in_ranges(whole1, b) ? 2u : 0u);
                    }
                }
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive(&sm.scanned[st]);
                    // keys too: S of the block that has the stage next then says that the values which had its values' stage have been looked over
                    if (C::AHEAD) mbar_arrive(&sm.empty[(pos - 1) % C::STAGES]);
                    mbar_arrive(&sm.empty[st]);
                }
                __syncwarp();
            }
            pos0 += 2 * blocks;
            if (lane == 0) {
                sm.bad_whole[slot] = bad_whole;
                mbar_arrive(&sm.item_scanned[slot]);
                mbar_arrive(&sm.item_empty[slot]);
            }
            __syncwarp();
        }
    } else if (warp >= 4) {
        // ---- softmax group i: thread = query row.  Probabilities are taken against a maximum that may be up to 2^8 behind the running one, which
        // changes nothing (sum and products carry the same factor) and spares nearly all passes over O.
        const int i = (warp - 4) >> 2, quarter = warp & 3, row = quarter * 32 + lane;
        const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
        const uint32_t s_at = tmem + lanes + i * 128, o_at = tmem + lanes + C::O_AT + i * DP, p_at = tmem + lanes + C::P_AT + i * C::P_STEP;
        const float scale = p.sh.scale_log2;
        const TokenBounds* bounds = pdl_acquire(p.sh.bounds);
        const int tok = row / ratio, head = row - tok * ratio;
        uint32_t pos0 = 0, s_count = 0;      // blocks of this tile so far: parity of s_full, pv_done
        bool ok = true;
        for (uint32_t n = 0; ok; ++n) {
            const uint32_t slot = n % FWD_SLOTS;
            if (!mbar_wait_warp(&sm.item_full[slot], (n / FWD_SLOTS) & 1u, abort_flag)) { ok = false; break; }
            const FwdItem& it = sm.items[slot];
            if (!it.valid) break;
            const int t = it.t0 + i * TOK + tok;
            const bool live = tok < it.tile[i].tokens;
            TokenBounds bd = {0, 0, 0, 0};
            if (live) bd = bounds[t];
            float m = -INFINITY, l = 0.f;
            bool have_o = false;
            const int4 need = it.tile[i].need, whole = it.tile[i].whole;
            const int n_pre = it.n_pre;
            int b = need.y > need.x ? need.x : need.z;
            bool masked = !in_ranges(whole, b);
            while (b < need.w) {
                const bool pre = b < n_pre;
                int lo = 0, len = FWD_BLOCK;
                if (masked) {
                    const int k0 = pre ? it.pre0 + b * FWD_BLOCK : it.own0 + (b - n_pre) * FWD_BLOCK;
                    lo = (pre ? bd.pre_lo : bd.own_lo) - k0;
                    len = !live ? 0 : (pre ? bd.pre_hi : t + 1) - k0 - lo;
                    if (lo < 0) { len += lo; lo = 0; }
                    len = min(max(len, 0), FWD_BLOCK - lo);
                }
                if (!mbar_wait_warp(&sm.s_full[i], s_count & 1u, abort_flag)) { ok = false; break; }
                if (C::AHEAD && i == 1 && !have_o && it.n >= APART_FROM) {
                    // half a block behind the other tile, once: in step, both groups would want the exponentials' unit at the same time and
                    // leave it idle at the same time
                    const long long c0 = clock64();
                    while (clock64() - c0 < APART_CYCLES) {}
                }
                tcgen05_fence_after();
                uint32_t s[4][32];
                __syncwarp();
#pragma unroll
                for (int c = 0; c < 4; ++c) tcgen05_ld_32x32_issue(s_at + c * 32, s[c]);
                uint32_t on[4] = {0xffffffffu, 0xffffffffu, 0xffffffffu, 0xffffffffu};     // this row's keys of the block
                if (masked) {
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        const int a = min(max(lo - c * 32, 0), 32), z = min(max(lo + len - c * 32, 0), 32);
                        on[c] = z > a ? (0xffffffffu >> (32 - z + a)) << a : 0u;
                    }
                }
#pragma unroll
                for (int c = 0; c < 4; ++c) tcgen05_ld_wait(s[c]);
                if (C::AHEAD) {                  // S is in registers: the next block's may take its place
                    tcgen05_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&sm.s_free[i]);
                    __syncwarp();
                }
                if (masked) {
#pragma unroll
                    for (int c = 0; c < 4; ++c)
                        if (!__all_sync(0xffffffffu, on[c] == 0xffffffffu)) {
#pragma unroll
                            for (int j = 0; j < 32; ++j)
                                if (!(on[c] >> j & 1u)) s[c][j] = 0xFF800000u;
                        }
                }
                float mx[4];
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    mx[c] = fmaxf(__uint_as_float(s[c][0]), __uint_as_float(s[c][1]));
#pragma unroll
                    for (int j = 2; j < 32; j += 2) mx[c] = max3(mx[c], __uint_as_float(s[c][j]), __uint_as_float(s[c][j + 1]));
                }
                const float top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * scale;
                float up = 1.f;
                if (top > m + RESCALE_AT) {  // the first finite score too
                    up = ex2_approx(m - top);
                    m = top;
                    l *= up;
                }
                const bool rescale = have_o && __any_sync(0xffffffffu, up != 1.f);
                if (have_o && (C::AHEAD || rescale)) {       // P V of the block before is done: P may be written over, O changed
                    if (!mbar_wait_warp(&sm.pv_done[i], (s_count - 1u) & 1u, abort_flag)) { ok = false; break; }
                    tcgen05_fence_after();
                }
                if (rescale) {
#pragma unroll 1
                    for (int c = 0; c < DP / 16; ++c) {
                        float v[16];
                        __syncwarp();
                        tcgen05_ld_32(o_at + c * 16, v);
#pragma unroll
                        for (int j = 0; j < 16; ++j) v[j] *= up;
                        tcgen05_st_32x16(o_at + c * 16, v);
                    }
                }
                const float sub = m == -INFINITY ? 0.f : -m;
                const uint64_t scale2 = pack_f32x2(scale, scale), sub2 = pack_f32x2(sub, sub);
                uint64_t sum[2] = {0, 0};
                uint32_t pk[4][16];
                auto quarter_of_p = [&](int c) {
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        float x, y;
                        unpack_f32x2(fma_f32x2(pack_f32x2(__uint_as_float(s[c][2 * j]), __uint_as_float(s[c][2 * j + 1])), scale2, sub2), x, y);
                        x = ex2_approx(x);
                        y = ex2_approx(y);
                        sum[j & 1] = add_f32x2(sum[j & 1], pack_f32x2(x, y));
                        pk[c][j] = pack_bf16(x, y);
                    }
                };
                auto publish = [&](uint64_t* bar) {
                    __syncwarp();
                    tcgen05_st_wait();
                    tcgen05_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar);
                    __syncwarp();
                };
                if (masked) {
                    // The values have been looked over before P V may begin.  Nothing here may wait for the scanner while it is still at the values that had the
                    // stage before: their phase's parity is what the wait would take for this one's, and S needs the keys alone.  A stage that has been
                    // filled again rules it out; where S runs ahead the keys' stage does, which the scanner hands back with the values (there 413 us with
                    // this wait, 399 with that; with heads of 128 458 with this, 472 to 487 with that).
                    const uint32_t pos = pos0 + 2 * b + 1, st = pos % C::STAGES, parity = (pos / C::STAGES) & 1u;
                    if (!C::AHEAD && !mbar_wait_warp(&sm.full[st], parity, abort_flag)) { ok = false; break; }
                    if (!mbar_wait_warp(&sm.scanned[st], parity, abort_flag)) { ok = false; break; }
                    const uint4 bad = *reinterpret_cast<const uint4*>(sm.bad_keys[st]);
                    if ((bad.x & on[0]) | (bad.y & on[1]) | (bad.z & on[2]) | (bad.w & on[3])) l = NAN;
                    __syncwarp();
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        if (__all_sync(0xffffffffu, on[c] == 0u)) {      // no key of any row of the warp
#pragma unroll
                            for (int j = 0; j < 16; ++j) pk[c][j] = 0u;
                        } else {
                            quarter_of_p(c);
                        }
                        __syncwarp();
                        tcgen05_st_32x16(p_at + c * 16, pk[c]);
                        if (c == 2 && !C::AHEAD) publish(&sm.p_most[i]);
                    }
                } else {
                    // no barrier and no store between the exponentials that could keep their pipeline from filling
                    quarter_of_p(0);
                    quarter_of_p(1);
                    quarter_of_p(2);
                    if (C::AHEAD) quarter_of_p(3);
                    __syncwarp();
#pragma unroll
                    for (int c = 0; c < (C::AHEAD ? 4 : 3); ++c) tcgen05_st_32x16(p_at + c * 16, pk[c]);
                    if (!C::AHEAD) {
                        publish(&sm.p_most[i]);
                        quarter_of_p(3);
                        __syncwarp();
                        tcgen05_st_32x16(p_at + 48, pk[3]);
                    }
                }
                b = b + 1 == need.y ? need.z : b + 1;
                masked = !in_ranges(whole, b);
                publish(&sm.p_full[i]);
                float x, y;
                unpack_f32x2(add_f32x2(sum[0], sum[1]), x, y);
                l += x + y;
                ++s_count;
                have_o = true;
            }
            pos0 += 2 * it.n;
            if (!ok) break;
            if (have_o) {
                if (!mbar_wait_warp(&sm.pv_done[i], (s_count - 1u) & 1u, abort_flag)) { ok = false; break; }
                tcgen05_fence_after();
                if (!mbar_wait_warp(&sm.item_scanned[slot], (n / FWD_SLOTS) & 1u, abort_flag)) { ok = false; break; }
                if (sm.bad_whole[slot] >> i & 1u) l = NAN;
                const int h = it.g * ratio + head;
                const float inv = 1.f / l;
                __nv_bfloat16* out = p.o + (int64_t)t * p.o_stride + (int64_t)h * p.sh.D;
                const int64_t part_row = ((int64_t)it.split * p.sh.T_max + t) * p.sh.Hq + h;
#pragma unroll 1
                for (int c = 0; c < DP / 32; ++c) {
                    uint32_t v[32];
                    __syncwarp();
                    tcgen05_ld_32x32_issue(o_at + c * 32, v);
                    tcgen05_ld_wait(v);
                    if (live) {
                        if constexpr (SPLIT) {
#pragma unroll
                            for (int j = 0; j < 32; j += 4)
                                if (c * 32 + j < p.sh.D)
                                    *reinterpret_cast<uint4*>(p.part_o + part_row * p.sh.D + c * 32 + j) = make_uint4(v[j], v[j + 1], v[j + 2], v[j + 3]);
                        } else {
#pragma unroll
                            for (int j = 0; j < 32; j += 8)
                                if (c * 32 + j < p.sh.D) {
                                    uint4 w;
                                    w.x = pack_bf16(__uint_as_float(v[j]) * inv, __uint_as_float(v[j + 1]) * inv);
                                    w.y = pack_bf16(__uint_as_float(v[j + 2]) * inv, __uint_as_float(v[j + 3]) * inv);
                                    w.z = pack_bf16(__uint_as_float(v[j + 4]) * inv, __uint_as_float(v[j + 5]) * inv);
                                    w.w = pack_bf16(__uint_as_float(v[j + 6]) * inv, __uint_as_float(v[j + 7]) * inv);
                                    *reinterpret_cast<uint4*>(out + c * 32 + j) = w;
                                }
                        }
                    }
                }
                __syncwarp();
                tcgen05_fence_before();
                if (!SPLIT && live) p.lse[(int64_t)t * p.sh.Hq + h] = (m + log2f(l)) * LN2;
            }
            if (SPLIT && live)           // a part without a key of this tile: nothing for the join
                p.part_ml[((int64_t)it.split * p.sh.T_max + t) * p.sh.Hq + it.g * ratio + head] = have_o ? make_float2(m, l) : make_float2(-INFINITY, 0.f);
            __syncwarp();
            if (lane == 0) mbar_arrive(&sm.item_empty[slot]);
            __syncwarp();
        }
    }
    tcgen05_fence_before();
    __syncthreads();
    if (threadIdx.x == 0 && *abort_flag) atomicOr(p.status, ARROL_DEV_WAIT_EXPIRED);
    if (warp == 1) {
        tcgen05_fence_after();
        tcgen05_dealloc(tmem, 512);
    }
}

// The parts of a row, in order: a warp per (token, query head), four dimensions a lane.
__global__ void __launch_bounds__(256) attention_join_kernel(const FwdParams p) {
    pdl_launch_dependents();
    pdl_wait();
    const int T = clamp_row(*pdl_acquire(p.sh.d_num + 1), 0, p.sh.T_max), lane = threadIdx.x & 31, d = lane * 4;
    const int64_t rows = (int64_t)T * p.sh.Hq, step = (int64_t)p.sh.T_max * p.sh.Hq;
    for (int64_t i = blockIdx.x * (int64_t)8 + (threadIdx.x >> 5); i < rows; i += (int64_t)gridDim.x * 8) {
        const float2* ml = pdl_acquire(p.part_ml) + i;
        const float* o = pdl_acquire(p.part_o) + i * p.sh.D + d;
        float top = -INFINITY, l = 0.f;
        for (int s = 0; s < p.splits; ++s) top = fmaxf(top, ml[s * step].x);
        float4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
        for (int s = 0; s < p.splits; ++s) {
            const float2 x = ml[s * step];
            if (x.x == -INFINITY && x.y == 0.f) continue;            // no key; its sums were not written
            const float by = x.x == -INFINITY ? 1.f : ex2_approx(x.x - top);       // a NaN without a reference stays one
            l += by * x.y;
            if (d < p.sh.D) {
                const float4 v = *reinterpret_cast<const float4*>(o + s * step * p.sh.D);
                sum.x += by * v.x; sum.y += by * v.y; sum.z += by * v.z; sum.w += by * v.w;
            }
        }
        const float inv = 1.f / l;
        const int64_t t = i / p.sh.Hq;
        if (d < p.sh.D)
            *reinterpret_cast<uint2*>(p.o + t * p.o_stride + (i - t * p.sh.Hq) * p.sh.D + d) = make_uint2(pack_bf16(sum.x * inv, sum.y * inv), pack_bf16(sum.z * inv, sum.w * inv));
        if (lane == 0) p.lse[i] = (top + log2f(l)) * LN2;
    }
}

template <int DP>
int launch_attention(arrol_ctx* ctx, const arrol_attention_args* a, const AttnWorkspace& w, cudaStream_t s) {
    using C = FwdConf<DP>;
    bool& set = ctx->attention_smem_set[DP == 128];
    if (!set) {
        ARROL_CUDA_OK(cudaFuncSetAttribute(attention_kernel<DP, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)C::SMEM));
        ARROL_CUDA_OK(cudaFuncSetAttribute(attention_kernel<DP, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)C::SMEM));
        set = true;
    }
    FwdParams p = {};
    p.sh = {a->d_num, w.bounds, nullptr, (int)a->T_max, (int)a->prompt_rows, a->Hq, a->Hkv, a->D, a->Hq / a->Hkv, a->scale, a->scale * LOG2E};
    p.o = static_cast<__nv_bfloat16*>(a->o);
    p.o_stride = a->o_stride;
    p.lse = a->lse;
    p.counter = w.counters;
    p.status = ctx->d_status;
    p.tile_tokens = 128 / p.sh.ratio;
    CUtensorMap q, k, v, pk, pv;
    if (make_map_heads(ctx, &q, a->q, a->T_max, a->Hq, a->D, a->q_stride, p.sh.ratio, p.tile_tokens) != ARROL_OK) return ARROL_ERR_CUDA;
    if (make_map_heads(ctx, &k, a->k, a->T_max, a->Hkv, a->D, a->k_stride, 1, FWD_BLOCK) != ARROL_OK) return ARROL_ERR_CUDA;
    if (make_map_heads(ctx, &v, a->v, a->T_max, a->Hkv, a->D, a->v_stride, 1, FWD_BLOCK) != ARROL_OK) return ARROL_ERR_CUDA;
    pk = k; pv = v;                          // never read without prompts
    if (a->prompt_rows > 0) {
        if (make_map_heads(ctx, &pk, a->prompt_k, a->prompt_rows, a->Hkv, a->D, a->prompt_k_stride, 1, FWD_BLOCK) != ARROL_OK) return ARROL_ERR_CUDA;
        if (make_map_heads(ctx, &pv, a->prompt_v, a->prompt_rows, a->Hkv, a->D, a->prompt_v_stride, 1, FWD_BLOCK) != ARROL_OK) return ARROL_ERR_CUDA;
    }
    // A form of its own: the parts' arithmetic spills 56 bytes of registers a thread with heads of 128 and 92 with 64, the form of whole keys 32 and none.
    p.splits = attn_key_splits(ctx->sm_count, a->T_max, a->prompt_rows, a->P, a->S_max, a->Hq, a->Hkv);
    p.part_o = w.part_o;
    p.part_ml = w.part_ml;
    int64_t items = (a->T_max + 2 * p.tile_tokens - 1) / (2 * p.tile_tokens) * a->Hkv * p.splits;
    const unsigned grid = (unsigned)(items < ctx->sm_count ? items : ctx->sm_count);
    ARROL_CUDA_OK(arrol_launch_pdl(p.splits > 1 ? attention_kernel<DP, true> : attention_kernel<DP, false>, dim3(grid), dim3(FWD_THREADS), C::SMEM, s, q, k, v, pk, pv, p));
    ctx->launches += 1;
    if (p.splits > 1) {
        const int64_t blocks = (a->T_max * a->Hq + 7) / 8;
        ARROL_CUDA_OK(arrol_launch_pdl(attention_join_kernel, dim3((unsigned)(blocks < 8 * ctx->sm_count ? blocks : 8 * ctx->sm_count)), dim3(256), 0, s, p));
        ctx->launches += 1;
    }
    return ARROL_OK;
}

}  // namespace

int arrol_internal_check_attention(const arrol_attention_args* a) {
    if (a->T_max < 0 || a->S_max < 0 || a->P < 0 || a->prompt_rows < 0 || a->G < 1) return ARROL_ERR_INVALID_ARG;
    if (a->Hq < 1 || a->Hkv < 1 || a->D < 1 || a->Hq % a->Hkv) return ARROL_ERR_INVALID_ARG;
    if (!(a->scale > 0.f) || !isfinite(a->scale)) return ARROL_ERR_INVALID_ARG;
    if (!attn_heads_ok(a->Hq, a->Hkv, a->D) || a->T_max >= ATTN_MAX_ROWS || a->prompt_rows >= ATTN_MAX_ROWS) return ARROL_ERR_UNSUPPORTED;
    if (a->T_max == 0 && a->prompt_rows == 0) return ARROL_OK;
    if (!a->d_num || !a->cu_seqlens) return ARROL_ERR_INVALID_ARG;
    if (a->T_max > 0 && (!attn_rows_ok(a->q, a->q_stride, a->Hq, a->D) || !attn_rows_ok(a->k, a->k_stride, a->Hkv, a->D) ||
                         !attn_rows_ok(a->v, a->v_stride, a->Hkv, a->D) || !attn_rows_ok(a->o, a->o_stride, a->Hq, a->D) || !a->lse))
        return ARROL_ERR_INVALID_ARG;
    if (a->P > 0 ? !a->cu_prompts : a->prompt_rows > 0) return ARROL_ERR_INVALID_ARG;
    if (a->prompt_rows > 0 && (!attn_rows_ok(a->prompt_k, a->prompt_k_stride, a->Hkv, a->D) || !attn_rows_ok(a->prompt_v, a->prompt_v_stride, a->Hkv, a->D)))
        return ARROL_ERR_INVALID_ARG;
    if (!a->workspace || !arrol_aligned(a->workspace, 256)) return ARROL_ERR_WORKSPACE;
    return ARROL_OK;
}

int arrol_internal_attention_bounds(arrol_ctx* ctx, const arrol_attention_args* a, const AttnWorkspace& w, bool backward, cudaStream_t s) {
    int64_t items = a->T_max > a->prompt_rows ? a->T_max : a->prompt_rows;
    int64_t blocks = (items + BOUNDS_THREADS - 1) / BOUNDS_THREADS;
    RowStats rs = {};
    if (backward && a->T_max > 0) {
        rs = {static_cast<const __nv_bfloat16*>(a->o), static_cast<const __nv_bfloat16*>(a->d_o), a->o_stride, a->d_o_stride, a->lse, w.stats, a->Hq, a->D};
        const int64_t rows_a_block = BOUNDS_THREADS / (a->D <= 64 ? 8 : 16) * 2;
        if (blocks < (a->T_max * a->Hq + rows_a_block - 1) / rows_a_block) blocks = (a->T_max * a->Hq + rows_a_block - 1) / rows_a_block;
    }
    if (blocks > 8 * ctx->sm_count) blocks = 8 * ctx->sm_count;
    if (blocks < 1) blocks = 1;
    ARROL_CUDA_OK(arrol_launch_pdl(attention_bounds_kernel, dim3((unsigned)blocks), dim3(BOUNDS_THREADS), 0, s, a->cu_seqlens, a->d_num,
                                   a->cu_prompts, a->survivor_idx, a->S_max, (int)a->T_max, a->P, a->G, (int)a->prompt_rows, w.bounds,
                                   backward ? w.prompt_range : nullptr, w.counters, ctx->d_status, rs));
    ctx->launches += 1;
    return ARROL_OK;
}

extern "C" size_t arrol_attention_workspace(arrol_ctx* ctx, int32_t S_max, int64_t T_max, int64_t prompt_rows, int32_t Hq, int32_t Hkv,
                                            int32_t D, int32_t backward) {
    if (!ctx || S_max < 0 || T_max < 0 || prompt_rows < 0 || T_max >= ATTN_MAX_ROWS || prompt_rows >= ATTN_MAX_ROWS || !attn_heads_ok(Hq, Hkv, D)) return 0;
    return attn_workspace(nullptr, ctx->sm_count, T_max, prompt_rows, Hq, Hkv, D, backward != 0).bytes;
}

extern "C" int arrol_attention(arrol_ctx* ctx, const arrol_attention_args* a, void* stream) {
    if (!ctx || !a) return ARROL_ERR_INVALID_ARG;
    const int rc = arrol_internal_check_attention(a);
    if (rc != ARROL_OK) return rc;
    if (a->T_max == 0) return ARROL_OK;
    const AttnWorkspace w = attn_workspace(a->workspace, ctx->sm_count, a->T_max, a->prompt_rows, a->Hq, a->Hkv, a->D, false);
    if (a->workspace_bytes < w.bytes) return ARROL_ERR_WORKSPACE;
    ArrolDeviceGuard guard(ctx->device);
    if (!guard.ok) return ARROL_ERR_CUDA;
    cudaStream_t s = (cudaStream_t)stream;
    const int rb = arrol_internal_attention_bounds(ctx, a, w, false, s);
    if (rb != ARROL_OK) return rb;
    return a->D <= 64 ? launch_attention<64>(ctx, a, w, s) : launch_attention<128>(ctx, a, w, s);
}
