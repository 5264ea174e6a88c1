// arrol_attention: attention of the packed survivors over their shared prompts and their own tokens.
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
// One thread per packed token and per prompt row.  Everything that the other kernels follow is clamped to the buffers here, so numbers out
// of order give wrong results and a status bit, never an access outside.
__global__ void __launch_bounds__(BOUNDS_THREADS)
attention_bounds_kernel(const int64_t* __restrict__ cu_seqlens, const int64_t* __restrict__ d_num, const int64_t* __restrict__ cu_prompts,
                        const int32_t* __restrict__ survivor_idx, int S_max, int T_max, int P, int G, int prompt_rows,
                        TokenBounds* __restrict__ bounds, int2* __restrict__ prompt_range, uint32_t* __restrict__ counters,
                        uint32_t* __restrict__ status) {
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
}

// What the backward needs of a query row: lse log2(e) and delta = sum_d d_o[t, h, d] o[t, h, d].  A warp per row.
__global__ void __launch_bounds__(BOUNDS_THREADS)
attention_stats_kernel(const __nv_bfloat16* __restrict__ o, int64_t o_stride, const __nv_bfloat16* __restrict__ d_o, int64_t d_o_stride,
                       const float* __restrict__ lse, const int64_t* __restrict__ d_num, int T_max, int Hq, int D, float2* __restrict__ stats) {
    pdl_launch_dependents();
    pdl_wait();
    o = pdl_acquire(o); d_o = pdl_acquire(d_o); lse = pdl_acquire(lse); d_num = pdl_acquire(d_num);
    const int T = clamp_row(d_num[1], 0, T_max);
    const int lane = threadIdx.x & 31;
    const int64_t rows = (int64_t)T * Hq, warps = (int64_t)gridDim.x * (BOUNDS_THREADS / 32);
    for (int64_t i = blockIdx.x * (int64_t)(BOUNDS_THREADS / 32) + (threadIdx.x >> 5); i < rows; i += warps) {
        const int64_t t = i / Hq;
        const int h = (int)(i - t * Hq);
        float sum = 0.f;
        for (int c = lane * 4; c < D; c += 128) {
            const uint2 x = *reinterpret_cast<const uint2*>(o + t * o_stride + (int64_t)h * D + c);
            const uint2 y = *reinterpret_cast<const uint2*>(d_o + t * d_o_stride + (int64_t)h * D + c);
            const float2 x0 = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&x.x)), x1 = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&x.y));
            const float2 y0 = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&y.x)), y1 = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&y.y));
            sum += x0.x * y0.x + x0.y * y0.y + (x1.x * y1.x + x1.y * y1.y);
        }
#pragma unroll
        for (int m = 16; m > 0; m >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, m);
        if (lane == 0) stats[i] = make_float2(lse[i] * LOG2E, sum);
    }
}

// ---- the tensor-core kernel ------------------------------------------------------------------------------------------------------
// Work item = (2 TOK consecutive packed tokens, key head).  Its query rows are all of these tokens' heads of the group, token-major, so a group of
// any size fills the 128 rows of a tile (TOK = 128 / ratio tokens, rounded down) and keys are loaded once per group; two tiles share the loads.
// Keys come in blocks of 128: those of the tiles' prompts (consecutive prompts are consecutive rows), then the own ones; a block
// that lies inside every row's range is not masked at all.
constexpr int FWD_BLOCK = 128;
constexpr int FWD_THREADS = 320;             // producer, MMA issuer, two softmax groups of four warps
constexpr int FWD_SLOTS = 2;                 // work items announced ahead
constexpr uint32_t HALF_BYTES = 128 * 128;   // 128 rows x 64 dimensions
constexpr float RESCALE_AT = 8.0f;           // the running maximum follows once it is 2^8 behind

struct FwdTile {
    int tokens;                              // live tokens of the tile
    int pre_lo, pre_hi, own_lo, own_hi;      // keys that any row needs
    int pre_in_lo, pre_in_hi, own_in_lo, own_in_hi;   // keys that every row needs
};
struct FwdItem {
    int t0, g, valid;
    int pre0, n_pre, own0, n;                // block b < n_pre: prompt rows pre0 + 128 b .., then own rows own0 + 128 (b - n_pre) ..
    FwdTile tile[2];
};
__device__ __forceinline__ int fwd_block_start(const FwdItem& it, int b) { return b < it.n_pre ? it.pre0 + b * FWD_BLOCK : it.own0 + (b - it.n_pre) * FWD_BLOCK; }
__device__ __forceinline__ bool fwd_needs(const FwdItem& it, int i, int b) {
    const FwdTile& t = it.tile[i];
    const int k0 = fwd_block_start(it, b), lo = b < it.n_pre ? t.pre_lo : t.own_lo, hi = b < it.n_pre ? t.pre_hi : t.own_hi;
    return k0 < hi && k0 + FWD_BLOCK > lo;
}
__device__ __forceinline__ bool fwd_masked(const FwdItem& it, int i, int b) {
    const FwdTile& t = it.tile[i];
    const int k0 = fwd_block_start(it, b), lo = b < it.n_pre ? t.pre_in_lo : t.own_in_lo, hi = b < it.n_pre ? t.pre_in_hi : t.own_in_hi;
    return k0 < lo || k0 + FWD_BLOCK > hi;
}

template <int DP>
struct FwdConf {
    static constexpr int HALVES = DP / 64;
    static constexpr uint32_t TILE_BYTES = HALVES * HALF_BYTES;
    static constexpr int STAGES = DP == 128 ? 4 : 8;
    static constexpr size_t SMEM = 1024 + (2 + STAGES) * (size_t)TILE_BYTES;
};

struct FwdParams {
    AttnShape sh;
    __nv_bfloat16* o;
    int64_t o_stride;
    float* lse;
    uint32_t* counter;
    uint32_t* status;
    int tile_tokens;                         // TOK
};

struct FwdShared {
    uint64_t full[8], empty[8], q_full, q_empty, s_full[2], p_full[2], pv_done[2], item_full[FWD_SLOTS], item_empty[FWD_SLOTS], scanned[2], drain;
    uint32_t bad_keys[8][4];                 // per stage with values: keys of an edge block that are not finite
    FwdItem items[FWD_SLOTS];
    uint32_t tmem, abort;
};

template <int DP>
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
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int i = 0; i < C::STAGES; ++i) { mbar_init(&sm.full[i], 1); mbar_init(&sm.empty[i], 1); }
        mbar_init(&sm.q_full, 1);
        mbar_init(&sm.q_empty, 1);
        for (int i = 0; i < 2; ++i) { mbar_init(&sm.s_full[i], 1); mbar_init(&sm.p_full[i], 4); mbar_init(&sm.pv_done[i], 1); mbar_init(&sm.scanned[i], 4); }
        for (int i = 0; i < FWD_SLOTS; ++i) { mbar_init(&sm.item_full[i], 1); mbar_init(&sm.item_empty[i], 9); }
        mbar_init(&sm.drain, 1);
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
    const uint32_t tmem = sm.tmem;           // S of the two tiles (P in its place), then O
    pdl_launch_dependents();
    pdl_wait();
    const int T = clamp_row(*pdl_acquire(p.sh.d_num + 1), 0, p.sh.T_max);
    const int ratio = p.sh.ratio, TOK = p.tile_tokens;
    const int pairs = (T + 2 * TOK - 1) / (2 * TOK);
    const int64_t items = (int64_t)pairs * p.sh.Hkv;

    if (warp == 0) {
        // ---- producer: fetches work items, announces them, loads queries, keys and values
        const TokenBounds* bounds = pdl_acquire(p.sh.bounds);
        uint32_t pos = 0, q_loads = 0;       // ring positions filled so far, items whose queries were asked for
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
                const int t0 = (pairs - 1 - (int)(idx / (uint32_t)p.sh.Hkv)) * 2 * TOK;
                FwdTile tl = {0, 0, 0, 0, 0, 0, 0, 0, 0};
                if (lane < 2) {
                    const int first = t0 + lane * TOK;
                    tl.tokens = min(TOK, T - first);
                    if (tl.tokens > 0) {
                        const int last = first + tl.tokens - 1;
                        const TokenBounds a = bounds[first], z = bounds[last];
                        tl = {tl.tokens, a.pre_lo, z.pre_hi, a.own_lo, last + 1, z.pre_lo, a.pre_hi, z.own_lo, first + 1};
                        if (tl.pre_hi <= tl.pre_lo) tl.pre_hi = tl.pre_lo = 0;
                    } else {
                        tl.tokens = 0;
                    }
                    it.tile[lane] = tl;
                }
                __syncwarp();
                if (lane == 0) {
                    const FwdTile &a = it.tile[0], &z = it.tile[1];
                    int pl = a.pre_lo, ph = a.pre_hi;
                    if (z.pre_hi > z.pre_lo) {
                        pl = ph > pl ? min(pl, z.pre_lo) : z.pre_lo;
                        ph = max(ph, z.pre_hi);
                    }
                    const int ol = a.own_lo, oh = z.tokens > 0 ? z.own_hi : a.own_hi;
                    it.t0 = t0;
                    it.g = (int)(idx % (uint32_t)p.sh.Hkv);
                    it.pre0 = pl;
                    it.n_pre = (ph - pl + FWD_BLOCK - 1) / FWD_BLOCK;
                    it.own0 = ol;
                    it.n = it.n_pre + (oh - ol + FWD_BLOCK - 1) / FWD_BLOCK;
                }
            }
            if (lane == 0) it.valid = valid;
            __syncwarp();
            if (lane == 0) mbar_arrive(&sm.item_full[slot]);
            __syncwarp();
            if (!valid) break;
            const int g = it.g, t0 = it.t0, blocks = it.n;
            if (!mbar_wait_warp(&sm.q_empty, (n & 1u) ^ 1u, abort_flag)) { ok = false; break; }
            if (elect_one()) {
                mbar_expect_tx(&sm.q_full, 2u * C::HALVES * (uint32_t)(TOK * ratio) * 128u);
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int h = 0; h < C::HALVES; ++h)
                        tma_load_3d(q_tiles + i * C::TILE_BYTES + h * HALF_BYTES, &map_q, h * 64, g * ratio, t0 + i * TOK, &sm.q_full);
            }
            __syncwarp();
            ++q_loads;
            for (int b = 0; b < blocks && ok; ++b) {
                const bool pre = b < it.n_pre;
                const int row = fwd_block_start(it, b);
#pragma unroll
                for (int kv = 0; kv < 2; ++kv, ++pos) {
                    const uint32_t st = pos % C::STAGES;
                    if (!mbar_wait_warp(&sm.empty[st], ((pos / C::STAGES) & 1u) ^ 1u, abort_flag)) { ok = false; break; }
                    if (lane < 4) sm.bad_keys[st][lane] = 0u;
                    __syncwarp();
                    if (elect_one()) {
                        mbar_expect_tx(&sm.full[st], C::TILE_BYTES);
                        const CUtensorMap* m = kv == 0 ? (pre ? &map_pk : &map_k) : (pre ? &map_pv : &map_v);
#pragma unroll
                        for (int h = 0; h < C::HALVES; ++h) tma_load_3d(ring + st * C::TILE_BYTES + h * HALF_BYTES, m, h * 64, g, row, &sm.full[st]);
                    }
                    __syncwarp();
                }
            }
        }
        if (!ok) {                           // let the copies in flight land before the block's shared memory goes away
            for (uint32_t i = 1; i <= C::STAGES && i <= pos; ++i)
                for (uint32_t spin = 0; spin < SPIN_LIMIT; ++spin)
                    if (mbar_try_wait(&sm.full[(pos - i) % C::STAGES], ((pos - i) / C::STAGES) & 1u)) break;
            if (q_loads > 0)
                for (uint32_t spin = 0; spin < SPIN_LIMIT; ++spin)
                    if (mbar_try_wait(&sm.q_full, (q_loads - 1u) & 1u)) break;
        }
        __syncwarp();
    } else if (warp == 1) {
        // ---- MMA issuer.  Per tile and block: S = Q K^T, and once the softmax group has put P in its place, O += P V, directly followed by
        // the next block's S; while one tile's softmax runs, the tensor cores work for the other one.
        constexpr uint32_t idesc_s = make_idesc(128, FWD_BLOCK), idesc_o = make_idesc(128, DP, false, true);
        const uint32_t q_base = smem_u32(q_tiles), ring_base = smem_u32(ring);
        uint32_t pos0 = 0, parity_p[2] = {0, 0};
        bool ok = true;
        for (uint32_t n = 0; ok; ++n) {
            const uint32_t slot = n % FWD_SLOTS;
            if (!mbar_wait_warp(&sm.item_full[slot], (n / FWD_SLOTS) & 1u, abort_flag)) { ok = false; break; }
            const FwdItem& it = sm.items[slot];
            if (!it.valid) break;
            if (!mbar_wait_warp(&sm.q_full, n & 1u, abort_flag)) { ok = false; break; }
            tcgen05_fence_after();
            int pending[2] = {-1, -1};       // block whose P V is still to be issued
            bool first[2] = {true, true};
            // a stage is free after the last tile that needs it: tile 1 where it does, as its MMAs are issued behind tile 0's
            auto issue_pv = [&](int i) {
                const uint32_t pos = pos0 + 2 * pending[i] + 1, st = pos % C::STAGES;
                if (!mbar_wait_warp(&sm.p_full[i], parity_p[i], abort_flag)) return false;
                parity_p[i] ^= 1u;
                if (!mbar_wait_warp(&sm.full[st], (pos / C::STAGES) & 1u, abort_flag)) return false;
                tcgen05_fence_after();
                if (elect_one()) {
                    const uint64_t b_desc = make_smem_desc_mn(ring_base + st * C::TILE_BYTES, 128);
#pragma unroll
                    for (int k = 0; k < FWD_BLOCK / UMMA_K; ++k)
                        tcgen05_mma_bf16_tmem_a(tmem + 256 + i * 128, tmem + i * 128 + k * (UMMA_K / 2), b_desc + (uint64_t)(k * (UMMA_K * 128 >> 4)), idesc_o,
                                                first[i] && k == 0 ? 0u : 1u);
                    if (i == 1 || !fwd_needs(it, 1, pending[i])) tcgen05_commit(&sm.empty[st]);
                    tcgen05_commit(&sm.pv_done[i]);
                }
                __syncwarp();
                first[i] = false;
                pending[i] = -1;
                return true;
            };
            for (int b = 0; b < it.n && ok; ++b) {
                const uint32_t pos = pos0 + 2 * b, st = pos % C::STAGES;
                if (!fwd_needs(it, 0, b) && !fwd_needs(it, 1, b)) {      // only where row numbers are out of order
                    const uint32_t sv = (pos + 1) % C::STAGES;
                    if (!mbar_wait_warp(&sm.full[st], (pos / C::STAGES) & 1u, abort_flag) ||
                        !mbar_wait_warp(&sm.full[sv], ((pos + 1) / C::STAGES) & 1u, abort_flag)) { ok = false; break; }
                    if (elect_one()) { mbar_arrive(&sm.empty[st]); mbar_arrive(&sm.empty[sv]); }
                    __syncwarp();
                    continue;
                }
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    if (!ok) break;
                    if (pending[i] >= 0 && !issue_pv(i)) { ok = false; break; }
                    if (!fwd_needs(it, i, b)) continue;
                    if (!mbar_wait_warp(&sm.full[st], (pos / C::STAGES) & 1u, abort_flag)) { ok = false; break; }
                    tcgen05_fence_after();
                    if (elect_one()) {
#pragma unroll
                        for (int h = 0; h < C::HALVES; ++h) {
                            const uint64_t a_desc = make_smem_desc(q_base + i * C::TILE_BYTES + h * HALF_BYTES);
                            const uint64_t b_desc = make_smem_desc(ring_base + st * C::TILE_BYTES + h * HALF_BYTES);
#pragma unroll
                            for (int k = 0; k < 64 / UMMA_K; ++k)
                                tcgen05_mma_bf16(tmem + i * 128, a_desc + (uint64_t)(k * (UMMA_K * 2 >> 4)), b_desc + (uint64_t)(k * (UMMA_K * 2 >> 4)), idesc_s, (h | k) != 0 ? 1u : 0u);
                        }
                        tcgen05_commit(&sm.s_full[i]);
                        if (i == 1 || !fwd_needs(it, 1, b)) tcgen05_commit(&sm.empty[st]);
                    }
                    __syncwarp();
                    pending[i] = b;
                }
            }
            if (ok && elect_one()) tcgen05_commit(&sm.q_empty);      // the item's last use of its queries
            __syncwarp();
#pragma unroll
            for (int i = 0; i < 2; ++i)
                if (ok && pending[i] >= 0 && !issue_pv(i)) ok = false;
            pos0 += 2 * it.n;
            if (ok && elect_one()) mbar_arrive(&sm.item_empty[slot]);
            __syncwarp();
        }
        if (!ok) {
            if (elect_one()) tcgen05_commit(&sm.drain);
            __syncwarp();
            for (uint32_t spin = 0; spin < SPIN_LIMIT; ++spin)
                if (mbar_try_wait(&sm.drain, 0u)) break;
        }
        __syncwarp();
    } else {
        // ---- softmax group i: thread = query row.  Probabilities are taken against a maximum that may be up to 2^8 behind the running one, which
        // changes nothing (sum and products carry the same factor) and spares nearly all passes over O.
        const int i = (warp - 2) >> 2, quarter = warp & 3, row = quarter * 32 + lane;
        const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
        const uint32_t s_at = tmem + lanes + i * 128, o_at = tmem + lanes + 256 + i * 128;
        const float scale = p.sh.scale_log2;
        const TokenBounds* bounds = pdl_acquire(p.sh.bounds);
        const int tok = row / ratio, head = row - tok * ratio;
        uint32_t pos0 = 0, s_count = 0, scans = 0;   // blocks of this tile so far: parity of s_full, pv_done
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
            for (int b = 0; b < it.n && ok; ++b) {
                if (!fwd_needs(it, i, b)) continue;
                const bool masked = fwd_masked(it, i, b);
                const bool edge = masked || (fwd_needs(it, 1 - i, b) && fwd_masked(it, 1 - i, b));
                const int k0 = fwd_block_start(it, b);
                int lo = 0, len = FWD_BLOCK;
                if (masked) {
                    lo = (b < it.n_pre ? bd.pre_lo : bd.own_lo) - k0;
                    len = !live ? 0 : (b < it.n_pre ? bd.pre_hi : t + 1) - k0 - lo;
                }
                if (!mbar_wait_warp(&sm.s_full[i], s_count & 1u, abort_flag)) { ok = false; break; }
                tcgen05_fence_after();
                uint32_t s[4][32];
                __syncwarp();
#pragma unroll
                for (int c = 0; c < 4; ++c) tcgen05_ld_32x32_issue(s_at + c * 32, s[c]);
#pragma unroll
                for (int c = 0; c < 4; ++c) tcgen05_ld_wait(s[c]);
                if (masked) {
#pragma unroll
                    for (int c = 0; c < 4; ++c)
#pragma unroll
                        for (int j = 0; j < 32; ++j)
                            if (len <= 0 || (uint32_t)(c * 32 + j - lo) >= (uint32_t)len) s[c][j] = 0xFF800000u;
                }
                float mx[4];
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    mx[c] = __uint_as_float(s[c][0]);
#pragma unroll
                    for (int j = 1; j < 32; ++j) mx[c] = fmaxf(mx[c], __uint_as_float(s[c][j]));
                }
                const float top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * scale;
                float up = 1.f;
                if (top > m + RESCALE_AT) {  // the first finite score too
                    up = ex2_approx(m - top);
                    m = top;
                    l *= up;
                }
                const float sub = m == -INFINITY ? 0.f : -m;
                const uint64_t scale2 = pack_f32x2(scale, scale), sub2 = pack_f32x2(sub, sub);
                uint64_t sum[2] = {0, 0};
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    uint32_t pk[32];
#pragma unroll
                    for (int j = 0; j < 32; ++j) {
                        const int cc = c * 2 + j / 16, jj = (j % 16) * 2;
                        float x, y;
                        unpack_f32x2(fma_f32x2(pack_f32x2(__uint_as_float(s[cc][jj]), __uint_as_float(s[cc][jj + 1])), scale2, sub2), x, y);
                        x = ex2_approx(x);
                        y = ex2_approx(y);
                        sum[j & 1] = add_f32x2(sum[j & 1], pack_f32x2(x, y));
                        pk[j] = pack_bf16(x, y);
                    }
                    __syncwarp();
                    tcgen05_st_32x32(s_at + c * 32, pk);
                }
                float x, y;
                unpack_f32x2(add_f32x2(sum[0], sum[1]), x, y);
                l += x + y;
                if (have_o && __any_sync(0xffffffffu, up != 1.f)) {
                    if (!mbar_wait_warp(&sm.pv_done[i], (s_count - 1u) & 1u, abort_flag)) { ok = false; break; }
                    tcgen05_fence_after();
#pragma unroll 1
                    for (int c = 0; c < DP / 32; ++c) {
                        uint32_t v[32];
                        __syncwarp();
                        tcgen05_ld_32x32_issue(o_at + c * 32, v);
                        tcgen05_ld_wait(v);
#pragma unroll
                        for (int j = 0; j < 32; ++j) v[j] = __float_as_uint(__uint_as_float(v[j]) * up);
                        tcgen05_st_32x32(o_at + c * 32, v);
                    }
                }
                if (edge) {
                    // 0 times an infinity or a NaN would carry values of keys that a row does not attend to into its sum: they become zeros here,
                    // and rows that do attend to them NaN
                    const uint32_t pos = pos0 + 2 * b + 1, st = pos % C::STAGES;
                    if (!mbar_wait_warp(&sm.full[st], (pos / C::STAGES) & 1u, abort_flag)) { ok = false; break; }
                    bool wrote = false;
#pragma unroll
                    for (int h = 0; h < C::HALVES; ++h)
                        wrote |= drop_not_finite(ring + st * C::TILE_BYTES + h * HALF_BYTES + row * 128, lane, [&] {
                            atomicOr(&sm.bad_keys[st][quarter], 1u << lane);
                            __threadfence_block();
                        });
                    if (wrote) fence_proxy_async_smem();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&sm.scanned[i]);
                    __syncwarp();
                    if (!mbar_wait_warp(&sm.scanned[i], scans++ & 1u, abort_flag)) { ok = false; break; }
#pragma unroll
                    for (int w = 0; w < 4; ++w) {
                        const uint32_t bad = *reinterpret_cast<volatile uint32_t*>(&sm.bad_keys[st][w]);
                        if (bad)
                            for (int j = 0; j < 32; ++j)
                                if ((bad >> j & 1u) && len > 0 && (uint32_t)(w * 32 + j - lo) < (uint32_t)len) l = NAN;
                    }
                }
                __syncwarp();
                tcgen05_st_wait();
                tcgen05_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&sm.p_full[i]);
                __syncwarp();
                ++s_count;
                have_o = true;
            }
            pos0 += 2 * it.n;
            if (ok && have_o) {
                if (!mbar_wait_warp(&sm.pv_done[i], (s_count - 1u) & 1u, abort_flag)) { ok = false; break; }
                tcgen05_fence_after();
                const int h = it.g * ratio + head;
                const float inv = 1.f / l;
                __nv_bfloat16* out = p.o + (int64_t)t * p.o_stride + (int64_t)h * p.sh.D;
#pragma unroll 1
                for (int c = 0; c < DP / 32; ++c) {
                    uint32_t v[32];
                    __syncwarp();
                    tcgen05_ld_32x32_issue(o_at + c * 32, v);
                    tcgen05_ld_wait(v);
                    if (live) {
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
                __syncwarp();
                tcgen05_fence_before();
                if (live) p.lse[(int64_t)t * p.sh.Hq + h] = (m + log2f(l)) * LN2;
            }
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

template <int DP>
int launch_attention(arrol_ctx* ctx, const arrol_attention_args* a, const AttnWorkspace& w, cudaStream_t s) {
    using C = FwdConf<DP>;
    bool& set = ctx->attention_smem_set[DP == 128];
    if (!set) {
        ARROL_CUDA_OK(cudaFuncSetAttribute(attention_kernel<DP>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)C::SMEM));
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
    int64_t items = (a->T_max + 2 * p.tile_tokens - 1) / (2 * p.tile_tokens) * a->Hkv;
    const unsigned grid = (unsigned)(items < ctx->sm_count ? items : ctx->sm_count);
    ARROL_CUDA_OK(arrol_launch_pdl(attention_kernel<DP>, dim3(grid), dim3(FWD_THREADS), C::SMEM, s, q, k, v, pk, pv, p));
    ctx->launches += 1;
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
    if (blocks > 4 * ctx->sm_count) blocks = 4 * ctx->sm_count;
    if (blocks < 1) blocks = 1;
    ARROL_CUDA_OK(arrol_launch_pdl(attention_bounds_kernel, dim3((unsigned)blocks), dim3(BOUNDS_THREADS), 0, s, a->cu_seqlens, a->d_num,
                                   a->cu_prompts, a->survivor_idx, a->S_max, (int)a->T_max, a->P, a->G, (int)a->prompt_rows, w.bounds,
                                   backward ? w.prompt_range : nullptr, w.counters, ctx->d_status));
    ctx->launches += 1;
    if (backward && a->T_max > 0) {
        int64_t rows = (a->T_max * a->Hq + 7) / 8;
        if (rows > 16 * ctx->sm_count) rows = 16 * ctx->sm_count;
        ARROL_CUDA_OK(arrol_launch_pdl(attention_stats_kernel, dim3((unsigned)rows), dim3(BOUNDS_THREADS), 0, s,
                                       static_cast<const __nv_bfloat16*>(a->o), a->o_stride, static_cast<const __nv_bfloat16*>(a->d_o),
                                       a->d_o_stride, static_cast<const float*>(a->lse), a->d_num, (int)a->T_max, a->Hq, a->D, w.stats));
        ctx->launches += 1;
    }
    return ARROL_OK;
}

extern "C" size_t arrol_attention_workspace(arrol_ctx* ctx, int32_t S_max, int64_t T_max, int64_t prompt_rows, int32_t Hq, int32_t Hkv,
                                            int32_t D, int32_t backward) {
    if (!ctx || S_max < 0 || T_max < 0 || prompt_rows < 0 || T_max >= ATTN_MAX_ROWS || prompt_rows >= ATTN_MAX_ROWS || !attn_heads_ok(Hq, Hkv, D)) return 0;
    return attn_workspace(nullptr, T_max, prompt_rows, Hq, backward != 0).bytes;
}

extern "C" int arrol_attention(arrol_ctx* ctx, const arrol_attention_args* a, void* stream) {
    if (!ctx || !a) return ARROL_ERR_INVALID_ARG;
    const int rc = arrol_internal_check_attention(a);
    if (rc != ARROL_OK) return rc;
    if (a->T_max == 0) return ARROL_OK;
    const AttnWorkspace w = attn_workspace(a->workspace, a->T_max, a->prompt_rows, a->Hq, false);
    if (a->workspace_bytes < w.bytes) return ARROL_ERR_WORKSPACE;
    ArrolDeviceGuard guard(ctx->device);
    if (!guard.ok) return ARROL_ERR_CUDA;
    cudaStream_t s = (cudaStream_t)stream;
    const int rb = arrol_internal_attention_bounds(ctx, a, w, false, s);
    if (rb != ARROL_OK) return rb;
    return a->D <= 64 ? launch_attention<64>(ctx, a, w, s) : launch_attention<128>(ctx, a, w, s);
}
