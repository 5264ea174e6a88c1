// arrol_attention_backward: gradients of the packed survivors' attention.
//
// P and dS are recomputed from q, k, the logarithms of the sums and delta = d_o . o, twice: once for the keys' gradients and once for the
// queries', 7 products of 2 D flops a pair where 5 would do with sums of dq in memory.  Those sums would be atomics, whose order would change the
// result; this way each tile of gradients has one block that adds in a fixed order in tensor memory.
//
// One kernel, two sides: a block takes items of the keys' side until there are none, then of the queries' side, which needs nothing of the other.
// 128 rows stay (two operands a1, a2), 64 rows a block stream past (b1, b2):
//     x = a1 b1^T,  y = a2 b2^T  (128 x 64),  p = exp(scale x - lse),  ds = p (y - delta),
//   keys' gradients (KEYS):  rows are keys, a1 = k, a2 = v; columns are query rows (tokens x heads of the group), b1 = q, b2 = d_o;
//       dv += p b2,  dk += ds b1;  lse and delta belong to columns;
//   queries' gradients:      rows are query rows, a1 = q, a2 = d_o; columns are keys, b1 = k, b2 = v;
//       dq += ds b1;  lse and delta belong to rows.
// x and y are double-buffered in tensor memory (2 x 128 columns beside the accumulators' 2 x D), p and ds replace them as bf16 and are read from
// there by the second products; two groups of four warps take the blocks in turn.  p and ds are the roundings beside the results'; delta is that of
// the o that was written.
// Bounded by the tensor cores and by what feeds them: with 128 dimensions a block is 512 cycles of first products and 512 of second ones for the keys' side,
// but 64 columns a product make the first ones wait for shared memory (96 KB at 128 a cycle), unless the rows that stay are in tensor memory.
// Measured with 4,096 tokens, 32 heads of 128 on 8: the sides as launches of their own 297 us (keys; tensor pipe busy 0.53 of the cycles, its feeding 0.70)
// and 195 us (queries; 0.58, 0.62); forward and backward together 571 us from a graph, 0.84 PFLOP/s of the 14 D flops a pair that cannot be done without (18
// are done).
#include "attention_common.cuh"

namespace {

constexpr int BWD_THREADS = 384;                  // producer, MMA issuer, scanner, a spare warp; two groups of four warps
constexpr int BWD_BLOCK = 64;                     // columns: query rows or keys a block
constexpr int BWD_SLOTS = 2;
constexpr uint32_t ROWS_HALF_BYTES = 128 * 128;   // 128 rows x 64 dimensions
constexpr uint32_t COLS_HALF_BYTES = 64 * 128;

struct BwdParams {
    AttnShape sh;
    const float2* stats;                          // [T_max, Hq]: lse log2(e), delta
    const int64_t* cu_prompts;
    int P;
    __nv_bfloat16 *dv, *dk, *dq;
    int64_t dv_stride, dk_stride, dq_stride;
    __nv_bfloat16 *shared1, *shared2;             // dprompt_v, dprompt_k
    int64_t shared1_stride, shared2_stride;
    int splits;                                   // parts of the tokens that pass by a prompt's tile, each an item; with more than one their sums go to
    float *part1, *part2;                         // [splits][prompt tiles][Hkv][128][DP]
    uint32_t* counter[2];                         // of the queries' items, the keys' items
    uint32_t* status;
};

struct BwdMaps {
    CUtensorMap q_rows, do_rows, q_cols, do_cols, k_rows, v_rows, k_cols, v_cols, pk_rows, pv_rows, pk_cols, pv_cols;
};

struct BwdItem {
    int valid, g, shared, row0, rows;             // rows row0 .. of keys (prompt rows where shared) or tokens
    int split;
    int pre0, n_pre, own0, n;                     // blocks, as in the forward kernel; KEYS: tokens own0 + TOKQ b ..
    int pre_in_lo, pre_in_hi, in_lo, in_hi;       // columns (keys or tokens) that every row has
};

template <int DP>
struct BwdConf {
    static constexpr int HALVES = DP / 64;
    static constexpr uint32_t ROWS_BYTES = HALVES * ROWS_HALF_BYTES, COLS_BYTES = HALVES * COLS_HALF_BYTES;
    static constexpr int STAGES = DP == 128 ? 4 : 8;
    // The rows that stay are put into tensor memory where there is room (not for keys' gradients of 128 dimensions): read from shared memory, 128 of them
    // with every 64 columns, they make the first products wait for its bandwidth (96 KB at 128 a cycle against 512 cycles of products).
    template <bool KEYS> static constexpr bool A_IN_TMEM = !(KEYS && DP == 128);
    static constexpr uint32_t A_AT = DP == 128 ? 0 : 64, A_STEP = DP == 128 ? 64 : 128;
    static constexpr size_t SMEM = 1024 + 2 * (size_t)ROWS_BYTES + STAGES * 2 * (size_t)COLS_BYTES;
};

struct BwdBarriers {
    uint64_t full[8], empty[8], scanned[8];                    // per stage
    uint64_t a_full, a_ready, a_empty, xy_full[2], ps_full[2], acc_full, acc_empty, item_full[BWD_SLOTS], item_empty[BWD_SLOTS], drain;
};
struct BwdShared {
    BwdBarriers of[2];                            // of the queries' side, the keys' side: the last arrivals of one may come while the other begins
    alignas(16) float lse[8][BWD_BLOCK];          // negative, as delta; read four at a time
    alignas(16) float delta[8][BWD_BLOCK];
    uint32_t bad[8][2], bad_stats[8][2];          // per stage: rows of an edge block that are not finite, or whose statistics are not
    BwdItem items[BWD_SLOTS];
    uint32_t tmem, abort;
};

// Block b's first column and whether some row does not have all of it.
template <bool KEYS>
__device__ __forceinline__ int bwd_start(const BwdItem& it, int b, int TOKQ) {
    if (KEYS) return it.own0 + b * TOKQ;
    return b < it.n_pre ? it.pre0 + b * BWD_BLOCK : it.own0 + (b - it.n_pre) * BWD_BLOCK;
}
template <bool KEYS>
__device__ __forceinline__ bool bwd_masked(const BwdItem& it, int b, int TOKQ) {
    const int c0 = bwd_start<KEYS>(it, b, TOKQ);
    const bool pre = !KEYS && b < it.n_pre;
    return c0 < (pre ? it.pre_in_lo : it.in_lo) || c0 + (KEYS ? TOKQ : BWD_BLOCK) > (pre ? it.pre_in_hi : it.in_hi);
}

template <int DP, bool KEYS>
__device__ __forceinline__ void init_barriers(BwdBarriers& bar) {
    using C = BwdConf<DP>;
    for (int i = 0; i < C::STAGES; ++i) { mbar_init(&bar.full[i], 1); mbar_init(&bar.empty[i], 2); mbar_init(&bar.scanned[i], 1); }
    mbar_init(&bar.a_full, 1);
    mbar_init(&bar.a_ready, 8);
    mbar_init(&bar.a_empty, C::template A_IN_TMEM<KEYS> ? 8 : 1);
    for (int i = 0; i < 2; ++i) { mbar_init(&bar.xy_full[i], 1); mbar_init(&bar.ps_full[i], 4); }
    mbar_init(&bar.acc_full, 1);
    mbar_init(&bar.acc_empty, 8);
    for (int i = 0; i < BWD_SLOTS; ++i) { mbar_init(&bar.item_full[i], 1); mbar_init(&bar.item_empty[i], 10); }
    mbar_init(&bar.drain, 1);
}

// All items of one side that this block gets.  The prompts' keys and values (p1, p2) are rows of KEYS items, columns otherwise.
template <int DP, bool KEYS>
__device__ __forceinline__ void backward_side(const CUtensorMap& map_a1, const CUtensorMap& map_a2, const CUtensorMap& map_b1, const CUtensorMap& map_b2,
                                              const CUtensorMap& map_p1, const CUtensorMap& map_p2, const BwdParams& p, BwdShared& sm, uint8_t* const smem,
                                              const uint32_t tmem) {
    using C = BwdConf<DP>;
    constexpr bool A_TMEM = C::template A_IN_TMEM<KEYS>;
    BwdBarriers& bar = sm.of[KEYS];
    uint8_t* const rows_a = smem;
    uint8_t* const ring = smem + 2 * C::ROWS_BYTES;
    volatile uint32_t* abort_flag = &sm.abort;
    const int warp = uniform((int)threadIdx.x >> 5), lane = threadIdx.x & 31;
    const int ratio = p.sh.ratio, TOK = 128 / ratio, TOKQ = BWD_BLOCK / ratio;
    const int T = clamp_row(*pdl_acquire(p.sh.d_num + 1), 0, p.sh.T_max);
    const int live_prompt = KEYS && p.P > 0 ? clamp_row(pdl_acquire(p.cu_prompts)[p.P], 0, p.sh.prompt_rows) : 0;
    const TokenBounds* bounds = pdl_acquire(p.sh.bounds);
    const int2* prompt_range = pdl_acquire(p.sh.prompt_range);
    const int prompt_tiles = (live_prompt + 127) / 128;
    const int tiles = KEYS ? prompt_tiles * p.splits + (T + 127) / 128 : (T + TOK - 1) / TOK;
    const int64_t items = (int64_t)tiles * p.sh.Hkv;

    if (warp == 0) {
        // ---- producer
        const float2* stats = pdl_acquire(p.stats);
        const int col_tok[2] = {lane / ratio, (lane + 32) / ratio};       // tokens of columns lane and lane + 32 of a block (KEYS)
        uint32_t pos = 0, a_loads = 0;
        bool ok = true;
        for (uint32_t n = 0; ok; ++n) {
            const uint32_t slot = n % BWD_SLOTS, use = n / BWD_SLOTS;
            if (!mbar_wait_warp(&bar.item_empty[slot], (use & 1u) ^ 1u, abort_flag)) { ok = false; break; }
            uint32_t idx = 0;
            if (lane == 0) idx = atomicAdd(p.counter[KEYS], 1u);
            idx = __shfl_sync(0xffffffffu, idx, 0);
            BwdItem it = {};
            it.valid = (int64_t)idx < items;
            if (it.valid) {
                const int tile = (int)(idx / (uint32_t)p.sh.Hkv);
                it.g = (int)(idx % (uint32_t)p.sh.Hkv);
                if (KEYS) {
                    // the prompts' tiles first: every survivor's tokens pass by them; then the own ones from the first token on
                    it.shared = tile < prompt_tiles * p.splits;
                    it.split = it.shared ? tile % p.splits : 0;
                    it.row0 = (it.shared ? tile / p.splits : tile - prompt_tiles * p.splits) * 128;
                    it.rows = min(128, (it.shared ? live_prompt : T) - it.row0);
                    int lo = INT_MAX, hi = 0, in_lo = 0, in_hi = INT_MAX;
                    for (int r = lane; r < it.rows; r += 32) {
                        const int j = it.row0 + r;
                        const int2 x = it.shared ? prompt_range[j] : make_int2(j, bounds[j].own_hi);
                        if (x.x < x.y) { lo = min(lo, x.x); hi = max(hi, x.y); }
                        in_lo = max(in_lo, x.x);
                        in_hi = min(in_hi, x.y);
                    }
                    lo = __reduce_min_sync(0xffffffffu, lo);
                    hi = __reduce_max_sync(0xffffffffu, hi);
                    it.in_lo = __reduce_max_sync(0xffffffffu, in_lo);
                    it.in_hi = __reduce_min_sync(0xffffffffu, in_hi);
                    it.own0 = lo;
                    it.n = lo < hi ? (hi - lo + TOKQ - 1) / TOKQ : 0;
                    if (it.shared && p.splits > 1) {
                        const int each = (it.n + p.splits - 1) / p.splits, from = min(it.split * each, it.n);
                        it.own0 += from * TOKQ;
                        it.n = min(each, it.n - from);
                    }
                } else {
                    it.row0 = (tiles - 1 - tile) * TOK;      // last tokens first: theirs are the longest ranges
                    it.rows = min(TOK, T - it.row0);
                    const int last = it.row0 + it.rows - 1;
                    const TokenBounds a = bounds[it.row0], z = bounds[last];
                    it.pre0 = a.pre_lo;
                    it.n_pre = z.pre_hi > a.pre_lo ? (z.pre_hi - a.pre_lo + BWD_BLOCK - 1) / BWD_BLOCK : 0;
                    it.pre_in_lo = z.pre_lo;
                    it.pre_in_hi = a.pre_hi;
                    it.own0 = a.own_lo;
                    it.n = it.n_pre + (last + 1 - a.own_lo + BWD_BLOCK - 1) / BWD_BLOCK;
                    it.in_lo = z.own_lo;
                    it.in_hi = it.row0 + 1;
                }
            }
            if (lane == 0) sm.items[slot] = it;
            __syncwarp();
            if (lane == 0) mbar_arrive(&bar.item_full[slot]);
            __syncwarp();
            if (!it.valid) break;
            if (it.n == 0) continue;              // a prompt without survivors: nothing is loaded
            if (!mbar_wait_warp(&bar.a_empty, (a_loads & 1u) ^ 1u, abort_flag)) { ok = false; break; }
            if (elect_one()) {
                mbar_expect_tx(&bar.a_full, 2u * C::HALVES * (KEYS ? 128u : (uint32_t)(TOK * ratio)) * 128u);
#pragma unroll
                for (int o = 0; o < 2; ++o) {
                    const CUtensorMap* m = KEYS && it.shared ? (o ? &map_p2 : &map_p1) : (o ? &map_a2 : &map_a1);
#pragma unroll
                    for (int h = 0; h < C::HALVES; ++h)
                        tma_load_3d(rows_a + o * C::ROWS_BYTES + h * ROWS_HALF_BYTES, m, h * 64, KEYS ? it.g : it.g * ratio, it.row0, &bar.a_full);
                }
            }
            __syncwarp();
            ++a_loads;
            // the columns' statistics are asked for three blocks ahead; columns without a query row: p = exp(-inf)
            constexpr int BLOCKS_AHEAD = 3;
            float2 ahead[BLOCKS_AHEAD][2];
            auto ask = [&](int b, float2 (&into)[2]) {
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const int tok = col_tok[u], t = bwd_start<KEYS>(it, b, TOKQ) + tok;
                    into[u] = make_float2(INFINITY, 0.f);
                    if (b < it.n && tok < TOKQ && t < T) into[u] = stats[(int64_t)t * p.sh.Hq + it.g * ratio + (u * 32 + lane - tok * ratio)];
                }
            };
            if (KEYS) {
#pragma unroll
                for (int k = 0; k < BLOCKS_AHEAD; ++k) ask(k, ahead[k]);
            }
            for (int b = 0; b < it.n; ++b, ++pos) {
                const uint32_t st = pos % C::STAGES;
                if (!mbar_wait_warp(&bar.empty[st], ((pos / C::STAGES) & 1u) ^ 1u, abort_flag)) { ok = false; break; }
                if (KEYS) {
                    const bool masked = bwd_masked<KEYS>(it, b, TOKQ);
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        const float2 x = ahead[0][u];
                        const bool there = col_tok[u] < TOKQ && bwd_start<KEYS>(it, b, TOKQ) + col_tok[u] < T;
                        // where some row does not have the column, statistics that are not finite go the way of such values; rows behind the last token
                        // have none and may hold anything
                        const bool bad = masked && col_tok[u] < TOKQ && !(there && fabsf(x.x) < INFINITY && fabsf(x.y) < INFINITY);
                        sm.lse[st][u * 32 + lane] = bad ? 0.f : there && x.x == INFINITY ? NAN : -x.x;
                        sm.delta[st][u * 32 + lane] = bad ? 0.f : -x.y;
                        const uint32_t all = __ballot_sync(0xffffffffu, bad);
                        if (lane == 0) sm.bad_stats[st][u] = all;
                    }
                }
                __syncwarp();
                if (elect_one()) {
                    const bool pre = !KEYS && b < it.n_pre;
                    const int row = bwd_start<KEYS>(it, b, TOKQ);
                    mbar_expect_tx(&bar.full[st], 2u * C::HALVES * (KEYS ? (uint32_t)(TOKQ * ratio) : (uint32_t)BWD_BLOCK) * 128u);
#pragma unroll
                    for (int o = 0; o < 2; ++o) {
                        const CUtensorMap* m = pre ? (o ? &map_p2 : &map_p1) : (o ? &map_b2 : &map_b1);
#pragma unroll
                        for (int h = 0; h < C::HALVES; ++h)
                            tma_load_3d(ring + (st * 2 + o) * C::COLS_BYTES + h * COLS_HALF_BYTES, m, h * 64, KEYS ? it.g * ratio : it.g, row, &bar.full[st]);
                    }
                }
                __syncwarp();
                if (KEYS) {
#pragma unroll
                    for (int k = 0; k + 1 < BLOCKS_AHEAD; ++k) { ahead[k][0] = ahead[k + 1][0]; ahead[k][1] = ahead[k + 1][1]; }
                    ask(b + BLOCKS_AHEAD, ahead[BLOCKS_AHEAD - 1]);
                }
            }
        }
        if (!ok) {                                // let the copies in flight land before the block's shared memory goes away
            for (uint32_t i = 1; i <= C::STAGES && i <= pos; ++i)
                for (uint32_t spin = 0; spin < SPIN_LIMIT; ++spin)
                    if (mbar_try_wait(&bar.full[(pos - i) % C::STAGES], ((pos - i) / C::STAGES) & 1u)) break;
            if (a_loads > 0)
                for (uint32_t spin = 0; spin < SPIN_LIMIT; ++spin)
                    if (mbar_try_wait(&bar.a_full, (a_loads - 1u) & 1u)) break;
        }
        __syncwarp();
    } else if (warp == 1) {
        // ---- MMA issuer: x and y of a block, then the second products of the block before it
        constexpr uint32_t idesc_xy = make_idesc(128, BWD_BLOCK), idesc_acc = make_idesc(128, DP, false, true);
        const uint32_t a_base = smem_u32(rows_a), ring_base = smem_u32(ring);
        uint32_t c = 0, with_blocks = 0;          // blocks, items with blocks so far
        bool ok = true;
        for (uint32_t n = 0; ok; ++n) {
            const uint32_t slot = n % BWD_SLOTS;
            if (!mbar_wait_warp(&bar.item_full[slot], (n / BWD_SLOTS) & 1u, abort_flag)) { ok = false; break; }
            if (!sm.items[slot].valid) break;
            const int blocks = uniform(sm.items[slot].n);
            if (blocks > 0) {
                if (!mbar_wait_warp(A_TMEM ? &bar.a_ready : &bar.a_full, with_blocks & 1u, abort_flag)) { ok = false; break; }
                for (int b = 0; b <= blocks; ++b) {
                    if (b < blocks) {
                        const uint32_t cur = c + b, st = cur % C::STAGES, xy = tmem + 256 + (cur & 1u) * 128;
                        if (!mbar_wait_warp(&bar.full[st], (cur / C::STAGES) & 1u, abort_flag)) { ok = false; break; }
                        tcgen05_fence_after();
                        if (elect_one()) {
#pragma unroll
                            for (int o = 0; o < 2; ++o) {
                                const uint32_t cols = ring_base + (st * 2 + o) * C::COLS_BYTES;
                                if (A_TMEM) mma_over_dims_tmem_a<C::HALVES>(xy + o * 64, tmem + C::A_AT + o * C::A_STEP, cols, COLS_HALF_BYTES, idesc_xy);
                                else mma_over_dims<C::HALVES>(xy + o * 64, a_base + o * C::ROWS_BYTES, ROWS_HALF_BYTES, cols, COLS_HALF_BYTES, idesc_xy);
                            }
                            tcgen05_commit(&bar.xy_full[cur & 1u]);
                            if (!A_TMEM && b == blocks - 1) tcgen05_commit(&bar.a_empty);
                        }
                        __syncwarp();
                    }
                    if (b > 0) {
                        const uint32_t cur = c + b - 1, st = cur % C::STAGES, xy = tmem + 256 + (cur & 1u) * 128;
                        if (b == 1 && !mbar_wait_warp(&bar.acc_empty, (with_blocks & 1u) ^ 1u, abort_flag)) { ok = false; break; }
                        if (!mbar_wait_warp(&bar.ps_full[cur & 1u], (cur >> 1) & 1u, abort_flag)) { ok = false; break; }
                        tcgen05_fence_after();
                        if (elect_one()) {
#pragma unroll
                            for (int o = KEYS ? 0 : 1; o < 2; ++o)       // accumulator 1: p b2; accumulator 2: ds b1
                                mma_over_rows<BWD_BLOCK, 0, BWD_BLOCK / UMMA_K>(tmem + o * 128, xy + o * 64, ring_base + (st * 2 + 1 - o) * C::COLS_BYTES, idesc_acc, b == 1);
                            tcgen05_commit(&bar.empty[st]);
                            if (b == blocks) tcgen05_commit(&bar.acc_full);
                        }
                        __syncwarp();
                    }
                }
                c += blocks;
                ++with_blocks;
            }
            if (ok && elect_one()) mbar_arrive(&bar.item_empty[slot]);
            __syncwarp();
        }
        if (!ok) {
            if (elect_one()) tcgen05_commit(&bar.drain);
            __syncwarp();
            for (uint32_t spin = 0; spin < SPIN_LIMIT; ++spin)
                if (mbar_try_wait(&bar.drain, 0u)) break;
        }
        __syncwarp();
    } else if (warp == 2) {
        // ---- scanner: in a block that some row does not have all of, what a masked 0 would meet in the second products must be finite.
        // A query row or its d_o that is not leaves statistics that are not (its lse is a sum over its scores, its delta a sum over d_o), so query rows
        // are looked over only where some statistics are not finite, or missing; keys always.
        uint32_t c = 0;
        bool ok = true;
        for (uint32_t n = 0; ok; ++n) {
            const uint32_t slot = n % BWD_SLOTS;
            if (!mbar_wait_warp(&bar.item_full[slot], (n / BWD_SLOTS) & 1u, abort_flag)) break;
            const BwdItem& it = sm.items[slot];
            if (!it.valid) break;
            const int blocks = it.n;
            for (int b = 0; b < blocks; ++b) {
                const uint32_t cur = c + b, st = cur % C::STAGES;
                if (!mbar_wait_warp(&bar.full[st], (cur / C::STAGES) & 1u, abort_flag)) { ok = false; break; }
                const bool masked = bwd_masked<KEYS>(it, b, TOKQ);
                if (KEYS && masked && (sm.bad_stats[st][0] | sm.bad_stats[st][1]) == 0u) {
                    if (lane < 2) sm.bad[st][lane] = 0u;
                } else if (masked) {
#pragma unroll 1
                    for (int r = 0; r < 2; ++r) {
                        bool bad = false;
#pragma unroll
                        for (int piece = 0; piece < (KEYS ? 2 : 1) * C::HALVES; ++piece) {
                            uint8_t* at = ring + st * 2 * C::COLS_BYTES + piece * COLS_HALF_BYTES + (r * 32 + lane) * 128;
                            if (row_not_finite(at, lane)) {
                                bad = true;
                                drop_not_finite(at);
                                fence_proxy_async_smem();
                            }
                        }
                        const uint32_t all = __ballot_sync(0xffffffffu, bad);
                        if (lane == 0) sm.bad[st][r] = all;
                    }
                }
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive(&bar.scanned[st]);
                    mbar_arrive(&bar.empty[st]);
                }
                __syncwarp();
            }
            c += blocks;
            if (lane == 0) mbar_arrive(&bar.item_empty[slot]);
            __syncwarp();
        }
    } else if (warp >= 4) {
        // ---- groups w = 0, 1: blocks in turn; thread = row
        const int w = (warp - 4) >> 2, quarter = warp & 3, row = quarter * 32 + lane;
        const uint32_t lanes = (uint32_t)(quarter * 32) << 16;
        const float scale2 = p.sh.scale_log2;
        const uint64_t scale_x2 = pack_f32x2(scale2, scale2);
        const float2* stats = pdl_acquire(p.stats);
        uint32_t c = 0, with_blocks = 0;
        bool ok = true;
        // Group w puts the rows of operand w into tensor memory, a row a thread.  All products of the item before are done by then.
        uint32_t prepared = 0;
        auto prepare = [&](uint32_t n) {
            if (!A_TMEM) return true;
            const uint32_t slot = n % BWD_SLOTS;
            if (!mbar_wait_warp(&bar.item_full[slot], (n / BWD_SLOTS) & 1u, abort_flag)) return false;
            if (!sm.items[slot].valid || sm.items[slot].n == 0) return true;
            if (!mbar_wait_warp(&bar.a_full, prepared++ & 1u, abort_flag)) return false;
#pragma unroll 1
            for (int h = 0; h < C::HALVES; ++h) {
                const uint8_t* at = rows_a + w * C::ROWS_BYTES + h * ROWS_HALF_BYTES + row * 128;
                uint32_t v[32];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const uint4 x = *reinterpret_cast<const uint4*>(at + ((j ^ (row & 7)) << 4));
                    v[4 * j] = x.x; v[4 * j + 1] = x.y; v[4 * j + 2] = x.z; v[4 * j + 3] = x.w;
                }
                __syncwarp();
                tcgen05_st_32x32(tmem + lanes + C::A_AT + w * C::A_STEP + h * 32, v);
            }
            tcgen05_st_wait();
            tcgen05_fence_before();
            __syncwarp();
            if (lane == 0) {
                mbar_arrive(&bar.a_ready);
                mbar_arrive(&bar.a_empty);
            }
            __syncwarp();
            return true;
        };
        ok = prepare(0);
        for (uint32_t n = 0; ok; ++n) {
            const uint32_t slot = n % BWD_SLOTS;
            if (!mbar_wait_warp(&bar.item_full[slot], (n / BWD_SLOTS) & 1u, abort_flag)) { ok = false; break; }
            const BwdItem& it = sm.items[slot];
            if (!it.valid) break;
            const int blocks = it.n, tok = KEYS ? row : row / ratio, head = it.g * ratio + (KEYS ? 0 : row - tok * ratio);
            const int j = it.row0 + tok;              // key row or token of this thread
            const bool live = tok < it.rows;
            int lo = 0, hi = 0, pre_lo = 0, pre_hi = 0;
            float2 mine = make_float2(0.f, 0.f);      // the row's statistics
            if (live) {
                if (KEYS) {
                    const int2 x = it.shared ? prompt_range[j] : make_int2(j, bounds[j].own_hi);
                    lo = x.x; hi = x.y;
                } else {
                    const TokenBounds x = bounds[j];
                    pre_lo = x.pre_lo; pre_hi = x.pre_hi; lo = x.own_lo; hi = j + 1;
                    mine = stats[(int64_t)j * p.sh.Hq + head];
                }
            }
            const uint64_t neg_lse = pack_f32x2(-mine.x, -mine.x), neg_delta = pack_f32x2(-mine.y, -mine.y);
            for (int b = 0; b < blocks; ++b) {
                const uint32_t cur = c + b;
                if ((cur & 1u) != (uint32_t)w) continue;
                const uint32_t st = cur % C::STAGES, xy = tmem + lanes + 256 + w * 128;
                const bool masked = bwd_masked<KEYS>(it, b, TOKQ);
                int first = 0, len = BWD_BLOCK;       // this row's columns
                if (masked) {
                    const int c0 = bwd_start<KEYS>(it, b, TOKQ);
                    if (KEYS) {
                        first = min(max(lo - c0, 0), TOKQ) * ratio;
                        len = min(max(hi - c0, 0), TOKQ) * ratio - first;
                    } else {
                        const bool pre = b < it.n_pre;
                        first = (pre ? pre_lo : lo) - c0;
                        len = (pre ? pre_hi - pre_lo : hi - lo);
                        if (first < 0) { len += first; first = 0; }
                        len = min(len, BWD_BLOCK - first);        // of this block: a whole block's number is what leaves the selection out below
                    }
                    if (!live || len < 0) len = 0;
                }
                if (!mbar_wait_warp(&bar.full[st], (cur / C::STAGES) & 1u, abort_flag) ||      // the columns' statistics
                    !mbar_wait_warp(&bar.xy_full[w], (cur >> 1) & 1u, abort_flag)) { ok = false; break; }
                tcgen05_fence_after();
                uint32_t on[2] = {0xffffffffu, 0xffffffffu}, bad[2] = {0u, 0u};
                bool select = false, none_of_it = false;
                if (masked) {
                    if (!mbar_wait_warp(&bar.scanned[st], (cur / C::STAGES) & 1u, abort_flag)) { ok = false; break; }
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        const int a = min(max(first - u * 32, 0), 32), z = min(max(first + len - u * 32, 0), 32);
                        on[u] = z > a ? (0xffffffffu >> (32 - z + a)) << a : 0u;
                        bad[u] = (sm.bad[st][u] | (KEYS ? sm.bad_stats[st][u] : 0u)) & on[u];
                    }
                    none_of_it = __all_sync(0xffffffffu, len == 0);
                    select = !__all_sync(0xffffffffu, len == (KEYS ? TOKQ * ratio : BWD_BLOCK) && (bad[0] | bad[1]) == 0u);
                }
                // half of the columns at a time: both operands of all 64 would not leave room for the results.  p and ds take the first halves of x's and
                // y's columns, which have been read by then.
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    uint32_t pk[16], dk[16];
                    if (none_of_it) {
#pragma unroll
                        for (int i = 0; i < 16; ++i) pk[i] = dk[i] = 0u;
                    } else {
                        uint32_t x[32], y[32];
                        __syncwarp();
                        tcgen05_ld_32x32_issue(xy + u * 32, x);
                        tcgen05_ld_32x32_issue(xy + 64 + u * 32, y);
                        tcgen05_ld_wait(x);
                        tcgen05_ld_wait(y);
                        if (select) {
#pragma unroll
                            for (int v = 0; v < 32; ++v) {
                                if (!(on[u] >> v & 1u)) { x[v] = 0xFF800000u; y[v] = 0u; }      // p = 0, ds = 0
                                if (bad[u] >> v & 1u) x[v] = 0x7FC00000u;                       // a row that has a column which was not finite
                            }
                        }
#pragma unroll
                        for (int i = 0; i < 16; i += 2) {
                            float4 l4, d4;
                            if (KEYS) {
                                l4 = *reinterpret_cast<const float4*>(&sm.lse[st][u * 32 + 2 * i]);
                                d4 = *reinterpret_cast<const float4*>(&sm.delta[st][u * 32 + 2 * i]);
                            }
#pragma unroll
                            for (int k = 0; k < 2; ++k) {
                                const int v = 2 * (i + k);
                                const uint64_t nl = KEYS ? (k ? pack_f32x2(l4.z, l4.w) : pack_f32x2(l4.x, l4.y)) : neg_lse;
                                const uint64_t nd = KEYS ? (k ? pack_f32x2(d4.z, d4.w) : pack_f32x2(d4.x, d4.y)) : neg_delta;
                                float p0, p1, s0, s1;
                                unpack_f32x2(fma_f32x2(pack_f32x2(__uint_as_float(x[v]), __uint_as_float(x[v + 1])), scale_x2, nl), p0, p1);
                                p0 = ex2_approx(p0);
                                p1 = ex2_approx(p1);
                                const uint64_t dp = add_f32x2(pack_f32x2(__uint_as_float(y[v]), __uint_as_float(y[v + 1])), nd);
                                unpack_f32x2(mul_f32x2(pack_f32x2(p0, p1), dp), s0, s1);
                                if (KEYS) pk[i + k] = pack_bf16(p0, p1);
                                dk[i + k] = pack_bf16(s0, s1);
                            }
                        }
                    }
                    __syncwarp();
                    if (KEYS) tcgen05_st_32x16(xy + u * 16, pk);
                    tcgen05_st_32x16(xy + 64 + u * 16, dk);
                }
                tcgen05_st_wait();
                tcgen05_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&bar.ps_full[w]);
                __syncwarp();
            }
            if (!ok) break;
            c += blocks;
            // KEYS: group 0 writes dv, group 1 dk; else each half of dq
            if (blocks > 0) {
                if (!mbar_wait_warp(&bar.acc_full, with_blocks & 1u, abort_flag)) { ok = false; break; }
                tcgen05_fence_after();
                ++with_blocks;
            }
            if (!prepare(n + 1)) { ok = false; break; }
            __nv_bfloat16* out;
            if (KEYS) {
                out = w == 0 ? (it.shared ? p.shared1 + j * p.shared1_stride : p.dv + j * p.dv_stride)
                             : (it.shared ? p.shared2 + j * p.shared2_stride : p.dk + j * p.dk_stride);
                out += (int64_t)it.g * p.sh.D;
            } else {
                out = p.dq + j * p.dq_stride + (int64_t)head * p.sh.D;
            }
            const float by = KEYS && w == 0 ? 1.f : p.sh.scale;
            const bool to_parts = KEYS && it.shared && p.splits > 1;
            const int64_t part_tile = ((int64_t)it.split * ((p.sh.prompt_rows + 127) / 128) + it.row0 / 128) * p.sh.Hkv + it.g;
            float* const sums = !to_parts ? nullptr : (w == 0 ? p.part1 : p.part2) + (part_tile * 128 + row) * DP;
            constexpr int PIECES = DP / 32;
#pragma unroll 1
            for (int piece = KEYS ? 0 : w * (PIECES / 2); piece < (KEYS ? PIECES : (w + 1) * (PIECES / 2)); ++piece) {
                uint32_t v[32];
                __syncwarp();
                if (blocks > 0) {
                    tcgen05_ld_32x32_issue(tmem + lanes + (KEYS && w == 0 ? 0 : 128) + piece * 32, v);
                    tcgen05_ld_wait(v);
                } else {
#pragma unroll
                    for (int i = 0; i < 32; ++i) v[i] = 0u;
                }
                if (to_parts) {
                    if (live) {
#pragma unroll
                        for (int i = 0; i < 32; i += 4) {
                            auto f = [&](int k) { return __uint_as_float(v[i + k]) * by; };
                            *reinterpret_cast<float4*>(sums + piece * 32 + i) = make_float4(f(0), f(1), f(2), f(3));
                        }
                    }
                } else if (live) {
#pragma unroll
                    for (int i = 0; i < 32; i += 8)
                        if (piece * 32 + i < p.sh.D) {
                            uint4 o4;
                            o4.x = pack_bf16(__uint_as_float(v[i]) * by, __uint_as_float(v[i + 1]) * by);
                            o4.y = pack_bf16(__uint_as_float(v[i + 2]) * by, __uint_as_float(v[i + 3]) * by);
                            o4.z = pack_bf16(__uint_as_float(v[i + 4]) * by, __uint_as_float(v[i + 5]) * by);
                            o4.w = pack_bf16(__uint_as_float(v[i + 6]) * by, __uint_as_float(v[i + 7]) * by);
                            *reinterpret_cast<uint4*>(out + piece * 32 + i) = o4;
                        }
                }
            }
            __syncwarp();
            tcgen05_fence_before();
            __syncwarp();
            if (lane == 0) {
                if (blocks > 0) mbar_arrive(&bar.acc_empty);
                mbar_arrive(&bar.item_empty[slot]);
            }
            __syncwarp();
        }
    }
}

template <int DP>
__global__ void __launch_bounds__(BWD_THREADS, 1) attention_backward_kernel(const __grid_constant__ BwdMaps maps, const BwdParams p) {
    using C = BwdConf<DP>;
    extern __shared__ uint8_t smem_raw[];
    __shared__ BwdShared sm;
    uint8_t* const smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    const int warp = uniform((int)threadIdx.x >> 5);
    if (threadIdx.x == 0) {
        init_barriers<DP, true>(sm.of[1]);
        init_barriers<DP, false>(sm.of[0]);
        sm.abort = 0u;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        for (const CUtensorMap* m : {&maps.k_rows, &maps.v_rows, &maps.q_cols, &maps.do_cols}) asm volatile("prefetch.tensormap [%0];" ::"l"(m) : "memory");
    }
    if (BWD_BLOCK / p.sh.ratio * p.sh.ratio < BWD_BLOCK) {       // rows behind the last whole token are never loaded: zeros, for the keys' second products
        for (uint32_t i = threadIdx.x * 16; i < C::STAGES * 2 * C::COLS_BYTES; i += BWD_THREADS * 16)
            *reinterpret_cast<uint4*>(smem + 2 * C::ROWS_BYTES + i) = make_uint4(0, 0, 0, 0);
        fence_proxy_async_smem();
    }
    if (warp == 1) {
        tcgen05_alloc(&sm.tmem, 512);
        tcgen05_relinquish();
    }
    tcgen05_fence_before();
    __syncthreads();
    tcgen05_fence_after();
    const uint32_t tmem = uniform(sm.tmem);                // accumulators 1 and 2 at columns 0 and 128; x, y of buffer i at 256 + 128 i and + 64
    pdl_launch_dependents();
    pdl_wait();
    // The queries' side needs nothing of the keys' side, so a block goes on to it as soon as it finds no more of the keys' items.
    backward_side<DP, true>(maps.k_rows, maps.v_rows, maps.q_cols, maps.do_cols, maps.pk_rows, maps.pv_rows, p, sm, smem, tmem);
    tcgen05_fence_before();
    __syncthreads();
    tcgen05_fence_after();
    if (!*static_cast<volatile uint32_t*>(&sm.abort))
        backward_side<DP, false>(maps.q_rows, maps.do_rows, maps.k_cols, maps.v_cols, maps.pk_cols, maps.pv_cols, p, sm, smem, tmem);
    tcgen05_fence_before();
    __syncthreads();
    if (threadIdx.x == 0 && *static_cast<volatile uint32_t*>(&sm.abort)) atomicOr(p.status, ARROL_DEV_WAIT_EXPIRED);
    if (warp == 1) {
        tcgen05_fence_after();
        tcgen05_dealloc(tmem, 512);
    }
}

// The parts of a prompt tile's sums, in order.
template <int DP>
__global__ void __launch_bounds__(256) attention_add_parts_kernel(const BwdParams p) {
    pdl_launch_dependents();
    pdl_wait();
    const int live = p.P > 0 ? clamp_row(pdl_acquire(p.cu_prompts)[p.P], 0, p.sh.prompt_rows) : 0;
    const int tiles = (p.sh.prompt_rows + 127) / 128;
    const int64_t pieces = (int64_t)live * p.sh.Hkv * (DP / 8), step = (int64_t)tiles * p.sh.Hkv * 128 * DP;
    for (int64_t x = blockIdx.x * (int64_t)256 + threadIdx.x; x < 2 * pieces; x += (int64_t)gridDim.x * 256) {
        const bool second = x >= pieces;
        const int64_t y = second ? x - pieces : x;
        const int d = (int)(y % (DP / 8)) * 8, g = (int)(y / (DP / 8) % p.sh.Hkv), j = (int)(y / (DP / 8) / p.sh.Hkv);
        if (d >= p.sh.D) continue;
        const float* at = pdl_acquire(second ? p.part2 : p.part1) + (((int64_t)(j / 128) * p.sh.Hkv + g) * 128 + j % 128) * DP + d;
        float4 a = {0.f, 0.f, 0.f, 0.f}, b = a;
        for (int s = 0; s < p.splits; ++s, at += step) {
            const float4 u = *reinterpret_cast<const float4*>(at), v = *reinterpret_cast<const float4*>(at + 4);
            a.x += u.x; a.y += u.y; a.z += u.z; a.w += u.w;
            b.x += v.x; b.y += v.y; b.z += v.z; b.w += v.w;
        }
        __nv_bfloat16* out = (second ? p.shared2 + j * p.shared2_stride : p.shared1 + j * p.shared1_stride) + (int64_t)g * p.sh.D + d;
        *reinterpret_cast<uint4*>(out) = make_uint4(pack_bf16(a.x, a.y), pack_bf16(a.z, a.w), pack_bf16(b.x, b.y), pack_bf16(b.z, b.w));
    }
}

template <int DP>
int launch_backward(arrol_ctx* ctx, const arrol_attention_args* a, const AttnWorkspace& w, cudaStream_t s) {
    using C = BwdConf<DP>;
    bool& set = ctx->attention_backward_smem_set[DP == 128];
    if (!set) {
        ARROL_CUDA_OK(cudaFuncSetAttribute(attention_backward_kernel<DP>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)C::SMEM));
        set = true;
    }
    const int ratio = a->Hq / a->Hkv;
    BwdParams p = {};
    p.sh = {a->d_num, w.bounds, w.prompt_range, (int)a->T_max, (int)a->prompt_rows, a->Hq, a->Hkv, a->D, ratio, a->scale, a->scale * LOG2E};
    p.stats = w.stats;
    p.cu_prompts = a->cu_prompts;
    p.P = a->P;
    p.status = ctx->d_status;
    BwdMaps m;
    struct { CUtensorMap* map; const void* base; int64_t rows, stride; int heads, group, tokens; } maps[] = {
        {&m.q_rows, a->q, a->T_max, a->q_stride, a->Hq, ratio, 128 / ratio},       {&m.do_rows, a->d_o, a->T_max, a->d_o_stride, a->Hq, ratio, 128 / ratio},
        {&m.q_cols, a->q, a->T_max, a->q_stride, a->Hq, ratio, BWD_BLOCK / ratio}, {&m.do_cols, a->d_o, a->T_max, a->d_o_stride, a->Hq, ratio, BWD_BLOCK / ratio},
        {&m.k_rows, a->k, a->T_max, a->k_stride, a->Hkv, 1, 128},                  {&m.v_rows, a->v, a->T_max, a->v_stride, a->Hkv, 1, 128},
        {&m.k_cols, a->k, a->T_max, a->k_stride, a->Hkv, 1, BWD_BLOCK},            {&m.v_cols, a->v, a->T_max, a->v_stride, a->Hkv, 1, BWD_BLOCK},
        {&m.pk_rows, a->prompt_k, a->prompt_rows, a->prompt_k_stride, a->Hkv, 1, 128},
        {&m.pv_rows, a->prompt_v, a->prompt_rows, a->prompt_v_stride, a->Hkv, 1, 128},
        {&m.pk_cols, a->prompt_k, a->prompt_rows, a->prompt_k_stride, a->Hkv, 1, BWD_BLOCK},
        {&m.pv_cols, a->prompt_v, a->prompt_rows, a->prompt_v_stride, a->Hkv, 1, BWD_BLOCK}};
    for (auto& x : maps) {
        if (x.rows == 0) continue;
        if (make_map_heads(ctx, x.map, x.base, x.rows, x.heads, a->D, x.stride, x.group, x.tokens) != ARROL_OK) return ARROL_ERR_CUDA;
    }
    // never read then
    if (a->prompt_rows == 0) { m.pk_rows = m.k_rows; m.pv_rows = m.v_rows; m.pk_cols = m.k_cols; m.pv_cols = m.v_cols; }
    if (a->T_max == 0) { m.q_rows = m.do_rows = m.q_cols = m.do_cols = m.k_rows = m.v_rows = m.k_cols = m.v_cols = m.pk_rows; }
    p.dv = static_cast<__nv_bfloat16*>(a->dv); p.dv_stride = a->dv_stride;
    p.dk = static_cast<__nv_bfloat16*>(a->dk); p.dk_stride = a->dk_stride;
    p.dq = static_cast<__nv_bfloat16*>(a->dq); p.dq_stride = a->dq_stride;
    p.shared1 = static_cast<__nv_bfloat16*>(a->dprompt_v); p.shared1_stride = a->dprompt_v_stride;
    p.shared2 = static_cast<__nv_bfloat16*>(a->dprompt_k); p.shared2_stride = a->dprompt_k_stride;
    p.counter[0] = w.counters + 2;
    p.counter[1] = w.counters + 1;
    p.splits = attn_prompt_splits(ctx->sm_count, a->T_max, a->prompt_rows, a->P, a->Hq, a->Hkv);
    p.part1 = w.parts;
    p.part2 = w.parts + (int64_t)p.splits * ((a->prompt_rows + 127) / 128) * a->Hkv * 128 * DP;
    const int64_t items = ((a->T_max + 127) / 128 + (a->prompt_rows + 127) / 128 * p.splits + (a->T_max + 128 / ratio - 1) / (128 / ratio)) * a->Hkv;
    const auto blocks = [&](int64_t n, int64_t most) { return dim3((unsigned)(n < most ? n : most)); };
    ARROL_CUDA_OK(arrol_launch_pdl(attention_backward_kernel<DP>, blocks(items, ctx->sm_count), dim3(BWD_THREADS), C::SMEM, s, m, p));
    ctx->launches += 1;
    if (p.splits > 1) {
        const int64_t pieces = 2 * a->prompt_rows * a->Hkv * (DP / 8);
        ARROL_CUDA_OK(arrol_launch_pdl(attention_add_parts_kernel<DP>, blocks((pieces + 255) / 256, 8 * ctx->sm_count), dim3(256), 0, s, p));
        ctx->launches += 1;
    }
    return ARROL_OK;
}

}  // namespace

extern "C" int arrol_attention_backward(arrol_ctx* ctx, const arrol_attention_args* a, void* stream) {
    if (!ctx || !a) return ARROL_ERR_INVALID_ARG;
    const int rc = arrol_internal_check_attention(a);
    if (rc != ARROL_OK) return rc;
    if (a->T_max == 0 && a->prompt_rows == 0) return ARROL_OK;
    if (a->T_max > 0 && (!attn_rows_ok(a->d_o, a->d_o_stride, a->Hq, a->D) || !attn_rows_ok(a->dq, a->dq_stride, a->Hq, a->D) ||
                         !attn_rows_ok(a->dk, a->dk_stride, a->Hkv, a->D) || !attn_rows_ok(a->dv, a->dv_stride, a->Hkv, a->D)))
        return ARROL_ERR_INVALID_ARG;
    if (a->prompt_rows > 0 && (!attn_rows_ok(a->dprompt_k, a->dprompt_k_stride, a->Hkv, a->D) ||
                               !attn_rows_ok(a->dprompt_v, a->dprompt_v_stride, a->Hkv, a->D)))
        return ARROL_ERR_INVALID_ARG;
    const AttnWorkspace w = attn_workspace(a->workspace, ctx->sm_count, a->T_max, a->prompt_rows, a->Hq, a->Hkv, a->D, true);
    if (a->workspace_bytes < w.bytes) return ARROL_ERR_WORKSPACE;
    ArrolDeviceGuard guard(ctx->device);
    if (!guard.ok) return ARROL_ERR_CUDA;
    cudaStream_t s = (cudaStream_t)stream;
    const int rb = arrol_internal_attention_bounds(ctx, a, w, true, s);
    if (rb != ARROL_OK) return rb;
    return a->D <= 64 ? launch_backward<64>(ctx, a, w, s) : launch_backward<128>(ctx, a, w, s);
}
