// arrol_attention_decode: one generated token per rollout over its group's prompt and its own cache.
//
// Bound by HBM: every live rollout's cache and every group's prompt is read once.  decode_plan_kernel cuts them into units of about equal
// numbers of tokens (a rollout's own chunk with its `ratio` query rows, or a chunk of a prompt with the rows of up to 64 / ratio live
// rollouts), decode_units_kernel works through (unit, key head) pairs, which leave partial sums with their maxima, and decode_merge_kernel adds
// these up in order, so the result does not depend on who did what.  The plan follows lengths and mask on the device.
// The products are 16 x 8 x 16 mma.sync: 64 rows at most meet a key, which is too few flops a byte for tensor memory to pay, and a unit's 4 to 16
// rows would leave seven eighths of a 128-row tile empty.
// Measured (calls from a graph): 256 live rollouts of 2,200 tokens, 16 heads of 128 on 8 (2.46 GB) 381 to 394 us, 6.2 to 6.5 TB/s, 0.96 to 0.99 of the
// measured copy rate; 8 rollouts of 6,600 tokens, 32 heads (236 MB) 61 us; 384 rollouts of 160 tokens over 24 prompts of 5,800, 32 heads of 64 121 to 124 us
// (0.52): there it is latency, with 64 rows' products behind every key and eight consuming warps an SM (the products' pipe is active 0.30 of the cycles, a
// scheduler issues 0.33 instructions a cycle, no pipe is full); 16 rollouts of 30 tokens 14 us, three launches one behind another.
// More than one tile of keys at once per warp (for its latencies) left too little of the ring for the copies: 121 -> 136 us.
#include "attention_common.cuh"

namespace {

constexpr int DEC_ROWS = 64;                       // query rows a unit
constexpr int DEC_WARPS = 4;                       // consumers; one more warp loads keys and values, one looks up what comes next
constexpr int DEC_THREADS = 32 * (DEC_WARPS + 2);
constexpr int DEC_STAGES = 4;
// A warp waits for every fourth stage at most: were the ring shorter, it could wait for a fill that is two ahead of the last one, whose parity is the
// same as that of the one before, and would not wait at all.
static_assert(DEC_STAGES >= DEC_WARPS, "parity waits");
constexpr int DEC_SLOTS = 4;                       // pairs looked up ahead
constexpr int DEC_STAGE_BYTES = 16384;             // keys and values of 32 tokens of 128 dimensions, of 64 tokens of 64
// Tokens of a chunk: as many as make DEC_FEW_PER_SM (unit, head) pairs an SM, between 128 and 512; more where that would make more than
// DEC_OWN_PER_SM pairs (DEC_SHARED_PER_SM of prompts, whose partial sums are many).  One rollout of 8,000 tokens with 2 / 4 / 8 pairs an SM 18.7 / 27.7 / 27.8 us;
// 8 of 6,600 with chunks of 128 / 256 / 512 76.8 / 75.6 / 67.2; prompts with 8 / 12 / 16 121 / 126 / 131.
constexpr int DEC_MIN_CHUNK = 128, DEC_GOOD_CHUNK = 512;
constexpr int DEC_FEW_PER_SM = 2, DEC_OWN_PER_SM = 32, DEC_SHARED_PER_SM = 8;
constexpr int PLAN_THREADS = 1024;
constexpr float RESCALE_AT = 8.0f;                 // the running maximum follows once it is 2^8 behind

struct alignas(16) DecodeUnit {
    int tok0, ntok;        // rows of the cache, or of the prompts
    int rows, src;         // query rows; number of the first of its rollouts among the live ones
    int slot, shared;      // record of each of its rollouts: own chunk `slot`, or chunk `slot` of the prompt behind the own ones
    int pad[2];
};
// A live rollout and its records: own chunks, then the prompt's.
struct alignas(16) LiveRollout {
    int rollout, base, own, count;
};

struct DecodeWorkspace {
    int* head;             // [0] work counter, [1] units
    DecodeUnit* units;
    LiveRollout* live;     // in order
    int* live_before;      // [N]: live rollouts before each
    int* prompt_chunks;    // [P]
    float* o;              // [records][Hq][D]
    float2* ml;            // [records][Hq]: maximum (of scores log2 e), sum
    int64_t max_units, max_records;
    size_t bytes;
};

inline int dec_group(int ratio) { return ratio > DEC_ROWS ? 1 : DEC_ROWS / ratio; }       // rollouts a prompt unit

DecodeWorkspace decode_workspace(void* base, int sm_count, int N, int P, int Hq, int Hkv, int D) {
    // With W tokens in all, chunks of at least W Hkv / target tokens: units <= one each + target / Hkv, and as many records per rollout.
    const int ratio = Hq / Hkv, group = dec_group(ratio);
    const int64_t own = (int64_t)sm_count * DEC_OWN_PER_SM / Hkv + 1, shared = (int64_t)sm_count * DEC_SHARED_PER_SM / Hkv + 1;
    DecodeWorkspace w = {};
    w.max_units = (int64_t)N + own + (P > 0 ? (int64_t)N + P + shared : 0);
    w.max_records = (int64_t)N + own + (P > 0 ? (int64_t)N + shared * group : 0);
    uint8_t* p = static_cast<uint8_t*>(base);
    size_t at = 0;
    auto take = [&](size_t n) { uint8_t* q = p + at; at += attn_round(n); return q; };
    w.head = reinterpret_cast<int*>(take(256));
    w.units = reinterpret_cast<DecodeUnit*>(take((size_t)w.max_units * sizeof(DecodeUnit)));
    w.live = reinterpret_cast<LiveRollout*>(take((size_t)N * sizeof(LiveRollout)));
    w.live_before = reinterpret_cast<int*>(take((size_t)N * sizeof(int)));
    w.prompt_chunks = reinterpret_cast<int*>(take((size_t)P * sizeof(int)));
    w.ml = reinterpret_cast<float2*>(take((size_t)w.max_records * Hq * sizeof(float2)));
    w.o = reinterpret_cast<float*>(take((size_t)w.max_records * Hq * D * sizeof(float)));
    w.bytes = at;
    return w;
}

struct DecodeParams {
    arrol_decode_args a;
    DecodeWorkspace w;
    int ratio, group;
    int few_units, own_target, shared_target;
    float scale_log2;
    uint32_t* status;
};

// A rollout's own rows, or a prompt's; nothing where they are not inside the buffer.
__device__ __forceinline__ int own_tokens(const arrol_decode_args& a, int i, bool& bad) {
    if (a.keep && !a.keep[i]) return -1;
    const int64_t off = a.src_tok_off[i], n = a.lengths[i];
    if (off < 0 || n < 0 || off > a.cache_rows || n > a.cache_rows - off) { bad = true; return 0; }
    return (int)n;
}
__device__ __forceinline__ int prompt_tokens(const arrol_decode_args& a, int p, bool& bad) {
    const int64_t x = a.cu_prompts[p], y = a.cu_prompts[p + 1];
    if (x < 0 || y < x || y > a.prompt_rows) { bad = true; return 0; }
    return (int)(y - x);
}

// Sums of (x, y) over the block's threads before this one, and all of them.  Fixed order; PLAN_THREADS threads.
__device__ __forceinline__ int2 block_scan(int2 v, int2& total, int2* warp_sums) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int2 s = v;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int x = __shfl_up_sync(0xffffffffu, s.x, d), y = __shfl_up_sync(0xffffffffu, s.y, d);
        if (lane >= d) { s.x += x; s.y += y; }
    }
    if (lane == 31) warp_sums[warp] = s;
    __syncthreads();
    int2 w = warp_sums[lane];
    int2 ws = w;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const int x = __shfl_up_sync(0xffffffffu, ws.x, d), y = __shfl_up_sync(0xffffffffu, ws.y, d);
        if (lane >= d) { ws.x += x; ws.y += y; }
    }
    total = make_int2(__shfl_sync(0xffffffffu, ws.x, 31), __shfl_sync(0xffffffffu, ws.y, 31));
    const int before_x = __shfl_sync(0xffffffffu, ws.x - w.x, warp), before_y = __shfl_sync(0xffffffffu, ws.y - w.y, warp);
    __syncthreads();
    return make_int2(before_x + s.x - v.x, before_y + s.y - v.y);
}
__device__ __forceinline__ long long block_sum(long long v, long long* warp_sums) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    if ((threadIdx.x & 31) == 0) warp_sums[threadIdx.x >> 5] = v;
    __syncthreads();
    v = warp_sums[threadIdx.x & 31];
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    __syncthreads();
    return v;
}
__device__ __forceinline__ int chunk_tokens(long long tokens, int few, int target) {
    long long c = (tokens + few - 1) / few;
    if (c > DEC_GOOD_CHUNK) c = DEC_GOOD_CHUNK;
    c = max(c, (tokens + target - 1) / target);
    return c <= DEC_MIN_CHUNK ? DEC_MIN_CHUNK : c >= 1 << 30 ? 1 << 30 : (int)((c + 63) / 64 * 64);
}

// One block: lengths of the chunks, the live rollouts, units and records.
__global__ void __launch_bounds__(PLAN_THREADS) decode_plan_kernel(const DecodeParams p) {
    __shared__ long long sums[32];
    __shared__ int2 warp_sums[32];
    pdl_launch_dependents();
    pdl_wait();
    const arrol_decode_args& a = p.a;
    const int tid = threadIdx.x;
    bool bad = false;
    // live rollouts before each, own tokens
    int live_before = 0;
    long long own_total = 0;
    for (int i0 = 0; i0 < a.N; i0 += PLAN_THREADS) {
        const int i = i0 + tid, n = i < a.N ? own_tokens(a, i, bad) : -1;
        int2 total;
        const int2 before = block_scan(make_int2(n >= 0, 0), total, warp_sums);
        if (n >= 0) own_total += n;
        if (i < a.N) p.w.live_before[i] = live_before + before.x;
        live_before += total.x;
    }
    const int own_chunk = chunk_tokens(block_sum(own_total, sums), p.few_units, p.own_target);     // its barriers publish the numbers above
    // prompt tokens, once per group of live rollouts that a unit takes
    auto live_of = [&](int q) { return (q + 1 < a.P ? p.w.live_before[(q + 1) * a.G] : live_before) - p.w.live_before[q * a.G]; };
    long long shared_total = 0;
    for (int q = tid; q < a.P; q += PLAN_THREADS) {
        const int live = live_of(q);
        if (live > 0) shared_total += (long long)prompt_tokens(a, q, bad) * ((live + p.group - 1) / p.group);
    }
    const int shared_chunk = chunk_tokens(block_sum(shared_total, sums), p.few_units, p.shared_target);
    // prompt units: a thread writes those of its prompt
    int units = 0;
    for (int q0 = 0; q0 < a.P; q0 += PLAN_THREADS) {
        const int q = q0 + tid, live = q < a.P ? live_of(q) : 0, n = live > 0 ? prompt_tokens(a, q, bad) : 0;
        const int chunks = (n + shared_chunk - 1) / shared_chunk, groups = (live + p.group - 1) / p.group;
        int2 total;
        const int2 before = block_scan(make_int2(chunks * groups, 0), total, warp_sums);
        if (q < a.P) p.w.prompt_chunks[q] = chunks;
        if (n > 0) {
            const int first = p.w.live_before[q * a.G], x = (int)a.cu_prompts[q];
            int64_t at = units + before.x;
            for (int c = 0; c < chunks; ++c)
                for (int g = 0; g < groups && at < p.w.max_units; ++g, ++at) {        // a chunk's groups side by side: they read the same rows
                    const DecodeUnit d = {x + c * shared_chunk, min(shared_chunk, n - c * shared_chunk), min(p.group, live - g * p.group) * p.ratio,
                                          first + g * p.group, c, 1, {0, 0}};
                    p.w.units[at] = d;
                }
        }
        units += total.x;
    }
    __syncthreads();
    // own units and records
    int records = 0;
    for (int i0 = 0; i0 < a.N; i0 += PLAN_THREADS) {
        const int i = i0 + tid, n = i < a.N ? own_tokens(a, i, bad) : -1;
        const int own = n > 0 ? (n + own_chunk - 1) / own_chunk : 0;
        const int count = n < 0 ? 0 : own + (a.P > 0 ? p.w.prompt_chunks[i / a.G] : 0);
        int2 total;
        const int2 before = block_scan(make_int2(own, count), total, warp_sums);
        if (n >= 0) {
            const int number = p.w.live_before[i];
            LiveRollout r = {i, records + before.y, own, count};
            if (r.base + (int64_t)count > p.w.max_records) { r = {i, 0, 0, 0}; bad = true; }     // only past 2^30 tokens a unit
            p.w.live[number] = r;
            int64_t at = units + before.x;
            const int off = n > 0 ? (int)a.src_tok_off[i] : 0;
            for (int c = 0; c < r.own && at < p.w.max_units; ++c, ++at) {
                const DecodeUnit d = {off + c * own_chunk, min(own_chunk, n - c * own_chunk), p.ratio, number, c, 0, {0, 0}};
                p.w.units[at] = d;
            }
        }
        units += total.x;
        records += total.y;
    }
    if (tid == 0) {
        p.w.head[0] = 0;
        p.w.head[1] = (int)min((int64_t)units, p.w.max_units);
    }
    if (bad) atomicOr(p.status, ARROL_DEV_BAD_INDEX);
}

__device__ __forceinline__ void mma_16x8x16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void ldmatrix_x4(uint32_t addr, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldmatrix_x4_trans(uint32_t addr, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void mbar_arrive_n(uint64_t* bar, uint32_t n) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0], %1;" ::"r"(smem_u32(bar)), "r"(n) : "memory");
}

template <int DP>
struct DecConf {
    static constexpr int HALVES = DP / 64;
    static constexpr int TOKENS = DP == 128 ? 32 : 64;            // a stage
    static constexpr int HALF_BYTES = TOKENS * 128;
    static constexpr int KEYS_BYTES = HALVES * HALF_BYTES;        // values behind them
    static constexpr int PITCH = DP + 4;                          // floats of a partial row
    static constexpr int PART_BYTES = DEC_WARPS * 16 * PITCH * 4;
    static constexpr size_t SMEM = 1024 + DEC_STAGES * (size_t)DEC_STAGE_BYTES + PART_BYTES;
    static_assert(2 * KEYS_BYTES == DEC_STAGE_BYTES, "a stage holds keys and values");
};

struct DecodeItem {
    int tok0, ntok, rows, shared, g, valid;
    int2 of[DEC_ROWS];                             // per rollout of the unit: its number, the record
};
struct DecodeShared {
    uint64_t full[DEC_STAGES], empty[DEC_STAGES], item_full[DEC_SLOTS], item_empty[DEC_SLOTS], part_full, part_free;
    DecodeItem items[DEC_SLOTS];
    float2 ml[DEC_WARPS][16];
    uint32_t abort;
};

template <int DP>
__global__ void __launch_bounds__(DEC_THREADS, 2)
decode_units_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, const __grid_constant__ CUtensorMap map_pk,
                    const __grid_constant__ CUtensorMap map_pv, const DecodeParams p) {
    using C = DecConf<DP>;
    extern __shared__ uint8_t smem_raw[];
    __shared__ DecodeShared sm;
    uint8_t* const ring = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    float* const part = reinterpret_cast<float*>(ring + DEC_STAGES * DEC_STAGE_BYTES);
    volatile uint32_t* abort_flag = &sm.abort;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const arrol_decode_args& a = p.a;
    if (threadIdx.x == 0) {
        for (int i = 0; i < DEC_STAGES; ++i) { mbar_init(&sm.full[i], 1); mbar_init(&sm.empty[i], DEC_WARPS); }
        for (int i = 0; i < DEC_SLOTS; ++i) { mbar_init(&sm.item_full[i], 1); mbar_init(&sm.item_empty[i], DEC_WARPS + 1); }
        mbar_init(&sm.part_full, DEC_WARPS);
        mbar_init(&sm.part_free, DEC_WARPS);
        sm.abort = 0u;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&map_k) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&map_v) : "memory");
    }
    __syncthreads();
    pdl_launch_dependents();
    pdl_wait();
    const int* head = pdl_acquire(p.w.head);
    const int64_t items = (int64_t)head[1] * a.Hkv;

    if (warp == DEC_WARPS + 1) {
        // ---- looks up what comes next: while a pair's rollouts are fetched, the next one's unit is, and a number for the one after it
        const DecodeUnit* units = pdl_acquire(p.w.units);
        const LiveRollout* live = pdl_acquire(p.w.live);
        auto number = [&] {
            uint32_t idx = 0;
            if (lane == 0) idx = atomicAdd(reinterpret_cast<unsigned int*>(p.w.head), 1u);
            return idx;
        };
        uint32_t idx = __shfl_sync(0xffffffffu, number(), 0);
        bool valid = (int64_t)idx < items;
        DecodeUnit u = {};
        if (valid) u = units[idx / (uint32_t)a.Hkv];           // the heads of a unit side by side: they read the same rows
        uint32_t after = number();
        for (uint32_t n = 0;; ++n) {
            const uint32_t next = __shfl_sync(0xffffffffu, after, 0);
            const bool next_valid = valid && (int64_t)next < items;
            DecodeUnit next_u = {};
            if (next_valid) {
                next_u = units[next / (uint32_t)a.Hkv];
                after = number();
            }
            const int rollouts = u.rows / p.ratio;
            LiveRollout r[DEC_ROWS / 32];
#pragma unroll
            for (int k = 0; k < DEC_ROWS / 32; ++k)
                if (valid && k * 32 + lane < rollouts) r[k] = live[u.src + k * 32 + lane];
            const uint32_t slot = n % DEC_SLOTS;
            if (!mbar_wait_warp(&sm.item_empty[slot], ((n / DEC_SLOTS) & 1u) ^ 1u, abort_flag)) break;
            DecodeItem& it = sm.items[slot];
#pragma unroll
            for (int k = 0; k < DEC_ROWS / 32; ++k)
                if (valid && k * 32 + lane < rollouts) it.of[k * 32 + lane] = make_int2(r[k].rollout, r[k].base + (u.shared ? r[k].own : 0) + u.slot);
            if (lane == 0) {
                it.tok0 = u.tok0; it.ntok = u.ntok; it.rows = u.rows; it.shared = u.shared;
                it.g = (int)(idx % (uint32_t)a.Hkv);
                it.valid = valid;
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(&sm.item_full[slot]);
            __syncwarp();
            if (!valid) break;
            idx = next; valid = next_valid; u = next_u;
        }
    } else if (warp == DEC_WARPS) {
        uint32_t pos = 0;
        bool ok = true;
        for (uint32_t n = 0; ok; ++n) {
            const uint32_t slot = n % DEC_SLOTS;
            if (!mbar_wait_warp(&sm.item_full[slot], (n / DEC_SLOTS) & 1u, abort_flag)) { ok = false; break; }
            const DecodeItem& it = sm.items[slot];
            if (!it.valid) break;
            const int ntok = uniform(it.ntok), tok0 = uniform(it.tok0), g = uniform(it.g);
            const CUtensorMap* mk = it.shared ? &map_pk : &map_k;
            const CUtensorMap* mv = it.shared ? &map_pv : &map_v;
            for (int t = 0; t < ntok; t += C::TOKENS, ++pos) {
                const uint32_t st = pos % DEC_STAGES;
                if (!mbar_wait_warp(&sm.empty[st], ((pos / DEC_STAGES) & 1u) ^ 1u, abort_flag)) { ok = false; break; }
                if (elect_one()) {
                    mbar_expect_tx(&sm.full[st], DEC_STAGE_BYTES);
                    uint8_t* at = ring + st * DEC_STAGE_BYTES;
#pragma unroll
                    for (int h = 0; h < C::HALVES; ++h) {
                        tma_load_3d(at + h * C::HALF_BYTES, mk, h * 64, g, tok0 + t, &sm.full[st]);
                        tma_load_3d(at + C::KEYS_BYTES + h * C::HALF_BYTES, mv, h * 64, g, tok0 + t, &sm.full[st]);
                    }
                }
                __syncwarp();
            }
            if (ok && lane == 0) mbar_arrive(&sm.item_empty[slot]);
            __syncwarp();
        }
        if (!ok) {                           // let the copies in flight land before the block's shared memory goes away
            for (uint32_t i = 1; i <= DEC_STAGES && i <= pos; ++i)
                for (uint32_t spin = 0; spin < SPIN_LIMIT; ++spin)
                    if (mbar_try_wait(&sm.full[(pos - i) % DEC_STAGES], ((pos - i) / DEC_STAGES) & 1u)) break;
        }
        __syncwarp();
    } else {
        // ---- consumers.  A unit's rows are 1, 2 or 4 tiles of 16; the warps that are left share its tokens.
        // The next pair's queries are on their way while this one's sums are added up.
        const uint32_t ratio_inv = (65536u + p.ratio - 1) / p.ratio;          // row / ratio = row * ratio_inv >> 16 for rows below 64
        uint32_t pos0 = 0, merged = 0;
        uint32_t q[DP / 16][4];              // query rows (lane / 4) and (lane / 4) + 8 of the tile as fragments
        auto begin = [&](uint32_t n) {
            const uint32_t slot = n % DEC_SLOTS;
            if (!mbar_wait_warp(&sm.item_full[slot], (n / DEC_SLOTS) & 1u, abort_flag)) return false;
            const DecodeItem& it = sm.items[slot];
            if (!it.valid) return false;
            const int row_tiles = it.rows <= 16 ? 1 : it.rows <= 32 ? 2 : 4;
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const int row = (warp & (row_tiles - 1)) * 16 + (lane >> 2) + r * 8, l = (int)(row * ratio_inv >> 16);
                const bool there = row < it.rows;
                const int i = there ? it.of[l].x : 0;
                const __nv_bfloat16* at = static_cast<const __nv_bfloat16*>(a.q) + i * a.q_stride +
                                          (int64_t)(it.g * p.ratio + row - l * p.ratio) * a.D + (lane & 3) * 2;
#pragma unroll
                for (int k = 0; k < DP / 16; ++k)
#pragma unroll
                    for (int c = 0; c < 2; ++c)
                        q[k][c * 2 + r] = there && k * 16 + c * 8 < a.D ? *reinterpret_cast<const uint32_t*>(at + k * 16 + c * 8) : 0u;
            }
            return true;
        };
        bool more = begin(0);
        for (uint32_t n = 0; more; ++n) {
            const uint32_t slot = n % DEC_SLOTS;
            const DecodeItem& it = sm.items[slot];
            const int rows = it.rows, ntok = it.ntok, head0 = it.g * p.ratio;
            const int row_tiles = rows <= 16 ? 1 : rows <= 32 ? 2 : 4, parts = DEC_WARPS / row_tiles;
            const int tile = warp & (row_tiles - 1), share = warp / row_tiles;
            const int tiles = (ntok + C::TOKENS - 1) / C::TOKENS;
            float o[DP / 8][4], m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
#pragma unroll
            for (int d = 0; d < DP / 8; ++d) o[d][0] = o[d][1] = o[d][2] = o[d][3] = 0.f;
            bool ok = true;
            for (int t = share; t < tiles; t += parts) {
                const uint32_t pos = pos0 + t, st = pos % DEC_STAGES;
                if (!mbar_wait_warp(&sm.full[st], (pos / DEC_STAGES) & 1u, abort_flag)) { ok = false; break; }
                uint8_t* const stage = ring + st * DEC_STAGE_BYTES;
                const uint32_t keys = smem_u32(stage), values = keys + C::KEYS_BYTES;
                const int there = ntok - t * C::TOKENS;      // tokens of the unit from here on
                float s[C::TOKENS / 8][4];
                // dimensions outermost: a warp issues in order, and one score's products would each wait for the one before
                constexpr int AT_ONCE = 4;
#pragma unroll
                for (int j = 0; j < C::TOKENS / 8; ++j) s[j][0] = s[j][1] = s[j][2] = s[j][3] = 0.f;
#pragma unroll
                for (int k = 0; k < DP / 32; ++k)
#pragma unroll
                    for (int j0 = 0; j0 < C::TOKENS / 8; j0 += AT_ONCE) {
                        uint32_t b[AT_ONCE][4];
                        const int c = k * 4 + (lane >> 3);
#pragma unroll
                        for (int j = 0; j < AT_ONCE; ++j) {
                            const int row = (j0 + j) * 8 + (lane & 7);
                            ldmatrix_x4(keys + (c >> 3) * C::HALF_BYTES + row * 128 + (((c & 7) ^ (row & 7)) << 4), b[j]);
                        }
#pragma unroll
                        for (int j = 0; j < AT_ONCE; ++j) mma_16x8x16(s[j0 + j], q[2 * k], b[j][0], b[j][1]);
#pragma unroll
                        for (int j = 0; j < AT_ONCE; ++j) mma_16x8x16(s[j0 + j], q[2 * k + 1], b[j][2], b[j][3]);
                    }
                if (there < C::TOKENS) {
                    // tokens behind the unit: no weight, and nothing that 0 times it would not make 0
#pragma unroll
                    for (int j = 0; j < C::TOKENS / 8; ++j)
#pragma unroll
                        for (int c = 0; c < 4; ++c)
                            if (j * 8 + (lane & 3) * 2 + (c & 1) >= there) s[j][c] = -INFINITY;
                    for (int x = there * 8 + lane; x < C::TOKENS * 8; x += 32)
#pragma unroll
                        for (int h = 0; h < C::HALVES; ++h)
                            *reinterpret_cast<uint4*>(stage + C::KEYS_BYTES + h * C::HALF_BYTES + x * 16) = make_uint4(0, 0, 0, 0);
                    __syncwarp();
                }
                // The reference is let fall up to 2^8 behind the maximum, which changes nothing (sums and products carry the same factor): only where
                // some row is further behind do its four lanes settle on a new one.
                float mx[2];
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    mx[r] = fmaxf(s[0][2 * r], s[0][2 * r + 1]);
#pragma unroll
                    for (int j = 1; j < C::TOKENS / 8; ++j) mx[r] = fmaxf(mx[r], fmaxf(s[j][2 * r], s[j][2 * r + 1]));
                    mx[r] *= p.scale_log2;
                }
                if (__any_sync(0xffffffffu, mx[0] > m[0] + RESCALE_AT || mx[1] > m[1] + RESCALE_AT)) {
                    float up[2];
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        mx[r] = fmaxf(mx[r], __shfl_xor_sync(0xffffffffu, mx[r], 1));
                        mx[r] = fmaxf(mx[r], __shfl_xor_sync(0xffffffffu, mx[r], 2));
                        const float top = fmaxf(m[r], mx[r]);
                        up[r] = top == -INFINITY ? 1.f : ex2_approx(m[r] - top);
                        m[r] = top;
                        l[r] *= up[r];
                    }
#pragma unroll
                    for (int d = 0; d < DP / 8; ++d) { o[d][0] *= up[0]; o[d][1] *= up[0]; o[d][2] *= up[1]; o[d][3] *= up[1]; }
                }
                const float sub[2] = {m[0] == -INFINITY ? 0.f : m[0], m[1] == -INFINITY ? 0.f : m[1]};
#pragma unroll
                for (int j = 0; j < C::TOKENS / 8; ++j)
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        s[j][c] = ex2_approx(fmaf(s[j][c], p.scale_log2, -sub[c >> 1]));
                        l[c >> 1] += s[j][c];
                    }
#pragma unroll
                for (int k = 0; k < C::TOKENS / 16; ++k) {
                    const uint32_t w[4] = {pack_bf16(s[2 * k][0], s[2 * k][1]), pack_bf16(s[2 * k][2], s[2 * k][3]),
                                           pack_bf16(s[2 * k + 1][0], s[2 * k + 1][1]), pack_bf16(s[2 * k + 1][2], s[2 * k + 1][3])};
                    const int row = k * 16 + (lane & 15);
#pragma unroll
                    for (int d0 = 0; d0 < DP / 16; d0 += AT_ONCE) {
                        uint32_t b[AT_ONCE][4];
#pragma unroll
                        for (int d = 0; d < AT_ONCE; ++d) {
                            const int c = (d0 + d) * 2 + (lane >> 4);
                            ldmatrix_x4_trans(values + (c >> 3) * C::HALF_BYTES + row * 128 + (((c & 7) ^ (row & 7)) << 4), b[d]);
                        }
#pragma unroll
                        for (int d = 0; d < AT_ONCE; ++d) {
                            mma_16x8x16(o[2 * (d0 + d)], w, b[d][0], b[d][1]);
                            mma_16x8x16(o[2 * (d0 + d) + 1], w, b[d][2], b[d][3]);
                        }
                    }
                }
                // The next copy into the stage is the async proxy's: the arrival alone does not keep it behind this warp's reads (and zeros).  Without the
                // fence the last values were now and then those of the copy that followed.
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive_n(&sm.empty[st], (uint32_t)parts);     // row_tiles warps read it: DEC_WARPS in all
                __syncwarp();
            }
            if (!ok) break;
            pos0 += tiles;
            // the shares of a row tile add up in shared memory, in order
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                l[r] += __shfl_xor_sync(0xffffffffu, l[r], 1);
                l[r] += __shfl_xor_sync(0xffffffffu, l[r], 2);
            }
            int2 of[2];                      // head and record of this lane's two rows, before the slot is left
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const int row = tile * 16 + (lane >> 2) + r * 8, lr = (int)(row * ratio_inv >> 16);
                of[r] = make_int2(head0 + row - lr * p.ratio, row < rows ? it.of[lr].y : -1);
            }
            if (parts > 1) {
                if (!mbar_wait_warp(&sm.part_free, (merged & 1u) ^ 1u, abort_flag)) break;
                float* const mine = part + warp * 16 * C::PITCH;
#pragma unroll
                for (int d = 0; d < DP / 8; ++d) {
                    *reinterpret_cast<float2*>(mine + (lane >> 2) * C::PITCH + d * 8 + (lane & 3) * 2) = make_float2(o[d][0], o[d][1]);
                    *reinterpret_cast<float2*>(mine + ((lane >> 2) + 8) * C::PITCH + d * 8 + (lane & 3) * 2) = make_float2(o[d][2], o[d][3]);
                }
                if ((lane & 3) == 0) {
                    sm.ml[warp][lane >> 2] = make_float2(m[0], l[0]);
                    sm.ml[warp][(lane >> 2) + 8] = make_float2(m[1], l[1]);
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(&sm.part_full);
                __syncwarp();
                more = begin(n + 1);
                if (!mbar_wait_warp(&sm.part_full, merged++ & 1u, abort_flag)) break;
                for (int x = warp * 32 + lane; x < rows * (DP / 4); x += 32 * DEC_WARPS) {
                    const int row = x / (DP / 4), d = x % (DP / 4) * 4, t = row >> 4, r = row & 15;
                    if (d >= a.D) continue;
                    float2 ml[DEC_WARPS];
                    float top = -INFINITY;
#pragma unroll
                    for (int s = 0; s < DEC_WARPS; ++s) {
                        ml[s] = s < parts ? sm.ml[s * row_tiles + t][r] : make_float2(-INFINITY, 0.f);
                        top = fmaxf(top, ml[s].x);
                    }
                    float4 sum = {0.f, 0.f, 0.f, 0.f};
                    float total = 0.f;
#pragma unroll
                    for (int s = 0; s < DEC_WARPS; ++s)
                        if (s < parts) {
                            // a NaN without a maximum stays one
                            const float by = ml[s].x == -INFINITY ? (ml[s].y == 0.f ? 0.f : 1.f) : ex2_approx(ml[s].x - top);
                            const float4 v = *reinterpret_cast<const float4*>(part + ((s * row_tiles + t) * 16 + r) * C::PITCH + d);
                            sum.x += by * v.x; sum.y += by * v.y; sum.z += by * v.z; sum.w += by * v.w;
                            total += by * ml[s].y;
                        }
                    const int lr = (int)(row * ratio_inv >> 16);
                    const int64_t at = (int64_t)it.of[lr].y * a.Hq + head0 + row - lr * p.ratio;
                    if (at >= p.w.max_records * a.Hq) continue;
                    *reinterpret_cast<float4*>(p.w.o + at * a.D + d) = sum;
                    if (d == 0) p.w.ml[at] = make_float2(top, total);
                }
                __syncwarp();
                if (lane == 0) {
                    mbar_arrive(&sm.part_free);
                    mbar_arrive(&sm.item_empty[slot]);
                }
                __syncwarp();
            } else {                         // every warp has its rows to itself
                if (lane == 0) mbar_arrive(&sm.item_empty[slot]);
                __syncwarp();
                more = begin(n + 1);
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    const int64_t at = (int64_t)of[r].y * a.Hq + of[r].x;
                    if (of[r].y < 0 || at >= p.w.max_records * a.Hq) continue;
                    float* out = p.w.o + at * a.D + (lane & 3) * 2;
#pragma unroll
                    for (int d = 0; d < DP / 8; ++d)
                        if (d * 8 < a.D) *reinterpret_cast<float2*>(out + d * 8) = make_float2(o[d][2 * r], o[d][2 * r + 1]);
                    if ((lane & 3) == 0) p.w.ml[at] = make_float2(m[r], l[r]);
                }
                __syncwarp();
            }
        }
    }
    __syncthreads();
    if (threadIdx.x == 0 && *abort_flag) atomicOr(p.status, ARROL_DEV_WAIT_EXPIRED);
}

// A warp per (rollout, query head): its records in order, four dimensions a lane.
__global__ void __launch_bounds__(256) decode_merge_kernel(const DecodeParams p) {
    pdl_launch_dependents();
    pdl_wait();
    const arrol_decode_args& a = p.a;
    const int lane = threadIdx.x & 31;
    const int64_t row = blockIdx.x * (int64_t)8 + (threadIdx.x >> 5);
    if (row >= (int64_t)a.N * a.Hq) return;
    const int i = (int)(row / a.Hq), h = (int)(row - (int64_t)i * a.Hq);
    if (a.keep && !a.keep[i]) return;
    const LiveRollout rec = pdl_acquire(p.w.live)[pdl_acquire(p.w.live_before)[i]];
    const float2* ml = pdl_acquire(p.w.ml) + (int64_t)rec.base * a.Hq + h;
    const float* o = pdl_acquire(p.w.o) + ((int64_t)rec.base * a.Hq + h) * a.D;
    // eight records a round trip, each with its maximum; the sums follow the running one
    constexpr int AT_ONCE = 8;
    float top = -INFINITY, total = 0.f;
    float4 sum = {0.f, 0.f, 0.f, 0.f};
    const int d = lane * 4;
    for (int r0 = 0; r0 < rec.count; r0 += AT_ONCE) {
        float2 x[AT_ONCE];
        float4 v[AT_ONCE];
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) {
            x[k] = make_float2(-INFINITY, 0.f);
            v[k] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (r0 + k < rec.count) {
                x[k] = ml[(int64_t)(r0 + k) * a.Hq];
                if (d < a.D) v[k] = *reinterpret_cast<const float4*>(o + (int64_t)(r0 + k) * a.Hq * a.D + d);
            }
        }
        float next = top;
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) next = fmaxf(next, x[k].x);
        const float up = next == -INFINITY ? 1.f : ex2_approx(top - next);
        total *= up;
        sum.x *= up; sum.y *= up; sum.z *= up; sum.w *= up;
        top = next;
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) {
            const float by = x[k].x == -INFINITY ? (x[k].y == 0.f ? 0.f : 1.f) : ex2_approx(x[k].x - top);
            total += by * x[k].y;
            sum.x += by * v[k].x; sum.y += by * v[k].y; sum.z += by * v[k].z; sum.w += by * v[k].w;
        }
    }
    const bool none = rec.count == 0;        // no key; a sum of nothing over keys that are there (scores of minus infinity) gives NaN, as the formula does
    const float inv = none ? 0.f : 1.f / total;
    if (d < a.D)
        *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(a.o) + i * a.o_stride + (int64_t)h * a.D + d) =
            none ? make_uint2(0u, 0u) : make_uint2(pack_bf16(sum.x * inv, sum.y * inv), pack_bf16(sum.z * inv, sum.w * inv));
    if (lane == 0 && a.lse) a.lse[row] = none ? -INFINITY : (top + log2f(total)) * LN2;
}

template <int DP>
int launch_decode(arrol_ctx* ctx, const DecodeParams& p, cudaStream_t s) {
    using C = DecConf<DP>;
    const arrol_decode_args& a = p.a;
    bool& set = ctx->attention_decode_smem_set[DP == 128];
    if (!set) {
        ARROL_CUDA_OK(cudaFuncSetAttribute(decode_units_kernel<DP>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)C::SMEM));
        set = true;
    }
    CUtensorMap k = {}, v = {}, pk = {}, pv = {};
    if (a.cache_rows > 0 && (make_map_heads(ctx, &k, a.k, a.cache_rows, a.Hkv, a.D, a.k_stride, 1, C::TOKENS) != ARROL_OK ||
                             make_map_heads(ctx, &v, a.v, a.cache_rows, a.Hkv, a.D, a.v_stride, 1, C::TOKENS) != ARROL_OK))
        return ARROL_ERR_CUDA;
    if (a.prompt_rows > 0 && (make_map_heads(ctx, &pk, a.prompt_k, a.prompt_rows, a.Hkv, a.D, a.prompt_k_stride, 1, C::TOKENS) != ARROL_OK ||
                              make_map_heads(ctx, &pv, a.prompt_v, a.prompt_rows, a.Hkv, a.D, a.prompt_v_stride, 1, C::TOKENS) != ARROL_OK))
        return ARROL_ERR_CUDA;
    if (a.cache_rows == 0) { k = pk; v = pv; }            // never read then
    if (a.prompt_rows == 0) { pk = k; pv = v; }
    ARROL_CUDA_OK(arrol_launch_pdl(decode_plan_kernel, dim3(1), dim3(PLAN_THREADS), 0, s, p));
    if (a.cache_rows > 0 || a.prompt_rows > 0) {
        const int64_t most = p.w.max_units * a.Hkv;
        const unsigned grid = (unsigned)(most < 2 * ctx->sm_count ? most : 2 * ctx->sm_count);
        ARROL_CUDA_OK(arrol_launch_pdl(decode_units_kernel<DP>, dim3(grid), dim3(DEC_THREADS), C::SMEM, s, k, v, pk, pv, p));
        ctx->launches += 1;
    }
    ARROL_CUDA_OK(arrol_launch_pdl(decode_merge_kernel, dim3((unsigned)(((int64_t)a.N * a.Hq + 7) / 8)), dim3(256), 0, s, p));
    ctx->launches += 2;
    return ARROL_OK;
}

}  // namespace

extern "C" size_t arrol_attention_decode_workspace(arrol_ctx* ctx, int32_t N, int32_t P, int32_t Hq, int32_t Hkv, int32_t D) {
    if (!ctx || N < 0 || P < 0 || !attn_heads_ok(Hq, Hkv, D)) return 0;
    return decode_workspace(nullptr, ctx->sm_count, N, P, Hq, Hkv, D).bytes;
}

extern "C" int arrol_attention_decode(arrol_ctx* ctx, const arrol_decode_args* a, void* stream) {
    if (!ctx || !a) return ARROL_ERR_INVALID_ARG;
    if (a->N < 0 || a->P < 0 || a->G < 1 || a->cache_rows < 0 || a->prompt_rows < 0) return ARROL_ERR_INVALID_ARG;
    if (a->Hq < 1 || a->Hkv < 1 || a->D < 1 || a->Hq % a->Hkv) return ARROL_ERR_INVALID_ARG;
    if (!(a->scale > 0.f) || !isfinite(a->scale)) return ARROL_ERR_INVALID_ARG;
    if (!attn_heads_ok(a->Hq, a->Hkv, a->D) || a->cache_rows >= ATTN_MAX_ROWS || a->prompt_rows >= ATTN_MAX_ROWS) return ARROL_ERR_UNSUPPORTED;
    if (a->G > 1024 || a->N > (1 << 24)) return ARROL_ERR_UNSUPPORTED;
    if (a->P > 0 ? (int64_t)a->P * a->G != a->N || !a->cu_prompts : a->prompt_rows > 0) return ARROL_ERR_INVALID_ARG;
    if (a->N == 0) return ARROL_OK;
    if (!attn_rows_ok(a->q, a->q_stride, a->Hq, a->D) || !attn_rows_ok(a->o, a->o_stride, a->Hq, a->D)) return ARROL_ERR_INVALID_ARG;
    if (!a->src_tok_off || !a->lengths) return ARROL_ERR_INVALID_ARG;
    if (a->cache_rows > 0 && (!attn_rows_ok(a->k, a->k_stride, a->Hkv, a->D) || !attn_rows_ok(a->v, a->v_stride, a->Hkv, a->D))) return ARROL_ERR_INVALID_ARG;
    if (a->prompt_rows > 0 && (!attn_rows_ok(a->prompt_k, a->prompt_k_stride, a->Hkv, a->D) || !attn_rows_ok(a->prompt_v, a->prompt_v_stride, a->Hkv, a->D)))
        return ARROL_ERR_INVALID_ARG;
    if (!a->workspace || !arrol_aligned(a->workspace, 256)) return ARROL_ERR_WORKSPACE;
    DecodeParams p = {};
    p.a = *a;
    p.w = decode_workspace(a->workspace, ctx->sm_count, a->N, a->P, a->Hq, a->Hkv, a->D);
    if (a->workspace_bytes < p.w.bytes) return ARROL_ERR_WORKSPACE;
    p.ratio = a->Hq / a->Hkv;
    p.group = dec_group(p.ratio);
    p.few_units = ctx->sm_count * DEC_FEW_PER_SM / a->Hkv + 1;
    p.own_target = ctx->sm_count * DEC_OWN_PER_SM / a->Hkv + 1;
    p.shared_target = ctx->sm_count * DEC_SHARED_PER_SM / a->Hkv + 1;
    p.scale_log2 = a->scale * LOG2E;
    p.status = ctx->d_status;
    ArrolDeviceGuard guard(ctx->device);
    if (!guard.ok) return ARROL_ERR_CUDA;
    return a->D <= 64 ? launch_decode<64>(ctx, p, (cudaStream_t)stream) : launch_decode<128>(ctx, p, (cudaStream_t)stream);
}
