// arrol_attention_decode: one generated token per rollout over its group's prompt and its own cache.
//
// Bound by HBM: every live rollout's cache and every group's prompt is read once.  decode_plan_kernel cuts them into units of about equal
// numbers of tokens (a rollout's own chunk with its `ratio` query rows, or a chunk of a prompt with the rows of up to 64 / ratio live
// rollouts), decode_units_kernel works through (unit, key head) pairs, which leave partial sums with their maxima, and decode_merge_kernel adds
// these up in order, so the result does not depend on who did what.  The plan follows lengths and mask on the device.
// The products are 16 x 8 x 16 mma.sync: 64 rows at most meet a key, which is too few flops a byte for tensor memory to pay, and a unit's 4 to 16
// rows would leave seven eighths of a 128-row tile empty.
#include "attention_common.cuh"

namespace {

constexpr int DEC_ROWS = 64;                       // query rows a unit
constexpr int DEC_WARPS = 4;                       // consumers; one more warp loads
constexpr int DEC_THREADS = 32 * (DEC_WARPS + 1);
constexpr int DEC_STAGES = 4;
constexpr int DEC_SLOTS = 2;
constexpr int DEC_STAGE_BYTES = 16384;             // keys and values of 32 tokens of 128 dimensions, of 64 tokens of 64
constexpr int DEC_MIN_CHUNK = 128;                 // tokens
constexpr int DEC_OWN_PER_SM = 32, DEC_SHARED_PER_SM = 8;   // (unit, head) pairs that the chunks' lengths aim at; partial sums of prompt units are many
constexpr int PLAN_THREADS = 1024;

struct alignas(16) DecodeUnit {
    int tok0, ntok;        // rows of the cache, or of the prompts
    int rows, src;         // query rows; the rollout, or the first live rollout's number among the live ones
    int slot, shared;      // record of each of its rollouts: own chunk `slot`, or chunk `slot` of the prompt behind the own ones
    int pad[2];
};
// A rollout's records: own chunks, then the prompt's.
struct alignas(16) RolloutRecords {
    int base, own, count, pad;
};

struct DecodeWorkspace {
    int* head;             // [0] work counter, [1] units
    DecodeUnit* units;
    RolloutRecords* records;
    int* live;             // live rollouts in order
    int* scan;             // [N][2], of the plan: own units before, live before
    int2* scan_prompt;     // [P]: units before
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
    w.records = reinterpret_cast<RolloutRecords*>(take((size_t)N * sizeof(RolloutRecords)));
    w.live = reinterpret_cast<int*>(take((size_t)N * sizeof(int)));
    w.scan = reinterpret_cast<int*>(take((size_t)N * 2 * sizeof(int)));
    w.scan_prompt = reinterpret_cast<int2*>(take((size_t)P * sizeof(int2)));
    w.ml = reinterpret_cast<float2*>(take((size_t)w.max_records * Hq * sizeof(float2)));
    w.o = reinterpret_cast<float*>(take((size_t)w.max_records * Hq * D * sizeof(float)));
    w.bytes = at;
    return w;
}

struct DecodeParams {
    arrol_decode_args a;
    DecodeWorkspace w;
    int ratio, group;
    int own_target, shared_target;      // units
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
__device__ __forceinline__ int chunk_tokens(long long tokens, int target) {
    const long long c = (tokens + target - 1) / target;
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
        if (n >= 0) {
            own_total += n;
            p.w.live[live_before + before.x] = i;
        }
        if (i < a.N) p.w.scan[2 * i + 1] = live_before + before.x;
        live_before += total.x;
    }
    const int own_chunk = chunk_tokens(block_sum(own_total, sums), p.own_target);     // its barriers publish the numbers above
    // prompt tokens, once per group of live rollouts that a unit takes
    auto live_of = [&](int q) { return (q + 1 < a.P ? p.w.scan[2 * (q + 1) * a.G + 1] : live_before) - p.w.scan[2 * q * a.G + 1]; };
    long long shared_total = 0;
    for (int q = tid; q < a.P; q += PLAN_THREADS) {
        const int live = live_of(q);
        if (live > 0) shared_total += (long long)prompt_tokens(a, q, bad) * ((live + p.group - 1) / p.group);
    }
    const int shared_chunk = chunk_tokens(block_sum(shared_total, sums), p.shared_target);
    // prompt units
    int units = 0;
    for (int q0 = 0; q0 < a.P; q0 += PLAN_THREADS) {
        const int q = q0 + tid, live = q < a.P ? live_of(q) : 0;
        const int chunks = live > 0 ? (prompt_tokens(a, q, bad) + shared_chunk - 1) / shared_chunk : 0;
        int2 total;
        const int2 before = block_scan(make_int2(chunks * ((live + p.group - 1) / p.group), 0), total, warp_sums);
        if (q < a.P) p.w.scan_prompt[q] = make_int2(units + before.x, chunks);
        units += total.x;
    }
    __syncthreads();
    // own units and records
    int records = 0;
    for (int i0 = 0; i0 < a.N; i0 += PLAN_THREADS) {
        const int i = i0 + tid, n = i < a.N ? own_tokens(a, i, bad) : -1;
        const int own = n > 0 ? (n + own_chunk - 1) / own_chunk : 0;
        const int count = n < 0 ? 0 : own + (a.P > 0 ? p.w.scan_prompt[i / a.G].y : 0);
        int2 total;
        const int2 before = block_scan(make_int2(own, count), total, warp_sums);
        if (i < a.N) {
            RolloutRecords r = {records + before.y, own, count, 0};
            if (r.base + (int64_t)count > p.w.max_records) { r = {0, 0, 0, 0}; bad = true; }     // only past 2^30 tokens a unit
            p.w.records[i] = r;
            p.w.scan[2 * i] = units + before.x;
        }
        units += total.x;
        records += total.y;
    }
    __syncthreads();
    // the units themselves: a warp per prompt, then per rollout
    const int lane = tid & 31, warp = tid >> 5;
    for (int q = warp; q < a.P; q += PLAN_THREADS / 32) {
        const int2 at = p.w.scan_prompt[q];
        if (at.y == 0) continue;
        const int live = live_of(q), first = p.w.scan[2 * q * a.G + 1], groups = (live + p.group - 1) / p.group;
        const int64_t x = a.cu_prompts[q];
        const int n = (int)(a.cu_prompts[q + 1] - x);
        for (int u = lane; u < groups * at.y && at.x + u < p.w.max_units; u += 32) {
            const int c = u / groups, g = u - c * groups;          // a chunk's groups side by side: they read the same rows
            DecodeUnit d = {(int)x + c * shared_chunk, min(shared_chunk, n - c * shared_chunk), min(p.group, live - g * p.group) * p.ratio, first + g * p.group, c, 1, {0, 0}};
            p.w.units[at.x + u] = d;
        }
    }
    for (int i = warp; i < a.N; i += PLAN_THREADS / 32) {
        const int own = p.w.records[i].own, at = p.w.scan[2 * i];
        for (int c = lane; c < own && at + c < p.w.max_units; c += 32) {
            DecodeUnit d = {(int)a.src_tok_off[i] + c * own_chunk, min(own_chunk, a.lengths[i] - c * own_chunk), p.ratio, i, c, 0, {0, 0}};
            p.w.units[at + c] = d;
        }
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
    DecodeUnit unit;
    int g, valid;
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
        for (int i = 0; i < DEC_SLOTS; ++i) { mbar_init(&sm.item_full[i], 1); mbar_init(&sm.item_empty[i], DEC_WARPS); }
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

    if (warp == DEC_WARPS) {
        const DecodeUnit* units = pdl_acquire(p.w.units);
        uint32_t pos = 0;
        bool ok = true;
        for (uint32_t n = 0; ok; ++n) {
            const uint32_t slot = n % DEC_SLOTS;
            if (!mbar_wait_warp(&sm.item_empty[slot], ((n / DEC_SLOTS) & 1u) ^ 1u, abort_flag)) { ok = false; break; }
            uint32_t idx = 0;
            if (lane == 0) idx = atomicAdd(reinterpret_cast<unsigned int*>(p.w.head), 1u);
            idx = __shfl_sync(0xffffffffu, idx, 0);
            const bool valid = (int64_t)idx < items;
            DecodeUnit u = {};
            const int g = (int)(idx % (uint32_t)a.Hkv);
            if (valid) u = units[idx / (uint32_t)a.Hkv];       // the heads of a unit side by side: they read the same rows
            if (lane == 0) {
                sm.items[slot].unit = u;
                sm.items[slot].g = g;
                sm.items[slot].valid = valid;
                mbar_arrive(&sm.item_full[slot]);
            }
            __syncwarp();
            if (!valid) break;
            const CUtensorMap* mk = u.shared ? &map_pk : &map_k;
            const CUtensorMap* mv = u.shared ? &map_pv : &map_v;
            for (int t = 0; t < u.ntok; t += C::TOKENS, ++pos) {
                const uint32_t st = pos % DEC_STAGES;
                if (!mbar_wait_warp(&sm.empty[st], ((pos / DEC_STAGES) & 1u) ^ 1u, abort_flag)) { ok = false; break; }
                if (elect_one()) {
                    mbar_expect_tx(&sm.full[st], DEC_STAGE_BYTES);
                    uint8_t* at = ring + st * DEC_STAGE_BYTES;
#pragma unroll
                    for (int h = 0; h < C::HALVES; ++h) {
                        tma_load_3d(at + h * C::HALF_BYTES, mk, h * 64, g, u.tok0 + t, &sm.full[st]);
                        tma_load_3d(at + C::KEYS_BYTES + h * C::HALF_BYTES, mv, h * 64, g, u.tok0 + t, &sm.full[st]);
                    }
                }
                __syncwarp();
            }
        }
        if (!ok) {                           // let the copies in flight land before the block's shared memory goes away
            for (uint32_t i = 1; i <= DEC_STAGES && i <= pos; ++i)
                for (uint32_t spin = 0; spin < SPIN_LIMIT; ++spin)
                    if (mbar_try_wait(&sm.full[(pos - i) % DEC_STAGES], ((pos - i) / DEC_STAGES) & 1u)) break;
        }
        __syncwarp();
    } else {
        // ---- consumers.  A unit's rows are 1, 2 or 4 tiles of 16; the warps that are left share its tokens.
        const int* live = pdl_acquire(p.w.live);
        const RolloutRecords* records = pdl_acquire(p.w.records);
        uint32_t pos0 = 0;
        for (uint32_t n = 0;; ++n) {
            const uint32_t slot = n % DEC_SLOTS;
            if (!mbar_wait_warp(&sm.item_full[slot], (n / DEC_SLOTS) & 1u, abort_flag)) break;
            const DecodeItem& it = sm.items[slot];
            if (!it.valid) break;
            const DecodeUnit u = it.unit;
            const int g = it.g, ratio = p.ratio;
            const int row_tiles = u.rows <= 16 ? 1 : u.rows <= 32 ? 2 : 4, parts = DEC_WARPS / row_tiles;
            const int tile = warp % row_tiles, share = warp / row_tiles;
            const int tiles = (u.ntok + C::TOKENS - 1) / C::TOKENS;
            // query rows (lane / 4) and (lane / 4) + 8 of the tile as fragments
            uint32_t q[DP / 16][4];
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                const int row = tile * 16 + (lane >> 2) + r * 8, l = row / ratio;
                const bool there = row < u.rows;
                const int i = !there ? 0 : u.shared ? live[u.src + l] : u.src;
                const __nv_bfloat16* at = static_cast<const __nv_bfloat16*>(a.q) + i * a.q_stride + (int64_t)(g * ratio + row - l * ratio) * a.D + (lane & 3) * 2;
#pragma unroll
                for (int k = 0; k < DP / 16; ++k)
#pragma unroll
                    for (int c = 0; c < 2; ++c)
                        q[k][c * 2 + r] = there && k * 16 + c * 8 < a.D ? *reinterpret_cast<const uint32_t*>(at + k * 16 + c * 8) : 0u;
            }
            float o[DP / 8][4], m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
#pragma unroll
            for (int d = 0; d < DP / 8; ++d) o[d][0] = o[d][1] = o[d][2] = o[d][3] = 0.f;
            bool ok = true;
            for (int t = share; t < tiles; t += parts) {
                const uint32_t pos = pos0 + t, st = pos % DEC_STAGES;
                if (!mbar_wait_warp(&sm.full[st], (pos / DEC_STAGES) & 1u, abort_flag)) { ok = false; break; }
                uint8_t* const stage = ring + st * DEC_STAGE_BYTES;
                const uint32_t keys = smem_u32(stage), values = keys + C::KEYS_BYTES;
                const int there = u.ntok - t * C::TOKENS;      // tokens of the unit from here on
                float s[C::TOKENS / 8][4];
#pragma unroll
                for (int j = 0; j < C::TOKENS / 8; ++j) {
                    s[j][0] = s[j][1] = s[j][2] = s[j][3] = 0.f;
                    const int row = j * 8 + (lane & 7);
#pragma unroll
                    for (int k = 0; k < DP / 32; ++k) {
                        const int c = k * 4 + (lane >> 3);
                        uint32_t b[4];
                        ldmatrix_x4(keys + (c >> 3) * C::HALF_BYTES + row * 128 + (((c & 7) ^ (row & 7)) << 4), b);
                        mma_16x8x16(s[j], q[2 * k], b[0], b[1]);
                        mma_16x8x16(s[j], q[2 * k + 1], b[2], b[3]);
                    }
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
                        for (int h = 0; h < C::HALVES; ++h) *reinterpret_cast<uint4*>(stage + C::KEYS_BYTES + h * C::HALF_BYTES + x * 16) = make_uint4(0, 0, 0, 0);
                    fence_proxy_async_smem();
                    __syncwarp();
                }
                float up[2];
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    float mx = -INFINITY;
#pragma unroll
                    for (int j = 0; j < C::TOKENS / 8; ++j) mx = fmaxf(mx, fmaxf(s[j][2 * r], s[j][2 * r + 1]));
                    mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
                    mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2)) * p.scale_log2;
                    const float top = fmaxf(m[r], mx);
                    up[r] = top == -INFINITY ? 1.f : ex2_approx(m[r] - top);
                    m[r] = top;
                    l[r] *= up[r];
                }
                if (__any_sync(0xffffffffu, up[0] != 1.f || up[1] != 1.f)) {
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
                    const uint32_t w[4] = {pack_bf16(s[2 * k][0], s[2 * k][1]), pack_bf16(s[2 * k][2], s[2 * k][3]), pack_bf16(s[2 * k + 1][0], s[2 * k + 1][1]),
                                           pack_bf16(s[2 * k + 1][2], s[2 * k + 1][3])};
                    const int row = k * 16 + (lane & 15);
#pragma unroll
                    for (int d = 0; d < DP / 16; ++d) {
                        const int c = d * 2 + (lane >> 4);
                        uint32_t b[4];
                        ldmatrix_x4_trans(values + (c >> 3) * C::HALF_BYTES + row * 128 + (((c & 7) ^ (row & 7)) << 4), b);
                        mma_16x8x16(o[2 * d], w, b[0], b[1]);
                        mma_16x8x16(o[2 * d + 1], w, b[2], b[3]);
                    }
                }
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
            if (!mbar_wait_warp(&sm.part_free, (n & 1u) ^ 1u, abort_flag)) break;
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
            if (lane == 0) {
                mbar_arrive(&sm.part_full);
                mbar_arrive(&sm.item_empty[slot]);
            }
            __syncwarp();
            if (!mbar_wait_warp(&sm.part_full, n & 1u, abort_flag)) break;
            const int pieces = a.D / 4;
            for (int x = warp * 32 + lane; x < u.rows * pieces; x += 32 * DEC_WARPS) {
                const int row = x / pieces, d = (x - row * pieces) * 4, t = row >> 4, r = row & 15;
                float top = -INFINITY;
                for (int s = 0; s < parts; ++s) top = fmaxf(top, sm.ml[s * row_tiles + t][r].x);
                float4 sum = {0.f, 0.f, 0.f, 0.f};
                float total = 0.f;
                for (int s = 0; s < parts; ++s) {
                    const float2 ml = sm.ml[s * row_tiles + t][r];
                    const float by = ml.x == -INFINITY ? (ml.y == 0.f ? 0.f : 1.f) : ex2_approx(ml.x - top);       // a NaN without a maximum stays one
                    const float4 v = *reinterpret_cast<const float4*>(part + ((s * row_tiles + t) * 16 + r) * C::PITCH + d);
                    sum.x += by * v.x; sum.y += by * v.y; sum.z += by * v.z; sum.w += by * v.w;
                    total += by * ml.y;
                }
                const int lr = row / ratio, h = g * ratio + row - lr * ratio;
                const RolloutRecords rec = records[u.shared ? live[u.src + lr] : u.src];
                const int64_t at = (int64_t)(rec.base + (u.shared ? rec.own : 0) + u.slot) * a.Hq + h;
                if (at >= p.w.max_records * a.Hq) continue;
                *reinterpret_cast<float4*>(p.w.o + at * a.D + d) = sum;
                if (d == 0) p.w.ml[at] = make_float2(top, total);
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(&sm.part_free);
            __syncwarp();
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
    const RolloutRecords rec = *pdl_acquire(p.w.records + i);
    const float2* ml = pdl_acquire(p.w.ml) + (int64_t)rec.base * a.Hq + h;
    const float* o = pdl_acquire(p.w.o) + ((int64_t)rec.base * a.Hq + h) * a.D;
    float top = -INFINITY;
    for (int r = lane; r < rec.count; r += 32) top = fmaxf(top, ml[(int64_t)r * a.Hq].x);
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
    float4 sum = {0.f, 0.f, 0.f, 0.f};
    float total = 0.f;
    const int d = lane * 4;
#pragma unroll 4
    for (int r = 0; r < rec.count; ++r) {
        const float2 x = ml[(int64_t)r * a.Hq];
        const float by = x.x == -INFINITY ? (x.y == 0.f ? 0.f : 1.f) : ex2_approx(x.x - top);
        total += by * x.y;
        if (d < a.D) {
            const float4 v = *reinterpret_cast<const float4*>(o + (int64_t)r * a.Hq * a.D + d);
            sum.x += by * v.x; sum.y += by * v.y; sum.z += by * v.z; sum.w += by * v.w;
        }
    }
    const bool none = total == 0.f;
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
    if (a->N < 0 || a->P < 0 || a->G < 1 || a->cache_rows < 0 || a->prompt_rows < 0 || a->Hq < 1 || a->Hkv < 1 || a->D < 1 || a->Hq % a->Hkv) return ARROL_ERR_INVALID_ARG;
    if (!(a->scale > 0.f) || !isfinite(a->scale)) return ARROL_ERR_INVALID_ARG;
    if (!attn_heads_ok(a->Hq, a->Hkv, a->D) || a->cache_rows >= ATTN_MAX_ROWS || a->prompt_rows >= ATTN_MAX_ROWS || a->G > 1024 || a->N > (1 << 24)) return ARROL_ERR_UNSUPPORTED;
    if (a->P > 0 ? (int64_t)a->P * a->G != a->N || !a->cu_prompts : a->prompt_rows > 0) return ARROL_ERR_INVALID_ARG;
    if (a->N == 0) return ARROL_OK;
    if (!attn_rows_ok(a->q, a->q_stride, a->Hq, a->D) || !attn_rows_ok(a->o, a->o_stride, a->Hq, a->D) || !a->src_tok_off || !a->lengths) return ARROL_ERR_INVALID_ARG;
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
    p.own_target = ctx->sm_count * DEC_OWN_PER_SM / a->Hkv + 1;
    p.shared_target = ctx->sm_count * DEC_SHARED_PER_SM / a->Hkv + 1;
    p.scale_log2 = a->scale * LOG2E;
    p.status = ctx->d_status;
    ArrolDeviceGuard guard(ctx->device);
    if (!guard.ok) return ARROL_ERR_CUDA;
    return a->D <= 64 ? launch_decode<64>(ctx, p, (cudaStream_t)stream) : launch_decode<128>(ctx, p, (cudaStream_t)stream);
}
