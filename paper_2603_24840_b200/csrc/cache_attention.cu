// arrol_cache_attention: one generated token per rollout over its group's prompt and its own tokens, both in the paged 8-bit cache.
//
// Bound by HBM: every live rollout's pages and every group's prompt pages are read once, half of a bf16 cache's bytes.  The products with keys take the e4m3 numbers as
// they lie in memory (m16n8k32 mma.sync): a row of q becomes two e4m3 rows, q = 2^e (hi + lo / 16), which is exact for bf16 but for entries below 2^-22 of the row's
// largest, so eight query rows fill the sixteen of a product and nothing has to be converted.  Probabilities would not survive that (a long tail of keys at 2^-20 of the
// first's weight carries real weight), so they are fp16 and the values are widened to it, two per instruction, which also brings the two tokens of an operand register
// together.  With a few rows a key there is too little work for tensor memory to pay.
//
// Work is cut without a plan: the lengths make a line of pieces of equal cost, every block takes an equal part of it, and each finds its own by a scan over the lengths
// (shared pieces first: a chunk of 128 tokens for more than 16 query rows, four warps a row tile each; then single ones: 32 tokens for 16 rows or less, a warp each).
// Pieces of a unit (rows x key head) that fall to different blocks or warps leave partial sums, which cache_merge_kernel adds up in order, so the result does not
// depend on who was first.
#include "cache_common.cuh"
#include "tc_common.cuh"

namespace {

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr int CA_WARPS = 4, CA_THREADS = 32 * CA_WARPS;
constexpr int CA_PER_SM = 2;                       // blocks
constexpr int CA_ROWS = 64;                        // query rows of a shared unit
constexpr int CA_ALONE = 16;                       // query rows up to which a unit is a warp's
constexpr int CA_TOKENS = 32;                      // a warp's piece; a shared one is CA_WARPS of them
constexpr int CA_SHARED_COST = 5;                  // of a shared piece, in single ones
constexpr float CA_RESCALE_AT = 8.0f;              // the running maximum follows once it is 2^8 behind
constexpr float CA_P_SCALE = 128.0f;               // probabilities up to 2^8 times 2^7 stay below fp16's largest

// Tokens that one set of query rows has in common: a rollout's own (rows = Hq / Hkv), or a prompt with the rows of some of its live rollouts.
struct alignas(16) CacheEntry {
    int entry, tokens, rows, pieces;               // pieces of one key head
};

struct CacheWorkspace {
    long long* head;           // [0] pieces of the shared line, [1] of the single one
    long long* where;          // [entries]: where an entry's pieces begin on its line
    CacheEntry* shared;        // entries with pieces, in order
    CacheEntry* single;
    float2* ml;                // per record row: reference (of scores log2 e), sum
    float* o;                  // [record rows][D]
    int64_t rows_own, rows_prompt, rows_shared;    // record rows of the three kinds, one behind the other
    size_t bytes;
};

inline int ca_group(int ratio) { return CA_ROWS / ratio; }                         // rollouts a prompt entry
inline int ca_blocks(int G, int ratio) { return (G + ca_group(ratio) - 1) / ca_group(ratio); }

inline CacheWorkspace cache_workspace(void* base, int sm_count, int N, int P, int G, int Hq, int Hkv, int D) {
    const int ratio = Hq / Hkv;
    const int64_t grid = (int64_t)sm_count * CA_PER_SM, prompts = P > 0 ? (int64_t)P * ca_blocks(G, ratio) : 0, entries = prompts + N;
    CacheWorkspace w = {};
    // a unit has one record, and one more for every border between blocks (warps) that falls into it: numbers unit + block (warp)
    w.rows_own = ratio <= CA_ALONE ? ((int64_t)N * Hkv + grid * CA_WARPS) * ratio : 0;
    w.rows_prompt = P > 0 ? (prompts * Hkv + grid * CA_WARPS) * CA_ALONE : 0;
    w.rows_shared = ((ratio <= CA_ALONE ? prompts : entries) * Hkv + (P > 0 || ratio > CA_ALONE ? grid : 0)) * CA_ROWS;
    uint8_t* p = static_cast<uint8_t*>(base);
    size_t at = 0;
    auto take = [&](size_t n) { uint8_t* q = p + at; at += (n + 255) & ~(size_t)255; return q; };
    const int64_t rows = w.rows_own + w.rows_prompt + w.rows_shared;
    w.head = reinterpret_cast<long long*>(take(256));
    w.where = reinterpret_cast<long long*>(take((size_t)entries * sizeof(long long)));
    w.shared = reinterpret_cast<CacheEntry*>(take((size_t)entries * sizeof(CacheEntry)));
    w.single = reinterpret_cast<CacheEntry*>(take((size_t)entries * sizeof(CacheEntry)));
    w.ml = reinterpret_cast<float2*>(take((size_t)rows * sizeof(float2)));
    w.o = reinterpret_cast<float*>(take((size_t)rows * D * sizeof(float)));
    w.bytes = at;
    return w;
}

struct CacheParams {
    arrol_cache_attention_args a;
    CacheWorkspace w;
    int ratio, group, blocks, prompts, entries;    // rollouts a prompt entry, entries a prompt, prompt entries, all
    int page_shift, grid;
    float scale_log2;
    uint32_t* status;
};

// ---- the line of pieces
struct Line {
    long long shared, single;      // pieces
    long long per;                 // cost that a block takes
};
__device__ __forceinline__ Line make_line(long long shared, long long single, int grid) {
    const long long cost = shared * CA_SHARED_COST + single;
    return {shared, single, cost <= grid ? 1 : (cost + grid - 1) / grid};
}
// shared pieces from there on are block b's or a later one's
__device__ __forceinline__ long long shared_begin(const Line& l, long long b) {
    const long long x = (b * l.per + CA_SHARED_COST - 1) / CA_SHARED_COST;
    return x < l.shared ? x : l.shared;
}
__device__ __forceinline__ long long shared_block(const Line& l, long long x) { return x * CA_SHARED_COST / l.per; }
// single pieces of block b, before they are cut to those that there are, and of each of its warps
__device__ __forceinline__ void single_range(const Line& l, long long b, long long& lo, long long& each) {
    const long long at = l.shared * CA_SHARED_COST;
    lo = b * l.per - at;
    if (lo < 0) lo = 0;
    const long long hi = (b + 1) * l.per - at;
    each = hi > lo ? (hi - lo + CA_WARPS - 1) / CA_WARPS : 0;
}
__device__ __forceinline__ void warp_range(const Line& l, long long warp, long long& y0, long long& y1) {
    long long lo, each;
    const long long b = warp / CA_WARPS, k = warp % CA_WARPS;
    single_range(l, b, lo, each);
    long long hi = (b + 1) * l.per - l.shared * CA_SHARED_COST;
    if (hi > l.single) hi = l.single;
    y0 = lo + k * each;
    y1 = y0 + each < hi ? y0 + each : hi;
}
__device__ __forceinline__ long long single_warp(const Line& l, long long y) {
    const long long b = (l.shared * CA_SHARED_COST + y) / l.per;
    long long lo, each;
    single_range(l, b, lo, each);
    return b * CA_WARPS + (y - lo) / each;
}

// Live rollouts of group p.
__device__ __forceinline__ int live_of(const CacheParams& p, int q) {
    const int G = p.a.G;
    if (!p.a.keep) return G;
    const uint8_t* keep = p.a.keep + (int64_t)q * G;
    int n = 0, i = 0;
    if ((reinterpret_cast<uintptr_t>(keep) & 15) == 0)
        for (; i + 16 <= G; i += 16) {
            const uint4 w = *reinterpret_cast<const uint4*>(keep + i);
            n += __popc(__vcmpne4(w.x, 0)) + __popc(__vcmpne4(w.y, 0)) + __popc(__vcmpne4(w.z, 0)) + __popc(__vcmpne4(w.w, 0));
        }
    n >>= 3;                       // a byte that is not zero gave eight bits
    for (; i < G; ++i) n += keep[i] != 0;
    return n;
}
__device__ __forceinline__ CacheEntry make_entry(const CacheParams& p, int e, bool& bad) {
    const arrol_cache_attention_args& a = p.a;
    CacheEntry x = {e, 0, 0, 0};
    if (e < p.prompts) {
        const int q = e / p.blocks, rollouts = min(live_of(p, q) - (e - q * p.blocks) * p.group, p.group);
        if (rollouts <= 0) return x;
        x.rows = rollouts * p.ratio;
        x.tokens = cache_tokens(a.prompt_lengths, q, a.prompt_table_pages, a.cache.page, bad);
    } else {
        const int i = e - p.prompts;
        if (a.keep && !a.keep[i]) return x;
        x.rows = p.ratio;
        x.tokens = cache_tokens(a.lengths, i, a.table_pages, a.cache.page, bad);
    }
    const int of = x.rows > CA_ALONE ? CA_TOKENS * CA_WARPS : CA_TOKENS;
    x.pieces = (int)(((int64_t)x.tokens + of - 1) / of);
    return x;
}

struct ScanSums {
    long long shared, single;      // pieces
    int shared_entries, single_entries;
};
__device__ __forceinline__ ScanSums operator+(const ScanSums& a, const ScanSums& b) {
    return {a.shared + b.shared, a.single + b.single, a.shared_entries + b.shared_entries, a.single_entries + b.single_entries};
}
__device__ __forceinline__ ScanSums shfl_up(const ScanSums& a, int d) {
    return {__shfl_up_sync(0xffffffffu, a.shared, d), __shfl_up_sync(0xffffffffu, a.single, d), __shfl_up_sync(0xffffffffu, a.shared_entries, d),
            __shfl_up_sync(0xffffffffu, a.single_entries, d)};
}

struct Start {
    int entry;                     // number in the list
    long long offset;              // pieces of it before
};

__device__ __forceinline__ void cp_async_zfill_16(uint32_t dst, const void* src, bool there) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp_async_zfill_8(uint32_t dst, const void* src, bool there) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;" ::"r"(dst), "l"(src), "r"(there ? 8 : 0) : "memory");
}
__device__ __forceinline__ void cp_async_4(uint32_t dst, const void* src) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

__device__ __forceinline__ void mma_e4m3(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k32.row.col.f32.e4m3.e4m3.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_f16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack_half(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

// What a warp copies and reads of 32 tokens.  Keys: a lane (g, t) = (lane / 4, lane % 4) has, of the tokens 8 j + g, the 16-byte chunks t and t + 4 of their rows; as the
// order of a product's dimensions is free as long as q has the same, these are the operand registers of two (DP = 64) or four products.  Values: of the tokens that the
// lane's own columns of the scores are, 8 j + 2 t and the next, the dimensions VB g .. VB g + VB - 1.  Each lane reads what it copied, 16 (8) bytes beside its neighbours'.
template <int DP>
struct CacheConf {
    static constexpr int CHUNKS = DP / 64;                        // of keys, per token and lane
    static constexpr int VB = DP / 8;                             // bytes of a token's values, per lane
    static constexpr int KEYS = CA_TOKENS * DP, BYTES = 2 * KEYS + 128;      // scales behind: keys' of the first and second 16 tokens, values'
    static constexpr int STAGES = DP == 128 ? 3 : 4;
    static constexpr int NT = DP / 8;
    static constexpr size_t SMEM = (size_t)STAGES * CA_WARPS * BYTES;
};

// Walks over a line's pieces.  What comes next is asked for before it is needed.
struct Cursor {
    CacheEntry e, next;
    const CacheEntry* list;
    int number, last;              // of the list's entries
    int head, piece;
    __device__ __forceinline__ void fetch() {
        if (number + 1 <= last) next = list[number + 1];
    }
    __device__ __forceinline__ void begin(const CacheEntry* l, const Start& s, int n) {
        list = l;
        number = s.entry;
        last = n - 1;
        e = list[number];
        head = (int)(s.offset / e.pieces);
        piece = (int)(s.offset - (long long)head * e.pieces);
        fetch();
    }
    __device__ __forceinline__ void advance(int heads) {
        if (++piece < e.pieces) return;
        piece = 0;
        if (++head < heads) return;
        head = 0;
        e = next;
        ++number;
        fetch();
    }
};

// The rows of the page table that an entry follows.
__device__ __forceinline__ const int32_t* entry_table(const CacheParams& p, int e) {
    return e < p.prompts ? p.a.prompt_table + (int64_t)(e / p.blocks) * p.a.prompt_table_stride : p.a.page_table + (int64_t)(e - p.prompts) * p.a.table_stride;
}
struct PagePair {
    int first, second;             // pages of the piece's first and second 16 tokens, -1 where there are none
};
__device__ __forceinline__ PagePair find_pages(const CacheParams& p, const Cursor& c, int tok) {
    const int32_t* table = entry_table(p, c.e.entry);
    PagePair g = {-1, -1};
    if (tok < c.e.tokens) g.first = table[tok >> p.page_shift];
    if (tok + 16 < c.e.tokens) g.second = table[(tok + 16) >> p.page_shift];
    return g;
}

template <int DP>
__device__ __forceinline__ void copy_piece(const CacheParams& p, const Cursor& c, int tok, PagePair pages, uint8_t* stage, int lane) {
    using C = CacheConf<DP>;
    const arrol_cache& cache = p.a.cache;
    const int D = cache.D, g = lane >> 2, t = lane & 3, there = c.e.tokens - tok, in_page = cache.page - 1;
    if ((pages.first < 0 && there > 0) || pages.first >= cache.pages || (pages.second < 0 && there > 16) || pages.second >= cache.pages) {
        if (lane == 0) atomicOr(p.status, ARROL_DEV_BAD_INDEX);
        if ((unsigned)pages.first >= (unsigned)cache.pages) pages.first = -1;
        if ((unsigned)pages.second >= (unsigned)cache.pages) pages.second = -1;
    }
    const uint32_t to = smem_u32(stage) + lane * 16;
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        const int page = half ? pages.second : pages.first, slot = (tok + half * 16) & in_page, left = there - half * 16;
        const bool is = page >= 0;
        const int64_t at = (int64_t)c.head * cache.page * D + slot * D;
        const uint8_t* const none = reinterpret_cast<const uint8_t*>(p.w.head);       // of a copy that reads nothing
        const uint8_t* k = is ? static_cast<const uint8_t*>(cache.k_cache) + page * cache.k_page_stride + at : none;
        const uint8_t* v = is ? static_cast<const uint8_t*>(cache.v_cache) + page * cache.v_page_stride + at : none;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int token = 8 * j + g;
            const bool copy = is && token < left;
#pragma unroll
            for (int x = 0; x < C::CHUNKS; ++x)
                if ((t + 4 * x) * 16 < D) cp_async_zfill_16(to + ((half * 2 + j) * C::CHUNKS + x) * 512, k + (copy ? token * D + (t + 4 * x) * 16 : 0), copy);
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int token = (j >> 1) * 8 + 2 * t + (j & 1);
            const bool copy = is && token < left;
            if (g * C::VB < D) {
                const uint8_t* from = v + (copy ? token * D + g * C::VB : 0);
                if (C::VB == 16) cp_async_zfill_16(to + C::KEYS + (half * 4 + j) * 512, from, copy);
                else cp_async_zfill_8(smem_u32(stage) + C::KEYS + (half * 4 + j) * 256 + lane * 8, from, copy);
            }
        }
        if (lane < 2) {                                       // lane 0 the keys' scale, lane 1 the values'
            uint8_t* s = stage + 2 * C::KEYS + lane * 8 + half * 4;
            if (is) cp_async_4(smem_u32(s), lane ? cache.v_scale + page * cache.v_scale_stride + c.head : cache.k_scale + page * cache.k_scale_stride + c.head);
            else *reinterpret_cast<float*>(s) = lane ? 0.f : -1.f;
        }
    }
}

// A tile of up to 16 query rows against the pieces of its unit.  Rows g and g + 8 of the tile are this lane's.
template <int DP>
struct RowTile {
    using C = CacheConf<DP>;
    uint32_t q[2][DP / 32][4];        // rows 0 .. 7 and 8 .. 15 as operands: upper parts above, lower parts below
    float by[2];                      // what a product's sum times the key's scale is multiplied by
    float o[C::NT][4], m[2], l[2];
    float v_scale;                    // largest scale of the values so far: o is in units of it / CA_P_SCALE

    __device__ __forceinline__ void load(const CacheParams& p, int lane, const __nv_bfloat16* row0, const __nv_bfloat16* row1) {
        const int t = lane & 3, D = p.a.cache.D;
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            const __nv_bfloat16* row = r ? row1 : row0;
            uint32_t raw[C::CHUNKS][8];
            float most = 0.f, odd = 0.f;
#pragma unroll
            for (int x = 0; x < C::CHUNKS; ++x) {
                const bool there = row && (t + 4 * x) * 16 < D;
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    const uint4 w = there ? *reinterpret_cast<const uint4*>(row + (t + 4 * x) * 16 + y * 8) : make_uint4(0, 0, 0, 0);
                    raw[x][y * 4] = w.x; raw[x][y * 4 + 1] = w.y; raw[x][y * 4 + 2] = w.z; raw[x][y * 4 + 3] = w.w;
                }
#pragma unroll
                for (int y = 0; y < 8; ++y) {
                    const float a = __uint_as_float(raw[x][y] << 16), b = __uint_as_float(raw[x][y] & 0xFFFF0000u);
                    most = finite_max(finite_max(most, a), b);
                    odd += (a - a) + (b - b);                 // NaN where one is not finite
                }
            }
#pragma unroll
            for (int s = 1; s < 4; s <<= 1) {
                most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, s));
                odd += __shfl_xor_sync(0xffffffffu, odd, s);
            }
            const int e = cache_exponent(most);
            const float down = cache_power(-e);
            by[r] = cache_power(e) * p.scale_log2 + odd;      // a query that is not finite makes its scores NaN
#pragma unroll
            for (int x = 0; x < C::CHUNKS; ++x)
#pragma unroll
                for (int y = 0; y < 4; ++y) {                 // four dimensions: registers (2 x + y / 2), rows above and below
                    uint32_t upper = 0, lower = 0;
#pragma unroll
                    for (int z = 0; z < 2; ++z) {
                        const uint32_t w = raw[x][y * 2 + z];
                        const float a = __uint_as_float(w << 16) * down, b = __uint_as_float(w & 0xFFFF0000u) * down;
                        const uint16_t hi = e4m3_pair(a, b);
                        const float2 h = e4m3_pair_to_float(hi);
                        upper |= (uint32_t)hi << (z * 16);
                        lower |= (uint32_t)e4m3_pair((a - h.x) * 16.f, (b - h.y) * 16.f) << (z * 16);
                    }
                    q[r][2 * x + (y >> 1)][(y & 1) * 2] = upper;
                    q[r][2 * x + (y >> 1)][(y & 1) * 2 + 1] = lower;
                }
        }
#pragma unroll
        for (int d = 0; d < C::NT; ++d) o[d][0] = o[d][1] = o[d][2] = o[d][3] = 0.f;
        m[0] = m[1] = -INFINITY;
        l[0] = l[1] = 0.f;
        v_scale = 0.f;
    }

    // `there` tokens of the piece (at least one).  BOTH: rows 8 .. 15 are there.
    template <bool BOTH>
    __device__ __forceinline__ void piece(const uint8_t* stage, int there, int lane) {
        constexpr int ROWS = BOTH ? 2 : 1;
        const int t = lane & 3;
        const uint8_t* const mine = stage + lane * 16;
        const float4 scales = *reinterpret_cast<const float4*>(stage + 2 * C::KEYS);
        float s[ROWS][4][2];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            float acc[ROWS][4];
#pragma unroll
            for (int r = 0; r < ROWS; ++r) acc[r][0] = acc[r][1] = acc[r][2] = acc[r][3] = 0.f;
#pragma unroll
            for (int x = 0; x < C::CHUNKS; ++x) {
                const uint4 w = *reinterpret_cast<const uint4*>(mine + (j * C::CHUNKS + x) * 512);
#pragma unroll
                for (int r = 0; r < ROWS; ++r) mma_e4m3(acc[r], q[r][2 * x], w.x, w.y);
#pragma unroll
                for (int r = 0; r < ROWS; ++r) mma_e4m3(acc[r], q[r][2 * x + 1], w.z, w.w);
            }
            const float ks = j < 2 ? scales.x : scales.y;
#pragma unroll
            for (int r = 0; r < ROWS; ++r) {
                const float f = by[r] * ks;
                s[r][j][0] = fmaf(acc[r][2], 0.0625f, acc[r][0]) * f;
                s[r][j][1] = fmaf(acc[r][3], 0.0625f, acc[r][1]) * f;
            }
        }
        if (there < CA_TOKENS || scales.x < 0.f || scales.y < 0.f) {
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int c = 0; c < 2; ++c)
                    if (8 * j + 2 * t + c >= there || (j < 2 ? scales.x : scales.y) < 0.f)
#pragma unroll
                        for (int r = 0; r < ROWS; ++r) s[r][j][c] = -INFINITY;
        }
        // The reference is let fall up to 2^8 behind the maximum: only where some row is further behind do its four lanes settle on a new one.
        float mx[2] = {-INFINITY, -INFINITY};
#pragma unroll
        for (int r = 0; r < ROWS; ++r)
#pragma unroll
            for (int j = 0; j < 4; ++j) mx[r] = fmaxf(mx[r], fmaxf(s[r][j][0], s[r][j][1]));
        const float vs = fmaxf(scales.z, scales.w);
        if (vs > v_scale || __any_sync(0xffffffffu, mx[0] > m[0] + CA_RESCALE_AT || mx[1] > m[1] + CA_RESCALE_AT)) {
            const float shrink = vs > v_scale ? v_scale / vs : 1.f;
            v_scale = fmaxf(vs, v_scale);
            float up[2] = {1.f, 1.f};
#pragma unroll
            for (int r = 0; r < ROWS; ++r) {
                mx[r] = fmaxf(mx[r], __shfl_xor_sync(0xffffffffu, mx[r], 1));
                mx[r] = fmaxf(mx[r], __shfl_xor_sync(0xffffffffu, mx[r], 2));
                if (mx[r] > m[r] + CA_RESCALE_AT) {
                    up[r] = ex2_approx(m[r] - mx[r]);
                    m[r] = mx[r];
                    l[r] *= up[r];
                }
                up[r] *= shrink;
            }
#pragma unroll
            for (int d = 0; d < C::NT; ++d) { o[d][0] *= up[0]; o[d][1] *= up[0]; o[d][2] *= up[1]; o[d][3] *= up[1]; }
        }
        const float inv = v_scale > 0.f ? CA_P_SCALE / v_scale : 0.f, w0 = scales.z * inv, w1 = scales.w * inv;
        uint32_t a[2][4];
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            const float sub = m[r] == -INFINITY ? 0.f : m[r];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float e0 = ex2_approx(s[r][j][0] - sub), e1 = ex2_approx(s[r][j][1] - sub), w = j < 2 ? w0 : w1;
                l[r] += e0 + e1;
                a[j >> 1][(j & 1) * 2 + r] = pack_half(e0 * w, e1 * w);
            }
        }
        if (!BOTH) a[0][1] = a[0][3] = a[1][1] = a[1][3] = 0u;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            uint32_t v[4][C::VB / 4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (C::VB == 16) {
                    const uint4 w = *reinterpret_cast<const uint4*>(mine + C::KEYS + (half * 4 + j) * 512);
                    v[j][0] = w.x; v[j][1] = w.y; v[j][C::VB / 4 - 2] = w.z; v[j][C::VB / 4 - 1] = w.w;
                } else {
                    const uint2 w = *reinterpret_cast<const uint2*>(stage + C::KEYS + (half * 4 + j) * 256 + lane * 8);
                    v[j][0] = w.x; v[j][1] = w.y;
                }
            }
#pragma unroll
            for (int x = 0; x < C::VB / 4; ++x)
#pragma unroll
                for (int y = 0; y < 2; ++y) {                  // dimensions 4 x + 2 y and the next: their numbers of two tokens side by side
                    const uint32_t b0 = __byte_perm(v[0][x], v[1][x], y ? 0x7362 : 0x5140), b1 = __byte_perm(v[2][x], v[3][x], y ? 0x7362 : 0x5140);
                    mma_f16(o[4 * x + 2 * y], a[half], e4m3_pair_to_half((uint16_t)b0), e4m3_pair_to_half((uint16_t)b1));
                    mma_f16(o[4 * x + 2 * y + 1], a[half], e4m3_pair_to_half((uint16_t)(b0 >> 16)), e4m3_pair_to_half((uint16_t)(b1 >> 16)));
                }
        }
    }

    // Sums of the tile's first `rows` rows to record rows `at`, ...
    __device__ __forceinline__ void store(const CacheParams& p, int64_t at, int rows, int lane) {
        const int t = lane & 3, D = p.a.cache.D;
        const float unit = v_scale * (1.f / CA_P_SCALE);
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            l[r] += __shfl_xor_sync(0xffffffffu, l[r], 1);
            l[r] += __shfl_xor_sync(0xffffffffu, l[r], 2);
            const int row = (lane >> 2) + 8 * r;
            if (row >= rows) continue;
            float* out = p.w.o + (at + row) * D + t * 2 * C::VB;      // columns 2 t and 2 t + 1 of the products: dimensions VB 2 t .. + 2 VB
#pragma unroll
            for (int c = 0; c < 2; ++c)
                if ((2 * t + c) * C::VB < D)
#pragma unroll
                    for (int d = 0; d < C::VB; d += 4)
                        *reinterpret_cast<float4*>(out + c * C::VB + d) =
                            make_float4(o[d][2 * r + c] * unit, o[d + 1][2 * r + c] * unit, o[d + 2][2 * r + c] * unit, o[d + 3][2 * r + c] * unit);
            if (t == 0) p.w.ml[at + row] = make_float2(m[r], l[r]);
        }
    }
};

struct CacheShared {
    ScanSums warp_sums[CA_WARPS];
    Start shared, single[CA_WARPS];
    int live[CA_WARPS][CA_ROWS];       // rollouts of a prompt entry, per warp
};

// Query rows `row0`, `row0` + 8 of the entry's unit (rows of them), for this lane.
__device__ __forceinline__ const __nv_bfloat16* query_row(const CacheParams& p, const CacheEntry& e, int head, const int* live, int row) {
    if (row >= e.rows) return nullptr;
    const int of = row / p.ratio, i = e.entry < p.prompts ? live[of] : e.entry - p.prompts;
    return static_cast<const __nv_bfloat16*>(p.a.q) + i * p.a.q_stride + (int64_t)(head * p.ratio + row - of * p.ratio) * p.a.cache.D;
}
// The live rollouts of a prompt entry, in order; by a warp.
__device__ __forceinline__ void find_live(const CacheParams& p, int e, int* live, int lane) {
    const int q = e / p.blocks, first = (e - q * p.blocks) * p.group, G = p.a.G;
    __syncwarp();
    int n = 0;
    for (int i0 = 0; i0 < G && n < first + p.group; i0 += 32) {
        const int i = i0 + lane;
        const bool is = i < G && (!p.a.keep || p.a.keep[(int64_t)q * G + i]);
        const uint32_t all = __ballot_sync(0xffffffffu, is);
        const int number = n + __popc(all & ((1u << lane) - 1u)) - first;
        if (is && number >= 0 && number < p.group) live[number] = q * G + i;
        n += __popc(all);
    }
    __syncwarp();
}

template <int DP>
__global__ void __launch_bounds__(CA_THREADS, CA_PER_SM) cache_units_kernel(const CacheParams p) {
    using C = CacheConf<DP>;
    extern __shared__ __align__(128) uint8_t ring[];
    __shared__ CacheShared sm;
    pdl_launch_dependents();
    pdl_wait();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, Hkv = p.a.cache.Hkv, D = p.a.cache.D;
    const long long b = blockIdx.x;
    // dimensions that no copy fills are zeros
    if (D < DP)
        for (int x = threadIdx.x * 16; x < (int)C::SMEM; x += CA_THREADS * 16) *reinterpret_cast<uint4*>(ring + x) = make_uint4(0, 0, 0, 0);

    // ---- the scan: a thread has `each` entries in a row, twice (sums, then what is this block's)
    const int each = (p.entries + CA_THREADS - 1) / CA_THREADS;
    const int e0 = min((int)threadIdx.x * each, p.entries), e1 = min(e0 + each, p.entries);
    bool bad = false;
    ScanSums mine = {0, 0, 0, 0};
    for (int e = e0; e < e1; ++e) {
        const CacheEntry x = make_entry(p, e, bad);
        if (x.pieces == 0) continue;
        if (x.rows > CA_ALONE) { mine.shared += (long long)x.pieces * Hkv; ++mine.shared_entries; }
        else { mine.single += (long long)x.pieces * Hkv; ++mine.single_entries; }
    }
    if (bad && b == 0) atomicOr(p.status, ARROL_DEV_BAD_INDEX);
    ScanSums sum = mine;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const ScanSums x = shfl_up(sum, d);
        if (lane >= d) sum = sum + x;
    }
    if (lane == 31) sm.warp_sums[warp] = sum;
    __syncthreads();
    ScanSums total = {0, 0, 0, 0}, at = {sum.shared - mine.shared, sum.single - mine.single, sum.shared_entries - mine.shared_entries, sum.single_entries - mine.single_entries};
#pragma unroll
    for (int w = 0; w < CA_WARPS; ++w) {
        if (w < warp) at = at + sm.warp_sums[w];
        total = total + sm.warp_sums[w];
    }
    const Line line = make_line(total.shared, total.single, p.grid);
    if (b == 0 && threadIdx.x == 0) { p.w.head[0] = total.shared; p.w.head[1] = total.single; }
    const long long x0 = shared_begin(line, b), x1 = shared_begin(line, b + 1);
    long long y0, y1, block_y0, block_y1;
    warp_range(line, b * CA_WARPS + warp, y0, y1);
    {
        long long other;
        warp_range(line, b * CA_WARPS, block_y0, other);
        block_y1 = (b + 1) * line.per - line.shared * CA_SHARED_COST;
        if (block_y1 > line.single) block_y1 = line.single;
    }
    const bool tell = (int)(threadIdx.x % gridDim.x) == (int)b;            // where the entries' pieces begin, for the merge: each thread's by one block
    for (int e = e0; e < e1; ++e) {
        const CacheEntry x = make_entry(p, e, bad);
        if (x.pieces == 0) continue;
        const long long n = (long long)x.pieces * Hkv;
        if (x.rows > CA_ALONE) {
            if (tell) p.w.where[e] = at.shared;
            if (at.shared < x1 && at.shared + n > x0) p.w.shared[at.shared_entries] = x;      // neighbours write the same
            if (at.shared <= x0 && at.shared + n > x0) sm.shared = {at.shared_entries, x0 - at.shared};
            at.shared += n;
            ++at.shared_entries;
        } else {
            if (tell) p.w.where[e] = at.single;
            if (at.single < block_y1 && at.single + n > block_y0) p.w.single[at.single_entries] = x;
#pragma unroll
            for (int w = 0; w < CA_WARPS; ++w) {
                long long w0, w1;
                warp_range(line, b * CA_WARPS + w, w0, w1);
                if (w0 < w1 && at.single <= w0 && at.single + n > w0) sm.single[w] = {at.single_entries, w0 - at.single};
            }
            at.single += n;
            ++at.single_entries;
        }
    }
    __syncthreads();

    // ---- shared pieces: four warps, a tile of 16 rows each; with two tiles two warps share a tile's tokens
    RowTile<DP> tile;
    if (x0 < x1) {
        Cursor ahead, now;
        ahead.begin(p.w.shared, sm.shared, total.shared_entries);
        now = ahead;
        long long left = x1 - x0;                             // pieces to copy
        PagePair pages = find_pages(p, ahead, (ahead.piece * CA_WARPS + warp) * CA_TOKENS);
        uint32_t slot = 0;
        auto copy = [&](uint32_t to) {
            if (left > 0) {
                copy_piece<DP>(p, ahead, (ahead.piece * CA_WARPS + warp) * CA_TOKENS, pages, ring + (size_t)(to * CA_WARPS + warp) * C::BYTES, lane);
                if (--left > 0) {
                    ahead.advance(Hkv);
                    pages = find_pages(p, ahead, (ahead.piece * CA_WARPS + warp) * CA_TOKENS);
                }
            }
            cp_async_commit();
        };
#pragma unroll
        for (int i = 0; i < C::STAGES - 1; ++i) copy(i);
        bool first = true;
        for (long long x = x0; x < x1; ++x) {
            const int row_tiles = now.e.rows <= 32 ? 2 : 4, mine_tile = warp & (row_tiles - 1), share = warp / row_tiles;
            if (first || now.piece == 0) {
                if (now.e.entry < p.prompts) find_live(p, now.e.entry, sm.live[warp], lane);
                const int row = mine_tile * 16 + (lane >> 2);
                tile.load(p, lane, query_row(p, now.e, now.head, sm.live[warp], row), query_row(p, now.e, now.head, sm.live[warp], row + 8));
                first = false;
            }
            cp_async_wait<C::STAGES - 2>();
            __syncthreads();
            copy(slot == 0 ? C::STAGES - 1 : slot - 1);       // the stage that every warp has left before the barrier
            if (mine_tile * 16 < now.e.rows)
                for (int w = share; w < CA_WARPS; w += CA_WARPS / row_tiles) {
                    const int there = now.e.tokens - (now.piece * CA_WARPS + w) * CA_TOKENS;
                    if (there <= 0) break;
                    tile.template piece<true>(ring + (size_t)(slot * CA_WARPS + w) * C::BYTES, there, lane);
                }
            if (now.piece == now.e.pieces - 1 || x == x1 - 1) {
                const int64_t record = ((int64_t)now.e.entry * Hkv + now.head + b) * CA_ROWS + (row_tiles == 2 ? share * 32 : 0) + mine_tile * 16;
                tile.store(p, p.w.rows_own + p.w.rows_prompt + record, now.e.rows - mine_tile * 16, lane);
            }
            if (x < x1 - 1) now.advance(Hkv);
            slot = slot == C::STAGES - 1 ? 0 : slot + 1;
        }
        cp_async_wait<0>();
        __syncthreads();
    }

    // ---- single pieces: a warp each
    if (y0 < y1) {
        const long long global_warp = b * CA_WARPS + warp;
        Cursor ahead, now;
        ahead.begin(p.w.single, sm.single[warp], total.single_entries);
        now = ahead;
        long long left = y1 - y0;
        PagePair pages = find_pages(p, ahead, ahead.piece * CA_TOKENS);
        uint32_t slot = 0;
        uint8_t* const stages = ring + (size_t)warp * C::BYTES;
        auto copy = [&](uint32_t to) {
            if (left > 0) {
                copy_piece<DP>(p, ahead, ahead.piece * CA_TOKENS, pages, stages + (size_t)to * CA_WARPS * C::BYTES, lane);
                if (--left > 0) {
                    ahead.advance(Hkv);
                    pages = find_pages(p, ahead, ahead.piece * CA_TOKENS);
                }
            }
            cp_async_commit();
        };
#pragma unroll
        for (int i = 0; i < C::STAGES - 1; ++i) copy(i);
        bool first = true;
        for (long long y = y0; y < y1; ++y) {
            if (first || now.piece == 0) {
                if (now.e.entry < p.prompts) find_live(p, now.e.entry, sm.live[warp], lane);
                tile.load(p, lane, query_row(p, now.e, now.head, sm.live[warp], lane >> 2), query_row(p, now.e, now.head, sm.live[warp], (lane >> 2) + 8));
                first = false;
            }
            cp_async_wait<C::STAGES - 2>();
            __syncwarp();
            copy(slot == 0 ? C::STAGES - 1 : slot - 1);
            const int there = now.e.tokens - now.piece * CA_TOKENS;
            const uint8_t* stage = stages + (size_t)slot * CA_WARPS * C::BYTES;
            if (now.e.rows > 8) tile.template piece<true>(stage, there, lane);
            else tile.template piece<false>(stage, there, lane);
            if (now.piece == now.e.pieces - 1 || y == y1 - 1) {
                const int64_t record = now.e.entry < p.prompts ? p.w.rows_own + ((int64_t)now.e.entry * Hkv + now.head + global_warp) * CA_ALONE
                                                               : ((int64_t)(now.e.entry - p.prompts) * Hkv + now.head + global_warp) * p.ratio;
                tile.store(p, record, now.e.rows, lane);
            }
            if (y < y1 - 1) now.advance(Hkv);
            slot = slot == C::STAGES - 1 ? 0 : slot + 1;
        }
    }
    cp_async_wait_all();
}

// Running sum of records.
struct Merged {
    float top, total;
    float4 sum;
    __device__ __forceinline__ void add(float2 ml, float4 v) {
        const float next = fmaxf(top, ml.x), up = next == -INFINITY ? 1.f : ex2_approx(top - next);
        const float by = ml.x == -INFINITY ? (ml.y == 0.f ? 0.f : 1.f) : ex2_approx(ml.x - next);      // a NaN without a maximum stays one
        total = total * up + by * ml.y;
        sum.x = sum.x * up + by * v.x; sum.y = sum.y * up + by * v.y; sum.z = sum.z * up + by * v.z; sum.w = sum.w * up + by * v.w;
        top = next;
    }
};

// A warp per (rollout, query head): the prompt's records, then its own, in order; four dimensions a lane.
__global__ void __launch_bounds__(256) cache_merge_kernel(const CacheParams p) {
    pdl_launch_dependents();
    pdl_wait();
    const arrol_cache_attention_args& a = p.a;
    const int lane = threadIdx.x & 31, D = a.cache.D, Hkv = a.cache.Hkv, d = lane * 4;
    const int64_t row = blockIdx.x * (int64_t)8 + (threadIdx.x >> 5);
    if (row >= (int64_t)a.N * a.Hq) return;
    const int i = (int)(row / a.Hq), hq = (int)(row - (int64_t)i * a.Hq), h = hq / p.ratio, r = hq - h * p.ratio;
    if (a.keep && !a.keep[i]) return;
    const long long* head = pdl_acquire(p.w.head);
    const long long* where = pdl_acquire(p.w.where);
    const float2* ml = pdl_acquire(p.w.ml);
    const float* o = pdl_acquire(p.w.o);
    const Line line = make_line(head[0], head[1], p.grid);
    Merged m = {-INFINITY, 0.f, {0.f, 0.f, 0.f, 0.f}};
    bool any = false, bad = false;
    auto record = [&](int64_t at) { m.add(ml[at], d < D ? *reinterpret_cast<const float4*>(o + at * D + d) : make_float4(0.f, 0.f, 0.f, 0.f)); };
    auto entry = [&](const CacheEntry& e, int row_in) {
        if (e.pieces == 0) return;
        any = true;
        const long long from = where[e.entry] + (long long)h * e.pieces, to = from + e.pieces - 1;
        if (e.rows > CA_ALONE) {
            const long long b1 = shared_block(line, to);
            for (long long b = shared_block(line, from); b <= b1; ++b) {
                if (shared_begin(line, b) >= shared_begin(line, b + 1)) continue;
                const int64_t at = p.w.rows_own + p.w.rows_prompt + ((int64_t)e.entry * Hkv + h + b) * CA_ROWS + row_in;
                record(at);
                if (e.rows <= 32) record(at + 32);
            }
        } else {
            const long long w1 = single_warp(line, to);
            for (long long w = single_warp(line, from); w <= w1; ++w) {
                long long y0, y1;
                warp_range(line, w, y0, y1);
                if (y0 >= y1) continue;
                record(e.entry < p.prompts ? p.w.rows_own + ((int64_t)e.entry * Hkv + h + w) * CA_ALONE + row_in
                                           : ((int64_t)(e.entry - p.prompts) * Hkv + h + w) * p.ratio + row_in);
            }
        }
    };
    if (p.prompts) {
        const int q = i / a.G, G = a.G;
        int before = 0;                                       // live rollouts of the group before this one
        for (int j = lane; j < i - q * G; j += 32) before += !a.keep || a.keep[(int64_t)q * G + j];
        before = __reduce_add_sync(0xffffffffu, before);
        entry(make_entry(p, q * p.blocks + before / p.group, bad), before % p.group * p.ratio + r);
    }
    entry(make_entry(p, p.prompts + i, bad), r);
    const float inv = any ? 1.f / m.total : 0.f;
    if (d < D) {
        uint2 w = make_uint2(0u, 0u);
        if (any) {
            asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w.x) : "f"(m.sum.y * inv), "f"(m.sum.x * inv));
            asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w.y) : "f"(m.sum.w * inv), "f"(m.sum.z * inv));
        }
        *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(a.o) + i * a.o_stride + (int64_t)hq * D + d) = w;
    }
    if (lane == 0 && a.lse) a.lse[row] = any ? (m.top + log2f(m.total)) * LN2 : -INFINITY;
}

template <int DP>
int launch_cache_attention(arrol_ctx* ctx, const CacheParams& p, cudaStream_t s) {
    using C = CacheConf<DP>;
    bool& set = ctx->cache_attention_smem_set[DP == 128];
    if (!set) {
        ARROL_CUDA_OK(cudaFuncSetAttribute(cache_units_kernel<DP>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)C::SMEM));
        set = true;
    }
    ARROL_CUDA_OK(arrol_launch_pdl(cache_units_kernel<DP>, dim3((unsigned)p.grid), dim3(CA_THREADS), C::SMEM, s, p));
    ARROL_CUDA_OK(arrol_launch_pdl(cache_merge_kernel, dim3((unsigned)(((int64_t)p.a.N * p.a.Hq + 7) / 8)), dim3(256), 0, s, p));
    ctx->launches += 2;
    return ARROL_OK;
}

bool cache_heads_ok(int Hq, int Hkv, int D) {
    return Hkv >= 1 && Hq >= Hkv && Hq <= 65536 && Hq % Hkv == 0 && Hq / Hkv <= CA_ROWS && D >= 16 && D <= CACHE_MAX_D && D % 16 == 0;
}

}  // namespace

extern "C" size_t arrol_cache_attention_workspace(arrol_ctx* ctx, int32_t N, int32_t P, int32_t G, int32_t Hq, int32_t Hkv, int32_t D) {
    if (!ctx || N < 0 || P < 0 || G < 1 || !cache_heads_ok(Hq, Hkv, D)) return 0;
    return cache_workspace(nullptr, ctx->sm_count, N, P, G, Hq, Hkv, D).bytes;
}

extern "C" int arrol_cache_attention(arrol_ctx* ctx, const arrol_cache_attention_args* a, void* stream) {
    if (!ctx || !a) return ARROL_ERR_INVALID_ARG;
    const int cache = cache_check(a->cache);
    if (cache == ARROL_ERR_INVALID_ARG) return cache;
    if (a->N < 0 || a->P < 0 || a->G < 1 || a->Hq < 1 || a->Hq % a->cache.Hkv || !(a->scale > 0.f) || !isfinite(a->scale)) return ARROL_ERR_INVALID_ARG;
    if (a->table_pages < 0 || a->table_stride < a->table_pages) return ARROL_ERR_INVALID_ARG;
    if (cache != ARROL_OK || !cache_heads_ok(a->Hq, a->cache.Hkv, a->cache.D) || a->G > 1024 || a->N > (1 << 24)) return ARROL_ERR_UNSUPPORTED;
    if (a->P > 0 ? (int64_t)a->P * a->G != a->N || !a->prompt_lengths || a->prompt_table_pages < 0 || (a->prompt_table_pages > 0 && !a->prompt_table) || a->prompt_table_stride < a->prompt_table_pages
                 : a->prompt_table || a->prompt_lengths)
        return ARROL_ERR_INVALID_ARG;
    if (a->N == 0) return ARROL_OK;
    if (!cache_rows_ok(a->q, a->q_stride, a->Hq, a->cache.D) || !cache_rows_ok(a->o, a->o_stride, a->Hq, a->cache.D) || !a->lengths ||
        (a->table_pages > 0 && !a->page_table))
        return ARROL_ERR_INVALID_ARG;
    if (!a->workspace || !arrol_aligned(a->workspace, 256)) return ARROL_ERR_WORKSPACE;
    CacheParams p = {};
    p.a = *a;
    p.w = cache_workspace(a->workspace, ctx->sm_count, a->N, a->P, a->G, a->Hq, a->cache.Hkv, a->cache.D);
    if (a->workspace_bytes < p.w.bytes) return ARROL_ERR_WORKSPACE;
    p.ratio = a->Hq / a->cache.Hkv;
    p.group = ca_group(p.ratio);
    p.blocks = ca_blocks(a->G, p.ratio);
    p.prompts = a->P * p.blocks;
    p.entries = p.prompts + a->N;
    p.page_shift = __builtin_ctz((unsigned)a->cache.page);
    p.grid = ctx->sm_count * CA_PER_SM;
    p.scale_log2 = a->scale * LOG2E;
    p.status = ctx->d_status;
    ArrolDeviceGuard guard(ctx->device);
    if (!guard.ok) return ARROL_ERR_CUDA;
    return a->cache.D <= 64 ? launch_cache_attention<64>(ctx, p, (cudaStream_t)stream) : launch_cache_attention<128>(ctx, p, (cudaStream_t)stream);
}
