// arrol_cache_attention: one generated token per rollout over its group's prompt and its own tokens, both in the paged 8-bit cache.
//
// Bound by HBM in the large: every live rollout's pages and every group's prompt pages are read once, half of a bf16 cache's bytes.  Measured (calls one behind another):
// 256 live rollouts of 2,200 tokens over 32 prompts, 16 heads of 128 on 8 (1.23 GB) 235 us, 5.2 TB/s.  By clocks in the kernel the first pieces are there after 11 us (a scan
// of 4, then loads that depend on one another, and everybody's copies at once), warps end between 184 and 215, the merge takes 10.  8 rollouts of 6,600 tokens, 32 heads
// (118 MB) 55 us: pieces from 10 to 38, the merge behind them.  384 rollouts of 160 tokens over 24 prompts of 4,850, 32 heads of 64 (188 MB) 140 us: there it is the work of
// 64 query rows behind every key, each warp a chain of 2,000 cycles for 32 tokens of 16 rows, three of them an SM's quarter.  168 registers (heads up to 64: 128), at the edge: 28
// bytes are spilled, and instructions in the pieces' loops, run or jumped over, show in all calls.
//
// The products are m16n8k16 mma.sync in fp16, transposed: tokens (of S^T = K Q^T) and dimensions (of O^T = V^T P^T) are the sixteen rows, query rows the eight columns, so that
// eight query heads waste nothing.  e4m3 numbers widen to fp16 exactly, two an instruction, and q, scaled by a power of two for each row, is exact in fp16 too (bf16 has
// fewer bits; what is below 2^-27 of the row's largest is rounded at 2^-39 of it).  Probabilities are rounded to fp16, which holds a long tail of keys at 2^-20 of the
// largest one's weight as well as that one; its smallest steps are 2^-31 of that weight.  Scales of pages and heads join the scores and the probabilities, the latter in front of
// their rounding, in units of the largest: where they lie more than 2^8 apart small values would be rounded away, and the merge computes such rows anew in fp32.  (Products of
// e4m3 operands by mma.sync are widened by the compiler, at each use: 12 instructions for one.)
//
// Work is cut without a plan: the lengths make a line of pieces and units' setups by their cost, every block takes an equal part of it, and each finds its own by a scan over
// the lengths.  Shared pieces come first: tokens that more than 16 query rows have in common, four warps a tile of 16 rows each (or two for two tiles); then single ones, 32
// tokens for 16 rows or less, a warp each.  Pieces of a unit (rows x key head) that fall to different blocks or warps leave partial sums, which cache_merge_kernel adds up in
// order, so the result does not depend on who was first.
#include <type_traits>

#include "cache_common.cuh"
#include "tc_common.cuh"

namespace {

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr int CA_WARPS = 4, CA_THREADS = 32 * (CA_WARPS + 1);      // consumers; one more warp brings their pieces
constexpr int CA_ROWS = 64;                        // query rows of a shared unit
constexpr int CA_ALONE = 16;                       // query rows up to which a unit is a warp's
constexpr int CA_TOKENS = 32;                      // a single piece; a shared one is four of them, two for more than 32 rows, so that a warp has two to compute
// The line that the work is cut along: what a shared piece costs, a unit before its first single piece (queries, results), a single piece of up to eight rows and one of more.
// A shared unit's setup counts as one of its pieces.  By the ends of all blocks and whole calls over {36 .. 80, 12 .. 36, 4, 4 .. 6}; against {48, 12, 4, 4} heads of 128 take
// 231 us instead of 256 (256 rollouts of 2,200 tokens; pieces of nine rows or more ended last), 252 instead of 265 (24 prompts of 5,100 with 14 rollouts of 160 tokens, 32 heads on 8).
constexpr int CA_SHARED_SETUP = 1;
struct LineCosts {
    int shared, single_setup, few, many;
};
constexpr LineCosts CA_COSTS_64 = {44, 24, 4, 5}, CA_COSTS_128 = {54, 28, 4, 5};
// The same in steps of a piece, where tables are so long that the line could pass 32 bits.
constexpr LineCosts CA_COSTS_COARSE = {13, 7, 1, 1};
constexpr int CA_SCANNED = 768;                    // entries that a block keeps in shared memory between the two passes of its scan
constexpr float CA_RESCALE_AT = 8.0f;              // the running maximum follows once it is 2^8 behind
constexpr float CA_P_SCALE = 128.0f;               // probabilities up to 2^8 times 2^7 stay below fp16's largest
// Scales of values join the probabilities down to 2^-8 of the largest, so that fp16 holds probabilities to half a step from 2^-13 on whatever their pages' scales.  A record with
// others is marked, by its sum's sign, and the merge computes its rows anew (row_apart).
constexpr float CA_NEAR = 0.00390625f;

// Tokens that one set of query rows has in common: a rollout's own (rows = Hq / Hkv), or a prompt with the rows of some of its live rollouts.
struct alignas(16) CacheEntry {
    int entry, tokens, rows, pieces;               // pieces of one key head
};

struct CacheWorkspace {
    int2* owners;              // [entries][Hkv]: the first and the last block (warp) that has some of the unit
    CacheEntry* shared;        // entries with pieces, in order
    CacheEntry* single;
    float2* ml;                // per record row: reference (of scores log2 e), sum, negative where the row is computed anew
    float* o;                  // [record rows][D]
    int64_t rows_own, rows_prompt, rows_shared;    // record rows of the three kinds, one behind the other
    size_t bytes;
};

inline int ca_per_sm(int D) { return D <= 64 ? 3 : 2; }                            // blocks
inline int ca_group(int ratio) { return CA_ROWS / ratio; }                         // rollouts a prompt entry
inline int ca_blocks(int G, int ratio) { return (G + ca_group(ratio) - 1) / ca_group(ratio); }

inline CacheWorkspace cache_workspace(void* base, int sm_count, int N, int P, int G, int Hq, int Hkv, int D) {
    const int ratio = Hq / Hkv;
    const int64_t grid = (int64_t)sm_count * ca_per_sm(D), prompts = P > 0 ? (int64_t)P * ca_blocks(G, ratio) : 0, entries = prompts + N;
    CacheWorkspace w = {};
    // a unit has one record, and one more for every border between blocks (warps) that falls into it: numbers unit + block (warp)
    w.rows_own = ratio <= CA_ALONE ? ((int64_t)N * Hkv + grid * CA_WARPS) * ratio : 0;
    w.rows_prompt = P > 0 ? (prompts * Hkv + grid * CA_WARPS) * CA_ALONE : 0;
    w.rows_shared = ((ratio <= CA_ALONE ? prompts : entries) * Hkv + (P > 0 || ratio > CA_ALONE ? grid : 0)) * CA_ROWS;
    uint8_t* p = static_cast<uint8_t*>(base);
    size_t at = 0;
    auto take = [&](size_t n) { uint8_t* q = p + at; at += (n + 255) & ~(size_t)255; return q; };
    const int64_t rows = w.rows_own + w.rows_prompt + w.rows_shared;
    w.owners = reinterpret_cast<int2*>(take((size_t)entries * Hkv * sizeof(int2)));
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
    bool merge_apart;                              // a block of the merge has rows from all over, not one behind another
    int own_most;                                  // tokens that a row of page_table holds
    LineCosts costs;
    float scale_log2;
    uint32_t* status;
};

// ---- the line of pieces.  The host sees to it that its length fits 31 bits.
struct Line {
    int shared, single;      // lengths: units' pieces and setups, the single ones' by their cost
    int per;                 // cost that a block takes
    int cost;                // of a shared piece
    int begin;               // of the single line
};
// Shares are such that every block (warp) between the first and the last that has some of a unit has one of its pieces: a share holds a shared piece, a warp's part of one any
// single piece (`many`: some are of more than eight rows), and the single line begins where four warps have as much of it each, at the next block if that were less.
__device__ __forceinline__ Line make_line(int shared, int single, bool many, int grid, const LineCosts& costs) {
    const int least = CA_WARPS * (many ? costs.many : costs.few);
    Line l = {shared, single, 0, costs.shared, (shared * costs.shared + CA_WARPS - 1) / CA_WARPS * CA_WARPS};
    const int each = max((l.begin + single + least + grid - 1) / grid, max(shared > 0 ? costs.shared : 0, least));
    l.per = (each + CA_WARPS - 1) / CA_WARPS * CA_WARPS;
    const int used = l.begin % l.per;
    if (used > 0 && l.per - used < least) l.begin += l.per - used;
    return l;
}
// the shared line from there on is block b's or a later one's
__device__ __forceinline__ int shared_begin(const Line& l, int b) {
    const int x = (b * l.per + l.cost - 1) / l.cost;
    return x < l.shared ? x : l.shared;
}
// a warp's part of the single line, from y0 to y1 (none where that is not more); warps are counted over all blocks
__device__ __forceinline__ void warp_range(const Line& l, int warp, int& y0, int& y1) {
    const int b = warp / CA_WARPS, k = warp % CA_WARPS;
    const int lo = max(b * l.per - l.begin, 0), each = max((b + 1) * l.per - l.begin - lo, 0) / CA_WARPS;
    y0 = lo + k * each;
    y1 = min(y0 + each, l.single);
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
// Parts of 32 tokens of a piece.
__device__ __forceinline__ int piece_parts(int rows) { return rows > 32 ? 2 : rows > CA_ALONE ? 4 : 1; }
__device__ __forceinline__ int entry_pieces(int rows, int tokens) {
    const int of = CA_TOKENS * piece_parts(rows);             // a power of two
    return (int)(((int64_t)tokens + of - 1) / of);
}
__device__ __forceinline__ int unit_setup(const CacheParams& p, int rows) { return rows > CA_ALONE ? CA_SHARED_SETUP : p.costs.single_setup; }
// of a piece, on its line
__device__ __forceinline__ int piece_length(const CacheParams& p, int rows) { return rows > CA_ALONE ? 1 : rows > 8 ? p.costs.many : p.costs.few; }
// {tokens, rows} of an entry; no rows where it is left out.
__device__ __forceinline__ int2 entry_size(const CacheParams& p, int e, bool& bad) {
    const arrol_cache_attention_args& a = p.a;
    if (e < p.prompts) {
        const int q = e / p.blocks, rollouts = min(live_of(p, q) - (e - q * p.blocks) * p.group, p.group);
        bool wrong = false;
        const int tokens = cache_tokens(a.prompt_lengths, q, a.prompt_table_pages, a.cache.page, wrong);
        if (rollouts <= 0) return make_int2(0, 0);
        bad |= wrong;
        return make_int2(tokens, rollouts * p.ratio);
    }
    const int i = e - p.prompts;
    bool wrong = false;
    const int tokens = cache_tokens(a.lengths, i, a.table_pages, a.cache.page, wrong);      // asked for with the mask, not behind it
    if (a.keep && !a.keep[i]) return make_int2(0, 0);
    bad |= wrong;
    return make_int2(tokens, p.ratio);
}

struct ScanSums {
    int shared, single;      // lengths of the lines
    int shared_entries, single_entries;
};
__device__ __forceinline__ ScanSums operator+(const ScanSums& a, const ScanSums& b) {
    return {a.shared + b.shared, a.single + b.single, a.shared_entries + b.shared_entries, a.single_entries + b.single_entries};
}
__device__ __forceinline__ ScanSums shfl_up(const ScanSums& a, int d) {
    return {__shfl_up_sync(0xffffffffu, a.shared, d), __shfl_up_sync(0xffffffffu, a.single, d), __shfl_up_sync(0xffffffffu, a.shared_entries, d),
            __shfl_up_sync(0xffffffffu, a.single_entries, d)};
}

// Where a block (warp) begins: an entry, its number in the list, how much of it lies before.
struct Start {
    CacheEntry e;
    int offset;
    int number;
};

// bytes that the barrier's phase waits for, without an arrival
__device__ __forceinline__ void mbar_expect_bytes(uint64_t* bar, uint32_t bytes) {
    asm volatile("mbarrier.expect_tx.relaxed.cta.shared::cta.b64 [%0], %1;" ::"r"(smem_u32(bar)), "r"(bytes) : "memory");
}
__device__ __forceinline__ void mbar_arrive_n(uint64_t* bar, uint32_t n) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0], %1;" ::"r"(smem_u32(bar)), "r"(n) : "memory");
}
__device__ __forceinline__ void tma_load_4d(uint32_t dst, const CUtensorMap* map, int y, int z, int w, uint64_t* bar) {
    asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
        ::"r"(dst), "l"(map), "r"(0), "r"(y), "r"(z), "r"(w), "r"(smem_u32(bar)) : "memory");
}
// Four 8 x 16 byte matrices as they lie: a lane (g, t) gets bytes 4 t .. 4 t + 3 of row g of each.
__device__ __forceinline__ void ldmatrix_rows(uint32_t addr, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
// Two 16 x 16 byte matrices transposed: a lane gets bytes g and g + 8 of rows 4 t .. 4 t + 3, a register each.
__device__ __forceinline__ void ldmatrix_columns(uint32_t addr, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m16n16.x2.trans.shared.b8 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}

__device__ __forceinline__ void mma_f16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// An 8 x 8 matrix of pairs of halves transposed: from (row g, columns 2 t and the next) to (column g, rows 2 t and the next).
__device__ __forceinline__ uint32_t transpose_halves(uint32_t v) {
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}
// Four numbers of each of two registers as an operand of sixteen rows: (row g, first two), (row g + 8, first two), (row g, others), (row g + 8, others).
__device__ __forceinline__ void widen(uint32_t (&a)[4], uint32_t v0, uint32_t v1) {
    a[0] = e4m3_pair_to_half((uint16_t)v0);
    a[1] = e4m3_pair_to_half((uint16_t)v1);
    a[2] = e4m3_pair_to_half((uint16_t)(v0 >> 16));
    a[3] = e4m3_pair_to_half((uint16_t)(v1 >> 16));
}
__device__ __forceinline__ uint32_t pack_half(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

// A stage: 32 tokens' keys, then their values, as rows of DP bytes, swizzled by the copies over as many (chunk c of 16 bytes of row r lies where c ^ swizzle(r) would), and
// the four scales (keys' of the first and the second 16 tokens, values') in front of the ring.
template <int DP>
struct CacheConf {
    static constexpr int KEYS = CA_TOKENS * DP, BYTES = 2 * KEYS;
    // Heads up to 64 leave room for a third block (long prompts 191 -> 178 us).  Six consumers a block at 128 registers spill with heads of 128 (283 -> 307 us).
    static constexpr int STAGES = 3, PER_SM = DP == 128 ? 2 : 3;
    static constexpr int CHUNKS = DP / 16;
    static constexpr size_t SMEM = 1024 + (size_t)STAGES * CA_WARPS * BYTES;
    static __device__ __forceinline__ uint32_t at(int row, int chunk) { return row * DP + ((chunk ^ (DP == 128 ? row & 7 : row >> 1 & 3)) << 4); }
};

// Walks over a part of a line, piece by piece: those that begin in it.  What comes next is asked for before it is needed.
struct Cursor {
    CacheEntry e, next;
    const CacheEntry* list;
    int left;                // of the part, from the beginning of the cursor's piece on
    int number, last;        // of the list's entries
    int head, piece, setup, length;
    __device__ __forceinline__ void fetch() {
        if (number + 1 <= last) next = list[number + 1];
    }
    __device__ __forceinline__ void begin(const CacheParams& p, const CacheEntry* l, const Start& s, int entries, int part, int heads) {
        list = l;
        e = s.e;
        number = s.number;
        last = entries - 1;
        left = part;
        setup = unit_setup(p, e.rows);
        length = piece_length(p, e.rows);
        const int unit = e.pieces * length + setup;
        head = s.offset / unit;
        const int at = s.offset - head * unit - setup;
        piece = at > 0 ? (at + length - 1) / length : 0;
        left += at - piece * length;                     // negative: before the unit's first piece
        fetch();
        if (piece == e.pieces) {                         // its last one began before the part
            --piece;
            left += length;
            advance(p, heads);
        }
    }
    __device__ __forceinline__ void advance(const CacheParams& p, int heads) {
        left -= length;
        if (++piece < e.pieces) return;
        piece = 0;
        left -= setup;
        if (++head < heads) return;
        head = 0;
        e = next;
        length = piece_length(p, e.rows);
        ++number;
        fetch();
    }
    // so many pieces on, or past the part's end
    __device__ __forceinline__ void skip(const CacheParams& p, int n, int heads) {
        if (left > 0 && piece + n < e.pieces) {
            piece += n;
            left -= n * length;
            return;
        }
#pragma unroll 1
        for (; n > 0 && left > 0; --n) advance(p, heads);
    }
    // whether the piece is the part's last one
    __device__ __forceinline__ bool is_last() const { return left <= length || (piece == e.pieces - 1 && left <= length + setup); }
};

// Pages of the first and the second 16 tokens from `tok` on, -1 where there are none.
struct PagePair {
    int first, second;
};
__device__ __forceinline__ PagePair find_pages(const CacheParams& p, const Cursor& c, int tok) {
    const int32_t* table = c.e.entry < p.prompts ? p.a.prompt_table + (int64_t)(c.e.entry / p.blocks) * p.a.prompt_table_stride
                                                 : p.a.page_table + (int64_t)(c.e.entry - p.prompts) * p.a.table_stride;
    PagePair g = {-1, -1};
    if (tok < c.e.tokens) g.first = table[tok >> p.page_shift];
    if (tok + 16 < c.e.tokens) g.second = p.page_shift > 4 ? g.first : table[(tok >> 4) + 1];
    return g;
}

// What a consumer has to know of a piece.
struct alignas(16) PieceInfo {
    float scales[4];               // of the keys of the first and the second 16 tokens (below 0: none there), of the values
    int entry, head, there, flags; // there: tokens from its first one to the entry's end
};
// The last of a unit in this block or warp; the first and the last of the unit; no piece, but the end; query rows from bit 8 on.
constexpr int PIECE_LAST = 1, PIECE_BEGIN = 2, PIECE_END = 4, PIECE_NONE = 8, PIECE_ROWS = 8;

// A piece on its way: first its page numbers are asked for, then its scales, then its copies.
struct Fetch {
    PagePair pages;
    int tok;
    PieceInfo info;
    __device__ __forceinline__ void find(const CacheParams& p, const Cursor& c, int token) {
        tok = token;
        pages = find_pages(p, c, token);
        info.entry = c.e.entry;
        info.head = c.head;
        info.there = c.e.tokens - token;
        info.flags = (c.piece == 0 ? PIECE_BEGIN : 0) | (c.piece == c.e.pieces - 1 ? PIECE_LAST | PIECE_END : 0) |
                     (c.is_last() ? PIECE_LAST : 0) | c.e.rows << PIECE_ROWS;
    }
    // pages that are none are reported and left out
    __device__ __forceinline__ void check(const CacheParams& p) {
        const arrol_cache& c = p.a.cache;
        if ((pages.first < 0 && info.there > 0) || pages.first >= c.pages || (pages.second < 0 && info.there > 16) || pages.second >= c.pages) {
            atomicOr(p.status, ARROL_DEV_BAD_INDEX);
            if (pages.first >= c.pages) pages.first = -1;
            if (pages.second >= c.pages) pages.second = -1;
        }
    }
    __device__ __forceinline__ void find_scales(const CacheParams& p) {
        const arrol_cache& c = p.a.cache;
        check(p);
        info.scales[0] = info.scales[1] = -1.f;
        info.scales[2] = info.scales[3] = 0.f;
        if (pages.first >= 0) {
            info.scales[0] = c.k_scale[pages.first * c.k_scale_stride + info.head];
            info.scales[2] = c.v_scale[pages.first * c.v_scale_stride + info.head];
        }
        if (pages.second >= 0) {
            info.scales[1] = c.k_scale[pages.second * c.k_scale_stride + info.head];
            info.scales[3] = c.v_scale[pages.second * c.v_scale_stride + info.head];
        }
        // values that are not there have the others' scale, not one of their own
        if (pages.second < 0) info.scales[3] = info.scales[2];
        if (pages.first < 0) info.scales[2] = info.scales[3];
    }
    // The copies; the arrival that lets the stage be read is the caller's.
    template <int DP>
    __device__ __forceinline__ void copy(const CacheParams& p, const CUtensorMap* map_k, const CUtensorMap* map_v, uint32_t to, uint64_t* full) const {
        using C = CacheConf<DP>;
        const bool whole = p.page_shift > 4;                  // 32 tokens side by side
        if (pages.first >= 0) {
            const int slot = tok & (p.a.cache.page - 1);
            mbar_expect_bytes(full, whole ? C::BYTES : C::KEYS);
            tma_load_4d(to, map_k, slot, info.head, pages.first, full);
            tma_load_4d(to + C::KEYS, map_v, slot, info.head, pages.first, full);
        }
        if (!whole && pages.second >= 0) {
            mbar_expect_bytes(full, C::KEYS);
            tma_load_4d(to + C::KEYS / 2, map_k, 0, info.head, pages.second, full);
            tma_load_4d(to + C::KEYS + C::KEYS / 2, map_v, 0, info.head, pages.second, full);
        }
    }
};

// A tile of up to 16 query rows against the pieces of its unit.  A lane (g, t) = (lane / 4, lane % 4) has the scores of query rows 2 t and 2 t + 1 (of each eight) with
// tokens g and, of the second eight of sixteen, 8 + (g + 4) % 8: in that order eight rows of keys, and the sixteen of values that a lane's four scores belong to, are read
// without two in a bank.
template <int DP>
struct RowTile {
    using C = CacheConf<DP>;
    uint32_t q[C::CHUNKS][2][2];      // per 16 dimensions and eight rows: row g's dimensions 4 t .. 4 t + 3
    float by[2][2];                   // what a product's sum times the key's scale is multiplied by
    float o[C::CHUNKS][2][4], m[2][2], l[2][2];
    float v_scale, v_least;           // largest scale of the values so far, o is in units of it / CA_P_SCALE; the smallest

    // `row`: this lane's row g, or null; r: of the first or the second eight
    __device__ __forceinline__ void load(const CacheParams& p, int lane, const __nv_bfloat16* row, int r) {
        const int t = lane & 3, D = p.a.cache.D;
        uint2 raw[C::CHUNKS];
#pragma unroll
        for (int x = 0; x < C::CHUNKS; ++x) raw[x] = row && x * 16 < D ? *reinterpret_cast<const uint2*>(row + x * 16 + t * 4) : make_uint2(0, 0);
        {
            float most = 0.f, odd = 0.f;
#pragma unroll
            for (int x = 0; x < C::CHUNKS; ++x)
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    const uint32_t w = y ? raw[x].y : raw[x].x;
                    const float a = __uint_as_float(w << 16), b = __uint_as_float(w & 0xFFFF0000u);
                    most = finite_max(finite_max(most, a), b);
                    odd += (a - a) + (b - b);                 // NaN where one is not finite
                }
#pragma unroll
            for (int s = 1; s < 4; s <<= 1) {
                most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, s));
                odd += __shfl_xor_sync(0xffffffffu, odd, s);
            }
            const int e = cache_exponent(most) - 5;           // up to 448 x 2^5 = 14,336, a quarter of fp16's largest
            const float down = cache_power(-e), mine = cache_power(e) * p.scale_log2 + odd;      // a query that is not finite makes its scores NaN
            by[r][0] = __shfl_sync(0xffffffffu, mine, t * 8);
            by[r][1] = __shfl_sync(0xffffffffu, mine, t * 8 + 4);
#pragma unroll
            for (int x = 0; x < C::CHUNKS; ++x)
#pragma unroll
                for (int y = 0; y < 2; ++y) {
                    const uint32_t w = y ? raw[x].y : raw[x].x;
                    q[x][r][y] = pack_half(__uint_as_float(w << 16) * down, __uint_as_float(w & 0xFFFF0000u) * down);
                }
        }
#pragma unroll
        for (int c = 0; c < C::CHUNKS; ++c) o[c][r][0] = o[c][r][1] = o[c][r][2] = o[c][r][3] = 0.f;
        m[r][0] = m[r][1] = -INFINITY;
        l[r][0] = l[r][1] = 0.f;
        v_scale = 0.f;
        v_least = INFINITY;
    }

    // The second eight rows as rows without a query: scores 0 against a reference of 0, which asks for nothing.  (Loading them as such took 142 us where this took 140.7, long prompts.)
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int x = 0; x < C::CHUNKS; ++x) { q[x][1][0] = q[x][1][1] = 0u; o[x][1][0] = o[x][1][1] = o[x][1][2] = o[x][1][3] = 0.f; }
        by[1][0] = by[1][1] = 0.f;
        m[1][0] = m[1][1] = l[1][0] = l[1][1] = 0.f;
    }

    // A piece with at least one token, ROWS x 8 query rows.
    template <int ROWS>
    __device__ __forceinline__ void piece(uint8_t* stage, const PieceInfo& info, int lane) {
        const int g = lane >> 2, there = info.there;
        const float4 scales = *reinterpret_cast<const float4*>(info.scales);
        const uint32_t keys = smem_u32(stage), values = keys + C::KEYS;
        const int later = (lane >> 3) & 1, row = later * 8 + ((lane + 4 * later) & 7);
        float s[2][ROWS][4];
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
            for (int r = 0; r < ROWS; ++r) s[half][r][0] = s[half][r][1] = s[half][r][2] = s[half][r][3] = 0.f;
#pragma unroll
        for (int c = 0; c < C::CHUNKS; c += 2)
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                uint32_t w[4], a[4];
                ldmatrix_rows(keys + C::at(half * 16 + row, c + (lane >> 4)), w);
                widen(a, w[0], w[1]);
#pragma unroll
                for (int r = 0; r < ROWS; ++r) mma_f16(s[half][r], a, q[c][r][0], q[c][r][1]);
                widen(a, w[2], w[3]);
#pragma unroll
                for (int r = 0; r < ROWS; ++r) mma_f16(s[half][r], a, q[c + 1][r][0], q[c + 1][r][1]);
            }
        float f[2][ROWS][2];
#pragma unroll
        for (int r = 0; r < ROWS; ++r)
#pragma unroll
            for (int b = 0; b < 2; ++b) { f[0][r][b] = by[r][b] * scales.x; f[1][r][b] = by[r][b] * scales.y; }
        if (__builtin_expect(there < CA_TOKENS || scales.x < 0.f || scales.y < 0.f, 0)) {
            // tokens behind the unit's last, or on a page that is none: no weight, and nothing that 0 times it would not make 0
            const int most[2] = {scales.x < 0.f ? 0 : there, scales.y < 0.f ? 0 : there};      // tokens below these are there, in either half
#pragma unroll
            for (int half = 0; half < 2; ++half)
#pragma unroll
                for (int x = 0; x < 2; ++x)
                    if (half * 16 + (x ? 8 + ((g + 4) & 7) : g) >= most[half])
#pragma unroll
                        for (int r = 0; r < ROWS; ++r) s[half][r][2 * x] = s[half][r][2 * x + 1] = -INFINITY;
#pragma unroll
            for (int half = 0; half < 2; ++half)              // minus infinity stays that
#pragma unroll
                for (int r = 0; r < ROWS; ++r)
#pragma unroll
                    for (int b = 0; b < 2; ++b) f[half][r][b] = f[half][r][b] <= 0.f ? 1e-37f : f[half][r][b];
            for (int x = lane; x < CA_TOKENS * C::CHUNKS; x += 32) {
                const int token = x / C::CHUNKS;
                if (token >= most[token >> 4]) *reinterpret_cast<uint4*>(stage + C::KEYS + x * 16) = make_uint4(0, 0, 0, 0);
            }
            __syncwarp();
        }
        // The reference is let fall up to 2^8 behind the maximum: only where some row is further behind do its eight lanes settle on a new one.
        float mx[ROWS][2];
        bool behind = false;
#pragma unroll
        for (int r = 0; r < ROWS; ++r)
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                mx[r][b] = fmaxf(fmaxf(s[0][r][b], s[0][r][2 + b]) * f[0][r][b], fmaxf(s[1][r][b], s[1][r][2 + b]) * f[1][r][b]);
                behind |= mx[r][b] > m[r][b] + CA_RESCALE_AT;
            }
        const float vs = fmaxf(scales.z, scales.w);
        v_least = fminf(v_least, fminf(scales.z, scales.w));
        if (__builtin_expect(__any_sync(0xffffffffu, behind || vs > v_scale), 0)) {
            const float shrink = vs > v_scale ? v_scale / vs : 1.f;
            v_scale = fmaxf(vs, v_scale);
#pragma unroll
            for (int r = 0; r < ROWS; ++r)
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    float top = mx[r][b], up = shrink;
#pragma unroll
                    for (int d = 4; d < 32; d <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
                    if (top > m[r][b] + CA_RESCALE_AT) {
                        const float fall = ex2_approx(m[r][b] - top);
                        m[r][b] = top;
                        l[r][b] *= fall;
                        up *= fall;
                    }
#pragma unroll
                    for (int c = 0; c < C::CHUNKS; ++c) { o[c][r][b] *= up; o[c][r][2 + b] *= up; }
                }
        }
        const float inv = v_scale > 0.f ? CA_P_SCALE / v_scale : 0.f, w[2] = {scales.z * inv, scales.w * inv};
        uint32_t pt[2][ROWS][2];
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
            for (int r = 0; r < ROWS; ++r) {
                float e[4];
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const float sub = m[r][x & 1] == -INFINITY ? 0.f : m[r][x & 1];
                    e[x] = ex2_approx(fmaf(s[half][r][x], f[half][r][x & 1], -sub));
                    l[r][x & 1] += e[x];
                }
                pt[half][r][0] = transpose_halves(pack_half(e[0] * w[half], e[1] * w[half]));
                pt[half][r][1] = transpose_halves(pack_half(e[2] * w[half], e[3] * w[half]));
            }
        // row i of 16: tokens 2 t and the next (i % 4 < 2) and their likes of the second eight, t = i / 4
        const int i = lane & 15, of = (i >> 2) * 2 + (i & 1), token = i & 2 ? 8 + ((of + 4) & 7) : of;
#pragma unroll
        for (int c = 0; c < C::CHUNKS; c += 2)
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                uint32_t v[4], a[4];
                ldmatrix_columns(values + C::at(half * 16 + token, c + (lane >> 4)), v);
                widen(a, v[0], v[1]);
#pragma unroll
                for (int r = 0; r < ROWS; ++r) mma_f16(o[c][r], a, pt[half][r][0], pt[half][r][1]);
                widen(a, v[2], v[3]);
#pragma unroll
                for (int r = 0; r < ROWS; ++r) mma_f16(o[c + 1][r], a, pt[half][r][0], pt[half][r][1]);
            }
    }

    // Sums of the first or the second eight rows, as far as the tile has them, to record rows `at`, ...
    __device__ __forceinline__ void store(const CacheParams& p, int64_t at, int rows, int lane, int r) {
        const int g = lane >> 2, t = lane & 3, D = p.a.cache.D;
        const float unit = v_scale * (1.f / CA_P_SCALE);
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                float sum = l[r][b];
#pragma unroll
                for (int d = 4; d < 32; d <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
                const int row = 8 * r + 2 * t + b;
                if (row < rows) {
                    float* out = p.w.o + (at + row) * D + g;
#pragma unroll
                    for (int c = 0; c < C::CHUNKS; ++c)
                        if (c * 16 < D) {
                            out[c * 16] = o[c][r][b] * unit;
                            out[c * 16 + 8] = o[c][r][2 + b] * unit;
                        }
                    if (g == 0) p.w.ml[at + row] = make_float2(m[r][b], v_least < v_scale * CA_NEAR ? -sum : sum);      // marked
                }
            }
    }
};

struct CacheShared {
    PieceInfo info[4][CA_WARPS];       // per stage and warp, as the barriers
    uint64_t full[4][CA_WARPS], empty[4][CA_WARPS];
    ScanSums warp_sums[CA_WARPS + 1];
    Start shared, single[CA_WARPS];
    int live[CA_WARPS][CA_ROWS];       // rollouts of a prompt entry, per warp
    int2 sizes[CA_SCANNED];            // the entries' tokens and rows
    uint32_t abort;
};

// Who has the unit's first and last piece, for the merge.
__device__ __forceinline__ void tell_owner(const CacheParams& p, const PieceInfo& e, int owner) {
    int2* const at = p.w.owners + (int64_t)e.entry * p.a.cache.Hkv + e.head;
    if (e.flags & PIECE_BEGIN) at->x = owner;
    if (e.flags & PIECE_END) at->y = owner;
}
// Query row `row` of an entry's unit, if it has so many.
__device__ __forceinline__ const __nv_bfloat16* query_row(const CacheParams& p, const PieceInfo& e, const int* live, int row) {
    if (row >= e.flags >> PIECE_ROWS) return nullptr;
    const int of = row / p.ratio, i = e.entry < p.prompts ? live[of] : e.entry - p.prompts;
    return static_cast<const __nv_bfloat16*>(p.a.q) + i * p.a.q_stride + (int64_t)(e.head * p.ratio + row - of * p.ratio) * p.a.cache.D;
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
__global__ void __launch_bounds__(CA_THREADS, CacheConf<DP>::PER_SM) cache_units_kernel(const __grid_constant__ CUtensorMap map_k, const __grid_constant__ CUtensorMap map_v, const CacheParams p) {
    using C = CacheConf<DP>;
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(16) CacheShared sm;
    uint8_t* const ring = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    volatile uint32_t* abort_flag = &sm.abort;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, Hkv = p.a.cache.Hkv;
    if (threadIdx.x == 0) {
        for (int i = 0; i < C::STAGES * CA_WARPS; ++i) {
            mbar_init(&sm.full[i / CA_WARPS][i % CA_WARPS], 1);
            mbar_init(&sm.empty[i / CA_WARPS][i % CA_WARPS], CA_WARPS);
        }
        sm.abort = 0u;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        if (p.a.cache.pages > 0) {
            asm volatile("prefetch.tensormap [%0];" ::"l"(&map_k) : "memory");
            asm volatile("prefetch.tensormap [%0];" ::"l"(&map_v) : "memory");
        }
    }
    __syncthreads();
    pdl_launch_dependents();
    pdl_wait();
    const int b = blockIdx.x;

    // ---- the scan: sizes of the entries, side by side; then a thread has `each` entries in a row, twice (sums, and what is this block's)
    bool bad = false;
    constexpr int AT_ONCE = 4;                                // entries of a thread whose lengths are on their way together
    for (int e0 = threadIdx.x; e0 < min(p.entries, CA_SCANNED); e0 += AT_ONCE * CA_THREADS) {
        int n[AT_ONCE], kept[AT_ONCE];
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i) {
            const int own = e0 + i * CA_THREADS - p.prompts;
            n[i] = kept[i] = 0;
            if (own >= 0 && own < p.a.N) {
                n[i] = p.a.lengths[own];
                kept[i] = p.a.keep ? p.a.keep[own] : 1;
            }
        }
#pragma unroll
        for (int i = 0; i < AT_ONCE; ++i) {
            const int e = e0 + i * CA_THREADS;
            if (e >= min(p.entries, CA_SCANNED)) break;
            if (e < p.prompts) {
                sm.sizes[e] = entry_size(p, e, bad);
            } else {
                const bool fits = n[i] >= 0 && n[i] <= p.own_most;
                bad |= kept[i] && !fits;
                sm.sizes[e] = kept[i] && fits ? make_int2(n[i], p.ratio) : make_int2(0, 0);
            }
        }
    }
    __syncthreads();
    const int each = (p.entries + CA_THREADS - 1) / CA_THREADS;
    const int e0 = min((int)threadIdx.x * each, p.entries), e1 = min(e0 + each, p.entries);
    auto size = [&](int e) { return e < CA_SCANNED ? sm.sizes[e] : entry_size(p, e, bad); };
    auto length = [&](int2 x) { return (entry_pieces(x.y, x.x) * piece_length(p, x.y) + unit_setup(p, x.y)) * Hkv; };
    ScanSums mine = {0, 0, 0, 0};
    bool many = false;
    for (int e = e0; e < e1; ++e) {
        const int2 x = size(e);
        if (x.x == 0) continue;
        many |= x.y > 8 && x.y <= CA_ALONE;
        if (x.y > CA_ALONE) { mine.shared += length(x); ++mine.shared_entries; }
        else { mine.single += length(x); ++mine.single_entries; }
    }
    if (bad && b == 0) atomicOr(p.status, ARROL_DEV_BAD_INDEX);
    ScanSums sum = mine;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const ScanSums x = shfl_up(sum, d);
        if (lane >= d) sum = sum + x;
    }
    if (lane == 31) sm.warp_sums[warp] = sum;
    many = __syncthreads_or(many);
    ScanSums total = {0, 0, 0, 0}, at = {sum.shared - mine.shared, sum.single - mine.single, sum.shared_entries - mine.shared_entries, sum.single_entries - mine.single_entries};
#pragma unroll
    for (int w = 0; w < CA_WARPS + 1; ++w) {
        if (w < warp) at = at + sm.warp_sums[w];
        total = total + sm.warp_sums[w];
    }
    const Line line = make_line(total.shared, total.single, many, p.grid, p.costs);
    const int x0 = shared_begin(line, b), x1 = shared_begin(line, b + 1);
    int y0[CA_WARPS], y1[CA_WARPS];
#pragma unroll
    for (int w = 0; w < CA_WARPS; ++w) warp_range(line, b * CA_WARPS + w, y0[w], y1[w]);
    const int block_y1 = max(max(y1[0], y1[1]), max(y1[2], y1[3]));
    if (mine.shared > 0 && at.shared < x1 && at.shared + mine.shared > x0)
        for (int e = e0; e < e1; ++e) {
            const int2 x = size(e);
            if (x.x == 0 || x.y <= CA_ALONE) continue;
            const int n = length(x);
            const CacheEntry entry = {e, x.x, x.y, entry_pieces(x.y, x.x)};
            if (at.shared < x1 && at.shared + n > x0) p.w.shared[at.shared_entries] = entry;                 // neighbours write the same
            if (at.shared <= x0 && at.shared + n > x0) sm.shared = {entry, x0 - at.shared, at.shared_entries};
            at.shared += n;
            ++at.shared_entries;
        }
    if (mine.single > 0 && at.single < block_y1 && at.single + mine.single > y0[0])
        for (int e = e0; e < e1; ++e) {
            const int2 x = size(e);
            if (x.x == 0 || x.y > CA_ALONE) continue;
            const int n = length(x);
            if (at.single < block_y1 && at.single + n > y0[0]) {
                const CacheEntry entry = {e, x.x, x.y, entry_pieces(x.y, x.x)};
                p.w.single[at.single_entries] = entry;
#pragma unroll
                for (int w = 0; w < CA_WARPS; ++w)
                    if (at.single <= y0[w] && at.single + n > y0[w]) sm.single[w] = {entry, y0[w] - at.single, at.single_entries};
            }
            at.single += n;
            ++at.single_entries;
        }
    __syncthreads();

    // Stages are filled and read in turn, from the first shared piece to the last single one, behind which comes one that says so.  A consumer of shared pieces waits for all
    // four parts of a stage, those that it does not read too: a later wait for one of them by its parity alone would otherwise pass for a filling that is two ahead.
    auto stage = [&](uint32_t n, int w) { return ring + (size_t)(n % C::STAGES * CA_WARPS + w) * C::BYTES; };
    bool ok = true;
    if (warp == CA_WARPS) {
        // ---- the producer: eight lanes for each consumer, which look up eight pieces at once, the next eight while these are copied, and copy one after another
        const int of = lane >> 3, k = lane & 7;
        const uint32_t eight = 0xFFu << (of * 8);
        uint32_t n = 0, asked = 0;                            // pieces of this consumer before the eight, asked for so far
        for (int phase = 0; phase < 2 && ok; ++phase) {
            int from, to;
            warp_range(line, b * CA_WARPS + of, from, to);
            if (phase == 0) { from = x0; to = x1; }
            Cursor c;
            c.left = 0;
            if (from < to) c.begin(p, phase ? p.w.single : p.w.shared, phase ? sm.single[of] : sm.shared, phase ? total.single_entries : total.shared_entries, to - from, Hkv);
            // a part that its piece does not have begins where no tokens are
            auto token = [&] { const int parts = piece_parts(c.e.rows); return phase ? c.piece * CA_TOKENS : of < parts ? (c.piece * parts + of) * CA_TOKENS : c.e.tokens; };
            for (int i = 0; i < k && c.left > 0; ++i) c.advance(p, Hkv);
            Fetch now, next;
            bool there = c.left > 0, more = false;
            bool copied = false;
            if (there) {
                now.find(p, c, token());
                // The very first pieces find their stages free: their copies need not wait for the scales.
                if (n == 0 && k < C::STAGES) {
                    now.check(p);
                    now.copy<DP>(p, &map_k, &map_v, smem_u32(stage(k, of)), &sm.full[k][of]);
                    copied = true;
                }
                now.find_scales(p);
            }
            // Each consumer's eight lanes go on by themselves: `at` is the lane whose turn it is, a stage that is not free yet is asked for again in the next round.
            int at = 8;
            uint32_t fresh = 0;                               // rounds without any progress
            bool begun = false;
            for (;;) {
                const uint32_t all = __ballot_sync(0xffffffffu, there) & eight;
                if (at == 8 || at >= __popc(all)) {           // the next eight
                    if (begun) {
                        n += __popc(all);
                        there = more;
                        now = next;
                    }
                    begun = true;
                    at = 0;
                    c.skip(p, 8, Hkv);
                    more = there && c.left > 0;
                    if (more) next.find(p, c, token());
                }
                if (!__any_sync(0xffffffffu, there)) break;
                const uint32_t mine = n + k, st = mine % C::STAGES;
                const bool turn = there && k == at, go = turn && mbar_try_wait(&sm.empty[st][of], ((mine / C::STAGES) & 1u) ^ 1u);
                if (go) {
                    if (!copied) now.copy<DP>(p, &map_k, &map_v, smem_u32(stage(mine, of)), &sm.full[st][of]);
                    copied = false;
                    sm.info[st][of] = now.info;
                    mbar_arrive(&sm.full[st][of]);
                    if (phase || of == 0) tell_owner(p, now.info, (int)(phase ? b * CA_WARPS + of : b));
                }
                const uint32_t went = __ballot_sync(0xffffffffu, go);
                if (went & eight) {
                    ++at;
                    ++asked;
                    if (at == 4 && more) next.find_scales(p);
                }
                fresh = went ? 0 : fresh + 1;
                if (fresh > SPIN_LIMIT || ((fresh & 1023u) == 1023u && __any_sync(0xffffffffu, *abort_flag != 0u))) { *abort_flag = 1u; ok = false; break; }
            }
            if (!ok && copied) {                              // a copy whose stage nobody has been told of
                mbar_arrive(&sm.full[k][of]);
                for (uint32_t spin = 0; spin < SPIN_LIMIT; ++spin)
                    if (mbar_try_wait(&sm.full[k][of], 0u)) break;
            }
        }
        if (k == 0) {
            if (ok && mbar_wait(&sm.empty[n % C::STAGES][of], ((n / C::STAGES) & 1u) ^ 1u, abort_flag)) {
                sm.info[n % C::STAGES][of].flags = PIECE_NONE;
                mbar_arrive(&sm.full[n % C::STAGES][of]);
            } else {
                // let the copies in flight land before the block's shared memory goes away (all have, unless a wait ran out)
                for (uint32_t i = asked > C::STAGES ? asked - C::STAGES : 0; i < asked; ++i)
                    for (uint32_t spin = 0; spin < SPIN_LIMIT; ++spin)
                        if (mbar_try_wait(&sm.full[i % C::STAGES][of], (i / C::STAGES) & 1u)) break;
            }
        }
        __syncwarp();
    } else {
        // Units one behind another.  What a unit's pieces have in common stands outside their loop, which is kept short: a warp that jumps over code that it seldom needs waits
        // for instructions each time.
        RowTile<DP> tile;
        for (uint32_t n = 0; ok;) {
            if (!mbar_wait_warp(&sm.full[n % C::STAGES][warp], (n / C::STAGES) & 1u, abort_flag)) break;
            const PieceInfo& e = sm.info[n % C::STAGES][warp];
            const int rows = e.flags >> PIECE_ROWS, entry = e.entry, head = e.head;
            if (e.flags & PIECE_NONE) break;
            // a shared piece: a tile of 16 rows a warp; with two tiles two warps share a tile's tokens
            const bool shared = rows > CA_ALONE;
            const int row_tiles = rows > 32 ? 4 : 2, row0 = shared ? (warp & (row_tiles - 1)) * 16 : 0, left = rows - row0, share = shared ? warp / row_tiles : warp;
            if (left > 0) {
                if (entry < p.prompts) find_live(p, entry, sm.live[warp], lane);
                tile.load(p, lane, query_row(p, e, sm.live[warp], row0 + (lane >> 2)), 0);
                if (left > 8) tile.load(p, lane, query_row(p, e, sm.live[warp], row0 + 8 + (lane >> 2)), 1);
            }
            auto single_pieces = [&](auto eights) {
                for (;;) {
                    const uint32_t st = n % C::STAGES;
                    const PieceInfo& piece = sm.info[st][warp];
                    tile.template piece<decltype(eights)::value>(stage(n, warp), piece, lane);
                    const bool last = piece.flags & PIECE_LAST;
                    // what was read by instructions comes before the copies that fill the stage again
                    fence_proxy_async_smem();
                    __syncwarp();
                    if (lane == 0) mbar_arrive_n(&sm.empty[st][warp], CA_WARPS);
                    ++n;
                    if (last) break;
                    if (!mbar_wait_warp(&sm.full[n % C::STAGES][warp], (n / C::STAGES) & 1u, abort_flag)) { ok = false; break; }
                }
            };
            if (shared) {
                if (left <= 8) tile.clear();
                for (;;) {
                    const uint32_t st = n % C::STAGES, parity = (n / C::STAGES) & 1u;
                    ok = mbar_wait_warp(&sm.full[st][lane % CA_WARPS], parity, abort_flag);       // all four at once, a lane each
                    if (!ok) break;
                    __syncwarp();                             // the vote orders nothing: each lane has learnt of one part only
                    for (int w = share; w < CA_WARPS; w += CA_WARPS / row_tiles)
                        if (sm.info[st][w].there > 0 && left > 0) tile.template piece<2>(stage(n, w), sm.info[st][w], lane);
                    const bool last = sm.info[st][warp].flags & PIECE_LAST;
                    fence_proxy_async_smem();
                    __syncwarp();
                    if (lane < CA_WARPS) mbar_arrive(&sm.empty[st][lane]);
                    ++n;
                    if (last) break;
                }
            } else if (left > 8) {
                single_pieces(std::integral_constant<int, 2>());
            } else {
                single_pieces(std::integral_constant<int, 1>());
            }
            if (!ok) break;
            if (left > 0) {
                const int64_t unit = (int64_t)entry * Hkv + head, owner = b * CA_WARPS + warp;
                const int64_t record = shared ? p.w.rows_own + p.w.rows_prompt + (unit + b) * CA_ROWS + (row_tiles == 2 ? share * 32 : 0) + row0
                                     : entry < p.prompts ? p.w.rows_own + (unit + owner) * CA_ALONE : (unit - (int64_t)p.prompts * Hkv + owner) * p.ratio;
                tile.store(p, record, left, lane, 0);
                if (left > 8) tile.store(p, record, left, lane, 1);
            }
        }
    }
    __syncthreads();
    if (threadIdx.x == 0 && *abort_flag) atomicOr(p.status, ARROL_DEV_WAIT_EXPIRED);
}

// A warp, or with heads up to 64 half a warp, per (rollout, query head): the prompt's records, then its own, in order; four dimensions a lane.  Records are asked for eight
// at a time.
struct Merged {
    static constexpr int AT_ONCE = 8;
    float top, total;
    float4 sum;
    float least;               // of the records' sums: below 0 where one is marked
    __device__ __forceinline__ void add(const float2 (&x)[AT_ONCE], const float4 (&v)[AT_ONCE]) {
        float next = top;
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) next = fmaxf(next, x[k].x);
        const float up = next == -INFINITY ? 1.f : ex2_approx(top - next);
        total *= up;
        sum.x *= up; sum.y *= up; sum.z *= up; sum.w *= up;
        top = next;
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) {
            const float by = x[k].x == -INFINITY ? (x[k].y == 0.f ? 0.f : 1.f) : ex2_approx(x[k].x - top);      // a NaN without a maximum stays one
            least = fminf(least, x[k].y);
            total += by * x[k].y;
            sum.x += by * v[k].x; sum.y += by * v[k].y; sum.z += by * v[k].z; sum.w += by * v[k].w;
        }
    }
    // `any`: there are keys
    __device__ __forceinline__ void write(const arrol_cache_attention_args& a, int64_t row, int i, int hq, int lane, bool any) const {
        const int D = a.cache.D, d = lane * 4;
        const float inv = any ? 1.f / total : 0.f;
        if (d < D) {
            uint2 w = make_uint2(0u, 0u);
            if (any) {
                asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w.x) : "f"(sum.y * inv), "f"(sum.x * inv));
                asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w.y) : "f"(sum.w * inv), "f"(sum.z * inv));
            }
            *reinterpret_cast<uint2*>(static_cast<__nv_bfloat16*>(a.o) + i * a.o_stride + (int64_t)hq * D + d) = w;
        }
        if (lane == 0 && a.lse) a.lse[row] = any ? (top + log2f(total)) * LN2 : -INFINITY;
    }
};

constexpr int MERGE_THREADS = 256, MERGE_WARPS = MERGE_THREADS / 32;
struct ApartShared {
    int apart[MERGE_THREADS / 16];
    float q[CACHE_MAX_D], m[MERGE_WARPS], l[MERGE_WARPS];
    float4 o[MERGE_WARPS][32];
};
// A row from the pages themselves, all in fp32, by a whole block, for rows with a marked record: 32 tokens a warp, a lane a token for the scores, four dimensions a lane for the values.
// Slow (about 10 us a row for every 500 tokens, eight rows a block one behind another), for caches whose values hardly occur.  Forms for such pieces among the products (sums of
// their own, joined in fp32; a unit that follows the scales; records that are added to) took 5 to 60 % from all other calls, by instructions and registers alone; this takes 1 to 4.
__device__ __noinline__ void row_apart(const CacheParams& p, int64_t row, ApartShared& sm) {
    const arrol_cache_attention_args& a = p.a;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, D = a.cache.D, d = lane * 4;
    const int i = (int)(row / a.Hq), hq = (int)(row - (int64_t)i * a.Hq), h = hq / p.ratio;
    // the query as in RowTile::load
    uint2 raw = make_uint2(0u, 0u);
    if (d < D) raw = *reinterpret_cast<const uint2*>(static_cast<const __nv_bfloat16*>(a.q) + i * a.q_stride + (int64_t)hq * D + d);
    const float x[4] = {__uint_as_float(raw.x << 16), __uint_as_float(raw.x & 0xFFFF0000u), __uint_as_float(raw.y << 16), __uint_as_float(raw.y & 0xFFFF0000u)};
    float most = 0.f, odd = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) { most = finite_max(most, x[j]); odd += x[j] - x[j]; }
#pragma unroll
    for (int s = 1; s < 32; s <<= 1) { most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, s)); odd += __shfl_xor_sync(0xffffffffu, odd, s); }
    const int exponent = cache_exponent(most) - 5;
    const float by = cache_power(exponent) * p.scale_log2 + odd;
    if (warp == 0 && d < D)
#pragma unroll
        for (int j = 0; j < 4; ++j) sm.q[d + j] = x[j] * cache_power(-exponent);
    __syncthreads();
    bool bad = false;
    const int own = cache_tokens(a.lengths, i, a.table_pages, a.cache.page, bad);
    const int prompt = p.prompts ? cache_tokens(a.prompt_lengths, i / a.G, a.prompt_table_pages, a.cache.page, bad) : 0;
    const uint8_t* const k_cache = static_cast<const uint8_t*>(a.cache.k_cache);
    const uint8_t* const v_cache = static_cast<const uint8_t*>(a.cache.v_cache);
    const int64_t tokens = (int64_t)prompt + own;
    float m = -INFINITY, l = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
    for (int64_t t0 = warp * 32; t0 < tokens; t0 += MERGE_THREADS) {
        const int64_t token = t0 + lane;
        int page = -1, slot = 0;
        if (token < tokens) {
            const bool shared = token < prompt;
            const int at = (int)(shared ? token : token - prompt);
            page = shared ? a.prompt_table[(int64_t)(i / a.G) * a.prompt_table_stride + (at >> p.page_shift)] : a.page_table[(int64_t)i * a.table_stride + (at >> p.page_shift)];
            slot = at & (a.cache.page - 1);
            if (page >= a.cache.pages) page = -1;
        }
        float z = -INFINITY, vs = 0.f;
        const int64_t inside = ((int64_t)h * a.cache.page + slot) * D;
        if (page >= 0) {
            const uint8_t* const key = k_cache + page * a.cache.k_page_stride + inside;
            float dot = 0.f;
#pragma unroll 4
            for (int c = 0; c < D; c += 16) {
                const uint4 w = *reinterpret_cast<const uint4*>(key + c);
                const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float2 lo = e4m3_pair_to_float((uint16_t)u[j]), hi = e4m3_pair_to_float((uint16_t)(u[j] >> 16));
                    const float4 q = *reinterpret_cast<const float4*>(&sm.q[c + 4 * j]);
                    dot = fmaf(lo.x, q.x, fmaf(lo.y, q.y, fmaf(hi.x, q.z, fmaf(hi.y, q.w, dot))));
                }
            }
            z = dot * (by * a.cache.k_scale[page * a.cache.k_scale_stride + h]);
            vs = a.cache.v_scale[page * a.cache.v_scale_stride + h];
        }
        float top = fmaxf(m, z);                              // a NaN is passed over
#pragma unroll
        for (int s = 1; s < 32; s <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, s));
        const float e = ex2_approx(z - (top == -INFINITY ? 0.f : top)), fall = top == m ? 1.f : ex2_approx(m - top), weight = e * vs;
        m = top;
        l = fmaf(l, fall, e);
#pragma unroll
        for (int j = 0; j < 4; ++j) o[j] *= fall;
        const uint64_t value = reinterpret_cast<uint64_t>(v_cache) + (page >= 0 ? page * a.cache.v_page_stride + inside : 0);
        const uint32_t there = __ballot_sync(0xffffffffu, page >= 0);
#pragma unroll 1
        for (int t = 0; t < 32 && there >> t; t += 8) {
            uint32_t u[8];
            float w[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                w[j] = __shfl_sync(0xffffffffu, weight, t + j);
                const uint64_t at = __shfl_sync(0xffffffffu, value, t + j);
                u[j] = d < D && (there >> (t + j) & 1u) ? *reinterpret_cast<const uint32_t*>(at + d) : 0u;
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float2 lo = e4m3_pair_to_float((uint16_t)u[j]), hi = e4m3_pair_to_float((uint16_t)(u[j] >> 16));
                o[0] = fmaf(w[j], lo.x, o[0]); o[1] = fmaf(w[j], lo.y, o[1]); o[2] = fmaf(w[j], hi.x, o[2]); o[3] = fmaf(w[j], hi.y, o[3]);
            }
        }
    }
#pragma unroll
    for (int s = 1; s < 32; s <<= 1) l += __shfl_xor_sync(0xffffffffu, l, s);
    if (lane == 0) { sm.m[warp] = m; sm.l[warp] = l; }
    sm.o[warp][lane] = make_float4(o[0], o[1], o[2], o[3]);
    __syncthreads();
    if (warp == 0) {
        float top = -INFINITY, total = 0.f;
        float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
        for (int w = 0; w < MERGE_WARPS; ++w) top = fmaxf(top, sm.m[w]);
#pragma unroll 1
        for (int w = 0; w < MERGE_WARPS; ++w) {
            const float by = sm.m[w] == -INFINITY ? (sm.l[w] == 0.f ? 0.f : 1.f) : ex2_approx(sm.m[w] - top);
            const float4 v = sm.o[w][lane];
            total += by * sm.l[w];
            sum.x += by * v.x; sum.y += by * v.y; sum.z += by * v.z; sum.w += by * v.w;
        }
        const Merged all = {top, total, sum, 0.f};
        all.write(a, row, i, hq, lane, true);
    }
    __syncthreads();
}

template <int LANES>
__global__ void __launch_bounds__(MERGE_THREADS, 3) cache_merge_kernel(const __grid_constant__ CacheParams p) {
    pdl_launch_dependents();
    pdl_wait();
    const arrol_cache_attention_args& a = p.a;
    const int lane = threadIdx.x % LANES, part = (threadIdx.x & 31) - lane, D = a.cache.D, Hkv = a.cache.Hkv, d = lane * 4;
    const int64_t step = p.merge_apart ? gridDim.x : 1, first = p.merge_apart ? blockIdx.x : (int64_t)blockIdx.x * (MERGE_THREADS / LANES);
    const int64_t rows = (int64_t)a.N * a.Hq, asked = first + (int64_t)(threadIdx.x / LANES) * step, row = asked < rows ? asked : rows - 1;      // both halves go on together
    const int i = (int)(row / a.Hq), hq = (int)(row - (int64_t)i * a.Hq), h = hq / p.ratio, r = hq - h * p.ratio;
    const int2* owners = pdl_acquire(p.w.owners);
    const float2* ml = pdl_acquire(p.w.ml);
    const float* o = pdl_acquire(p.w.o);
    bool bad = false;
    const int own_tokens = cache_tokens(a.lengths, i, a.table_pages, a.cache.page, bad);
    const int2 own = owners[(int64_t)(p.prompts + i) * Hkv + h];       // nothing known where there are no tokens: not used there
    int prompt_tokens = 0, prompt_rows = 0, prompt_row = 0, entry = 0;
    int2 shared = {0, 0};
    if (p.prompts) {
        const int q = i / a.G, G = a.G;
        prompt_tokens = cache_tokens(a.prompt_lengths, q, a.prompt_table_pages, a.cache.page, bad);
        int before = 0, live = 0;                             // live rollouts of the group: before this one, all
        for (int j0 = 0; j0 < G; j0 += LANES) {
            const int j = j0 + lane;
            const uint32_t all = (__ballot_sync(0xffffffffu, j < G && (!a.keep || a.keep[(int64_t)q * G + j])) >> part) & (0xffffffffu >> (32 - LANES));
            const int left = i - q * G - j0;
            live += __popc(all);
            before += __popc(left >= LANES ? all : left <= 0 ? 0u : all & ((1u << left) - 1u));
        }
        entry = q * p.blocks + before / p.group;
        prompt_rows = min(live - before / p.group * p.group, p.group) * p.ratio;
        prompt_row = before % p.group * p.ratio + r;
        shared = owners[(int64_t)entry * Hkv + h];
    }
    const bool wanted = asked < rows && (!a.keep || a.keep[i]);
    Merged m = {-INFINITY, 0.f, {0.f, 0.f, 0.f, 0.f}, 0.f};
    // The records of a unit: `count` of the blocks (warps) that have some of it, `step` rows apart; of shared units of up to 32 rows two each, CA_ROWS / 2 apart.
    struct Records { int64_t first; int count, step, twice; };
    const int64_t own_number = (int64_t)i * Hkv + h, prompt_number = (int64_t)entry * Hkv + h, shared_rows = p.w.rows_own + p.w.rows_prompt;
    auto records = [&](int rows, int2 of, int64_t shared_first, int64_t first, int step) {
        const bool in_blocks = rows > CA_ALONE;
        const int twice = in_blocks && rows <= 32 ? 1 : 0;
        if (in_blocks) { first = shared_first; step = CA_ROWS; }
        // inside the workspace even where a wait ran out, so that nobody told of the unit
        const int most = (in_blocks ? p.grid : p.grid * CA_WARPS) - 1, from = min(max(of.x, 0), most), to = min(max(of.y, from - 1), most);
        return Records{first + (int64_t)from * step, (to - from + 1) << twice, step, twice};
    };
    Records a_prompt = {0, 0, 0, 0}, an_own = {0, 0, 0, 0};
    if (wanted && prompt_tokens > 0)
        a_prompt = records(prompt_rows, shared, shared_rows + prompt_number * CA_ROWS + prompt_row, p.w.rows_own + prompt_number * CA_ALONE + prompt_row, CA_ALONE);
    if (wanted && own_tokens > 0) an_own = records(p.ratio, own, shared_rows + ((int64_t)p.prompts * Hkv + own_number) * CA_ROWS + r, own_number * p.ratio + r, p.ratio);
    for (int w = 0; w < a_prompt.count + an_own.count; w += Merged::AT_ONCE) {
        float2 x[Merged::AT_ONCE];
        float4 v[Merged::AT_ONCE];
#pragma unroll
        for (int k = 0; k < Merged::AT_ONCE; ++k) {
            x[k] = make_float2(-INFINITY, 0.f);
            v[k] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (w + k < a_prompt.count + an_own.count) {
                const bool of_prompt = w + k < a_prompt.count;
                const Records& u = of_prompt ? a_prompt : an_own;
                const int number = of_prompt ? w + k : w + k - a_prompt.count;
                const int64_t at = u.first + (int64_t)(number >> u.twice) * u.step + (number & u.twice) * (CA_ROWS / 2);
                x[k] = ml[at];
                if (d < D) v[k] = *reinterpret_cast<const float4*>(o + at * D + d);
            }
        }
        m.add(x, v);
    }
    if (wanted && !(m.least < 0.f)) m.write(a, row, i, hq, lane, prompt_tokens > 0 || own_tokens > 0);
    __shared__ ApartShared sm;
    if (__builtin_expect(__syncthreads_or(wanted && m.least < 0.f), 0)) {
        if (lane == 0) sm.apart[threadIdx.x / LANES] = wanted && m.least < 0.f;
        __syncthreads();
#pragma unroll 1
        for (int x = 0; x < MERGE_THREADS / LANES; ++x)
            if (sm.apart[x]) row_apart(p, first + x * step, sm);
    }
}

// [pages, Hkv, page, D] numbers as boxes of up to 32 tokens x DP bytes of one page and head, rows of DP bytes in shared memory, swizzled over as many; dimensions past D are zeros.
int make_map_pages(arrol_ctx* ctx, CUtensorMap* map, const arrol_cache& c, const void* base, int64_t page_stride, int DP) {
    const cuuint64_t dims[4] = {(cuuint64_t)c.D, (cuuint64_t)c.page, (cuuint64_t)c.Hkv, (cuuint64_t)c.pages};
    const cuuint64_t strides[3] = {(cuuint64_t)c.D, (cuuint64_t)c.page * c.D, (cuuint64_t)page_stride};
    const cuuint32_t box[4] = {(cuuint32_t)DP, (cuuint32_t)(c.page < CA_TOKENS ? c.page : CA_TOKENS), 1, 1};
    const cuuint32_t elem_strides[4] = {1, 1, 1, 1};
    CUresult r = reinterpret_cast<EncodeTiledFn>(ctx->encode_tiled)(
        map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 4, const_cast<void*>(base), dims, strides, box, elem_strides, CU_TENSOR_MAP_INTERLEAVE_NONE,
        DP == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? ARROL_OK : ARROL_ERR_CUDA;
}

template <int DP>
int launch_cache_attention(arrol_ctx* ctx, CacheParams& p, cudaStream_t s) {
    using C = CacheConf<DP>;
    bool& set = ctx->cache_attention_smem_set[DP == 128];
    if (!set) {
        ARROL_CUDA_OK(cudaFuncSetAttribute(cache_units_kernel<DP>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)C::SMEM));
        set = true;
    }
    CUtensorMap k = {}, v = {};                              // without pages nothing is copied
    if (p.a.cache.pages > 0 && (make_map_pages(ctx, &k, p.a.cache, p.a.cache.k_cache, p.a.cache.k_page_stride, DP) != ARROL_OK ||
                                make_map_pages(ctx, &v, p.a.cache, p.a.cache.v_cache, p.a.cache.v_page_stride, DP) != ARROL_OK))
        return ARROL_ERR_CUDA;
    constexpr int LANES = DP / 4;
    const int64_t blocks = ((int64_t)p.a.N * p.a.Hq * LANES + MERGE_THREADS - 1) / MERGE_THREADS;
    // Few blocks: rows of one rollout over many of them, so that those that are not live, or computed anew, leave none idle (16 rollouts of 32 heads 56.3 -> 55.3 us; scales far apart in one of
    // them 1,504 -> 267).  Many: side by side, for what their rollouts have in common (512 rollouts of 16 heads 235, all over 237.5).
    p.merge_apart = blocks <= 2 * ctx->sm_count;
    ARROL_CUDA_OK(arrol_launch_pdl(cache_units_kernel<DP>, dim3((unsigned)p.grid), dim3(CA_THREADS), C::SMEM, s, k, v, p));
    ARROL_CUDA_OK(arrol_launch_pdl(cache_merge_kernel<LANES>, dim3((unsigned)blocks), dim3(MERGE_THREADS), 0, s, p));
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
    CacheParams p = {};
    p.a = *a;
    p.ratio = a->Hq / a->cache.Hkv;
    p.group = ca_group(p.ratio);
    p.blocks = ca_blocks(a->G, p.ratio);
    p.prompts = a->P * p.blocks;
    p.entries = p.prompts + a->N;
    p.page_shift = __builtin_ctz((unsigned)a->cache.page);
    p.grid = ctx->sm_count * ca_per_sm(a->cache.D);
    // The line is counted in 32 bits: with every table full it stays below 2^30.
    const int64_t own_most = (int64_t)a->table_pages * a->cache.page, prompt_most = (int64_t)a->prompt_table_pages * a->cache.page;
    if (own_most > INT32_MAX || prompt_most > INT32_MAX) return ARROL_ERR_UNSUPPORTED;
    auto fits = [&](const LineCosts& c) {
        auto longest = [&](int64_t units, int64_t tokens, bool shared) {
            return (double)units * a->cache.Hkv * (shared ? (double)(tokens / 64 + 2) * c.shared : (double)(tokens / 32 + 1) * c.many + c.single_setup);
        };
        return longest(a->N, own_most, p.ratio > CA_ALONE) + longest(p.prompts, prompt_most, true) < 1073741824.0;
    };
    p.costs = a->cache.D <= 64 ? CA_COSTS_64 : CA_COSTS_128;
    if (!fits(p.costs)) p.costs = CA_COSTS_COARSE;
    if (!fits(p.costs)) return ARROL_ERR_UNSUPPORTED;
    if (!a->workspace || !arrol_aligned(a->workspace, 256)) return ARROL_ERR_WORKSPACE;
    p.w = cache_workspace(a->workspace, ctx->sm_count, a->N, a->P, a->G, a->Hq, a->cache.Hkv, a->cache.D);
    if (a->workspace_bytes < p.w.bytes) return ARROL_ERR_WORKSPACE;
    p.own_most = (int)own_most;
    p.scale_log2 = a->scale * LOG2E;
    p.status = ctx->d_status;
    ArrolDeviceGuard guard(ctx->device);
    if (!guard.ok) return ARROL_ERR_CUDA;
    return a->cache.D <= 64 ? launch_cache_attention<64>(ctx, p, (cudaStream_t)stream) : launch_cache_attention<128>(ctx, p, (cudaStream_t)stream);
}
