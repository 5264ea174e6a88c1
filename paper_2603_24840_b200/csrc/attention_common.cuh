// Shared parts of the attention kernels: the packed tokens' key ranges, checks of the arguments, the workspace.
#pragma once
#include <cuda_bf16.h>
#include <limits.h>
#include <math.h>

#include "tc_common.cuh"

// Keys of one packed token: prompt rows [pre_lo, pre_hi), own rows [own_lo, token]; its sequence ends at own_hi.
struct alignas(16) TokenBounds {
    int pre_lo, pre_hi, own_lo, own_hi;
};

// The pieces of a packed call's workspace.
struct AttnWorkspace {
    uint32_t* counters;           // 64 words, zeroed by the bounds kernel
    TokenBounds* bounds;
    int2* prompt_range;
    float2* stats;                // per packed token and query head: lse log2(e), d_o . o
    float* parts;                 // partial sums of the prompts' gradients
    float* part_o;                // of o, where an item's keys are split, with
    float2* part_ml;              // their references and sums
    size_t bytes;
};

namespace {

constexpr int ATTN_MAX_D = 128;
constexpr int ATTN_MAX_RATIO = 64;                        // query heads per key head
constexpr int64_t ATTN_MAX_ROWS = ((int64_t)1 << 31) - 512;   // row numbers plus a tile fit 32 bits
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

// What the kernels of the packed calls share; built by the host, passed by value.
struct AttnShape {
    const int64_t* d_num;
    const TokenBounds* bounds;    // [T_max]
    const int2* prompt_range;     // [prompt_rows]: packed tokens [x, y) that attend to the prompt row; backward only
    int T_max, prompt_rows;
    int Hq, Hkv, D, ratio;        // ratio = Hq / Hkv
    float scale, scale_log2;      // scale_log2 = scale log2(e)
};

inline size_t attn_round(size_t n) { return (n + 255) & ~(size_t)255; }

// Items per tile of 128 prompt rows in the backward: every survivor's tokens pass by such a tile, which would make it the longest piece of work by far.
// Parts of about 48 blocks of 64 query rows (30 to 40 us); of 4 where the other tiles leave SMs free; and no more items than four an SM, whose
// partial sums take 128 KB each.
inline int attn_prompt_splits(int sm_count, int64_t T_max, int64_t prompt_rows, int P, int Hq, int Hkv) {
    if (prompt_rows == 0 || P < 1 || T_max == 0) return 1;
    const int64_t blocks = T_max * (Hq / Hkv) / P / 64, tiles = (prompt_rows + 127) / 128 * Hkv, others = (T_max + 127) / 128 * Hkv;
    int64_t n = (blocks + 47) / 48, fine = (sm_count - others) / tiles;
    if (fine > blocks / 4) fine = blocks / 4;
    if (n < fine) n = fine;
    const int64_t most = (4 * (int64_t)sm_count + tiles - 1) / tiles;
    if (n > most) n = most;
    return (int)(n < 1 ? 1 : n > 16 ? 16 : n);
}

// The most tiles of partial sums that a call of up to so many tokens and prompt rows has, so that a workspace for the largest call serves the smaller
// ones, which may have more parts.  With n > 1 parts n <= ceil(4 SMs / tiles), so there are fewer than 4 SMs tiles and less than 4 SMs + tiles parts.
inline int64_t attn_prompt_parts(int sm_count, int64_t T_max, int64_t prompt_rows, int Hq, int Hkv) {
    const int64_t blocks = T_max * (Hq / Hkv) / 64, tiles = (prompt_rows + 127) / 128 * Hkv, all = 4 * (int64_t)sm_count;
    const int64_t n = (blocks + 47) / 48 > blocks / 4 ? (blocks + 47) / 48 : blocks / 4;
    if (n <= 1) return 0;
    const int64_t few = (n < 16 ? n : 16) * tiles, many = all + (tiles < all ? tiles : all);
    return few < many ? few : many;
}

// Parts of an item's keys in the forward: as many as give every SM an item, of about four blocks of 128 keys at least (what the arrays' sizes say of a
// prompt and a sequence on average; the lengths are on the device, and a part may turn out to have none).  Few rows over long keys are bound by one
// block's walk over them otherwise: 64 tokens over a prompt of 6,000, 4 heads of 128 on one 100 -> 29 us, two prompts of 3,000 with 4 sequences of 30
// 98 -> 37, one sequence of 4,096 with 4 heads of 64 53 -> 49.  Where half of the SMs have an item already the walk is left whole.
inline int attn_key_splits(int sm_count, int64_t T_max, int64_t prompt_rows, int P, int S_max, int Hq, int Hkv) {
    const int64_t tokens = 2 * (128 / (Hq / Hkv)), items = (T_max + tokens - 1) / tokens * Hkv;
    if (items == 0 || items * 2 > sm_count) return 1;
    const int64_t blocks = (prompt_rows / (P > 0 ? P : 1) + T_max / (S_max > 0 ? S_max : 1) / 2) / 128;
    int64_t n = sm_count / items;
    if (n > blocks / 4) n = blocks / 4;
    return (int)(n < 1 ? 1 : n > 32 ? 32 : n);
}

// The most rows (part, token) of partial sums, likewise: n parts of `items` give n items <= SMs.
inline int64_t attn_key_parts(int sm_count, int64_t T_max, int64_t prompt_rows, int Hq, int Hkv) {
    const int64_t n = (prompt_rows + T_max / 2) / 512, most = sm_count / Hkv * (int64_t)(2 * (128 / (Hq / Hkv)));
    if (n <= 1 || sm_count / Hkv < 2) return 0;
    const int64_t few = (n < 32 ? n : 32) * T_max;
    return few < most ? few : most;
}

inline AttnWorkspace attn_workspace(void* base, int sm_count, int64_t T_max, int64_t prompt_rows, int Hq, int Hkv, int D, bool backward) {
    AttnWorkspace w = {};
    uint8_t* p = static_cast<uint8_t*>(base);
    size_t at = 0;
    auto take = [&](size_t n) { uint8_t* q = p + at; at += attn_round(n); return q; };
    w.counters = reinterpret_cast<uint32_t*>(take(256));
    w.bounds = reinterpret_cast<TokenBounds*>(take((size_t)T_max * sizeof(TokenBounds)));
    const size_t key_rows = (size_t)attn_key_parts(sm_count, T_max, prompt_rows, Hq, Hkv) * Hq;
    w.part_ml = reinterpret_cast<float2*>(take(key_rows * sizeof(float2)));
    w.part_o = reinterpret_cast<float*>(take(key_rows * D * sizeof(float)));
    if (backward) {
        w.prompt_range = reinterpret_cast<int2*>(take((size_t)prompt_rows * sizeof(int2)));
        w.stats = reinterpret_cast<float2*>(take((size_t)T_max * Hq * sizeof(float2)));
        const size_t tile = (size_t)128 * (D <= 64 ? 64 : 128) * 2 * sizeof(float);
        w.parts = reinterpret_cast<float*>(take((size_t)attn_prompt_parts(sm_count, T_max, prompt_rows, Hq, Hkv) * tile));
    }
    w.bytes = at;
    return w;
}

inline bool attn_heads_ok(int Hq, int Hkv, int D) {
    return Hkv >= 1 && Hq >= Hkv && Hq <= 65536 && Hq % Hkv == 0 && Hq / Hkv <= ATTN_MAX_RATIO && D >= 8 && D <= ATTN_MAX_D && D % 8 == 0;
}
inline bool attn_rows_ok(const void* p, int64_t stride, int heads, int D) {
    return p && arrol_aligned(p, 16) && stride % 8 == 0 && stride >= (int64_t)heads * D && stride < ((int64_t)1 << 38);
}

// [rows, heads, D] bf16, rows `stride` elements apart, as boxes of `tokens` rows x `group` heads x 64 dimensions: a box lands as tokens * group rows
// of 128 bytes, 128-byte swizzle; dimensions past D and rows outside are zeros.
int make_map_heads(arrol_ctx* ctx, CUtensorMap* map, const void* base, int64_t rows, int heads, int D, int64_t stride, int group, int tokens) {
    const cuuint64_t dims[3] = {(cuuint64_t)D, (cuuint64_t)heads, (cuuint64_t)rows};
    const cuuint64_t strides[2] = {(cuuint64_t)D * 2, (cuuint64_t)stride * 2};
    const cuuint32_t box[3] = {64, (cuuint32_t)group, (cuuint32_t)tokens};
    const cuuint32_t elem_strides[3] = {1, 1, 1};
    CUresult r = reinterpret_cast<EncodeTiledFn>(ctx->encode_tiled)(
        map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), dims, strides, box, elem_strides,
        CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
        CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? ARROL_OK : ARROL_ERR_CUDA;
}

__device__ __forceinline__ int clamp_row(int64_t x, int lo, int hi) { return (int)(x < lo ? lo : x > hi ? hi : x); }
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

// ---- products.  Operands with 64 HALVES dimensions lie as halves of 64 (128-byte swizzled rows), `half` bytes apart.
// d = A B^T, rows of both in shared memory
template <int HALVES>
__device__ __forceinline__ void mma_over_dims(uint32_t d, uint32_t a, uint32_t a_half, uint32_t b, uint32_t b_half, uint32_t idesc) {
#pragma unroll
    for (int h = 0; h < HALVES; ++h) {
        const uint64_t a_desc = make_smem_desc(a + h * a_half), b_desc = make_smem_desc(b + h * b_half);
#pragma unroll
        for (int k = 0; k < 64 / UMMA_K; ++k) {
            const uint64_t step = (uint64_t)(k * (UMMA_K * 2 >> 4));
            tcgen05_mma_bf16(d, a_desc + step, b_desc + step, idesc, (h | k) != 0 ? 1u : 0u);
        }
    }
}
// the same with A's rows in tensor memory
template <int HALVES>
__device__ __forceinline__ void mma_over_dims_tmem_a(uint32_t d, uint32_t a, uint32_t b, uint32_t b_half, uint32_t idesc) {
#pragma unroll
    for (int h = 0; h < HALVES; ++h) {
        const uint64_t b_desc = make_smem_desc(b + h * b_half);
#pragma unroll
        for (int k = 0; k < 64 / UMMA_K; ++k)
            tcgen05_mma_bf16_tmem_a(d, a + h * 32 + k * (UMMA_K / 2), b_desc + (uint64_t)(k * (UMMA_K * 2 >> 4)), idesc, (h | k) != 0 ? 1u : 0u);
    }
}
// d += A B over steps [K0, K1) of 16 of B's rows, A in tensor memory, B's rows in shared memory (ROWS of them); d = A B from step 0 on where `first`
template <int ROWS, int K0, int K1>
__device__ __forceinline__ void mma_over_rows(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, bool first) {
    const uint64_t b_desc = make_smem_desc_mn(b, ROWS);
#pragma unroll
    for (int k = K0; k < K1; ++k)
        tcgen05_mma_bf16_tmem_a(d, a + k * (UMMA_K / 2), b_desc + (uint64_t)(k * (UMMA_K * 128 >> 4)), idesc, first && k == 0 ? 0u : 1u);
}
__device__ __forceinline__ float2 bf16_pair(uint32_t v) { return __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&v)); }

// A row of 128 bytes (64 bf16) of a tile in shared memory: whether any value is an infinity or NaN (times 0 they leave NaN in the sum, everything
// else leaves 0).  Called for consecutive rows by consecutive lanes, which start at different 16-byte words so that they do not meet in a bank.
__device__ __forceinline__ bool row_not_finite(const uint8_t* row, int lane) {
    const __nv_bfloat162 zero = __floats2bfloat162_rn(0.f, 0.f);
    __nv_bfloat162 sum[4] = {zero, zero, zero, zero};
#pragma unroll
    for (int c = 0; c < 8; ++c) {
        const uint4 w = *reinterpret_cast<const uint4*>(row + (((c + lane) & 7) << 4));
        sum[0] = __hfma2(*reinterpret_cast<const __nv_bfloat162*>(&w.x), zero, sum[0]);
        sum[1] = __hfma2(*reinterpret_cast<const __nv_bfloat162*>(&w.y), zero, sum[1]);
        sum[2] = __hfma2(*reinterpret_cast<const __nv_bfloat162*>(&w.z), zero, sum[2]);
        sum[3] = __hfma2(*reinterpret_cast<const __nv_bfloat162*>(&w.w), zero, sum[3]);
    }
    const __nv_bfloat162 all = __hadd2(__hadd2(sum[0], sum[1]), __hadd2(sum[2], sum[3]));
    return __hisnan(__low2bfloat16(all)) || __hisnan(__high2bfloat16(all));
}
// Puts zeros in their place.
__device__ __forceinline__ void drop_not_finite(uint8_t* row) {
    uint32_t* w = reinterpret_cast<uint32_t*>(row);
    for (int c = 0; c < 32; ++c) {
        const uint32_t x = w[c];
        uint32_t y = x;
        if ((x & 0x7F80u) == 0x7F80u) y &= 0xFFFF0000u;
        if ((x & 0x7F800000u) == 0x7F800000u) y &= 0x0000FFFFu;
        if (y != x) w[c] = y;
    }
}

}  // namespace

// attention.cu: the packed tokens' bounds (for the backward the prompt rows' ranges and the statistics too); zeroes the counters.
int arrol_internal_attention_bounds(arrol_ctx* ctx, const arrol_attention_args* a, const AttnWorkspace& w, bool backward, cudaStream_t s);
int arrol_internal_check_attention(const arrol_attention_args* a);
