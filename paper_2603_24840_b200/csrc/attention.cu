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
__device__ __forceinline__ int clamp_row(int64_t x, int lo, int hi) { return (int)(x < lo ? lo : x > hi ? hi : x); }

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

// delta[t, h] = sum_d d_o[t, h, d] o[t, h, d]: a warp per row.
__global__ void __launch_bounds__(BOUNDS_THREADS)
attention_delta_kernel(const __nv_bfloat16* __restrict__ o, int64_t o_stride, const __nv_bfloat16* __restrict__ d_o, int64_t d_o_stride,
                       const int64_t* __restrict__ d_num, int T_max, int Hq, int D, float* __restrict__ delta) {
    pdl_launch_dependents();
    pdl_wait();
    o = pdl_acquire(o); d_o = pdl_acquire(d_o); d_num = pdl_acquire(d_num);
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
        if (lane == 0) delta[i] = sum;
    }
}

// First form: a warp per (token, query head), four dimensions a lane, one key at a time.
__global__ void __launch_bounds__(BOUNDS_THREADS)
attention_rows_kernel(AttnShape sh, const __nv_bfloat16* q, int64_t q_stride, const __nv_bfloat16* k, int64_t k_stride,
                      const __nv_bfloat16* v, int64_t v_stride, const __nv_bfloat16* pk, int64_t pk_stride, const __nv_bfloat16* pv,
                      int64_t pv_stride, __nv_bfloat16* o, int64_t o_stride, float* lse) {
    pdl_launch_dependents();
    pdl_wait();
    const int T = clamp_row(sh.d_num[1], 0, sh.T_max);
    const int lane = threadIdx.x & 31, c = lane * 4;
    const bool on = c < sh.D;
    const int64_t rows = (int64_t)T * sh.Hq, warps = (int64_t)gridDim.x * (BOUNDS_THREADS / 32);
    auto load4 = [&](const __nv_bfloat16* p) {
        float4 f = {0.f, 0.f, 0.f, 0.f};
        if (on) {
            const uint2 x = *reinterpret_cast<const uint2*>(p + c);
            const float2 a = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&x.x)), b = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&x.y));
            f = {a.x, a.y, b.x, b.y};
        }
        return f;
    };
    for (int64_t i = blockIdx.x * (int64_t)(BOUNDS_THREADS / 32) + (threadIdx.x >> 5); i < rows; i += warps) {
        const int t = (int)(i / sh.Hq), h = (int)(i - (int64_t)t * sh.Hq), g = h / sh.ratio;
        const TokenBounds b = sh.bounds[t];
        const float4 qf = load4(q + t * q_stride + (int64_t)h * sh.D);
        float m = -INFINITY, l = 0.f;
        float4 acc = {0.f, 0.f, 0.f, 0.f};
        auto visit = [&](const __nv_bfloat16* kr, const __nv_bfloat16* vr) {
            const float4 kf = load4(kr), vf = load4(vr);
            float z = qf.x * kf.x + qf.y * kf.y + (qf.z * kf.z + qf.w * kf.w);
#pragma unroll
            for (int x = 16; x > 0; x >>= 1) z += __shfl_xor_sync(0xffffffffu, z, x);
            z *= sh.scale_log2;
            const float m1 = fmaxf(m, z), up = exp2f(m - m1), p = exp2f(z - m1);
            m = m1;
            l = l * up + p;
            acc.x = acc.x * up + p * vf.x; acc.y = acc.y * up + p * vf.y; acc.z = acc.z * up + p * vf.z; acc.w = acc.w * up + p * vf.w;
        };
        for (int j = b.pre_lo; j < b.pre_hi; ++j) visit(pk + j * pk_stride + (int64_t)g * sh.D, pv + j * pv_stride + (int64_t)g * sh.D);
        for (int j = b.own_lo; j <= t; ++j) visit(k + j * k_stride + (int64_t)g * sh.D, v + j * v_stride + (int64_t)g * sh.D);
        const float inv = 1.f / l;
        if (on) {
            __nv_bfloat162 r[2] = {__floats2bfloat162_rn(acc.x * inv, acc.y * inv), __floats2bfloat162_rn(acc.z * inv, acc.w * inv)};
            *reinterpret_cast<uint2*>(o + t * o_stride + (int64_t)h * sh.D + c) = *reinterpret_cast<uint2*>(r);
        }
        if (lane == 0) lse[i] = (m + log2f(l)) * LN2;
    }
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
        ARROL_CUDA_OK(arrol_launch_pdl(attention_delta_kernel, dim3((unsigned)rows), dim3(BOUNDS_THREADS), 0, s,
                                       static_cast<const __nv_bfloat16*>(a->o), a->o_stride, static_cast<const __nv_bfloat16*>(a->d_o),
                                       a->d_o_stride, a->d_num, (int)a->T_max, a->Hq, a->D, w.delta));
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
    const AttnShape sh = {a->d_num, w.bounds, nullptr, (int)a->T_max, (int)a->prompt_rows, a->Hq, a->Hkv, a->D, a->Hq / a->Hkv, a->scale, a->scale * LOG2E};
    using bf = const __nv_bfloat16*;
    ARROL_CUDA_OK(arrol_launch_pdl(attention_rows_kernel, dim3((unsigned)(8 * ctx->sm_count)), dim3(BOUNDS_THREADS), 0, s, sh, (bf)a->q, a->q_stride,
                                   (bf)a->k, a->k_stride, (bf)a->v, a->v_stride, (bf)a->prompt_k, a->prompt_k_stride, (bf)a->prompt_v,
                                   a->prompt_v_stride, static_cast<__nv_bfloat16*>(a->o), a->o_stride, a->lse));
    ctx->launches += 1;
    return ARROL_OK;
}
