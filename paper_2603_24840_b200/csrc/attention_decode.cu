// arrol_attention_decode: one generated token per rollout over its group's prompt and its own cache.
#include "attention_common.cuh"

namespace {

constexpr int AD_THREADS = 256;

// First form: a warp per (rollout, query head), four dimensions a lane, one key at a time.
__global__ void __launch_bounds__(AD_THREADS) decode_rows_kernel(arrol_decode_args a, uint32_t* status) {
    pdl_launch_dependents();
    pdl_wait();
    using bf = const __nv_bfloat16*;
    const int lane = threadIdx.x & 31, c = lane * 4, ratio = a.Hq / a.Hkv;
    const bool on = c < a.D;
    const float scale_log2 = a.scale * LOG2E;
    auto load4 = [&](bf p) {
        float4 f = {0.f, 0.f, 0.f, 0.f};
        if (on) {
            const uint2 x = *reinterpret_cast<const uint2*>(p);
            const float2 u = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&x.x)), w = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&x.y));
            f = {u.x, u.y, w.x, w.y};
        }
        return f;
    };
    const int64_t rows = (int64_t)a.N * a.Hq, warps = (int64_t)gridDim.x * (AD_THREADS / 32);
    for (int64_t i = blockIdx.x * (int64_t)(AD_THREADS / 32) + (threadIdx.x >> 5); i < rows; i += warps) {
        const int n = (int)(i / a.Hq), h = (int)(i - (int64_t)n * a.Hq);
        if (a.keep && !a.keep[n]) continue;
        const int64_t gc = (int64_t)(h / ratio) * a.D + c;
        int64_t p0 = 0, p1 = 0, k0 = a.src_tok_off[n], k1 = k0 + a.lengths[n];
        if (a.P > 0) { p0 = a.cu_prompts[n / a.G]; p1 = a.cu_prompts[n / a.G + 1]; }
        bool bad = k0 < 0 || k1 < k0 || k1 > a.cache_rows;
        if (bad) k1 = k0;
        if (p0 < 0 || p1 < p0 || p1 > a.prompt_rows) { bad = true; p1 = p0; }
        if (bad && lane == 0) atomicOr(status, ARROL_DEV_BAD_INDEX);
        const float4 qf = load4((bf)a.q + n * a.q_stride + (int64_t)h * a.D + c);
        float m = -INFINITY, l = 0.f;
        float4 acc = {0.f, 0.f, 0.f, 0.f};
        auto visit = [&](bf kr, bf vr) {
            const float4 kf = load4(kr), vf = load4(vr);
            float z = qf.x * kf.x + qf.y * kf.y + (qf.z * kf.z + qf.w * kf.w);
#pragma unroll
            for (int x = 16; x > 0; x >>= 1) z += __shfl_xor_sync(0xffffffffu, z, x);
            z *= scale_log2;
            const float m1 = fmaxf(m, z), up = exp2f(m - m1), p = exp2f(z - m1);
            m = m1;
            l = l * up + p;
            acc.x = acc.x * up + p * vf.x; acc.y = acc.y * up + p * vf.y; acc.z = acc.z * up + p * vf.z; acc.w = acc.w * up + p * vf.w;
        };
        for (int64_t j = p0; j < p1; ++j) visit((bf)a.prompt_k + j * a.prompt_k_stride + gc, (bf)a.prompt_v + j * a.prompt_v_stride + gc);
        for (int64_t j = k0; j < k1; ++j) visit((bf)a.k + j * a.k_stride + gc, (bf)a.v + j * a.v_stride + gc);
        const float inv = m == -INFINITY ? 0.f : 1.f / l;
        if (on) {
            __nv_bfloat162 r[2] = {__floats2bfloat162_rn(acc.x * inv, acc.y * inv), __floats2bfloat162_rn(acc.z * inv, acc.w * inv)};
            *reinterpret_cast<uint2*>((__nv_bfloat16*)a.o + n * a.o_stride + (int64_t)h * a.D + c) = *reinterpret_cast<uint2*>(r);
        }
        if (lane == 0 && a.lse) a.lse[i] = m == -INFINITY ? -INFINITY : (m + log2f(l)) * LN2;
    }
}

}  // namespace

extern "C" size_t arrol_attention_decode_workspace(arrol_ctx* ctx, int32_t N, int32_t P, int32_t Hq, int32_t Hkv, int32_t D) {
    if (!ctx || N < 0 || P < 0 || !attn_heads_ok(Hq, Hkv, D)) return 0;
    return 256;
}

extern "C" int arrol_attention_decode(arrol_ctx* ctx, const arrol_decode_args* a, void* stream) {
    if (!ctx || !a) return ARROL_ERR_INVALID_ARG;
    if (a->N < 0 || a->P < 0 || a->G < 1 || a->cache_rows < 0 || a->prompt_rows < 0 || a->Hq < 1 || a->Hkv < 1 || a->D < 1 || a->Hq % a->Hkv) return ARROL_ERR_INVALID_ARG;
    if (!(a->scale > 0.f) || !isfinite(a->scale)) return ARROL_ERR_INVALID_ARG;
    if (!attn_heads_ok(a->Hq, a->Hkv, a->D) || a->cache_rows >= ATTN_MAX_ROWS || a->prompt_rows >= ATTN_MAX_ROWS || a->G > 1024) return ARROL_ERR_UNSUPPORTED;
    if (a->P > 0 ? (int64_t)a->P * a->G != a->N || !a->cu_prompts : a->prompt_rows > 0) return ARROL_ERR_INVALID_ARG;
    if (a->N == 0) return ARROL_OK;
    if (!attn_rows_ok(a->q, a->q_stride, a->Hq, a->D) || !attn_rows_ok(a->o, a->o_stride, a->Hq, a->D) || !a->src_tok_off || !a->lengths) return ARROL_ERR_INVALID_ARG;
    if (a->cache_rows > 0 && (!attn_rows_ok(a->k, a->k_stride, a->Hkv, a->D) || !attn_rows_ok(a->v, a->v_stride, a->Hkv, a->D))) return ARROL_ERR_INVALID_ARG;
    if (a->prompt_rows > 0 && (!attn_rows_ok(a->prompt_k, a->prompt_k_stride, a->Hkv, a->D) || !attn_rows_ok(a->prompt_v, a->prompt_v_stride, a->Hkv, a->D)))
        return ARROL_ERR_INVALID_ARG;
    if (!a->workspace || !arrol_aligned(a->workspace, 256) || a->workspace_bytes < arrol_attention_decode_workspace(ctx, a->N, a->P, a->Hq, a->Hkv, a->D))
        return ARROL_ERR_WORKSPACE;
    ArrolDeviceGuard guard(ctx->device);
    if (!guard.ok) return ARROL_ERR_CUDA;
    ARROL_CUDA_OK(arrol_launch_pdl(decode_rows_kernel, dim3((unsigned)(8 * ctx->sm_count)), dim3(AD_THREADS), 0, (cudaStream_t)stream, *a, ctx->d_status));
    ctx->launches += 1;
    return ARROL_OK;
}
