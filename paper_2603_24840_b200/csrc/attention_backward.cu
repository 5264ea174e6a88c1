// arrol_attention_backward: gradients of the packed survivors' attention.
#include "attention_common.cuh"

namespace {

constexpr int AB_THREADS = 256;

__device__ __forceinline__ float4 load_bf4(const __nv_bfloat16* p, bool on) {
    float4 f = {0.f, 0.f, 0.f, 0.f};
    if (on) {
        const uint2 x = *reinterpret_cast<const uint2*>(p);
        const float2 a = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&x.x)), b = __bfloat1622float2(*reinterpret_cast<const __nv_bfloat162*>(&x.y));
        f = {a.x, a.y, b.x, b.y};
    }
    return f;
}
__device__ __forceinline__ void store_bf4(__nv_bfloat16* p, bool on, float4 f, float by) {
    if (!on) return;
    __nv_bfloat162 r[2] = {__floats2bfloat162_rn(f.x * by, f.y * by), __floats2bfloat162_rn(f.z * by, f.w * by)};
    *reinterpret_cast<uint2*>(p) = *reinterpret_cast<uint2*>(r);
}
__device__ __forceinline__ float dot4_warp(float4 a, float4 b) {
    float z = a.x * b.x + a.y * b.y + (a.z * b.z + a.w * b.w);
#pragma unroll
    for (int x = 16; x > 0; x >>= 1) z += __shfl_xor_sync(0xffffffffu, z, x);
    return z;
}
__device__ __forceinline__ void axpy4(float4& y, float a, float4 x) { y.x += a * x.x; y.y += a * x.y; y.z += a * x.z; y.w += a * x.w; }

// First form: a warp per (token, query head) for dq.
__global__ void __launch_bounds__(AB_THREADS) attention_dq_rows_kernel(AttnShape sh, arrol_attention_args a, const float* delta) {
    pdl_launch_dependents();
    pdl_wait();
    using bf = const __nv_bfloat16*;
    const int64_t n = sh.d_num[1];
    const int T = (int)(n < 0 ? 0 : n > sh.T_max ? sh.T_max : n), lane = threadIdx.x & 31, c = lane * 4;
    const bool on = c < sh.D;
    const int64_t rows = (int64_t)T * sh.Hq, warps = (int64_t)gridDim.x * (AB_THREADS / 32);
    for (int64_t i = blockIdx.x * (int64_t)(AB_THREADS / 32) + (threadIdx.x >> 5); i < rows; i += warps) {
        const int t = (int)(i / sh.Hq), h = (int)(i - (int64_t)t * sh.Hq);
        const int64_t gc = (int64_t)(h / sh.ratio) * sh.D + c, hc = (int64_t)h * sh.D + c;
        const TokenBounds b = sh.bounds[t];
        const float4 q = load_bf4((bf)a.q + t * a.q_stride + hc, on), go = load_bf4((bf)a.d_o + t * a.d_o_stride + hc, on);
        const float lse = a.lse[i], del = delta[i];
        float4 acc = {0.f, 0.f, 0.f, 0.f};
        auto visit = [&](bf kr, bf vr) {
            const float4 k = load_bf4(kr, on);
            const float z = dot4_warp(q, k) * sh.scale, dp = dot4_warp(go, load_bf4(vr, on));
            axpy4(acc, expf(z - lse) * (dp - del), k);
        };
        for (int j = b.pre_lo; j < b.pre_hi; ++j) visit((bf)a.prompt_k + j * a.prompt_k_stride + gc, (bf)a.prompt_v + j * a.prompt_v_stride + gc);
        for (int j = b.own_lo; j <= t; ++j) visit((bf)a.k + j * a.k_stride + gc, (bf)a.v + j * a.v_stride + gc);
        store_bf4((__nv_bfloat16*)a.dq + t * a.dq_stride + hc, on, acc, sh.scale);
    }
}

// First form: a warp per (key row, key head) for dk and dv; prompt rows after the packed ones.
__global__ void __launch_bounds__(AB_THREADS) attention_dkv_rows_kernel(AttnShape sh, arrol_attention_args a, const float* delta) {
    pdl_launch_dependents();
    pdl_wait();
    using bf = const __nv_bfloat16*;
    const int64_t n = sh.d_num[1];
    const int T = (int)(n < 0 ? 0 : n > sh.T_max ? sh.T_max : n), lane = threadIdx.x & 31, c = lane * 4;
    const int64_t pn = a.P > 0 ? a.cu_prompts[a.P] : 0;
    const int live = (int)(pn < 0 ? 0 : pn > sh.prompt_rows ? sh.prompt_rows : pn);
    const bool on = c < sh.D;
    const int64_t items = ((int64_t)T + live) * sh.Hkv, warps = (int64_t)gridDim.x * (AB_THREADS / 32);
    for (int64_t i = blockIdx.x * (int64_t)(AB_THREADS / 32) + (threadIdx.x >> 5); i < items; i += warps) {
        int64_t j = i / sh.Hkv;
        const int g = (int)(i - j * sh.Hkv);
        const int64_t gc = (int64_t)g * sh.D + c;
        const bool shared = j >= T;
        if (shared) j -= T;
        const int lo = shared ? sh.prompt_range[j].x : (int)j, hi = shared ? sh.prompt_range[j].y : sh.bounds[j].own_hi;
        const float4 k = load_bf4(shared ? (bf)a.prompt_k + j * a.prompt_k_stride + gc : (bf)a.k + j * a.k_stride + gc, on);
        const float4 v = load_bf4(shared ? (bf)a.prompt_v + j * a.prompt_v_stride + gc : (bf)a.v + j * a.v_stride + gc, on);
        float4 dk = {0.f, 0.f, 0.f, 0.f}, dv = {0.f, 0.f, 0.f, 0.f};
        for (int t = lo; t < hi; ++t)
            for (int h = g * sh.ratio; h < (g + 1) * sh.ratio; ++h) {
                const int64_t hc = (int64_t)h * sh.D + c, r = (int64_t)t * sh.Hq + h;
                const float4 q = load_bf4((bf)a.q + t * a.q_stride + hc, on), go = load_bf4((bf)a.d_o + t * a.d_o_stride + hc, on);
                const float p = expf(dot4_warp(q, k) * sh.scale - a.lse[r]), ds = p * (dot4_warp(go, v) - delta[r]);
                axpy4(dv, p, go);
                axpy4(dk, ds, q);
            }
        store_bf4(shared ? (__nv_bfloat16*)a.dprompt_k + j * a.dprompt_k_stride + gc : (__nv_bfloat16*)a.dk + j * a.dk_stride + gc, on, dk, sh.scale);
        store_bf4(shared ? (__nv_bfloat16*)a.dprompt_v + j * a.dprompt_v_stride + gc : (__nv_bfloat16*)a.dv + j * a.dv_stride + gc, on, dv, 1.f);
    }
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
    if (a->prompt_rows > 0 && (!attn_rows_ok(a->dprompt_k, a->dprompt_k_stride, a->Hkv, a->D) || !attn_rows_ok(a->dprompt_v, a->dprompt_v_stride, a->Hkv, a->D)))
        return ARROL_ERR_INVALID_ARG;
    const AttnWorkspace w = attn_workspace(a->workspace, a->T_max, a->prompt_rows, a->Hq, true);
    if (a->workspace_bytes < w.bytes) return ARROL_ERR_WORKSPACE;
    ArrolDeviceGuard guard(ctx->device);
    if (!guard.ok) return ARROL_ERR_CUDA;
    cudaStream_t s = (cudaStream_t)stream;
    const int rb = arrol_internal_attention_bounds(ctx, a, w, true, s);
    if (rb != ARROL_OK) return rb;
    const AttnShape sh = {a->d_num, w.bounds, w.prompt_range, (int)a->T_max, (int)a->prompt_rows, a->Hq, a->Hkv, a->D, a->Hq / a->Hkv, a->scale, a->scale * LOG2E};
    ARROL_CUDA_OK(arrol_launch_pdl(attention_dkv_rows_kernel, dim3((unsigned)(8 * ctx->sm_count)), dim3(AB_THREADS), 0, s, sh, *a, static_cast<const float*>(w.delta)));
    ARROL_CUDA_OK(arrol_launch_pdl(attention_dq_rows_kernel, dim3((unsigned)(8 * ctx->sm_count)), dim3(AB_THREADS), 0, s, sh, *a, static_cast<const float*>(w.delta)));
    ctx->launches += 2;
    return ARROL_OK;
}
