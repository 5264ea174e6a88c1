// arrol_rotary, arrol_rotary_backward: queries and keys of packed tokens turned by their positions.
//
// Bound by HBM: every entry is read and written once, 4 D bytes a token and head.  A thread has one unit (two chunks, 16 bytes each in the usual case) of one token,
// forms its cosines and sines once and goes through the heads with them in registers, so that a token's angles are computed once and not once a head.  Where that
// makes too few threads the heads are split over blocks, each of which forms the angles again.
#include <math.h>

#include "rotary_common.cuh"

namespace {

// Two heads loaded at once and eight blocks of 128 threads an SM: 15,400 tokens of 24 heads of 80 22 to 26 us, 138,000 of 24 heads of 128 259.  Four at once take 80 registers:
// six blocks, 27 and 255 (one of 256 threads at 88 registers 29 and 264).
constexpr int ROT_THREADS = 128, ROT_PER_SM = 8;
constexpr int ROT_AT_ONCE = 2;
constexpr int64_t ROT_MAX_ROWS = ((int64_t)1 << 31) - 512;

struct RotaryParams {
    arrol_rotary_args a;
    RotaryPairs pairs;
    int units, heads;                             // of a head; of a block
    uint32_t* status;
};

// Position of packed token t; `s`: no later sequence's number than its own.
__device__ __forceinline__ int64_t packed_position(const arrol_rotary_args& a, int64_t t, int64_t s, int64_t S, bool& bad) {
    while (s < S && a.cu_seqlens[s + 1] <= t) ++s;
    if (s >= S) { bad = true; return 0; }
    const int64_t own = t - a.cu_seqlens[s];
    if (own < 0) { bad = true; return 0; }
    if (a.P == 0) return own;
    const int64_t p = (a.survivor_idx ? a.survivor_idx[s] : (int)s) / a.G;
    if ((a.survivor_idx && a.survivor_idx[s] < 0) || p >= a.P) { bad = true; return 0; }
    return own + a.cu_prompts[p + 1] - a.cu_prompts[p];
}

template <int V>
__global__ void __launch_bounds__(ROT_THREADS, ROT_PER_SM) rotary_kernel(const RotaryParams p) {
    typedef typename Bf16Chunk<V>::type Chunk;
    pdl_launch_dependents();
    pdl_wait();
    const arrol_rotary_args& a = p.a;
    const int64_t* num = pdl_acquire(a.d_num);
    int64_t T = a.T_max, S = a.S_max;
    if (num) {
        T = num[1] < T ? num[1] : T;
        S = num[0] < S ? num[0] : S;
    }
    const int64_t first = (int64_t)blockIdx.x * ROT_THREADS;
    const int64_t t0 = first / p.units;
    if (t0 >= T) return;
    int64_t s0 = 0;
    if (!a.positions) s0 = block_search(S, [&](int64_t i) { return a.cu_seqlens[i + 1] <= t0; });
    const int64_t t = (first + threadIdx.x) / p.units;
    if (t >= T) return;
    RotaryUnit<V> unit(p.pairs, (int)(first + threadIdx.x - t * p.units));
    if (unit.turns) {
        bool bad = false;
        const int64_t position = a.positions ? (int64_t)a.positions[t] : packed_position(a, t, s0, S, bad);
        if (bad) atomicOr(p.status, ARROL_DEV_BAD_INDEX);
        unit.at(p.pairs, position);
    }
    const int h0 = blockIdx.y * p.heads, h1 = min(h0 + p.heads, a.Hq + a.Hkv);
    const __nv_bfloat16* const q = static_cast<const __nv_bfloat16*>(a.q) + t * a.q_stride;
    const __nv_bfloat16* const k = static_cast<const __nv_bfloat16*>(a.k) + t * a.k_stride;
    __nv_bfloat16* const qo = static_cast<__nv_bfloat16*>(a.q_out) + t * a.q_out_stride;
    __nv_bfloat16* const ko = static_cast<__nv_bfloat16*>(a.k_out) + t * a.k_out_stride;
    for (int h = h0; h < h1; h += ROT_AT_ONCE) {
        Chunk ca[ROT_AT_ONCE], cb[ROT_AT_ONCE];
#pragma unroll
        for (int j = 0; j < ROT_AT_ONCE; ++j)
            if (h + j < h1) {
                const __nv_bfloat16* at = h + j < a.Hq ? q + (h + j) * a.D : k + (h + j - a.Hq) * a.D;
                ca[j] = *reinterpret_cast<const Chunk*>(at + unit.a);
                cb[j] = *reinterpret_cast<const Chunk*>(at + unit.b);
            }
#pragma unroll
        for (int j = 0; j < ROT_AT_ONCE; ++j)
            if (h + j < h1) {
                __nv_bfloat16* to = h + j < a.Hq ? qo + (h + j) * a.D : ko + (h + j - a.Hq) * a.D;
                if (unit.turns) {
                    float x[V], y[V];
                    chunk_to_floats<V>(ca[j], x);
                    chunk_to_floats<V>(cb[j], y);
                    unit.turn(p.pairs, x, y);
                    ca[j] = floats_to_chunk<V>(x);
                    cb[j] = floats_to_chunk<V>(y);
                }
                *reinterpret_cast<Chunk*>(to + unit.a) = ca[j];
                *reinterpret_cast<Chunk*>(to + unit.b) = cb[j];
            }
    }
}

bool rotary_rows_ok(const void* p, int64_t stride, int heads, int D) {
    return heads == 0 || (p && arrol_aligned(p, 16) && stride % 8 == 0 && stride >= (int64_t)heads * D && stride < ((int64_t)1 << 38));
}

int rotary_call(arrol_ctx* ctx, const arrol_rotary_args* a, float sign, void* stream) {
    if (!ctx || !a) return ARROL_ERR_INVALID_ARG;
    if (a->T_max < 0 || a->Hq < 0 || a->Hkv < 0 || a->D < 1 || a->R < 2 || a->R % 2 || a->R > a->D || !isfinite(a->factor)) return ARROL_ERR_INVALID_ARG;
    if (!a->positions && (a->S_max < 0 || a->P < 0 || a->G < 1)) return ARROL_ERR_INVALID_ARG;
    if (a->D % 8 || a->D > 256 || a->Hq > 65536 || a->Hkv > 65536 || a->T_max >= ROT_MAX_ROWS) return ARROL_ERR_UNSUPPORTED;
    if (a->T_max == 0 || a->Hq + a->Hkv == 0) return ARROL_OK;
    if (!rotary_rows_ok(a->q, a->q_stride, a->Hq, a->D) || !rotary_rows_ok(a->q_out, a->q_out_stride, a->Hq, a->D) ||
        !rotary_rows_ok(a->k, a->k_stride, a->Hkv, a->D) || !rotary_rows_ok(a->k_out, a->k_out_stride, a->Hkv, a->D))
        return ARROL_ERR_INVALID_ARG;
    if ((a->Hq && a->q == a->q_out && a->q_stride != a->q_out_stride) || (a->Hkv && a->k == a->k_out && a->k_stride != a->k_out_stride)) return ARROL_ERR_INVALID_ARG;
    if (!a->frequencies || !arrol_aligned(a->frequencies, 8)) return ARROL_ERR_INVALID_ARG;
    if (!a->positions && (!a->cu_seqlens || !a->d_num || (a->P > 0) != (a->cu_prompts != nullptr))) return ARROL_ERR_INVALID_ARG;
    RotaryParams p = {};
    p.a = *a;
    p.pairs = {a->frequencies, a->R, a->interleaved != 0, a->factor, sign};
    const int V = rotary_vector(a->D, a->R), heads = a->Hq + a->Hkv;
    p.units = a->D / (2 * V);
    p.status = ctx->d_status;
    const int64_t blocks = (a->T_max * p.units + ROT_THREADS - 1) / ROT_THREADS;
    // Four blocks an SM or more where the heads allow it, a few heads a block at least: with eight or sixteen the angles cost more than the waiting (22 -> 26, 27 us).
    int64_t split = (4 * (int64_t)ctx->sm_count + blocks - 1) / blocks;
    const int64_t most = (heads + ROT_AT_ONCE - 1) / ROT_AT_ONCE;
    if (split > most) split = most;
    p.heads = (int)((heads + split - 1) / split);
    split = (heads + p.heads - 1) / p.heads;
    ArrolDeviceGuard guard(ctx->device);
    if (!guard.ok) return ARROL_ERR_CUDA;
    void (*kernel)(RotaryParams) = V == 8 ? rotary_kernel<8> : V == 4 ? rotary_kernel<4> : V == 2 ? rotary_kernel<2> : rotary_kernel<1>;
    ARROL_CUDA_OK(arrol_launch_pdl(kernel, dim3((unsigned)blocks, (unsigned)split), dim3(ROT_THREADS), 0, (cudaStream_t)stream, p));
    ctx->launches += 1;
    return ARROL_OK;
}

}  // namespace

extern "C" int arrol_rotary(arrol_ctx* ctx, const arrol_rotary_args* args, void* stream) { return rotary_call(ctx, args, 1.0f, stream); }
extern "C" int arrol_rotary_backward(arrol_ctx* ctx, const arrol_rotary_args* args, void* stream) { return rotary_call(ctx, args, -1.0f, stream); }

extern "C" int arrol_rotary_frequencies(int32_t R, double base, int32_t kind, double stretch, double low, double high, double original,
                                        double* frequencies, double* factor) {
    if (R < 2 || R % 2 || !frequencies || !(base > 1.0) || !isfinite(base) || kind < ARROL_ROTARY_PLAIN || kind > ARROL_ROTARY_RAMP) return ARROL_ERR_INVALID_ARG;
    if (kind != ARROL_ROTARY_PLAIN && (!(stretch > 0.0) || !isfinite(stretch))) return ARROL_ERR_INVALID_ARG;
    const bool limits = kind == ARROL_ROTARY_BANDS || kind == ARROL_ROTARY_RAMP;
    if (limits && (!(low > 0.0) || !(high > low) || !isfinite(high) || !(original > 0.0) || !isfinite(original))) return ARROL_ERR_INVALID_ARG;
    const double two_pi = 6.283185307179586476925;
    double from = 0.0, to = 0.0;
    if (kind == ARROL_ROTARY_RAMP) {
        from = floor(R * log(original / (two_pi * high)) / (2.0 * log(base)));
        to = ceil(R * log(original / (two_pi * low)) / (2.0 * log(base)));
        if (from < 0.0) from = 0.0;
        if (to > R - 1) to = R - 1;
    }
    for (int i = 0; i < R / 2; ++i) {
        double f = pow(base, -2.0 * i / R);
        if (kind == ARROL_ROTARY_LINEAR) f /= stretch;
        if (limits) {
            double slow;
            if (kind == ARROL_ROTARY_BANDS) slow = 1.0 - (original * f / two_pi - low) / (high - low);
            else slow = (i - from) / (to - from > 0.001 ? to - from : 0.001);
            slow = slow < 0.0 ? 0.0 : slow > 1.0 ? 1.0 : slow;
            f = (1.0 - slow) * f + slow * (f / stretch);
        }
        frequencies[i] = f;
    }
    if (factor) *factor = kind == ARROL_ROTARY_RAMP && stretch > 1.0 ? 0.1 * log(stretch) + 1.0 : 1.0;
    return ARROL_OK;
}
