// Queries and keys of a packed batch: RMS norm of each head and rotation to the token's position, in one pass (moa_qk_norm_rope).
//
//   y = x / sqrt(mean(x^2) + eps) * g over a head's dh elements (without g: y = x),
//   (y_c, y_{c + r/2}) -> (y_c cos - y_{c + r/2} sin, y_{c + r/2} cos + y_c sin), angle pos theta^(-2c/r), for c < r/2; dims from r on pass.
// In single precision from end to end, rounded once to the storage type; only the angle is formed and reduced in double precision, since at
// position 2^20 a single-precision one is off by 0.06.  A token's cosines and sines are worked out once, by the threads of the workgroup
// that has it, and serve all of its heads.
#include "moa_common.h"
#include "../../include/moa.h"

#include <math.h>

namespace moa {

namespace {

struct RopeNormArgs {
    const void *x[2];                // queries, keys: row t at t * stride, heads dh apart
    void *y[2];
    const void *g[2];                // [dh] or NULL
    int64_t ldx[2], ldy[2];          // elements
    int heads[2];
    int64_t T;
    const int32_t *pos;              // [T]
    int dh, half;                    // elements of a head, pairs that are rotated
    float eps;
    double log_theta;
};

// cos and sin of the pairs of `tokens` tokens from t0 on, [tokens][half]
__device__ __forceinline__ void angles(const RopeNormArgs &a, int64_t t0, int tokens, float2 *cs)
{
    for (int i = threadIdx.x; i < tokens * a.half; i += blockDim.x) {
        const int t = i / a.half, c = i - t * a.half;
        // (in turns: what is left of them after the whole ones is exact)
        const double turns = (double)a.pos[t0 + t] * (exp((double)c / (double)a.half * -a.log_theta) * 0.15915494309189533577);
        double sn, cn;
        sincospi(2.0 * (turns - rint(turns)), &sn, &cn);
        cs[i] = make_float2((float)cn, (float)sn);
    }
}

// ---------------------------------------------------------------- any sizes: a wavefront a head, four elements a lane
template <typename T>
__global__ __launch_bounds__(256) void k_qk_norm_rope(RopeNormArgs a)
{
    __shared__ float2 cs[128];
    __shared__ float row_s[4][256];
    const int64_t t = blockIdx.x;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, dh = a.dh, half = a.half;
    angles(a, t, half ? 1 : 0, cs);
    __syncthreads();
    float *row = row_s[wave];
    for (int hh = wave; hh < a.heads[0] + a.heads[1]; hh += 4) {
        const int w = hh >= a.heads[0], h = w ? hh - a.heads[0] : hh;
        const T *x = (const T *)a.x[w] + t * a.ldx[w] + (int64_t)h * dh;
        const T *g = (const T *)a.g[w];
        float v[4], ss = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int e = lane + 64 * i;
            v[i] = e < dh ? ld(x + e) : 0.f;
            ss = fmaf(v[i], v[i], ss);
        }
        if (g) {
#pragma unroll
            for (int o = 32; o >= 1; o >>= 1) ss += __shfl_xor(ss, o);
            const float inv = 1.f / sqrtf(ss / (float)dh + a.eps);
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (lane + 64 * i < dh) v[i] = v[i] * inv * ld(g + lane + 64 * i);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) row[lane + 64 * i] = v[i];
        __builtin_amdgcn_wave_barrier();
        T *y = (T *)a.y[w] + t * a.ldy[w] + (int64_t)h * dh;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int e = lane + 64 * i;
            if (e >= dh) continue;
            float r = v[i];
            if (e < 2 * half) {
                const bool upper = e >= half;
                const float2 f = cs[upper ? e - half : e];
                const float other = row[upper ? e - half : e + half];
                r = upper ? fmaf(v[i], f.x, other * f.y) : fmaf(v[i], f.x, -other * f.y);
            }
            st(y + e, r);
        }
        __builtin_amdgcn_wave_barrier();
    }
}

template <typename T>
hipError_t launch(const RopeNormArgs &a, hipStream_t st)
{
    prof_begin(K_QK_NORM_ROPE, st);
    MOA_KLAUNCH(k_qk_norm_rope<T>, dim3((unsigned)a.T), dim3(256), 0, st, a);
    prof_end(st);
    return hipGetLastError();
}

}  // namespace
}  // namespace moa

using namespace moa;

extern "C" {

int32_t moa_qk_norm_rope(int32_t dtype, const void *q, int64_t q_stride, int32_t n_q_heads, const void *k, int64_t k_stride, int32_t n_kv_heads, int64_t T,
                         int32_t head_dim, const void *gq, const void *gk, float rms_eps, const int32_t *pos, float rope_theta, int32_t rot_dim,
                         void *q_out, int64_t q_out_stride, void *k_out, int64_t k_out_stride, void *stream)
{
    if (dtype != MOA_F32 && dtype != MOA_BF16) return api_fail(MOA_ERR_DTYPE, "qk_norm_rope: dtype is neither MOA_F32 nor MOA_BF16");
    if (head_dim < 1 || head_dim > 256 || n_q_heads < 0 || n_kv_heads < 0 || n_q_heads > (1 << 20) || n_kv_heads > (1 << 20) || T < 0 || T > (1 << 24))
        return api_fail(MOA_ERR_SHAPE, "qk_norm_rope: dimensions (1 <= head_dim <= 256, heads within 2^20, T within 2^24)");
    if (rot_dim < 0 || rot_dim > head_dim || rot_dim % 2) return api_fail(MOA_ERR_SHAPE, "qk_norm_rope: rot_dim must be even and at most head_dim");
    if (T == 0 || n_q_heads + n_kv_heads == 0) return MOA_OK;
    if ((n_q_heads && (!q || !q_out)) || (n_kv_heads && (!k || !k_out))) return api_fail(MOA_ERR_NULL, "qk_norm_rope: q / k / q_out / k_out is NULL");
    if (rot_dim && !pos) return api_fail(MOA_ERR_NULL, "qk_norm_rope: pos is NULL");
    if (rot_dim && !(rope_theta > 0.f && rope_theta < INFINITY)) return api_fail(MOA_ERR_RANGE, "qk_norm_rope: rope_theta must be positive and finite");
    if ((gq || gk) && !(rms_eps >= 0.f && rms_eps < INFINITY)) return api_fail(MOA_ERR_RANGE, "qk_norm_rope: rms_eps must be finite and not negative");
    const int64_t wq = (int64_t)n_q_heads * head_dim, wk = (int64_t)n_kv_heads * head_dim;
    if ((n_q_heads && (q_stride < wq || q_out_stride < wq)) || (n_kv_heads && (k_stride < wk || k_out_stride < wk)))
        return api_fail(MOA_ERR_SHAPE, "qk_norm_rope: rows closer to each other than their heads take");
    for (const int64_t s : {q_stride, q_out_stride, k_stride, k_out_stride})
        if (s > INT64_MAX / 8 / (T + 1)) return api_fail(MOA_ERR_SHAPE, "qk_norm_rope: strides beyond the address space");
    const uintptr_t es = dtype == MOA_BF16 ? 2 : 4;
    uintptr_t bits = 0;
    if (n_q_heads) bits |= (uintptr_t)q | (uintptr_t)q_out;
    if (n_kv_heads) bits |= (uintptr_t)k | (uintptr_t)k_out;
    bits |= (uintptr_t)gq | (uintptr_t)gk;
    if ((bits & (es - 1)) || ((uintptr_t)pos & 3)) return api_fail(MOA_ERR_SHAPE, "qk_norm_rope: pointers must be aligned to their elements");
    const RopeNormArgs a = {{q, k}, {q_out, k_out}, {gq, gk}, {q_stride, k_stride}, {q_out_stride, k_out_stride}, {n_q_heads, n_kv_heads}, T, pos,
                            head_dim, rot_dim / 2, rms_eps, rot_dim ? log((double)rope_theta) : 0.0};
    prof_set_site(S_QK_NORM_ROPE);
    const hipError_t e = dtype == MOA_BF16 ? launch<bf16_t>(a, (hipStream_t)stream) : launch<float>(a, (hipStream_t)stream);
    return e == hipSuccess ? MOA_OK : api_fail(MOA_ERR_HIP, hipGetErrorString(e));
}

}  // extern "C"
