// Queries and keys of a packed batch: RMS norm of each head and rotation to the token's position, in one pass (moa_qk_norm_rope).
//
//   y = x / sqrt(mean(x^2) + eps) * g over a head's dh elements (without g: y = x),
//   (y_c, y_{c + r/2}) -> (y_c cos - y_{c + r/2} sin, y_{c + r/2} cos + y_c sin), angle pos theta^(-2c/r), for c < r/2; dims from r on pass.
// In single precision from end to end, rounded once to the storage type; only the angle is formed and reduced in double precision, since at
// position 2^20 a single-precision one is off by 0.06.  A token's cosines and sines are worked out once, by the threads of the workgroup
// that has it, and serve all of its heads.
#include "moa_kv_device.h"
#include "moa_rope_plan.h"

#include <math.h>

namespace moa {

namespace {

struct RopeNormArgs {
    const void *x[2];                // queries, keys: row t at t * stride, heads dh apart
    void *y[2];
    const void *g[2];                // [dh] or NULL
    int64_t ldx[2], ldy[2];          // elements
    int heads[2];
    FastDiv by_heads[2];
    int64_t T;
    const int32_t *pos;              // [T]
    int dh, half;                    // elements of a head, pairs that are rotated
    float eps;
    double power[7];                 // theta^(-2^i / half): the frequency of pair c is the product of those of c's bits
};

// cos and sin of the pairs of `tokens` tokens from t0 on, [tokens][half].  The angle in turns, and in double precision until what is left of it
// is at most an eighth of one, from there in single: as good as a cosine rounded from double precision to a unit in the last place, and a
// fifth of the instructions (8192 tokens of 40 heads, exp and sincospi in double: 44 us, 119 in the kernel below).
__device__ __forceinline__ void angles(const RopeNormArgs &a, int64_t t0, int tokens, float2 *cs)
{
    for (int i = threadIdx.x; i < tokens * a.half; i += blockDim.x) {
        const int t = i / a.half, c = i - t * a.half;
        double f = 0.15915494309189533577;                  // 1 / (2 pi)
#pragma unroll
        for (int k = 0; k < 7; ++k) f *= c >> k & 1 ? a.power[k] : 1.0;
        const double turns = (double)a.pos[t0 + t] * f, quarters = rint(4.0 * turns);
        float sn, cn;
        sincospif((float)(2.0 * fma(-0.25, quarters, turns)), &sn, &cn);
        const int q = (int)(quarters - 4.0 * floor(0.25 * quarters));
        cs[i] = q == 0 ? make_float2(cn, sn) : q == 1 ? make_float2(-sn, cn) : q == 2 ? make_float2(-cn, -sn) : make_float2(sn, -cn);
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

// ---------------------------------------------------------------- rows in pieces of W words of 4 bytes: 4, or 2 where the rotated pairs do not lie in pieces of 16 bytes
// HBM bounds it where there are many tokens: 8192 of 40 heads of 128 dims, 168 MB, 31.3 us, 5.4 TB/s (a copy of 1 GiB: 5.15); the work of the vector units
// comes next (with weights picked by lane and rows found by division 36.9, vector units busy 82 % of the time).  Of few, its chain: position,
// angle, rows; 16 tokens 4.3 us by trace.
// A head is spread over LPR lanes, two pieces each: the ones that are rotated against each other, so that no lane needs another's elements, or two
// that pass.  A workgroup has TPB tokens, whose angles are one or two a thread.
template <typename T, int W, int LPR, int TPB>
__global__ __launch_bounds__(256) void k_qk_norm_rope_pieces(RopeNormArgs a)
{
    typedef __attribute__((ext_vector_type(W))) uint32_t Piece;
    constexpr int VE = 4 * W / sizeof(T), U = 2;
    __shared__ __attribute__((aligned(16))) float2 cs[TPB * 128];
    const int64_t t0 = (int64_t)blockIdx.x * TPB;
    const int tokens = (int)(a.T - t0 < TPB ? a.T - t0 : TPB);
    const int c = threadIdx.x % LPR, pairs = a.dh / (2 * VE), turned = a.half / VE;
    const bool on = c < pairs, turn = c < turned;
    const int pa = turn ? c : turned + c, step = turn ? turned : pairs - turned;      // pieces: pa and pa + step
    auto value = [](const Piece &v, int e) {
        return sizeof(T) == 4 ? __uint_as_float(v[e]) : __uint_as_float(e & 1 ? v[e / 2] & 0xffff0000u : v[e / 2] << 16);
    };
    constexpr int RP = 256 / LPR;                        // rows at a time
    const int first = threadIdx.x / LPR;
    // queries, then keys (or in workgroups of their own): which of them, and with what weights, is the same for a whole workgroup
    const int w0 = gridDim.y > 1 ? (int)blockIdx.y : 0, w1 = gridDim.y > 1 ? w0 + 1 : 2;
#pragma unroll 1
    for (int w = w0; w < w1; ++w) {
        const int heads = a.heads[w], n = tokens * heads;
        const T *const g = (const T *)a.g[w];
        struct Row { Piece x[2]; int64_t y; int t; } row[U];
        auto load = [&](int r, Row &v) {
            v.x[0] = v.x[1] = Piece{};
            if (r >= n || !on) return;
            v.t = (int)a.by_heads[w]((uint32_t)r);
            const int64_t h = (int64_t)(r - v.t * heads) * a.dh + pa * VE;
            const T *p = (const T *)a.x[w] + (t0 + v.t) * a.ldx[w] + h;
            v.y = (t0 + v.t) * a.ldy[w] + h;
            v.x[0] = *(const Piece *)p;
            v.x[1] = *(const Piece *)(p + step * VE);
        };
#pragma unroll
        for (int u = 0; u < U; ++u) load(first + u * RP, row[u]);
        float gf[2][VE];
        if (g) {
            Piece gp[2] = {};
            if (on) {
                gp[0] = *(const Piece *)(g + pa * VE);
                gp[1] = *(const Piece *)(g + (pa + step) * VE);
            }
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int e = 0; e < VE; ++e) gf[i][e] = value(gp[i], e);
        }
        if (w == w0 && a.half) {
            angles(a, t0, tokens, cs);
            __syncthreads();
        }
        for (int r0 = first; r0 < n; r0 += U * RP) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int r = r0 + u * RP;
                float y[2][VE];
                float ss = 0.f;
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int e = 0; e < VE; ++e) {
                        y[i][e] = value(row[u].x[i], e);
                        if (g) ss = fmaf(y[i][e], y[i][e], ss);
                    }
                const int64_t to0 = row[u].y;
                const int t = row[u].t;
                load(r + U * RP, row[u]);
                if (g) {
#pragma unroll
                    for (int o = LPR / 2; o >= 1; o >>= 1) ss += __shfl_xor(ss, o);
                    const float inv = 1.f / sqrtf(ss / (float)a.dh + a.eps);
#pragma unroll
                    for (int i = 0; i < 2; ++i)
#pragma unroll
                        for (int e = 0; e < VE; ++e) y[i][e] = y[i][e] * inv * gf[i][e];
                }
                if (r >= n || !on) continue;
                if (turn) {
                    const f32x4 *f = (const f32x4 *)(cs + t * a.half + c * VE);
#pragma unroll
                    for (int e = 0; e < VE; e += 2) {
                        const f32x4 f2 = f[e / 2];
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            const float lo = y[0][e + i], hi = y[1][e + i], cn = f2[2 * i], sn = f2[2 * i + 1];
                            y[0][e + i] = fmaf(lo, cn, -hi * sn);
                            y[1][e + i] = fmaf(hi, cn, lo * sn);
                        }
                    }
                }
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    Piece o;
#pragma unroll
                    for (int e = 0; e < W; ++e) {
                        if constexpr (sizeof(T) == 4) o[e] = __float_as_uint(y[i][e]);
                        else o[e] = pack_bf16x2(y[i][2 * e], y[i][2 * e + 1]);
                    }
                    Piece *const to = (Piece *)((T *)a.y[w] + to0 + i * step * VE);
                    // (of many tokens no cache holds the results until they are read: 42.6 us without, 36.9 with, where reads said so too 38.8)
                    if constexpr (TPB > 1) __builtin_nontemporal_store(o, to);
                    else *to = o;
                }
            }
        }
    }
}

template <typename T, int W, int LPR>
hipError_t launch_pieces(const RopeNormArgs &a, const RopePlan &p, hipStream_t st)
{
    const dim3 grid((unsigned)((a.T + p.tokens - 1) / p.tokens), p.apart ? 2 : 1);
    prof_begin(K_QK_NORM_ROPE, st);
    if (p.tokens == 16) MOA_KLAUNCH((k_qk_norm_rope_pieces<T, W, LPR, 16>), grid, dim3(256), 0, st, a);
    else if (p.tokens == 4) MOA_KLAUNCH((k_qk_norm_rope_pieces<T, W, LPR, 4>), grid, dim3(256), 0, st, a);
    else MOA_KLAUNCH((k_qk_norm_rope_pieces<T, W, LPR, 1>), grid, dim3(256), 0, st, a);
    prof_end(st);
    return hipGetLastError();
}

template <typename T, int W>
hipError_t launch_width(const RopeNormArgs &a, const RopePlan &p, hipStream_t st)
{
    constexpr int MOST = 256 * sizeof(T) / (8 * W);      // pairs of pieces that a head can have
    if (p.lanes == 4) return launch_pieces<T, W, 4>(a, p, st);
    if (p.lanes == 8) return launch_pieces<T, W, 8>(a, p, st);
    if constexpr (MOST > 32)
        if (p.lanes == 64) return launch_pieces<T, W, 64>(a, p, st);
    if constexpr (MOST > 16)
        if (p.lanes == 32) return launch_pieces<T, W, 32>(a, p, st);
    return launch_pieces<T, W, 16>(a, p, st);
}

template <typename T>
hipError_t launch(const RopeNormArgs &a, hipStream_t st)
{
    uint64_t bits = 0, elems = 0;
    for (int w = 0; w < 2; ++w)
        if (a.heads[w]) {
            bits |= (uintptr_t)a.x[w] | (uintptr_t)a.y[w] | (uintptr_t)a.g[w];
            elems |= (uint64_t)(a.ldx[w] | a.ldy[w]);
        }
    const RopePlan p = rope_plan(sizeof(T), a.dh, a.half, bits, elems, a.T, a.heads[0] > a.heads[1] ? a.heads[0] : a.heads[1]);
    if (p.words == 4) return launch_width<T, 4>(a, p, st);
    if (p.words == 2) return launch_width<T, 2>(a, p, st);
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
    if (head_dim < 1 || head_dim > 256 || n_q_heads < 0 || n_kv_heads < 0 || n_q_heads > (1 << 20) || n_kv_heads > (1 << 20) || T < 0 || T > (1 << 23))
        return api_fail(MOA_ERR_SHAPE, "qk_norm_rope: dimensions (1 <= head_dim <= 256, heads within 2^20, T within 2^23)");
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
    RopeNormArgs a = {{q, k}, {q_out, k_out}, {gq, gk}, {q_stride, k_stride}, {q_out_stride, k_out_stride}, {n_q_heads, n_kv_heads},
                      {FastDiv(n_q_heads ? n_q_heads : 1), FastDiv(n_kv_heads ? n_kv_heads : 1)}, T, pos,
                            head_dim, rot_dim / 2, rms_eps, {}};
    for (int i = 0; i < 7 && rot_dim; ++i) a.power[i] = exp(-log((double)rope_theta) * ((1 << i) / (0.5 * rot_dim)));
    prof_set_site(S_QK_NORM_ROPE);
    const hipError_t e = dtype == MOA_BF16 ? launch<bf16_t>(a, (hipStream_t)stream) : launch<float>(a, (hipStream_t)stream);
    return e == hipSuccess ? MOA_OK : api_fail(MOA_ERR_HIP, hipGetErrorString(e));
}

}  // extern "C"
