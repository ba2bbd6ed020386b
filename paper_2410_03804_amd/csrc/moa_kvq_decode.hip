// Attention of one new token per sequence over its cache of pages held in 8 bits (moa_kvq_decode_attn).
//
// As moa_decode_attn.hip, with keys and values code * scale, a scale for each block of rows of a page and KV head:
//   s_j = (q . c_j) ks_j log2(e) / sqrt(dh),  l = sum 2^(s_j - m),  o = sum (2^(s_j - m) vs_j) d_j / l,
// c_j, d_j the codes of key and value j and ks_j, vs_j their blocks' scales: a scale is multiplied into the score or the weight, once
// a key, and not into every element.  The list of tiles, the runs and the second launch are moa_decode_attn's.
#include "moa_decode_device.h"
#include "moa_kvq_device.h"
#include "moa_kvq_plan.h"

namespace moa {

namespace {

struct KvqDecodeArgs {
    DecodeArgs d;
    const float *k_scale, *v_scale;
    int blocks;                       // of a page
};

// ---------------------------------------------------------------- element by element
// A row of keys or values is spread over LPR lanes, four codes each; 64 / LPR keys at a time.  WORDS: they can be read as one word.
template <typename T, int LPR, bool WORDS>
__global__ __launch_bounds__(256, 2) void k_kvq_decode(KvqDecodeArgs k)
{
    constexpr int HG = 4, VE = 4, KPW = 64 / LPR, U = 4;
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    const DecodeArgs &a = k.d;
    float *acc_s = (float *)smem, *ml_s = acc_s + WAVES * a.HG * a.c.dh, *fin = ml_s + WAVES * a.HG * 2;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, c = lane % LPR, grp = lane / LPR, dh = a.c.dh;
    const int e0 = c * VE, ne = min(max(dh - e0, 0), VE);
    for_each_pair(a, [&](int b, int len, int hb, uint32_t t0, uint32_t nt, bool whole, int64_t slot) {
        const int h = hb / a.rtiles, r0 = (hb - h * a.rtiles) * a.HG, rows = min(a.HG, a.G - r0);
        float qf[HG][VE], acc[HG][VE], m[HG], l[HG];
        uint64_t any = 0;                        // lanes that have had a key
#pragma unroll
        for (int r = 0; r < HG; ++r) {
            const T *qr = (const T *)a.q + ((int64_t)b * a.H + h * a.G + r0 + min(r, rows - 1)) * dh + e0;
#pragma unroll
            for (int e = 0; e < VE; ++e) {
                qf[r][e] = e < ne ? ld(qr + e) * a.scale : 0.f;
                acc[r][e] = 0.f;
            }
            m[r] = -INFINITY;
            l[r] = 0.f;
        }
        auto load = [&](const char *pool, int row) {
            const unsigned char *p = (const unsigned char *)pool + (int64_t)row * dh + e0;
            uint32_t x = 0;
            if (row < 0 || ne == 0) return x;
            if (WORDS) return *(const uint32_t *)p;
#pragma unroll
            for (int e = 0; e < VE; ++e)
                if (e < ne) x |= (uint32_t)p[e] << 8 * e;
            return x;
        };
        const int first = (int)t0 * TK, last = min(len, (int)(t0 + nt) * TK);
#pragma unroll 1
        for (int s0 = first + wave * KPW * U; s0 < last; s0 += WAVES * KPW * U) {
            int row[U];
            uint32_t kc[U], vc[U];
            float ks[U], vs[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int s = s0 + u * KPW + grp;
                row[u] = -1;
                ks[u] = vs[u] = 0.f;
                if (s < last) {
                    const int pg = (int)a.c.page((uint32_t)s), id = a.c.table[(int64_t)b * a.c.max_pages + pg];
                    row[u] = a.c.row_in(id, pg, h, s);
                    if (row[u] < 0) a.c.flag(MOA_DEV_BAD_PAGE);
                    else {
                        const int block = (id * a.c.Hkv + h) * k.blocks + (s - pg * (int)a.c.page.d) / MOA_KVQ_BLOCK;
                        ks[u] = k.k_scale[block];
                        vs[u] = k.v_scale[block];
                    }
                }
                any |= __ballot(row[u] >= 0);
                kc[u] = load(a.c.k, row[u]);
                vc[u] = load(a.c.v, row[u]);
            }
            float s[U][HG];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const float x[VE] = {code_value<0>(kc[u]), code_value<1>(kc[u]), code_value<2>(kc[u]), code_value<3>(kc[u])};
#pragma unroll
                for (int r = 0; r < HG; ++r) {
                    float d = 0.f;
#pragma unroll
                    for (int e = 0; e < VE; ++e) d = fmaf(qf[r][e], x[e], d);
#pragma unroll
                    for (int o = LPR / 2; o >= 1; o >>= 1) d += __shfl_xor(d, o);
                    s[u][r] = row[u] >= 0 ? d * ks[u] : -INFINITY;
                }
            }
#pragma unroll
            for (int r = 0; r < HG; ++r) {
                float mn = m[r];
#pragma unroll
                for (int u = 0; u < U; ++u) mn = fmaxf(mn, s[u][r]);
                const float ms = mn == -INFINITY ? 0.f : mn, corr = fast_exp2(m[r] - ms);
                m[r] = mn;
                l[r] *= corr;
#pragma unroll
                for (int e = 0; e < VE; ++e) acc[r][e] *= corr;
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const float p = fast_exp2(s[u][r] - ms), w = p * vs[u];
                    l[r] += p;
                    acc[r][0] = fmaf(w, code_value<0>(vc[u]), acc[r][0]);
                    acc[r][1] = fmaf(w, code_value<1>(vc[u]), acc[r][1]);
                    acc[r][2] = fmaf(w, code_value<2>(vc[u]), acc[r][2]);
                    acc[r][3] = fmaf(w, code_value<3>(vc[u]), acc[r][3]);
                }
            }
        }
        // the lane groups' parts of a head, then one per wavefront into LDS
#pragma unroll
        for (int r = 0; r < HG; ++r) {
            if (r >= a.HG) break;
            constexpr int FROM = LPR == 16 ? 4 : LPR == 32 ? 5 : 6;
            const float mn = over_lanes<FROM>(m[r], fmaxf), ms = mn == -INFINITY ? 0.f : mn, corr = fast_exp2(m[r] - ms);
            l[r] = over_lanes<FROM>(l[r] * corr, add);
#pragma unroll
            for (int e = 0; e < VE; ++e) {
                const float o = over_lanes<FROM>(acc[r][e] * corr, add);
                if (grp == 0 && e < ne) acc_s[(wave * a.HG + r) * dh + e0 + e] = o;
            }
            if (lane == 0) {
                ml_s[(wave * a.HG + r) * 2] = max_of_keys(mn, any != 0);
                ml_s[(wave * a.HG + r) * 2 + 1] = l[r];
            }
        }
        finish<T, 0>(a, b, len, hb, whole, slot, acc_s, a.HG * dh, ml_s, fin);
    });
}

// ---------------------------------------------------------------- host
template <typename T, int LPR>
hipError_t launch_elements(const KvqDecodeArgs &k, int grid, hipStream_t st)
{
    const DecodeArgs &a = k.d;
    const size_t lds = ((size_t)WAVES * a.HG * (a.c.dh + 2) + a.HG * 2) * 4;
    const bool words = a.c.dh % 4 == 0 && !(((uintptr_t)a.c.k | (uintptr_t)a.c.v) & 3);
    prof_begin(K_KVQ_DECODE, st);
    if (words) MOA_KLAUNCH((k_kvq_decode<T, LPR, true>), dim3(grid), dim3(64 * WAVES), lds, st, k);
    else MOA_KLAUNCH((k_kvq_decode<T, LPR, false>), dim3(grid), dim3(64 * WAVES), lds, st, k);
    prof_end(st);
    return hipGetLastError();
}

template <typename T>
hipError_t launch_decode(const KvqDecodeArgs &k, hipStream_t st)
{
    const DecodeArgs &a = k.d;
    const int grid = a.runs ? a.runs : a.c.B * a.HB;
    const hipError_t e = a.c.dh <= 64 ? launch_elements<T, 16>(k, grid, st) : a.c.dh <= 128 ? launch_elements<T, 32>(k, grid, st) : launch_elements<T, 64>(k, grid, st);
    if (e != hipSuccess || !a.runs) return e;
    return launch_decode_join(a, sizeof(T) == 2, st);
}

KvqPlan plan_of(const moa_kvq_cache_t &c, int H) { return kvq_plan(c.B, c.n_kv_heads, c.head_dim, c.max_pages * c.page_size, H); }

int32_t check_decode(const moa_kvq_cache_t *c, int32_t H, const char *who)
{
    int32_t rc = check_kvq_cache(c, who);
    if (rc) return rc;
    if (H < 1 || H % c->n_kv_heads) return api_fail(MOA_ERR_SHAPE, "kvq_decode_attn: n_q_heads must be a multiple of the cache's n_kv_heads");
    if ((int64_t)c->B * H > (1 << 20)) return api_fail(MOA_ERR_SHAPE, "kvq_decode_attn: more than 2^20 pairs of sequence and query head");
    const int64_t cap = (int64_t)c->max_pages * c->page_size;
    // tiles are counted in 32 bits
    if ((int64_t)c->B * H * ((cap + TK - 1) / TK) > INT32_MAX / 2)
        return api_fail(MOA_ERR_SHAPE, "kvq_decode_attn: B * n_q_heads * ceil(capacity / 128) above 2^30");
    return MOA_OK;
}

}  // namespace
}  // namespace moa

using namespace moa;

extern "C" {

int32_t moa_kvq_decode_attn_workspace_bytes(const moa_kvq_cache_t *cache, int32_t n_q_heads, size_t *bytes_host)
{
    if (!bytes_host) return api_fail(MOA_ERR_NULL, "kvq_decode_attn_workspace_bytes: bytes_host is NULL");
    const int32_t rc = check_decode(cache, n_q_heads, "kvq_decode_attn_workspace_bytes");
    if (rc) return rc;
    *bytes_host = plan_of(*cache, n_q_heads).total();
    return MOA_OK;
}

int32_t moa_kvq_decode_attn(const moa_kvq_cache_t *cache, int32_t n_q_heads, const void *q, void *out, int32_t *dev_status, void *ws,
                            size_t ws_bytes, void *stream)
{
    const int32_t rc = check_decode(cache, n_q_heads, "kvq_decode_attn");
    if (rc) return rc;
    if (!q || !out) return api_fail(MOA_ERR_NULL, "kvq_decode_attn: q / out is NULL");
    if (((uintptr_t)q | (uintptr_t)out) & (cache->dtype == MOA_BF16 ? 1 : 3)) return api_fail(MOA_ERR_SHAPE, "kvq_decode_attn: q / out not aligned to their elements");
    const KvqPlan p = plan_of(*cache, n_q_heads);
    const size_t need = p.total();
    if (need && (!ws || (((uintptr_t)ws) & 255) || ws_bytes < need))
        return api_fail(MOA_ERR_WORKSPACE, "kvq_decode_attn: workspace NULL, misaligned or smaller than moa_kvq_decode_attn_workspace_bytes");
    const KvqDecodeArgs k = {{KvDev(kvq_geometry(*cache), dev_status), q, out, n_q_heads, n_q_heads / cache->n_kv_heads, p.HG, p.rtiles, cache->n_kv_heads * p.rtiles,
                              p.runs, p.runs ? 31 - __builtin_clz((unsigned)p.runs) : 0, 1.4426950408889634f / sqrtf((float)cache->head_dim),
                              (float *)ws, (float *)((char *)ws + p.part_o), 0, nullptr},
                             cache->k_scale, cache->v_scale, kvq_blocks(cache->page_size)};
    prof_set_site(S_KVQ);
    hipStream_t st = (hipStream_t)stream;
    const hipError_t e = cache->dtype == MOA_BF16 ? launch_decode<bf16_t>(k, st) : launch_decode<float>(k, st);
    return e == hipSuccess ? MOA_OK : api_fail(MOA_ERR_HIP, hipGetErrorString(e));
}

}  // extern "C"
