// Attention of one new token per sequence over its cache of pages (moa_decode_attn).
//
// One pass over the keys and values with the running maximum m and sum l of a softmax per query head, scores in the log2 domain:
//   s_j = q . k_j log2(e) / sqrt(dh),  l = sum 2^(s_j - m),  o = sum 2^(s_j - m) v_j / l.
// The work is the list of all tiles of TK keys of all (sequence, KV head) pairs, in that order, cut into equal runs, one per
// workgroup: lengths are only known on the device, and a batch of very different ones is then as fast as an even one.  A run
// that has all tiles of a pair writes its result; other pairs leave m, l and the unnormalised o (single precision) of each run
// that touched them in the workspace for a second launch to join.
#include "moa_attn_device.h"
#include "moa_kv_device.h"

namespace moa {

namespace {

constexpr int TK = 128, WAVES = 4, WK = TK / WAVES;        // keys of a tile, wavefronts, keys of a tile that a wavefront takes

struct DecodeArgs {
    KvDev c;
    const void *q;                // [B, H, dh]
    void *out;                    // [B, H, dh]
    int H, G, HG, rtiles, HB;     // query heads, per KV head; of these in a tile; tiles per KV head; Hkv * rtiles
    int runs;                     // workgroups the tiles are dealt to; 0: one workgroup per pair
    int min_run;                  // tiles of a run, at least
    int wide;                     // rows can be read 16 bytes at a time
    float scale;                  // log2(e) / sqrt(dh)
    float *part_o;                // [runs + B HB][HG][dh]
    float *part_ml;               // [runs + B HB][HG][2]
    float *raw;                   // [B, H, cap] scores, where accounts are kept; else NULL
};

__device__ __forceinline__ uint32_t wave_scan(uint32_t x, int lane)
{
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const uint32_t y = __shfl_up(x, d);
        if (lane >= d) x += y;
    }
    return x;
}

__device__ __forceinline__ uint32_t uniform(uint32_t x) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)x); }

// Where the tiles of the sequences lie in the list of all tiles: every wavefront works this out for itself.
struct TileList {
    uint32_t total, per;          // tiles in all, of a run
    __device__ __forceinline__ uint32_t tiles(const DecodeArgs &a, int b) const
    {
        return b < a.c.B ? (uint32_t)(a.c.length(b, false) + TK - 1) / TK : 0u;
    }
    __device__ __forceinline__ explicit TileList(const DecodeArgs &a)
    {
        const int lane = threadIdx.x & 63;
        uint32_t x = 0;
        for (int b = lane; b < a.c.B; b += 64) x += tiles(a, b);
#pragma unroll
        for (int d = 32; d; d >>= 1) x += __shfl_xor(x, d);
        total = uniform(x) * (uint32_t)a.HB;
        const uint32_t even = (total + a.runs - 1) / a.runs;
        per = even > (uint32_t)a.min_run ? even : (uint32_t)a.min_run;
    }
    // the sequence of tile f < total and its first tile
    __device__ __forceinline__ void find(const DecodeArgs &a, uint32_t f, int &b, uint32_t &begin, uint32_t &nt) const
    {
        const int lane = threadIdx.x & 63;
        uint32_t base = 0;
        for (int b0 = 0;; b0 += 64) {
            const uint32_t mine = tiles(a, b0 + lane), upto = base + wave_scan(mine, lane);
            const uint64_t past = __ballot(f < upto * (uint32_t)a.HB);
            if (past || b0 + 64 >= a.c.B) {
                const int at = past ? __ffsll((unsigned long long)past) - 1 : 63;
                b = b0 + at;
                nt = uniform(__shfl(mine, at));
                begin = (uniform(__shfl(upto, at)) - nt) * (uint32_t)a.HB;
                return;
            }
            base = uniform(__shfl(upto, 63));
        }
    }
};

// ---------------------------------------------------------------- what either kernel does with a run's result
// LDS: acc [WAVES][HG][dh], ml [WAVES][HG][2] hold each wavefront's part.
template <typename T>
__device__ __forceinline__ void finish(const DecodeArgs &a, int b, int hb, uint32_t t0, uint32_t nt, bool whole, int64_t slot, const float *acc,
                                       const float *ml, float *fin)
{
    const int tid = threadIdx.x, dh = a.c.dh, h = hb / a.rtiles, rt = hb - h * a.rtiles;
    const int r0 = rt * a.HG, rows = min(a.HG, a.G - r0);
    __syncthreads();
    if (tid < rows) {
        float m = -INFINITY, l = 0.f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) m = fmaxf(m, ml[(w * a.HG + tid) * 2]);
        const float ms = m == -INFINITY ? 0.f : m;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) l += ml[(w * a.HG + tid) * 2 + 1] * fast_exp2(ml[(w * a.HG + tid) * 2] - ms);
        fin[tid * 2] = ms;
        fin[tid * 2 + 1] = whole ? (l == 0.f ? 0.f : 1.f / l) : 1.f;
        // (a pair with several row tiles has its accounts changed by the second launch in any case)
        if (!whole || (a.raw && a.rtiles > 1)) {
            a.part_ml[(slot * a.HG + tid) * 2] = m;
            a.part_ml[(slot * a.HG + tid) * 2 + 1] = l;
        }
        if (whole && l == 0.f) a.c.flag(MOA_DEV_EMPTY_KEYS);
    }
    __syncthreads();
    for (int i = tid; i < rows * dh; i += 64 * WAVES) {
        const int r = i / dh, d = i - r * dh;
        float o = 0.f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) o += acc[(w * a.HG + r) * dh + d] * fast_exp2(ml[(w * a.HG + r) * 2] - fin[r * 2]);
        o *= fin[r * 2 + 1];
        if (whole) st((T *)a.out + ((int64_t)b * a.H + h * a.G + r0 + r) * dh + d, o);
        else a.part_o[(slot * a.HG + r) * dh + d] = o;
    }
    // A pair's accounts are one workgroup's to change only where it has all its keys and all its query heads.
    if (a.raw && whole && a.rtiles == 1) {
        const int n = min((int)((t0 + nt) * TK), a.c.length(b, false));
        for (int s = (int)t0 * TK + tid; s < n; s += 64 * WAVES) {
            float p = 0.f;
            for (int r = 0; r < rows; ++r) p += fast_exp2(a.raw[((int64_t)b * a.H + h * a.G + r) * a.c.cap + s] - fin[r * 2]) * fin[r * 2 + 1];
            a.c.score[((int64_t)b * a.c.Hkv + h) * a.c.cap + s] += p;
        }
    }
    __syncthreads();
}

// The runs of a workgroup: each of the pairs that its tiles belong to, with process(b, hb, first tile, tiles, all of them, partial slot).
template <typename F>
__device__ __forceinline__ void for_each_pair(const DecodeArgs &a, const F &process)
{
    if (a.runs == 0) {
        const int b = (int)blockIdx.x / a.HB, hb = (int)blockIdx.x - b * a.HB;
        process(b, hb, 0u, (uint32_t)(a.c.length(b, hb == 0 && threadIdx.x == 0) + TK - 1) / TK, true, (int64_t)0);
        return;
    }
    const TileList list(a);
    uint32_t f = blockIdx.x * list.per;
    const uint32_t end = min(f + list.per, list.total);
    if (f >= end) return;
    int b;
    uint32_t begin, nt;
    list.find(a, f, b, begin, nt);
    for (;;) {
        const uint32_t in = f - begin, hb = in / nt, t = in - hb * nt, cnt = min(nt - t, end - f);
        process(b, (int)hb, t, cnt, cnt == nt, (int64_t)blockIdx.x + (int64_t)b * a.HB + hb);
        f += cnt;
        if (f >= end) return;
        if (f == begin + nt * (uint32_t)a.HB) {
            begin = f;
            do {
                ++b;
                nt = uniform(list.tiles(a, b));
            } while (nt == 0);                              // (f < total: there is one)
        }
    }
}

// ---------------------------------------------------------------- element by element: any head_dim, either type
template <int LPR>
__device__ __forceinline__ float sum_over_lanes(float x)
{
    x += dpp_move_f32<0xB1>(x);     // quad_perm [1, 0, 3, 2]
    x += dpp_move_f32<0x4E>(x);     // quad_perm [2, 3, 0, 1]
    x += dpp_move_f32<0x141>(x);    // row_half_mirror
    if (LPR >= 16) x += dpp_move_f32<0x140>(x);    // row_mirror
    if (LPR >= 32) x += __shfl_xor(x, 16);
    if (LPR >= 64) x += __shfl_xor(x, 32);
    return x;
}

// A row of keys or values is spread over LPR lanes, VE = 16 bytes' worth of elements each; 64 / LPR keys at a time.
template <typename T, int LPR, int HG>
__global__ __launch_bounds__(256) void k_decode_attn(DecodeArgs a)
{
    constexpr int VE = 16 / sizeof(T), KPW = 64 / LPR, U = 4;
    extern __shared__ float smem[];
    float *acc_s = smem, *ml_s = acc_s + WAVES * HG * a.c.dh, *fin = ml_s + WAVES * HG * 2;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, c = lane % LPR, grp = lane / LPR, dh = a.c.dh;
    const int e0 = c * VE, ne = min(max(dh - e0, 0), VE);
    for_each_pair(a, [&](int b, int hb, uint32_t t0, uint32_t nt, bool whole, int64_t slot) {
        const int h = hb / a.rtiles, r0 = (hb - h * a.rtiles) * HG, rows = min(HG, a.G - r0);
        const int len = a.c.length(b, hb == 0 && t0 == 0 && tid == 0);
        float qf[HG][VE], acc[HG][VE], m[HG], l[HG];
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
        auto load = [&](const char *pool, int row, float (&x)[VE]) {
            const T *p = (const T *)pool + (int64_t)row * dh + e0;
            union { u32x4 v; T t[VE]; } u;
            u.v = u32x4{0u, 0u, 0u, 0u};
            if (row >= 0 && ne > 0) {
                if (a.wide) u.v = *(const u32x4 *)p;
                else
                    for (int e = 0; e < ne; ++e) u.t[e] = p[e];
            }
#pragma unroll
            for (int e = 0; e < VE; ++e) x[e] = ld(&u.t[e]);
        };
        for (uint32_t t = t0; t < t0 + nt; ++t)
            for (int s0 = 0; s0 < WK; s0 += KPW * U) {
                int slots[U], row[U];
                float x[U][VE], s[U][HG];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    slots[u] = (int)t * TK + wave * WK + s0 + u * KPW + grp;
                    row[u] = -1;
                    if (slots[u] < len) {
                        row[u] = a.c.row(b, h, slots[u]);
                        if (row[u] < 0) a.c.flag(MOA_DEV_BAD_PAGE);
                    }
                    load(a.c.k, row[u], x[u]);
                }
#pragma unroll
                for (int u = 0; u < U; ++u)
#pragma unroll
                    for (int r = 0; r < HG; ++r) {
                        float d = 0.f;
#pragma unroll
                        for (int e = 0; e < VE; ++e) d = fmaf(qf[r][e], x[u][e], d);
                        d = sum_over_lanes<LPR>(d);
                        s[u][r] = row[u] >= 0 ? d : -INFINITY;
                        if (a.raw && c == 0 && slots[u] < len && r < rows)
                            a.raw[((int64_t)b * a.H + h * a.G + r0 + r) * a.c.cap + slots[u]] = s[u][r];
                    }
#pragma unroll
                for (int u = 0; u < U; ++u) load(a.c.v, row[u], x[u]);
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
                        const float p = fast_exp2(s[u][r] - ms);
                        l[r] += p;
#pragma unroll
                        for (int e = 0; e < VE; ++e) acc[r][e] = fmaf(p, x[u][e], acc[r][e]);
                    }
                }
            }
        // the lane groups' parts of a head, then one per wavefront into LDS
#pragma unroll
        for (int r = 0; r < HG; ++r) {
            float mn = m[r];
#pragma unroll
            for (int d = LPR; d < 64; d <<= 1) mn = fmaxf(mn, __shfl_xor(mn, d));
            const float ms = mn == -INFINITY ? 0.f : mn, corr = fast_exp2(m[r] - ms);
            l[r] *= corr;
#pragma unroll
            for (int d = LPR; d < 64; d <<= 1) l[r] += __shfl_xor(l[r], d);
#pragma unroll
            for (int e = 0; e < VE; ++e) {
                float o = acc[r][e] * corr;
#pragma unroll
                for (int d = LPR; d < 64; d <<= 1) o += __shfl_xor(o, d);
                if (grp == 0 && e < ne) acc_s[(wave * HG + r) * dh + e0 + e] = o;
            }
            if (lane == 0) {
                ml_s[(wave * HG + r) * 2] = mn;
                ml_s[(wave * HG + r) * 2 + 1] = l[r];
            }
        }
        finish<T>(a, b, hb, t0, nt, whole, slot, acc_s, ml_s, fin);
    });
}

// ---------------------------------------------------------------- the second launch
// Workgroups 0 .. B HB - 1 join the partial results of a pair; the others bring the accounts of 1024 slots of a (sequence, KV
// head) up to date from its scores, now that the sums are known.  Either leaves alone what the first launch finished.
constexpr int ACC_SLOTS = 1024;
template <typename T>
__global__ __launch_bounds__(256) void k_decode_join(DecodeArgs a)
{
    __shared__ float sm[2][16][16], fin[16][2];
    const int tid = threadIdx.x, dh = a.c.dh;
    const TileList list(a);
    const int nb = a.c.B * a.HB;
    const bool accounts = (int)blockIdx.x >= nb;
    int b, hb, chunk = 0;
    if (!accounts) {
        b = (int)blockIdx.x / a.HB;
        hb = (int)blockIdx.x - b * a.HB;
    } else {
        const int chunks = (a.c.cap + ACC_SLOTS - 1) / ACC_SLOTS, i = (int)blockIdx.x - nb, bh = i / chunks;
        chunk = i - bh * chunks;
        b = bh / a.c.Hkv;
        hb = (bh - b * a.c.Hkv) * a.rtiles;
    }
    const int len = a.c.length(b, !accounts && hb == 0 && tid == 0);
    const uint32_t nt = (uint32_t)(len + TK - 1) / TK;
    uint32_t before = 0;
    for (int i = tid & 63; i < b; i += 64) before += list.tiles(a, i);
#pragma unroll
    for (int d = 32; d; d >>= 1) before += __shfl_xor(before, d);
    const uint32_t begin = uniform(before) * (uint32_t)a.HB;
    float accs[ACC_SLOTS / 256] = {0.f, 0.f, 0.f, 0.f};      // of this thread's slots, over the row tiles
    for (int rt = 0; rt < (accounts ? a.rtiles : 1); ++rt, ++hb) {
        const int h = hb / a.rtiles, r0 = (hb - h * a.rtiles) * a.HG, rows = min(a.HG, a.G - r0);
        const uint32_t f0 = begin + (uint32_t)hb * nt;
        const uint32_t w0 = f0 / list.per, w1 = nt ? (f0 + nt - 1) / list.per : w0;
        if (!accounts && nt == 0) {
            for (int i = tid; i < rows * dh; i += 256) st((T *)a.out + ((int64_t)b * a.H + h * a.G + r0) * dh + i, 0.f);
            if (tid == 0) a.c.flag(MOA_DEV_EMPTY_KEYS);
            return;
        }
        if (accounts && chunk * ACC_SLOTS >= len) return;
        if (w0 == w1 && (!accounts || a.rtiles == 1)) return;        // the first launch had all of it
        // of each row the maximum and the sum: sixteen threads a row
        const int64_t slot0 = (int64_t)w0 + (int64_t)b * a.HB + hb, ns = (int64_t)w1 - w0 + 1;
        const int row = tid & 15, part = tid >> 4;
        float m = -INFINITY, l = 0.f;
        if (row < rows)
            for (int64_t s = part; s < ns; s += 16) m = fmaxf(m, a.part_ml[((slot0 + s) * a.HG + row) * 2]);
        __syncthreads();
        sm[0][row][part] = m;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 16; ++i) m = fmaxf(m, sm[0][row][i]);
        const float ms = m == -INFINITY ? 0.f : m;
        if (row < rows)
            for (int64_t s = part; s < ns; s += 16) {
                const float *ml = a.part_ml + ((slot0 + s) * a.HG + row) * 2;
                l += ml[1] * fast_exp2(ml[0] - ms);
            }
        sm[1][row][part] = l;
        __syncthreads();
        if (part == 0) {
            l = 0.f;
#pragma unroll
            for (int i = 0; i < 16; ++i) l += sm[1][row][i];
            fin[row][0] = ms;
            fin[row][1] = l == 0.f ? 0.f : 1.f / l;
            if (!accounts && row < rows && l == 0.f) a.c.flag(MOA_DEV_EMPTY_KEYS);
        }
        __syncthreads();
        if (!accounts) {
            for (int i = tid; i < rows * dh; i += 256) {
                const int r = i / dh, d = i - r * dh;
                float o = 0.f;
                for (int64_t s = 0; s < ns; ++s) o += a.part_o[((slot0 + s) * a.HG + r) * dh + d] * fast_exp2(a.part_ml[((slot0 + s) * a.HG + r) * 2] - fin[r][0]);
                st((T *)a.out + ((int64_t)b * a.H + h * a.G + r0 + r) * dh + d, o * fin[r][1]);
            }
        } else {
#pragma unroll
            for (int i = 0; i < ACC_SLOTS / 256; ++i) {
                const int s = chunk * ACC_SLOTS + i * 256 + tid;
                if (s < len)
                    for (int r = 0; r < rows; ++r)
                        accs[i] += fast_exp2(a.raw[((int64_t)b * a.H + h * a.G + r0 + r) * a.c.cap + s] - fin[r][0]) * fin[r][1];
            }
        }
    }
    if (accounts) {
        const int h = hb / a.rtiles - 1;                     // (the loop left hb one past the head's last row tile)
#pragma unroll
        for (int i = 0; i < ACC_SLOTS / 256; ++i) {
            const int s = chunk * ACC_SLOTS + i * 256 + tid;
            if (s < len) a.c.score[((int64_t)b * a.c.Hkv + h) * a.c.cap + s] += accs[i];
        }
    }
}

// ---------------------------------------------------------------- host
struct DecodePlan {
    int HG, rtiles, runs;
    size_t part_o, part_ml, raw;       // bytes
    size_t total() const { return part_o + part_ml + raw; }
};

size_t align256(size_t n) { return (n + 255) & ~(size_t)255; }

DecodePlan decode_plan(const moa_kv_cache_t &c, int H, bool accounts)
{
    DecodePlan p;
    const int G = H / c.n_kv_heads, cap = c.max_pages * c.page_size;
    p.HG = G <= 2 ? 2 : 8;
    p.rtiles = (G + p.HG - 1) / p.HG;
    const int64_t pairs = (int64_t)c.B * c.n_kv_heads * p.rtiles;
    // one workgroup per pair where that is a short walk, without a second launch; else four workgroups per compute unit
    p.runs = cap <= 4 * TK && !(accounts && p.rtiles > 1) ? 0 : 1024;
    p.part_o = p.runs ? align256((size_t)(p.runs + pairs) * p.HG * c.head_dim * 4) : 0;
    p.part_ml = p.runs ? align256((size_t)(p.runs + pairs) * p.HG * 2 * 4) : 0;
    p.raw = accounts ? align256((size_t)c.B * H * cap * 4) : 0;
    return p;
}

template <typename T, int LPR, int HG>
hipError_t launch_one(const DecodeArgs &a, int grid, hipStream_t st)
{
    const size_t lds = ((size_t)WAVES * HG * (a.c.dh + 2) + HG * 2) * 4;
    prof_begin(K_DECODE_ATTN, st);
    MOA_KLAUNCH((k_decode_attn<T, LPR, HG>), dim3(grid), dim3(64 * WAVES), lds, st, a);
    prof_end(st);
    return hipGetLastError();
}

template <typename T>
hipError_t launch_decode(const DecodeArgs &a, hipStream_t st)
{
    const int grid = a.runs ? a.runs : a.c.B * a.HB;
    constexpr int VE = 16 / sizeof(T), L1 = 64 / VE;
    hipError_t e;
    if (a.HG == 2) e = a.c.dh <= 64 ? launch_one<T, L1, 2>(a, grid, st) : a.c.dh <= 128 ? launch_one<T, 2 * L1, 2>(a, grid, st) : launch_one<T, 4 * L1, 2>(a, grid, st);
    else e = a.c.dh <= 64 ? launch_one<T, L1, 8>(a, grid, st) : a.c.dh <= 128 ? launch_one<T, 2 * L1, 8>(a, grid, st) : launch_one<T, 4 * L1, 8>(a, grid, st);
    if (e != hipSuccess || !a.runs) return e;
    const int64_t chunks = (a.c.cap + ACC_SLOTS - 1) / ACC_SLOTS;
    prof_begin(K_DECODE_JOIN, st);
    MOA_KLAUNCH(k_decode_join<T>, dim3((unsigned)(a.c.B * a.HB + (a.raw ? a.c.B * a.c.Hkv * chunks : 0))), dim3(256), 0, st, a);
    prof_end(st);
    return hipGetLastError();
}

int32_t check_decode(const moa_kv_cache_t *c, int32_t H, const char *who)
{
    int32_t rc = check_kv_cache(c, who);
    if (rc) return rc;
    if (H < 1 || H % c->n_kv_heads) return api_fail(MOA_ERR_SHAPE, "decode_attn: n_q_heads must be a multiple of the cache's n_kv_heads");
    if ((int64_t)c->B * H > (1 << 20)) return api_fail(MOA_ERR_SHAPE, "decode_attn: more than 2^20 pairs of sequence and query head");
    const int64_t cap = (int64_t)c->max_pages * c->page_size;
    // tiles are counted in 32 bits, and so are the workgroups of the second launch
    if ((int64_t)c->B * H * ((cap + TK - 1) / TK) > INT32_MAX / 2)
        return api_fail(MOA_ERR_SHAPE, "decode_attn: B * n_q_heads * ceil(capacity / 128) above 2^30");
    return MOA_OK;
}

}  // namespace
}  // namespace moa

using namespace moa;

extern "C" {

int32_t moa_decode_attn_workspace_bytes(const moa_kv_cache_t *cache, int32_t n_q_heads, size_t *bytes_host)
{
    if (!bytes_host) return api_fail(MOA_ERR_NULL, "decode_attn_workspace_bytes: bytes_host is NULL");
    int32_t rc = check_decode(cache, n_q_heads, "decode_attn_workspace_bytes");
    if (rc) return rc;
    const size_t without = decode_plan(*cache, n_q_heads, false).total(), with = cache->score ? decode_plan(*cache, n_q_heads, true).total() : 0;
    *bytes_host = with > without ? with : without;
    return MOA_OK;
}

int32_t moa_decode_attn(const moa_kv_cache_t *cache, int32_t n_q_heads, const void *q, void *out, int32_t accumulate,
                        int32_t *dev_status, void *ws, size_t ws_bytes, void *stream)
{
    int32_t rc = check_decode(cache, n_q_heads, "decode_attn");
    if (rc) return rc;
    if (!q || !out) return api_fail(MOA_ERR_NULL, "decode_attn: q / out is NULL");
    if (accumulate && !cache->score) return api_fail(MOA_ERR_NULL, "decode_attn: the cache keeps no accounts (score)");
    const size_t es = kv_esize(*cache);
    if (((uintptr_t)q | (uintptr_t)out) & (es - 1)) return api_fail(MOA_ERR_SHAPE, "decode_attn: q / out not aligned to their elements");
    const DecodePlan p = decode_plan(*cache, n_q_heads, accumulate != 0);
    if (p.total() && (!ws || (((uintptr_t)ws) & 255) || ws_bytes < p.total()))
        return api_fail(MOA_ERR_WORKSPACE, "decode_attn: workspace NULL, misaligned or smaller than moa_decode_attn_workspace_bytes");
    DecodeArgs a = {KvDev(*cache, dev_status), q, out, n_q_heads, n_q_heads / cache->n_kv_heads, p.HG, p.rtiles, cache->n_kv_heads * p.rtiles,
                    p.runs, 2, kv_rows16(*cache, {}) ? 1 : 0, 1.4426950408889634f / sqrtf((float)cache->head_dim),
                    (float *)ws, (float *)((char *)ws + p.part_o), p.raw ? (float *)((char *)ws + p.part_o + p.part_ml) : nullptr};
    prof_set_site(S_DECODE);
    hipStream_t st = (hipStream_t)stream;
    const hipError_t e = es == 2 ? launch_decode<bf16_t>(a, st) : launch_decode<float>(a, st);
    if (e != hipSuccess) return api_fail(MOA_ERR_HIP, hipGetErrorString(e));
    return MOA_OK;
}

}  // extern "C"
