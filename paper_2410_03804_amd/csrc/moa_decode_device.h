// What the kernels of the attention of one token per sequence share, over a cache of either kind: the list of tiles and how it is dealt
// to workgroups, sums and maxima over lanes, loads from pages straight into LDS, and what is done with a run's result.
#ifndef MOA_DECODE_DEVICE_H
#define MOA_DECODE_DEVICE_H
#include "moa_attn_device.h"
#include "moa_decode_plan.h"
#include "moa_kv_device.h"

#include <float.h>

namespace moa {

constexpr int WAVES = 4, WK = TK / WAVES;        // wavefronts, keys of a tile that a wavefront takes

struct DecodeArgs {
    KvDev c;
    const void *q;                // [B, H, dh]
    void *out;                    // [B, H, dh]
    int H, G, HG, rtiles, HB;     // query heads, per KV head; of these in a tile; tiles per KV head; Hkv * rtiles
    int runs, runs_log2;          // workgroups the tiles are dealt to, a power of two; 0: one workgroup per pair
    float scale;                  // log2(e) / sqrt(dh)
    float *part_o;                // [runs + B HB][HG][dh]
    float *part_ml;               // [runs + B HB][HG][2]
    int cap32;                    // the capacity in whole blocks of 32 slots
    float *raw;                   // [B, HB, cap32, HG] scores, where accounts are kept; else NULL
};

// the second launch (moa_decode_attn.hip): joins the partial results, and brings accounts up to date
hipError_t launch_decode_join(const DecodeArgs &a, bool bf16, hipStream_t st);

namespace {

__device__ __forceinline__ uint32_t uniform(uint32_t x) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)x); }
__device__ __forceinline__ uint32_t from_lane(uint32_t x, int lane) { return (uint32_t)__builtin_amdgcn_readlane((int)x, lane); }
template <int KEYS = TK>
__device__ __forceinline__ uint32_t tiles_of(int len)
{
    return (uint32_t)(len + KEYS - 1) / KEYS;
}

// f(x of this lane, x of the lane 16 (32) away), by exchanges inside the vector unit; f commutes
template <typename F>
__device__ __forceinline__ float with_lane16(float x, const F &f)
{
    const auto y = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return f(__uint_as_float(y[0]), __uint_as_float(y[1]));
}
template <typename F>
__device__ __forceinline__ float with_lane32(float x, const F &f)
{
    const auto y = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return f(__uint_as_float(y[0]), __uint_as_float(y[1]));
}
// over the lanes that differ in bits FROM .. 5 of their number only (FROM = 0: over all)
template <int FROM, typename F>
__device__ __forceinline__ float over_lanes(float x, const F &f)
{
    if (FROM <= 0) x = f(x, dpp_move_f32<0xB1>(x));      // quad_perm [1, 0, 3, 2]
    if (FROM <= 1) x = f(x, dpp_move_f32<0x4E>(x));      // quad_perm [2, 3, 0, 1]
    if (FROM <= 2) x = f(x, dpp_move_f32<0x141>(x));     // row_half_mirror: by now quads are uniform
    if (FROM <= 3) x = f(x, FROM == 3 ? dpp_move_f32<0x128>(x) : dpp_move_f32<0x140>(x));   // row_ror 8; row_mirror where halves of rows are uniform
    if (FROM <= 4) x = with_lane16(x, f);
    return FROM <= 5 ? with_lane32(x, f) : x;
}
__device__ __forceinline__ float add(float x, float y) { return x + y; }

// The maximum that keys whose scores are all -infinity leave, where no key at all leaves -infinity: below every other score, so that
// other keys' results stand when the two are joined.
__device__ __forceinline__ float max_of_keys(float m, bool any) { return any && m == -INFINITY ? -FLT_MAX : m; }
// what the sum is divided by: nothing where there was no key, and a softmax of nothing but -infinity is no number
__device__ __forceinline__ float inverse_sum(float m, float l) { return l != 0.f ? 1.f / l : m == -INFINITY ? 0.f : __builtin_nanf(""); }

// Where the tiles of the sequences lie in the list of all tiles: every wavefront works this out for itself.
struct TileList {
    uint32_t total, per;          // tiles in all, of a run
    __device__ __forceinline__ void set(const DecodeArgs &a, uint32_t all)       // all: tiles of the sequences, for one KV head
    {
        total = all * (uint32_t)a.HB;
        per = max((total + a.runs - 1) >> a.runs_log2, 1u);
    }
    // the sequence of the first tile of run w (if it has one), its length and its first tile
    __device__ __forceinline__ bool find(const DecodeArgs &a, uint32_t w, int &b, int &len, uint32_t &begin)
    {
        const int lane = threadIdx.x & 63;
        int mine = lane < a.c.B ? a.c.length(lane, false) : 0;
        uint32_t upto = wave_scan(tiles_of(mine)), all = from_lane(upto, 63);
        for (int i = lane + 64; i < (a.c.B + 63) / 64 * 64; i += 64) all += from_lane(wave_scan(i < a.c.B ? tiles_of(a.c.length(i, false)) : 0u), 63);
        set(a, all);
        const uint32_t f = w * per;
        if (f >= total) return false;
        uint32_t base = 0;
        for (int b0 = 0;; b0 += 64) {
            const uint64_t past = __ballot(f < (base + upto) * (uint32_t)a.HB);
            if (past) {
                const int at = __ffsll((unsigned long long)past) - 1;
                b = b0 + at;
                len = (int)from_lane((uint32_t)mine, at);
                begin = (base + from_lane(upto, at) - tiles_of(len)) * (uint32_t)a.HB;
                return true;
            }
            base += from_lane(upto, 63);
            mine = b0 + 64 + lane < a.c.B ? a.c.length(b0 + 64 + lane, false) : 0;
            upto = wave_scan(tiles_of(mine));
        }
    }
};

// ---------------------------------------------------------------- what either kernel does with a run's result
// (DH: the head_dim, 0 where it is not known here.)  LDS: acc [HG][dh] of each wavefront, `stride` floats apart, and ml [WAVES][HG][2].
template <typename T, int DH>
__device__ __forceinline__ void finish(const DecodeArgs &a, int b, int len, int hb, bool whole, int64_t slot, const float *acc,
                                       int stride, const float *ml, float *fin)
{
    const int tid = threadIdx.x, dh = DH ? DH : a.c.dh, h = hb / a.rtiles, rt = hb - h * a.rtiles;
    const int r0 = rt * a.HG, rows = min(a.HG, a.G - r0);
    __syncthreads();
    for (int i = tid; i < rows * dh; i += 64 * WAVES) {
        const int r = i / dh, d = i - r * dh;
        float mw[WAVES], m = -INFINITY, l = 0.f, o = 0.f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) m = fmaxf(m, mw[w] = ml[(w * a.HG + r) * 2]);
        const float ms = m == -INFINITY ? 0.f : m;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const float c = fast_exp2(mw[w] - ms);
            l = fmaf(ml[(w * a.HG + r) * 2 + 1], c, l);
            o = fmaf(acc[w * stride + i], c, o);
        }
        const float inv = inverse_sum(m, l);
        if (whole) st((T *)a.out + ((int64_t)b * a.H + h * a.G + r0 + r) * dh + d, o * inv);
        else a.part_o[(slot * a.HG + r) * dh + d] = o;
        if (d != 0) continue;
        // (a pair with several row tiles has its accounts changed by the second launch in any case)
        if (!whole || (a.raw && a.rtiles > 1)) {
            a.part_ml[(slot * a.HG + r) * 2] = m;
            a.part_ml[(slot * a.HG + r) * 2 + 1] = l;
        }
        if (whole && m == -INFINITY && l == 0.f) a.c.flag(MOA_DEV_EMPTY_KEYS);
        fin[r * 2] = ms;
        fin[r * 2 + 1] = inv;
    }
    __syncthreads();
    // A pair's accounts are one workgroup's to change only where it has all its keys and all its query heads.
    if (a.raw && whole && a.rtiles == 1) {
        for (int s = tid; s < len; s += 64 * WAVES) {
            float p = 0.f;
            const float *raw = a.raw + (((int64_t)b * a.HB + hb) * a.cap32 + s) * a.HG;
            for (int r = 0; r < rows; ++r) p += fast_exp2(raw[r] - fin[r * 2]) * fin[r * 2 + 1];
            a.c.score[((int64_t)b * a.c.Hkv + h) * a.c.cap + s] += p;
        }
    }
    __syncthreads();
}

// The run of a workgroup: each of the pairs that its tiles belong to, with process(b, length, hb, first tile, tiles, whether these are
// all of them, partial slot).
template <typename F>
__device__ __forceinline__ void for_each_pair(const DecodeArgs &a, const F &process)
{
    int b, len;
    uint32_t f = 0, end = 0, begin = 0, hb, t = 0, cnt;
    const bool one = a.runs == 0;
    if (one) {
        b = (int)blockIdx.x / a.HB;
        hb = blockIdx.x - (uint32_t)b * a.HB;
        len = (int)uniform((uint32_t)a.c.length(b, hb == 0 && threadIdx.x == 0));
        cnt = tiles_of(len);
    } else {
        TileList list;
        if (!list.find(a, blockIdx.x, b, len, begin)) return;
        f = blockIdx.x * list.per;
        end = min(f + list.per, list.total);
    }
    for (;;) {
        const uint32_t nt = tiles_of(len);
        if (!one) {
            const uint32_t in = f - begin;
            hb = in / nt;
            t = in - hb * nt;
            cnt = min(nt - t, end - f);
            if (hb == 0 && t == 0 && threadIdx.x == 0) (void)a.c.length(b, true);
        }
        process(b, len, (int)hb, t, cnt, cnt == nt, (int64_t)blockIdx.x + (int64_t)b * a.HB + hb);
        f += cnt;
        if (one || f >= end) return;
        if (f == begin + nt * (uint32_t)a.HB) {
            begin = f;
            do len = (int)uniform((uint32_t)a.c.length(++b, false));
            while (len == 0);                               // (f < total: there is one)
        }
    }
}

// ---------------------------------------------------------------- loads from pages straight into LDS
// 64 lanes x 16 (4) bytes, each from an address of its own, to 1 KB (256 bytes) of LDS at `lds`.  (As lds_dma16 in
// moa_gemm_device.h, but a pool of pages takes 64-bit addresses; the s_nop stands between the write of m0 and its use.)
// ONCE: said to be read once only.  Keys and values whose rows are whole lines: 8 x 32768 keys 180 us without, 159 with (6.7
// TB/s), 64 ragged sequences 193 and 171.  Rows of 160 bytes share lines: 11.7 us without, 13.9 with.  It is not true of every line
// that it is said of.  Where several tiles of query heads read a KV head's keys it costs: 128 heads on one KV head, 16 x 32000
// keys, 155 us without, 173 with; 31 heads of 256 dims, 8 x 8000, 31 and 34.5.  Where sequences share pages it does not: 64 x
// 4500 keys, the first 1024 of them common, 167 without, 149 with; 4096 of them 72 and 73.
template <bool ONCE>
__device__ __forceinline__ void lds_gather16(uint32_t lds, uint64_t at)
{
    if (ONCE) asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off nt" ::"s"(lds), "v"(at));
    else asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds), "v"(at));
}
__device__ __forceinline__ void lds_gather4(uint32_t lds, uint64_t at)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(lds), "v"(at));
}
template <int N>
__device__ __forceinline__ void wait_loads()
{
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

// what rows that do not count are read from
__device__ const u32x4 zero_row[32] = {};

}  // namespace
}  // namespace moa
#endif
