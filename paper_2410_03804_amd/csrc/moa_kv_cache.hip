// A cache of pages: rows appended to it (moa_kv_append) and cut down to a budget by accumulated attention weight (moa_kv_evict).
#include "moa_kv_device.h"

#include <stdio.h>

namespace moa {

int32_t check_kv_cache(const moa_kv_cache_t *c, const char *who)
{
    char msg[160];
    auto refuse = [&](int32_t code, const char *what) {
        snprintf(msg, sizeof msg, "%s: %s", who, what);
        return api_fail(code, msg);
    };
    if (!c) return refuse(MOA_ERR_NULL, "cache is NULL");
    if (c->dtype != MOA_F32 && c->dtype != MOA_BF16) return refuse(MOA_ERR_DTYPE, "cache dtype is neither MOA_F32 nor MOA_BF16");
    if (c->n_kv_heads < 1 || c->head_dim < 1 || c->head_dim > 256 || c->B < 1 || c->n_pages < 1 || c->page_size < 1 || c->max_pages < 1)
        return refuse(MOA_ERR_SHAPE, "cache dimensions (all >= 1, head_dim <= 256)");
    // slots and pool rows are counted in 32 bits on the device
    if ((int64_t)c->max_pages * c->page_size > (1 << 30)) return refuse(MOA_ERR_SHAPE, "more than 2^30 slots per sequence");
    if ((int64_t)c->n_kv_heads * c->page_size > INT32_MAX / c->n_pages) return refuse(MOA_ERR_SHAPE, "more than 2^31 - 1 rows in the pool");
    if ((int64_t)c->B * c->n_kv_heads > (1 << 20)) return refuse(MOA_ERR_SHAPE, "more than 2^20 pairs of sequence and KV head");
    if (!c->k || !c->v || !c->table || !c->len) return refuse(MOA_ERR_NULL, "cache k / v / table / len is NULL");
    if (!c->pos != !c->seen) return refuse(MOA_ERR_NULL, "cache pos and seen come together");
    const uintptr_t es = kv_esize(*c);
    if ((((uintptr_t)c->k | (uintptr_t)c->v) & (es - 1)) ||
        (((uintptr_t)c->table | (uintptr_t)c->len | (uintptr_t)c->pos | (uintptr_t)c->seen | (uintptr_t)c->score) & 3))
        return refuse(MOA_ERR_SHAPE, "cache pointers must be aligned to their elements");
    return MOA_OK;
}

namespace {

// ---------------------------------------------------------------- append
struct AppendArgs {
    KvDev c;
    const char *k_new, *v_new;       // [B, Hkv, M, dh]
    const int32_t *path, *n_new;     // [B, M], [B]; may be NULL
    int M;
    FastDiv units;                   // units of T per row
};

// rows that sequence b gets: those asked for, within M and the room there is
__device__ __forceinline__ int append_count(const AppendArgs &a, int b, int held, bool report)
{
    int n = a.n_new ? a.n_new[b] : a.M;
    if ((uint32_t)n > (uint32_t)a.M) {
        if (report) a.c.flag(MOA_DEV_BAD_LENGTH);
        n = n < 0 ? 0 : a.M;
    }
    if (n > a.c.cap - held) {
        if (report) a.c.flag(MOA_DEV_CACHE_FULL);
        n = a.c.cap - held;
    }
    return n;
}

// ONE: a workgroup per sequence, which may then also move its length on.  Else gridDim.x of them per sequence and KV head.
template <typename T, int THREADS, bool ONE>
__global__ __launch_bounds__(THREADS) void k_kv_append(AppendArgs a)
{
    const int b = blockIdx.z, units = (int)a.units.d;
    const bool first = blockIdx.x + blockIdx.y == 0 && threadIdx.x == 0;
    const int held = a.c.length(b, first), n = append_count(a, b, held, first);
    const int seen = a.c.seen ? a.c.seen[b] : 0;
    const int h0 = ONE ? 0 : blockIdx.y, h1 = ONE ? a.c.Hkv : h0 + 1;
    // item: a unit of a row of K and the same of V; the rows of a head one after the other, as they come
    const uint32_t per_head = (uint32_t)n * units, work = per_head * (uint32_t)(h1 - h0);
    for (uint32_t w = blockIdx.x * THREADS + threadIdx.x; w < work; w += gridDim.x * THREADS) {
        const uint32_t hh = ONE ? w / per_head : 0u, in = w - hh * per_head, i = a.units(in), u = in - i * units;
        const int h = h0 + (int)hh;
        int src = (int)i;
        if (a.path) {
            src = a.path[(int64_t)b * a.M + i];
            if ((uint32_t)src >= (uint32_t)a.M) {
                a.c.flag(MOA_DEV_BAD_PARENT);
                src = src < 0 ? 0 : a.M - 1;
            }
        }
        const int row = a.c.row(b, h, held + (int)i);
        const int64_t from = (((int64_t)b * a.c.Hkv + h) * a.M + src) * units + u;
        const T kx = ((const T *)a.k_new)[from], vx = ((const T *)a.v_new)[from];
        if (row >= 0) {
            ((T *)a.c.k)[(int64_t)row * units + u] = kx;
            ((T *)a.c.v)[(int64_t)row * units + u] = vx;
        } else a.c.flag(MOA_DEV_BAD_PAGE);
        if (u == 0) {
            const int64_t slot = ((int64_t)b * a.c.Hkv + h) * a.c.cap + held + i;
            if (a.c.pos) a.c.pos[slot] = seen + (int)i;
            if (a.c.score) a.c.score[slot] = 0.f;
        }
    }
    if (ONE) {
        __syncthreads();                     // every thread has read the length
        if (threadIdx.x == 0) {
            a.c.len[b] = held + n;
            if (a.c.seen) a.c.seen[b] = seen + n;
        }
    }
}

__global__ __launch_bounds__(256) void k_kv_append_len(AppendArgs a)
{
    const int b = blockIdx.x * 256 + threadIdx.x;
    if (b >= a.c.B) return;
    const int held = a.c.length(b, false), n = append_count(a, b, held, false);
    a.c.len[b] = held + n;
    if (a.c.seen) a.c.seen[b] += n;
}

template <typename T>
hipError_t launch_append(const AppendArgs &a, hipStream_t st)
{
    const int64_t per_head = (int64_t)a.M * a.units.d, work = per_head * a.c.Hkv;
    prof_begin(K_KV_APPEND, st);
    // One workgroup per sequence saves the second launch (5 us); up to eight items a thread that is the shorter way.  8b heads, us, one
    // workgroup against two launches: 60 rows of one sequence 9.0, 5.7 + 5.4, of 64 sequences 14.0, 10.4 + 5.3; 200 rows 20.6, 5.9 + 5.0.
    if (work <= 1024) MOA_KLAUNCH((k_kv_append<T, 256, true>), dim3(1, 1, a.c.B), dim3(256), 0, st, a);
    else if (work <= 8192) MOA_KLAUNCH((k_kv_append<T, 1024, true>), dim3(1, 1, a.c.B), dim3(1024), 0, st, a);
    else {
        const int64_t blocks = (per_head + 1023) / 1024;
        MOA_KLAUNCH((k_kv_append<T, 256, false>), dim3((unsigned)(blocks < 1024 ? blocks : 1024), a.c.Hkv, a.c.B), dim3(256), 0, st, a);
    }
    prof_end(st);
    if (work > 8192) {
        prof_begin(K_KV_APPEND_LEN, st);
        MOA_KLAUNCH(k_kv_append_len, dim3((a.c.B + 255) / 256), dim3(256), 0, st, a);
        prof_end(st);
    }
    return hipGetLastError();
}

// ---------------------------------------------------------------- evict
constexpr int EV_T = 1024, EV_BITS = 11, EV_BINS = 1 << EV_BITS, EV_KEYS = 32768;
constexpr int EV_U = 4;                // rounds of 64 slots of a wavefront at a time

struct EvictArgs {
    KvDev c;
    int budget, recent;
    int moves;                // room for moves per (sequence, KV head)
    int keys;                 // that LDS holds: a multiple of EV_U rounds per wavefront
    int32_t *count;           // [B, Hkv]
    int32_t *dst, *src;       // [B, Hkv, moves]
    uint32_t *spill;          // [B, Hkv, cap] the keys that LDS does not hold; NULL where it holds all
    FastDiv units;
};

// The order in which slots stay: the newest tokens' first, then by weight (ordered as its float is; NaN last).
__device__ __forceinline__ uint32_t stay_key(float w, bool newest)
{
    if (newest) return 0xffffffffu;
    if (!(w == w)) return 0u;
    const uint32_t u = __float_as_uint(w + 0.f);               // -0 becomes +0
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// one number of each of the 16 wavefronts: their sum over the ones before this one, and over all
struct Before { uint32_t mine, all; };
__device__ __forceinline__ Before sum_before(const uint32_t *s, int wave)
{
    const int lane = threadIdx.x & 63;
    const uint32_t upto = wave_scan(lane < 16 ? s[lane] : 0u);
    const uint32_t mine = (uint32_t)__builtin_amdgcn_readlane((int)upto, wave ? wave - 1 : 0);
    return {wave ? mine : 0u, (uint32_t)__builtin_amdgcn_readlane((int)upto, 15)};
}

__device__ __forceinline__ uint32_t lanes_below(uint64_t mask)
{
    return __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0u));
}

// One workgroup per (sequence, KV head).  Every wavefront has a stretch of the slots, whose keys it keeps in LDS, or in the
// workspace where there are more than that holds.  The key of the last slot that stays is found digit by digit from histograms
// (11, 11 and 10 bits; the newest, whose key is the largest there is, are only counted); slots with a larger key stay, and of
// those with an equal one the lowest, which only matters in the one wavefront where the equal ones that stay end.  Each
// wavefront then lists what its stretch frees below the budget and what stays beyond it; the i-th of either are one move.
// What bounds it is that one compute unit has all of a pair: its vector units are busy 45 % of the time at up to 16384 slots (32 % at
// 2112), and its wavefronts wait 54 % (64 %) of theirs, for barriers, LDS and the pass over 8 bytes a slot that it loads alone.  64 pairs of up to 16384 slots: 34 us with keys in registers and every pass unrolled (33 KB of code, fetched for one
// pass), 35 with loops but sums by shuffles, 19.5 now; 128 pairs of 2112 9.6 us.  Eight pairs of 131072: 206 us with accounts and positions read again
// in every pass, 149 with the keys in the workspace; of 32768 33.  (Those use eight compute units of 256.)
__global__ __launch_bounds__(EV_T) void k_kv_evict_select(EvictArgs a)
{
    constexpr int NW = EV_T / 64, U = EV_U, UL = 8;      // rounds at a time: keys, accounts
    static_assert(NW == 16 && EV_BINS == 2 * EV_T, "sum_before; two digits a thread");
    constexpr uint32_t NEWEST = 0xffffffffu;
    __shared__ __attribute__((aligned(8))) uint32_t hist[EV_BINS];
    __shared__ uint32_t sums[NW], chosen[2], per_wave[3][NW];
    extern __shared__ uint32_t keys[];         // a.keys of them
    const int bh = blockIdx.x, b = bh / a.c.Hkv, h = bh - b * a.c.Hkv, tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n = a.c.length(b, h == 0 && tid == 0);
    if (n <= a.budget) {
        if (tid == 0) a.count[bh] = 0;
        return;
    }
    for (int i = tid; i < EV_BINS; i += EV_T) hist[i] = 0;
    __syncthreads();
    const float *score = a.c.score + (int64_t)bh * a.c.cap;
    const int32_t *pos = a.c.pos + (int64_t)bh * a.c.cap;
    const int64_t oldest = (int64_t)a.c.seen[b] - a.recent;
    const int seg = ((n + NW - 1) / NW + 63) / 64 * 64, s0 = wave * seg, s1 = min(s0 + seg, n), rounds = s1 > s0 ? (s1 - s0 + 63) / 64 : 0;
    const int room = a.keys / NW, here = min(rounds, room / 64);
    // (said to be in LDS: as one of two places to read a key from it would become an address of either kind)
    __attribute__((address_space(3))) uint32_t *const mine = (__attribute__((address_space(3))) uint32_t *)keys + wave * room;
    uint32_t *const spill = a.spill + (int64_t)bh * a.c.cap;
    auto tally = [&](uint32_t d) {
        // sixty-four equal accounts would wait for each other at one address
        const uint32_t d0 = (uint32_t)__builtin_amdgcn_readfirstlane((int)d);
        const uint64_t all = __ballot(true);
        if (__ballot(d == d0) == all) {
            if (lanes_below(all) == 0) atomicAdd(&hist[d0], (uint32_t)__popcll(all));
        } else atomicAdd(&hist[d], 1u);
    };
    uint32_t newest = 0;
#pragma unroll 1
    for (int j = 0; j < rounds; j += UL) {
        float w[UL];
        int32_t p[UL];
#pragma unroll
        for (int q = 0; q < UL; ++q) {
            const int s = min(s0 + 64 * (j + q) + lane, s1 - 1);
            w[q] = score[s];
            p[q] = pos[s];
        }
#pragma unroll
        for (int q = 0; q < UL; ++q) {
            const bool in = s0 + 64 * (j + q) + lane < s1;
            const uint32_t x = stay_key(w[q], p[q] >= oldest);
            if (j + q < here) mine[64 * (j + q) + lane] = x;
            else if (in) __builtin_nontemporal_store(x, spill + s0 + 64 * (j + q) + lane);
            newest += __popcll(__ballot(in && x == NEWEST));
            if (in && x != NEWEST) tally(x >> 21);
        }
    }
    // f(first slot, this lane's key, whether it has one) for every round of 64 slots
    auto each = [&](auto f) {
#pragma unroll 1
        for (int j = 0; j < rounds; j += U) {
            uint32_t x[U];
            if (j + U <= room / 64) {
#pragma unroll
                for (int q = 0; q < U; ++q) x[q] = mine[64 * (j + q) + lane];
            } else {                                       // (written by this very thread)
#pragma unroll
                for (int q = 0; q < U; ++q) {
                    const int s = s0 + 64 * (j + q) + lane;
                    x[q] = 0;
                    if (j + q < here) x[q] = mine[64 * (j + q) + lane];
                    else if (s < s1) x[q] = __builtin_nontemporal_load(spill + s);
                }
            }
#pragma unroll
            for (int q = 0; q < U; ++q) f(s0 + 64 * (j + q), x[q], s0 + 64 * (j + q) + lane < s1);
        }
    };

    if (lane == 0) per_wave[0][wave] = newest;
    __syncthreads();
    newest = sum_before(per_wave[0], wave).all;
    uint32_t last = NEWEST, ties = (uint32_t)a.budget;                // of the slots whose key is `last` the lowest `ties` stay
    if (newest < ties) {
        uint32_t want = ties - newest, prefix = 0;                    // `want` slots are still to be found among keys that begin with prefix
        int shift = 21;
#pragma unroll 1
        for (;;) {
            // from the largest digit down; thread t has the digits 2 t and 2 t + 1, counted from the top
            const int top = EV_BINS - 1 - 2 * tid;
            u32x2 *const pair = (u32x2 *)(hist + top - 1);
            const uint32_t c0 = (*pair)[1], c1 = (*pair)[0];
            *pair = u32x2{0u, 0u};
            uint32_t upto = wave_scan(c0 + c1);
            if (lane == 63) sums[wave] = upto;
            __syncthreads();
            upto += sum_before(sums, wave).mine;
            const uint32_t before = upto - c0 - c1;
            if (before < want && want <= upto) {
                const bool second = want > before + c0;
                chosen[0] = (uint32_t)(second ? top - 1 : top);
                chosen[1] = want - before - (second ? c0 : 0u);
            }
            __syncthreads();
            prefix |= chosen[0] << shift;
            want = chosen[1];
            if (shift == 0) break;
            const int down = shift, bits = shift == 21 ? EV_BITS : 10;
            shift -= bits;
            each([&](int, uint32_t x, bool in) {
                if (in && x != NEWEST && x >> down == prefix >> down) tally((x >> shift) & ((1u << bits) - 1));
            });
            __syncthreads();
        }
        last = prefix;
        ties = want;
    }

    // of this stretch, below the budget (0) and beyond it (1): keys above the last one, and equal to it
    uint32_t more[2] = {0, 0}, same[2] = {0, 0};
    each([&](int s, uint32_t x, bool in) {
        const bool low = s + lane < a.budget;
        const uint64_t gt = __ballot(in && x > last), eq = __ballot(in && x == last), lows = __ballot(low);
        more[0] += __popcll(gt & lows);
        more[1] += __popcll(gt & ~lows);
        same[0] += __popcll(eq & lows);
        same[1] += __popcll(eq & ~lows);
    });
    if (lane == 0) per_wave[1][wave] = same[0] + same[1];
    __syncthreads();
    // those of the equal ones that stay are the stretch's first
    const uint32_t eq0 = sum_before(per_wave[1], wave).mine, left = eq0 < ties ? ties - eq0 : 0u;
    const uint32_t stay_low = min(same[0], left), stay_high = min(same[1], left - stay_low);
    const uint32_t holes = (uint32_t)max(min(s1, a.budget) - s0, 0) - more[0] - stay_low, movers = more[1] + stay_high;
    if (lane == 0) {
        per_wave[0][wave] = holes;
        per_wave[2][wave] = movers;
    }
    __syncthreads();
    const uint32_t h0 = sum_before(per_wave[0], wave).mine;
    int32_t *dst = a.dst + (int64_t)bh * a.moves + h0, *src = a.src + (int64_t)bh * a.moves + sum_before(per_wave[2], wave).mine;
    uint32_t e = 0;
    each([&](int s, uint32_t x, bool in) {
        const bool low = s + lane < a.budget;
        const uint64_t eq = __ballot(in && x == last);
        const bool stays = in && (x > last || (x == last && e + lanes_below(eq) < left));
        e += __popcll(eq);
        if (s < a.budget) {
            const bool is = in && low && !stays;
            const uint64_t hole = __ballot(is);
            if (is) dst[lanes_below(hole)] = s + lane;
            dst += __popcll(hole);
        }
        if (s + 63 >= a.budget) {
            const bool is = !low && stays;
            const uint64_t mover = __ballot(is);
            if (is) src[lanes_below(mover)] = s + lane;
            src += __popcll(mover);
        }
    });
    if (tid == EV_T - 1) a.count[bh] = (int32_t)(h0 + holes);
}

template <typename T>
__global__ __launch_bounds__(256) void k_kv_evict_move(EvictArgs a)
{
    constexpr int U = 4;                  // items in flight per thread: a unit of a row of K and the same of V
    const int bh = blockIdx.y, b = bh / a.c.Hkv, h = bh - b * a.c.Hkv, units = (int)a.units.d;
    const int64_t at = (int64_t)bh * a.moves, acc = (int64_t)bh * a.c.cap;
    const uint32_t step = gridDim.x * 256, room = (uint32_t)a.moves * units;
    T *const k = (T *)a.c.k, *const v = (T *)a.c.v;
    const int32_t *const count = a.count + bh;
    int d[U], s[U];
    auto read_moves = [&](uint32_t w0) {  // (beyond the last move there is room, with anything in it)
#pragma unroll
        for (int q = 0; q < U; ++q) {
            const uint32_t i = a.units(min(w0 + q * step, room - 1));
            d[q] = a.dst[at + i];
            s[q] = a.src[at + i];
        }
    };
    uint32_t w0 = blockIdx.x * 256 + threadIdx.x;
    read_moves(w0);                       // on their way together with how many there are
    const uint32_t work = (uint32_t)*count * units;
    for (; w0 < work; w0 += U * step, read_moves(w0)) {
        int64_t to[U];
        T kx[U], vx[U];
#pragma unroll
        for (int q = 0; q < U; ++q) {
            const uint32_t w = w0 + q * step, u = w - a.units(w) * units;
            to[q] = -1;
            if (w >= work) continue;
            const int rd = a.c.row(b, h, d[q]), rs = a.c.row(b, h, s[q]);
            if (rd >= 0 && rs >= 0) {
                to[q] = (int64_t)rd * units + u;
                // (nobody reads a row again where it was: 64 pairs of about 1700 moves 27.5 us so, 32 without)
                kx[q] = __builtin_nontemporal_load(k + (int64_t)rs * units + u);
                vx[q] = __builtin_nontemporal_load(v + (int64_t)rs * units + u);
            } else a.c.flag(MOA_DEV_BAD_PAGE);
            if (u == 0) {
                a.c.pos[acc + d[q]] = a.c.pos[acc + s[q]];
                a.c.score[acc + d[q]] = a.c.score[acc + s[q]];
            }
        }
#pragma unroll
        for (int q = 0; q < U; ++q)
            if (to[q] >= 0) {
                k[to[q]] = kx[q];
                v[to[q]] = vx[q];
            }
    }
    // nobody in this launch reads the lengths
    if (h == 0 && blockIdx.x == 0 && threadIdx.x == 0 && a.c.len[b] > a.budget) a.c.len[b] = a.budget;
}

template <typename T>
hipError_t launch_evict(const EvictArgs &a, hipStream_t st)
{
    const int bh = a.c.B * a.c.Hkv;
    static bool raised[16] = {};
    hipError_t e = raise_lds_limit_once(raised, (const void *)k_kv_evict_select, EV_KEYS * 4);
    if (e != hipSuccess) return e;
    prof_begin(K_KV_EVICT_SELECT, st);
    MOA_KLAUNCH(k_kv_evict_select, dim3(bh), dim3(EV_T), (size_t)a.keys * 4, st, a);
    prof_end(st);
    const int64_t work = (int64_t)a.moves * a.units.d, blocks = (work + 255) / 256;
    prof_begin(K_KV_EVICT_MOVE, st);
    MOA_KLAUNCH(k_kv_evict_move<T>, dim3((unsigned)(blocks < 64 ? blocks : 64), bh), dim3(256), 0, st, a);
    prof_end(st);
    return hipGetLastError();
}

int evict_moves(const moa_kv_cache_t &c, int budget)
{
    const int cap = c.max_pages * c.page_size;
    return budget < cap - budget ? budget : cap - budget;
}

}  // namespace
}  // namespace moa

using namespace moa;

extern "C" {

int32_t moa_kv_append(const moa_kv_cache_t *cache, const void *k_new, const void *v_new, int32_t M, const int32_t *path,
                      const int32_t *n_new, int32_t *dev_status, void *stream)
{
    int32_t rc = check_kv_cache(cache, "kv_append");
    if (rc) return rc;
    if (!k_new || !v_new) return api_fail(MOA_ERR_NULL, "kv_append: k_new / v_new is NULL");
    if (M < 1 || M > (1 << 24)) return api_fail(MOA_ERR_SHAPE, "kv_append: M outside [1, 2^24]");
    if ((int64_t)cache->head_dim * M > INT32_MAX) return api_fail(MOA_ERR_SHAPE, "kv_append: M * head_dim above 2^31 - 1");
    if (cache->B > 65535 || cache->n_kv_heads > 65535) return api_fail(MOA_ERR_SHAPE, "kv_append: more than 65535 sequences or KV heads");
    const size_t es = kv_esize(*cache);
    if (((uintptr_t)k_new | (uintptr_t)v_new) & (es - 1)) return api_fail(MOA_ERR_SHAPE, "kv_append: k_new / v_new not aligned to their elements");
    const bool wide = kv_rows16(*cache, {k_new, v_new});
    AppendArgs a = {KvDev(*cache, dev_status), (const char *)k_new, (const char *)v_new, path, n_new, M,
                    FastDiv((uint32_t)(wide ? cache->head_dim * es / 16 : cache->head_dim))};
    prof_set_site(S_KV_CACHE);
    hipStream_t st = (hipStream_t)stream;
    const hipError_t e = wide ? launch_append<u32x4>(a, st) : es == 2 ? launch_append<uint16_t>(a, st) : launch_append<uint32_t>(a, st);
    if (e != hipSuccess) return api_fail(MOA_ERR_HIP, hipGetErrorString(e));
    return MOA_OK;
}

int32_t moa_kv_evict_workspace_bytes(const moa_kv_cache_t *cache, int32_t budget, size_t *bytes_host)
{
    if (!bytes_host) return api_fail(MOA_ERR_NULL, "kv_evict_workspace_bytes: bytes_host is NULL");
    int32_t rc = check_kv_cache(cache, "kv_evict_workspace_bytes");
    if (rc) return rc;
    if (budget < 1) return api_fail(MOA_ERR_RANGE, "kv_evict_workspace_bytes: budget < 1");
    const int64_t bh = (int64_t)cache->B * cache->n_kv_heads;
    const int moves = evict_moves(*cache, budget);
    const size_t cap = (size_t)cache->max_pages * cache->page_size;
    *bytes_host = moves > 0 ? (size_t)bh * 4 * (1 + 2 * (size_t)moves + (cap > EV_KEYS ? cap : 0)) : 0;
    return MOA_OK;
}

int32_t moa_kv_evict(const moa_kv_cache_t *cache, int32_t budget, int32_t recent, int32_t *dev_status, void *ws, size_t ws_bytes,
                     void *stream)
{
    size_t need = 0;
    int32_t rc = check_kv_cache(cache, "kv_evict");
    if (rc) return rc;
    if (!cache->pos || !cache->score) return api_fail(MOA_ERR_NULL, "kv_evict: the cache keeps no positions (pos, seen) or no accounts (score)");
    if (budget < 1 || recent < 0 || recent > budget) return api_fail(MOA_ERR_RANGE, "kv_evict: 1 <= budget and 0 <= recent <= budget");
    if ((int64_t)cache->B * cache->n_kv_heads > 65535) return api_fail(MOA_ERR_SHAPE, "kv_evict: more than 65535 pairs of sequence and KV head");
    if ((int64_t)evict_moves(*cache, budget) * cache->head_dim > (1 << 30))
        return api_fail(MOA_ERR_SHAPE, "kv_evict: min(budget, capacity - budget) * head_dim above 2^30");
    (void)moa_kv_evict_workspace_bytes(cache, budget, &need);
    if (need == 0) return MOA_OK;                              // no sequence can hold more than the budget
    if (!ws || (((uintptr_t)ws) & 255) || ws_bytes < need)
        return api_fail(MOA_ERR_WORKSPACE, "kv_evict: workspace NULL, misaligned or smaller than moa_kv_evict_workspace_bytes");
    const size_t es = kv_esize(*cache);
    const bool wide = kv_rows16(*cache, {});
    const int64_t bh = (int64_t)cache->B * cache->n_kv_heads;
    const int moves = evict_moves(*cache, budget);
    const int cap = cache->max_pages * cache->page_size, whole = EV_U * EV_T;
    const int keys = cap < EV_KEYS ? (cap + whole - 1) / whole * whole : EV_KEYS;
    int32_t *w = (int32_t *)ws;
    EvictArgs a = {KvDev(*cache, dev_status), budget, recent, moves, keys, w, w + bh, w + bh + bh * moves,
                   cap > EV_KEYS ? (uint32_t *)(w + bh + 2 * bh * moves) : nullptr,
                   FastDiv((uint32_t)(wide ? cache->head_dim * es / 16 : cache->head_dim))};
    prof_set_site(S_KV_CACHE);
    hipStream_t st = (hipStream_t)stream;
    const hipError_t e = wide ? launch_evict<u32x4>(a, st) : es == 2 ? launch_evict<uint16_t>(a, st) : launch_evict<uint32_t>(a, st);
    if (e != hipSuccess) return api_fail(MOA_ERR_HIP, hipGetErrorString(e));
    return MOA_OK;
}

}  // extern "C"
