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
    int M, units;                    // units of T per row
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

// One workgroup (LAST) or gridDim.x of them per sequence.  Only where it is one may it move the sequence's length on itself.
template <typename T, bool LAST>
__global__ __launch_bounds__(256) void k_kv_append(AppendArgs a)
{
    const int b = blockIdx.y;
    const bool first = blockIdx.x == 0 && threadIdx.x == 0;
    const int held = a.c.length(b, first), n = append_count(a, b, held, first);
    const int seen = a.c.seen ? a.c.seen[b] : 0;
    const int64_t work = (int64_t)n * a.c.Hkv * a.units;
    for (int64_t w = (int64_t)blockIdx.x * 256 + threadIdx.x; w < work; w += (int64_t)gridDim.x * 256) {
        const int u = (int)(w % a.units);
        const int hi = (int)(w / a.units), h = hi % a.c.Hkv, i = hi / a.c.Hkv;
        int src = i;
        if (a.path) {
            src = a.path[(int64_t)b * a.M + i];
            if ((uint32_t)src >= (uint32_t)a.M) {
                a.c.flag(MOA_DEV_BAD_PARENT);
                src = src < 0 ? 0 : a.M - 1;
            }
        }
        const int row = a.c.row(b, h, held + i);
        const int64_t from = (((int64_t)b * a.c.Hkv + h) * a.M + src) * a.units + u;
        if (row >= 0) {
            ((T *)a.c.k)[(int64_t)row * a.units + u] = ((const T *)a.k_new)[from];
            ((T *)a.c.v)[(int64_t)row * a.units + u] = ((const T *)a.v_new)[from];
        } else a.c.flag(MOA_DEV_BAD_PAGE);
        if (u == 0) {
            const int64_t slot = ((int64_t)b * a.c.Hkv + h) * a.c.cap + held + i;
            if (a.c.pos) a.c.pos[slot] = seen + i;
            if (a.c.score) a.c.score[slot] = 0.f;
        }
    }
    if (LAST) {
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
    const int64_t work = (int64_t)a.M * a.c.Hkv * a.units;
    const bool one = work <= 8192;
    const int64_t blocks = one ? 1 : (work + 1023) / 1024 < 1024 ? (work + 1023) / 1024 : 1024;
    prof_begin(K_KV_APPEND, st);
    if (one) MOA_KLAUNCH((k_kv_append<T, true>), dim3(1, a.c.B), dim3(256), 0, st, a);
    else MOA_KLAUNCH((k_kv_append<T, false>), dim3((unsigned)blocks, a.c.B), dim3(256), 0, st, a);
    prof_end(st);
    if (!one) {
        prof_begin(K_KV_APPEND_LEN, st);
        MOA_KLAUNCH(k_kv_append_len, dim3((a.c.B + 255) / 256), dim3(256), 0, st, a);
        prof_end(st);
    }
    return hipGetLastError();
}

// ---------------------------------------------------------------- evict
constexpr int EV_T = 1024, EV_W = EV_T / 64, EV_BITS = 11, EV_BINS = 1 << EV_BITS;

struct EvictArgs {
    KvDev c;
    int budget, recent;
    int moves;                // room for moves per (sequence, KV head)
    int32_t *count;           // [B, Hkv]
    int32_t *dst, *src;       // [B, Hkv, moves]
    int units;
};

// The order in which slots stay: the newest tokens' first, then by weight (ordered as its float is; NaN last).
__device__ __forceinline__ uint32_t stay_key(float w, bool newest)
{
    if (newest) return 0xffffffffu;
    if (!(w == w)) return 0u;
    const uint32_t u = __float_as_uint(w + 0.f);               // -0 becomes +0
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// inclusive sums over the workgroup's threads; s: EV_W words of LDS
__device__ __forceinline__ uint32_t block_scan(uint32_t x, uint32_t *s)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const uint32_t y = __shfl_up(x, d);
        if (lane >= d) x += y;
    }
    __syncthreads();
    if (lane == 63) s[wave] = x;
    __syncthreads();
    for (int w = 0; w < wave; ++w) x += s[w];
    return x;
}

// One workgroup per (sequence, KV head).  The key of the last slot that stays is found digit by digit from histograms (11, 11
// and 10 bits); slots with a larger key stay, and of those with an equal one the lowest.  Each wavefront then lists what its
// stretch of slots frees below the budget and what stays beyond it; the i-th of either are one move.
__global__ __launch_bounds__(EV_T) void k_kv_evict_select(EvictArgs a)
{
    __shared__ uint32_t hist[EV_BINS];
    __shared__ uint32_t sums[EV_W], chosen[2], per_wave[3][EV_W];
    const int bh = blockIdx.x, b = bh / a.c.Hkv, h = bh - b * a.c.Hkv, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int n = a.c.length(b, h == 0 && tid == 0);
    if (n <= a.budget) {
        if (tid == 0) a.count[bh] = 0;
        return;
    }
    const float *score = a.c.score + (int64_t)bh * a.c.cap;
    const int32_t *pos = a.c.pos + (int64_t)bh * a.c.cap;
    const int64_t oldest = (int64_t)a.c.seen[b] - a.recent;
    auto key = [&](int s) { return stay_key(score[s], pos[s] >= oldest); };

    uint32_t want = (uint32_t)a.budget, prefix = 0, known = 0;        // `want` slots are still to be found among keys that begin with prefix
#pragma unroll
    for (int pass = 0; pass < 3; ++pass) {
        const int bits = pass == 2 ? 10 : EV_BITS, shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
        for (int i = tid; i < EV_BINS; i += EV_T) hist[i] = 0;
        __syncthreads();
        for (int s = tid; s < n; s += EV_T) {
            const uint32_t x = key(s);
            if ((x & known) == prefix) atomicAdd(&hist[(x >> shift) & ((1u << bits) - 1)], 1u);
        }
        __syncthreads();
        // from the largest digit down; thread t has the two digits 2 t, 2 t + 1 from the top
        const int hi = EV_BINS - 1 - 2 * tid;
        const uint32_t c0 = hist[hi], c1 = hist[hi - 1];
        const uint32_t upto = block_scan(c0 + c1, sums), before = upto - c0 - c1;
        if (before < want && want <= upto) {
            const bool second = want > before + c0;
            chosen[0] = (uint32_t)(second ? hi - 1 : hi);
            chosen[1] = want - before - (second ? c0 : 0u);
        }
        __syncthreads();
        prefix |= chosen[0] << shift;
        known |= ((1u << bits) - 1) << shift;
        want = chosen[1];
        __syncthreads();
    }
    const uint32_t last = prefix, ties = want;          // of the slots whose key is `last` the lowest `ties` stay

    const int seg = ((n + EV_W - 1) / EV_W + 63) / 64 * 64, s0 = wave * seg, s1 = min(s0 + seg, n);
    const uint64_t below = lane ? ~0ull >> (64 - lane) : 0ull;
    uint32_t eq = 0;
    for (int s = s0; s < s1; s += 64) eq += __popcll(__ballot(s + lane < s1 && key(s + lane) == last));
    if (lane == 0) per_wave[0][wave] = eq;
    __syncthreads();
    uint32_t eq0 = 0;
    for (int w = 0; w < wave; ++w) eq0 += per_wave[0][w];
    uint32_t holes = 0, movers = 0;
    // out: NULL while counting
    auto walk = [&](int32_t *dst, int32_t *src) {
        uint32_t e = eq0;
        holes = movers = 0;
        for (int s = s0; s < s1; s += 64) {
            const int slot = s + lane;
            const bool in = slot < s1;
            const uint32_t x = in ? key(slot) : 0u;
            const uint64_t same = __ballot(in && x == last);
            const bool stays = in && (x > last || (x == last && e + __popcll(same & below) < ties));
            e += __popcll(same);
            const bool hole = in && !stays && slot < a.budget, mover = stays && slot >= a.budget;
            const uint64_t bh_ = __ballot(hole), bm = __ballot(mover);
            if (dst) {
                if (hole) dst[holes + __popcll(bh_ & below)] = slot;
                if (mover) src[movers + __popcll(bm & below)] = slot;
            }
            holes += __popcll(bh_);
            movers += __popcll(bm);
        }
    };
    walk(nullptr, nullptr);
    if (lane == 0) {
        per_wave[1][wave] = holes;
        per_wave[2][wave] = movers;
    }
    __syncthreads();
    uint32_t h0 = 0, m0 = 0;
    for (int w = 0; w < wave; ++w) {
        h0 += per_wave[1][w];
        m0 += per_wave[2][w];
    }
    const int64_t at = (int64_t)bh * a.moves;
    walk(a.dst + at + h0, a.src + at + m0);
    if (tid == EV_T - 1) a.count[bh] = (int32_t)(h0 + holes);
}

template <typename T>
__global__ __launch_bounds__(256) void k_kv_evict_move(EvictArgs a)
{
    const int bh = blockIdx.y, b = bh / a.c.Hkv, h = bh - b * a.c.Hkv;
    const int n = a.count[bh];
    const int64_t at = (int64_t)bh * a.moves, acc = (int64_t)bh * a.c.cap;
    const int64_t work = (int64_t)n * a.units;
    for (int64_t w = (int64_t)blockIdx.x * 256 + threadIdx.x; w < work; w += (int64_t)gridDim.x * 256) {
        const int i = (int)(w / a.units), u = (int)(w - (int64_t)i * a.units);
        const int d = a.dst[at + i], s = a.src[at + i], rd = a.c.row(b, h, d), rs = a.c.row(b, h, s);
        if (rd >= 0 && rs >= 0) {
            ((T *)a.c.k)[(int64_t)rd * a.units + u] = ((T *)a.c.k)[(int64_t)rs * a.units + u];
            ((T *)a.c.v)[(int64_t)rd * a.units + u] = ((T *)a.c.v)[(int64_t)rs * a.units + u];
        } else a.c.flag(MOA_DEV_BAD_PAGE);
        if (u == 0) {
            a.c.pos[acc + d] = a.c.pos[acc + s];
            a.c.score[acc + d] = a.c.score[acc + s];
        }
    }
    // nobody in this launch reads the lengths
    if (h == 0 && blockIdx.x == 0 && threadIdx.x == 0 && a.c.len[b] > a.budget) a.c.len[b] = a.budget;
}

template <typename T>
hipError_t launch_evict(const EvictArgs &a, hipStream_t st)
{
    const int bh = a.c.B * a.c.Hkv;
    prof_begin(K_KV_EVICT_SELECT, st);
    MOA_KLAUNCH(k_kv_evict_select, dim3(bh), dim3(EV_T), 0, st, a);
    prof_end(st);
    const int64_t work = (int64_t)a.moves * a.units, blocks = (work + 1023) / 1024;
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
    if ((int64_t)cache->n_kv_heads * M > INT32_MAX) return api_fail(MOA_ERR_SHAPE, "kv_append: more than 2^31 - 1 rows per sequence");
    if (cache->B > 65535) return api_fail(MOA_ERR_SHAPE, "kv_append: more than 65535 sequences");
    const size_t es = kv_esize(*cache);
    if (((uintptr_t)k_new | (uintptr_t)v_new) & (es - 1)) return api_fail(MOA_ERR_SHAPE, "kv_append: k_new / v_new not aligned to their elements");
    const bool wide = kv_rows16(*cache, {k_new, v_new});
    AppendArgs a = {KvDev(*cache, dev_status), (const char *)k_new, (const char *)v_new, path, n_new, M,
                    (int)(wide ? cache->head_dim * es / 16 : cache->head_dim)};
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
    *bytes_host = moves > 0 ? (size_t)bh * 4 * (1 + 2 * (size_t)moves) : 0;
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
    (void)moa_kv_evict_workspace_bytes(cache, budget, &need);
    if (need == 0) return MOA_OK;                              // no sequence can hold more than the budget
    if (!ws || (((uintptr_t)ws) & 255) || ws_bytes < need)
        return api_fail(MOA_ERR_WORKSPACE, "kv_evict: workspace NULL, misaligned or smaller than moa_kv_evict_workspace_bytes");
    const size_t es = kv_esize(*cache);
    const bool wide = kv_rows16(*cache, {});
    const int64_t bh = (int64_t)cache->B * cache->n_kv_heads;
    const int moves = evict_moves(*cache, budget);
    int32_t *w = (int32_t *)ws;
    EvictArgs a = {KvDev(*cache, dev_status), budget, recent, moves, w, w + bh, w + bh + bh * moves,
                   (int)(wide ? cache->head_dim * es / 16 : cache->head_dim)};
    prof_set_site(S_KV_CACHE);
    hipStream_t st = (hipStream_t)stream;
    const hipError_t e = wide ? launch_evict<u32x4>(a, st) : es == 2 ? launch_evict<uint16_t>(a, st) : launch_evict<uint32_t>(a, st);
    if (e != hipSuccess) return api_fail(MOA_ERR_HIP, hipGetErrorString(e));
    return MOA_OK;
}

}  // extern "C"
