// Pages of a pool handed out to the sequences of a batch and taken back, on the device (moa_kv_reserve, moa_kv_release).
//
// All of it is sums over the sequences in their order: of new tokens (where each one's rows lie in the batch), of pages that they lack
// (which of the free ones each gets, and who goes without).  One workgroup does these, 1024 sequences at a time; what it costs is its
// chain of loads and barriers.  Positions and slots, one of each a token, are written by it too where they are few, and by a launch of
// their own beyond.
#include "moa_kv_device.h"

namespace moa {

namespace {

constexpr int PT = 1024, PW = PT / 64;             // threads, wavefronts

// Sums over the workgroup's threads in their order.  Two sets of LDS in turn, so that one barrier a sum is enough.
struct BlockScan {
    uint32_t (*s)[PW];                             // [2][PW]
    int turn = 0;
    struct Sum { uint32_t before, all; };
    __device__ __forceinline__ Sum operator()(uint32_t x)
    {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        const uint32_t upto = wave_scan(x);
        uint32_t *t = s[turn];
        turn ^= 1;
        if (lane == 63) t[wave] = upto;
        __syncthreads();
        const uint32_t of = wave_scan(lane < PW ? t[lane] : 0u);
        const uint32_t waves = wave ? (uint32_t)__builtin_amdgcn_readlane((int)of, wave - 1) : 0u;
        return {waves + upto - x, (uint32_t)__builtin_amdgcn_readlane((int)of, PW - 1)};
    }
};

struct ReserveArgs {
    const int32_t *len, *n_new, *seen;             // [B]; seen may be NULL
    int32_t *table, *free_pages, *n_free;          // [B, max_pages], [n_pages], [1]
    int32_t *tok_off, *n_got, *pos, *slot;         // [B + 1], [B], [T], [T]; pos, slot may be NULL
    int32_t *dev_status;
    int B, n_pages, max_pages, cap, T;
    FastDiv page;
    __device__ __forceinline__ void flag(int bit) const
    {
        if (dev_status) atomicOr(dev_status, bit);
    }
    __device__ __forceinline__ int length(int b, bool report) const
    {
        const int n = len[b];
        if ((uint32_t)n <= (uint32_t)cap) return n;
        if (report) flag(MOA_DEV_BAD_LENGTH);
        return n < 0 ? 0 : cap;
    }
    // where the new tokens of sequence b, rows off .. off + n - 1 of the batch, have their position and slot
    __device__ __forceinline__ void token(int t, int b, int off, bool got) const
    {
        const int i = t - off, at = length(b, false) + i, pg = (int)page((uint32_t)at);
        if (pos) pos[t] = seen ? (int)((uint32_t)seen[b] + (uint32_t)i) : at;
        if (!slot) return;
        const int id = got ? table[(int64_t)b * max_pages + pg] : -1;
        slot[t] = (uint32_t)id < (uint32_t)n_pages ? id * (int)page.d + (at - pg * (int)page.d) : -1;
    }
    __device__ __forceinline__ void no_token(int t) const
    {
        if (pos) pos[t] = 0;
        if (slot) slot[t] = -1;
    }
};

// the last of s[0 .. n - 1] (s[0] = 0, ascending) that is <= x
template <typename P>
__device__ __forceinline__ int last_upto(const P *s, int n, P x)
{
    int lo = 0;
    for (int step = 1 << (31 - __clz(n)); step; step >>= 1)
        if (lo + step < n && s[lo + step] <= x) lo += step;
    return lo;
}

// TOKENS: positions and slots are written here (B <= PT then).
// A token each of 16 sequences 2.9 us by trace; 64 prompts of 200 to 2048 tokens, 4500 table entries, 15 us with one entry a thread at a time, 13.5
// with four, 11 with eight.
template <bool TOKENS>
__global__ __launch_bounds__(PT) void k_kv_reserve(ReserveArgs a)
{
    constexpr int PU = TOKENS ? 2 : 8;             // table entries that a thread looks at
    __shared__ uint32_t sums[2][PW], items_s[PT], need_s[PT];
    __shared__ int32_t first_s[PT], off_s[PT];
    __shared__ unsigned char got_s[PT];
    const int tid = threadIdx.x;
    BlockScan scan{sums};
    int left = *a.n_free;
    if ((uint32_t)left > (uint32_t)a.n_pages) {
        if (tid == 0) a.flag(MOA_DEV_BAD_LENGTH);
        left = left < 0 ? 0 : a.n_pages;
    }
    uint32_t tokens = 0, needed = 0, taken = 0;    // of the sequences of the rounds before
    bool refused = false;
    for (int b0 = 0; b0 < a.B; b0 += PT) {
        const int b = b0 + tid;
        int n = 0, len = 0;
        if (b < a.B) {
            const int asked = a.n_new[b];
            len = a.length(b, true);
            n = max(asked, 0);
            if (n > a.cap - len) {
                a.flag(MOA_DEV_CACHE_FULL);
                n = a.cap - len;
            }
            if (asked < 0) a.flag(MOA_DEV_BAD_LENGTH);
        }
        // (sums of what is left of the batch at most, 2^21: 1024 of them fit)
        const int want = n;
        n = min(n, a.T);
        const BlockScan::Sum at = scan((uint32_t)n);
        const int off = (int)min(tokens + at.before, (uint32_t)a.T);
        n = min(n, a.T - off);
        if (n < want) a.flag(MOA_DEV_BAD_LENGTH);
        tokens = min(tokens + at.all, (uint32_t)a.T);
        if (b < a.B) a.tok_off[b] = off;
        off_s[tid] = off;
        // the table's entries that the new tokens lie in: items, those of a sequence one behind the other
        const int p0 = (int)a.page((uint32_t)len), pages = n > 0 ? (int)a.page((uint32_t)(len + n - 1)) - p0 + 1 : 0;
        const BlockScan::Sum item = scan((uint32_t)pages);
        items_s[tid] = item.before;
        first_s[tid] = p0;
        need_s[tid] = 0;
        __syncthreads();
        // PU of them a thread, one behind the other: their sequences and table entries; which of them name no page
        uint32_t lacks = 0;
        auto look_at = [&](uint32_t i0, int (&s)[PU], int32_t *(&e)[PU]) {
            const uint32_t i1 = i0 + PU * tid;
            lacks = 0;
            if (i1 >= item.all) return;
            s[0] = last_upto<uint32_t>(items_s, PT, i1);
#pragma unroll
            for (int u = 0; u < PU; ++u) {
                const uint32_t i = i1 + u;
                if (u > 0) s[u] = s[u - 1];
                if (i >= item.all) continue;
                while (s[u] + 1 < PT && items_s[s[u] + 1] <= i) ++s[u];
                e[u] = a.table + (int64_t)(b0 + s[u]) * a.max_pages + first_s[s[u]] + (int)(i - items_s[s[u]]);
            }
            int32_t id[PU];
#pragma unroll
            for (int u = 0; u < PU; ++u) id[u] = i1 + u < item.all ? *e[u] : 0;
#pragma unroll
            for (int u = 0; u < PU; ++u) {
                if (id[u] < 0) lacks |= 1u << u;
                else if (id[u] >= a.n_pages) a.flag(MOA_DEV_BAD_PAGE);
            }
        };
        int s[PU];
        int32_t *e[PU];
        for (uint32_t i0 = 0; i0 < item.all; i0 += PT * PU) {
            look_at(i0, s, e);
            // (one addition a thread and sequence: the entries of a long prompt would else all add to the same place)
            uint32_t sum = 0;
#pragma unroll
            for (int u = 0; u < PU; ++u) {
                sum += lacks >> u & 1;
                if (sum && (u + 1 == PU || i0 + PU * tid + u + 1 >= item.all || s[u + 1 < PU ? u + 1 : u] != s[u])) {
                    atomicAdd(&need_s[s[u]], sum);
                    sum = 0;
                }
            }
        }
        __syncthreads();
        // in their order, as long as the free pages last; who lacks none goes on in any case
        const uint32_t need = need_s[tid];
        const BlockScan::Sum lack = scan(need);
        const bool got = need == 0 || needed + lack.before + need <= (uint32_t)left;
        got_s[tid] = got;
        if (b < a.B) a.n_got[b] = got ? n : 0;
        const BlockScan::Sum give = scan(got ? need : 0u);
        refused |= give.all != lack.all;
        // (the barriers of the sums stand between got_s and its use)
        uint32_t rank = needed;
        for (uint32_t i0 = 0; i0 < item.all; i0 += PT * PU) {
            if (item.all > PT * PU) look_at(i0, s, e);         // (else as it was left)
            const BlockScan::Sum r = scan(__popc(lacks));
            uint32_t at = rank + r.before;
#pragma unroll
            for (int u = 0; u < PU; ++u)
                if (lacks >> u & 1) {
                    if (got_s[s[u]]) {
                        const int32_t id = a.free_pages[left - 1 - (int)at];
                        if ((uint32_t)id >= (uint32_t)a.n_pages) a.flag(MOA_DEV_BAD_PAGE);
                        *e[u] = id;
                    }
                    ++at;
                }
            rank += r.all;
        }
        needed += lack.all;
        taken += give.all;
        if (!TOKENS) __syncthreads();              // the next round writes what this one reads
    }
    if (tid == 0) {
        a.tok_off[a.B] = (int)tokens;
        *a.n_free = left - (int)taken;
        if (refused) a.flag(MOA_DEV_CACHE_FULL);
    }
    if (TOKENS) {
        __syncthreads();                           // the table is written
        for (int t = tid; t < a.T; t += PT) {
            if (t >= (int)tokens) {
                a.no_token(t);
                continue;
            }
            const int s = last_upto<int32_t>(off_s, a.B, t);
            a.token(t, s, off_s[s], got_s[s]);
        }
    }
}

__global__ __launch_bounds__(256) void k_kv_slots(ReserveArgs a)
{
    const int t = blockIdx.x * 256 + threadIdx.x;
    if (t >= a.T) return;
    if (t >= a.tok_off[a.B]) {
        a.no_token(t);
        return;
    }
    const int b = last_upto<int32_t>(a.tok_off, a.B, t);
    a.token(t, b, a.tok_off[b], a.n_got[b] > 0);
}

struct ReleaseArgs {
    const int32_t *len;
    int32_t *table, *free_pages, *n_free, *dev_status;
    int B, n_pages, max_pages, cap;
    FastDiv row, page;                             // by max_pages, by the rows of a page
};

// The table as one list of entries, walked from its end: what goes back first lies deepest in the list of free pages.
__global__ __launch_bounds__(PT) void k_kv_release(ReleaseArgs a)
{
    constexpr int U = 4;
    __shared__ uint32_t sums[2][PW];
    const int tid = threadIdx.x;
    BlockScan scan{sums};
    auto flag = [&](int bit) {
        if (a.dev_status) atomicOr(a.dev_status, bit);
    };
    int have = *a.n_free;
    if ((uint32_t)have > (uint32_t)a.n_pages) {
        if (tid == 0) flag(MOA_DEV_BAD_LENGTH);
        have = have < 0 ? 0 : a.n_pages;
    }
    const int64_t all = (int64_t)a.B * a.max_pages;
    uint32_t count = (uint32_t)have;
    for (int64_t done = 0; done < all; done += PT * U) {
        int32_t id[U];
        uint32_t mine = 0;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t back = done + tid * U + u;
            id[u] = -1;
            if (back >= all) continue;
            const uint32_t i = (uint32_t)(all - 1 - back), b = a.row(i), p = i - b * a.row.d;
            int n = a.len[b];
            if ((uint32_t)n > (uint32_t)a.cap) {
                if (p == 0) flag(MOA_DEV_BAD_LENGTH);
                n = n < 0 ? 0 : a.cap;
            }
            if (p * a.page.d < (uint32_t)n) continue;          // slots in use
            id[u] = a.table[i];
            if (id[u] < 0) continue;
            a.table[i] = -1;
            if (id[u] >= a.n_pages) {
                flag(MOA_DEV_BAD_PAGE);
                id[u] = -1;
            } else ++mine;
        }
        const BlockScan::Sum s = scan(mine);
        uint32_t at = count + s.before;
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (id[u] >= 0) {
                if (at < (uint32_t)a.n_pages) a.free_pages[at] = id[u];
                else flag(MOA_DEV_BAD_PAGE);                   // more pages than there are: one was in two places
                ++at;
            }
        count += s.all;
    }
    if (tid == 0) *a.n_free = (int)min(count, (uint32_t)a.n_pages);
}

int32_t check_pages(int32_t B, int32_t n_pages, int32_t page_size, int32_t max_pages, std::initializer_list<const void *> needed,
                    std::initializer_list<const void *> all)
{
    if (B < 1 || n_pages < 1 || page_size < 1 || max_pages < 1) return api_fail(MOA_ERR_SHAPE, "pages: dimensions (all >= 1)");
    if (B > (1 << 20)) return api_fail(MOA_ERR_SHAPE, "pages: more than 2^20 sequences");
    if ((int64_t)max_pages * page_size > (1 << 30)) return api_fail(MOA_ERR_SHAPE, "pages: more than 2^30 slots per sequence");
    if ((int64_t)n_pages * page_size > INT32_MAX) return api_fail(MOA_ERR_SHAPE, "pages: more than 2^31 - 1 rows in the pool");
    if ((int64_t)B * max_pages > INT32_MAX) return api_fail(MOA_ERR_SHAPE, "pages: more than 2^31 - 1 table entries");
    uintptr_t bits = 0;
    for (const void *p : needed)
        if (!p) return api_fail(MOA_ERR_NULL, "pages: a required pointer is NULL");
    for (const void *p : all) bits |= (uintptr_t)p;
    if (bits & 3) return api_fail(MOA_ERR_SHAPE, "pages: pointers must be aligned to their elements");
    return MOA_OK;
}

}  // namespace
}  // namespace moa

using namespace moa;

extern "C" {

int32_t moa_kv_reserve(int32_t B, int32_t n_pages, int32_t page_size, int32_t max_pages, const int32_t *len, const int32_t *n_new,
                       const int32_t *seen, int32_t *table, int32_t *free_pages, int32_t *n_free, int32_t T, int32_t *tok_off, int32_t *n_got,
                       int32_t *pos, int32_t *slot, int32_t *dev_status, void *stream)
{
    const int32_t rc = check_pages(B, n_pages, page_size, max_pages, {len, n_new, table, free_pages, n_free, tok_off, n_got},
                                   {len, n_new, seen, table, free_pages, n_free, tok_off, n_got, pos, slot, dev_status});
    if (rc) return rc;
    if (T < 0 || T > (1 << 21)) return api_fail(MOA_ERR_SHAPE, "kv_reserve: T outside [0, 2^21]");
    const ReserveArgs a = {len, n_new, seen, table, free_pages, n_free, tok_off, n_got, pos, slot, dev_status, B, n_pages, max_pages, max_pages * page_size, T,
                           FastDiv((uint32_t)page_size)};
    const bool any = T > 0 && (pos || slot), here = any && B <= PT && T <= 8192;
    prof_set_site(S_KV_PAGES);
    hipStream_t st = (hipStream_t)stream;
    prof_begin(K_KV_RESERVE, st);
    if (here) MOA_KLAUNCH(k_kv_reserve<true>, dim3(1), dim3(PT), 0, st, a);
    else MOA_KLAUNCH(k_kv_reserve<false>, dim3(1), dim3(PT), 0, st, a);
    prof_end(st);
    if (any && !here) {
        prof_begin(K_KV_SLOTS, st);
        MOA_KLAUNCH(k_kv_slots, dim3((T + 255) / 256), dim3(256), 0, st, a);
        prof_end(st);
    }
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? MOA_OK : api_fail(MOA_ERR_HIP, hipGetErrorString(e));
}

int32_t moa_kv_release(int32_t B, int32_t n_pages, int32_t page_size, int32_t max_pages, const int32_t *len, int32_t *table,
                       int32_t *free_pages, int32_t *n_free, int32_t *dev_status, void *stream)
{
    const int32_t rc = check_pages(B, n_pages, page_size, max_pages, {len, table, free_pages, n_free}, {len, table, free_pages, n_free, dev_status});
    if (rc) return rc;
    const ReleaseArgs a = {len, table, free_pages, n_free, dev_status, B, n_pages, max_pages, max_pages * page_size, FastDiv((uint32_t)max_pages), FastDiv((uint32_t)page_size)};
    prof_set_site(S_KV_PAGES);
    hipStream_t st = (hipStream_t)stream;
    prof_begin(K_KV_RELEASE, st);
    MOA_KLAUNCH(k_kv_release, dim3(1), dim3(PT), 0, st, a);
    prof_end(st);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? MOA_OK : api_fail(MOA_ERR_HIP, hipGetErrorString(e));
}

}  // extern "C"
