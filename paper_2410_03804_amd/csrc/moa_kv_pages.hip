// Pages of a pool handed out to the sequences of a batch and taken back, on the device (moa_kv_reserve, moa_kv_release).
//
// All of it is sums over the sequences in their order: of new tokens (where each one's rows lie in the batch), of pages that they lack
// (which of the free ones each gets, and who goes without), of pages that go back.  Where there is little of it one workgroup does
// everything, and what it costs is its chain of loads and barriers.  Beyond, a launch counts, sequence by sequence; one workgroup sums; and
// a third launch writes, again sequence by sequence.  What they hand on lies in the results themselves, until these are written.
#include "moa_kv_device.h"

namespace moa {

namespace {

constexpr int PT = 1024, PW = PT / 64;             // threads, wavefronts

// Sums over the workgroup's threads (or as many of its wavefronts as there are, PW at most) in their order.  Two sets of LDS in turn, so that one
// barrier a sum is enough.
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
        const uint32_t of = wave_scan(lane < (int)blockDim.x / 64 ? t[lane] : 0u);
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
    // free pages, within what there is
    __device__ __forceinline__ int pages_left(bool report) const
    {
        const int n = *n_free;
        if ((uint32_t)n <= (uint32_t)n_pages) return n;
        if (report) flag(MOA_DEV_BAD_LENGTH);
        return n < 0 ? 0 : n_pages;
    }
    // the new tokens of sequence b, within its capacity
    __device__ __forceinline__ int wanted(int b, int &len) const
    {
        const int asked = n_new[b];
        len = length(b, true);
        int n = max(asked, 0);
        if (asked < 0) flag(MOA_DEV_BAD_LENGTH);
        if (n > cap - len) {
            flag(MOA_DEV_CACHE_FULL);
            n = cap - len;
        }
        return n;
    }
    // table entries that n tokens behind slot len - 1 lie in, from that of slot len on
    __device__ __forceinline__ int pages_of(int len, int n) const
    {
        return n > 0 ? (int)page((uint32_t)(len + n - 1)) - (int)page((uint32_t)len) + 1 : 0;
    }
    __device__ __forceinline__ int32_t page_from(int place) const
    {
        const int32_t id = free_pages[place];
        if ((uint32_t)id >= (uint32_t)n_pages) flag(MOA_DEV_BAD_PAGE);
        return id;
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

__device__ __forceinline__ uint32_t from_last_lane(uint32_t x) { return (uint32_t)__builtin_amdgcn_readlane((int)x, 63); }

// the last of s[0 .. n - 1] (s[0] = 0, ascending) that is <= x
template <typename P>
__device__ __forceinline__ int last_upto(const P *s, int n, P x)
{
    int lo = 0;
    for (int step = 1 << (31 - __clz(n)); step; step >>= 1)
        if (lo + step < n && s[lo + step] <= x) lo += step;
    return lo;
}

// ---------------------------------------------------------------- in one launch: up to PT sequences, positions and slots of up to FEW_ROWS rows
// A token each of 16 sequences: 4.8 us by trace.
constexpr int FEW_ROWS = 8192;
__global__ __launch_bounds__(PT) void k_kv_reserve(ReserveArgs a)
{
    constexpr int PU = 2;                          // table entries that a thread looks at
    __shared__ uint32_t sums[2][PW], items_s[PT], need_s[PT];
    __shared__ int32_t first_s[PT], off_s[PT];
    __shared__ unsigned char got_s[PT];
    const int tid = threadIdx.x;
    BlockScan scan{sums};
    const int left = a.pages_left(tid == 0);
    int want = 0, len = 0;
    if (tid < a.B) want = a.wanted(tid, len);
    // (sums of what is left of the batch at most: 1024 of them fit)
    int n = min(want, a.T);
    const BlockScan::Sum at = scan((uint32_t)n);
    const int off = (int)min(at.before, (uint32_t)a.T), tokens = (int)min(at.all, (uint32_t)a.T);
    n = min(n, a.T - off);
    if (n < want) a.flag(MOA_DEV_BAD_LENGTH);
    if (tid < a.B) a.tok_off[tid] = off;
    off_s[tid] = off;
    // the table's entries that the new tokens lie in: items, those of a sequence one behind the other
    const int p0 = (int)a.page((uint32_t)len), pages = a.pages_of(len, n);
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
            e[u] = a.table + (int64_t)s[u] * a.max_pages + first_s[s[u]] + (int)(i - items_s[s[u]]);
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
    const bool got = need == 0 || lack.before + need <= (uint32_t)left;
    got_s[tid] = got;
    if (tid < a.B) a.n_got[tid] = got ? n : 0;
    const BlockScan::Sum give = scan(got ? need : 0u);
    // (the barrier of the sum stands between got_s and its use)
    uint32_t rank = 0;
    for (uint32_t i0 = 0; i0 < item.all; i0 += PT * PU) {
        if (item.all > PT * PU) look_at(i0, s, e);             // (else as it was left)
        const BlockScan::Sum r = scan(__popc(lacks));
        uint32_t k = rank + r.before;
#pragma unroll
        for (int u = 0; u < PU; ++u)
            if (lacks >> u & 1) {
                if (got_s[s[u]]) *e[u] = a.page_from(left - 1 - (int)k);
                ++k;
            }
        rank += r.all;
    }
    if (tid == 0) {
        a.tok_off[a.B] = tokens;
        *a.n_free = left - (int)give.all;
        if (give.all != lack.all) a.flag(MOA_DEV_CACHE_FULL);
    }
    if (!a.pos && !a.slot) return;
    __syncthreads();                                           // the table is written
    for (int t = tid; t < a.T; t += PT) {
        if (t >= tokens) {
            a.no_token(t);
            continue;
        }
        const int b = last_upto<int32_t>(off_s, a.B, t);
        a.token(t, b, off_s[b], got_s[b]);
    }
}

// ---------------------------------------------------------------- in three: a wavefront a sequence counts what it wants and lacks, into tok_off and n_got
// 64 prompts of 200 to 2048 tokens, 131072 rows of positions and slots: 2.7 + 3.7 + 4.8 us by trace (one workgroup for all but positions and slots 10.7
// + 4.0, and 283 + 5 for 668 prompts in pages of one row, which now take 13).
__device__ __forceinline__ int count_lacking(const ReserveArgs &a, int b, int len, int n)
{
    const int lane = threadIdx.x & 63, p0 = (int)a.page((uint32_t)len), pages = a.pages_of(len, n);
    const int32_t *row = a.table + (int64_t)b * a.max_pages + p0;
    int count = 0;
#pragma unroll 4
    for (int p = lane; p < pages; p += 64) count += row[p] < 0;
    return (int)from_last_lane(wave_scan((uint32_t)count));
}

__global__ __launch_bounds__(256) void k_kv_reserve_count(ReserveArgs a)
{
    const int b = __builtin_amdgcn_readfirstlane((int)(blockIdx.x * 4 + (threadIdx.x >> 6)));
    if (b >= a.B) return;
    int len;
    const int n = a.wanted(b, len), lacks = count_lacking(a, b, len, n);
    if ((threadIdx.x & 63) == 0) {
        a.tok_off[b] = n;
        a.n_got[b] = lacks;
    }
}

// One workgroup: tok_off becomes what it is to be; n_got says where, counted from the free pages that will be left, the first one of the
// sequence's pages lies, those behind it below it; -1 where it gets none.
__global__ __launch_bounds__(PT) void k_kv_reserve_sum(ReserveArgs a)
{
    __shared__ uint32_t sums[2][PW];
    __shared__ int cut_s[2];
    const int tid = threadIdx.x;
    BlockScan scan{sums};
    const int left = a.pages_left(tid == 0);
    uint32_t taken = 0;
    // twice over the sequences: how many pages are taken in all, then where each one's are
    for (int pass = 0; pass < 2; ++pass) {
        uint32_t tokens = 0, needed = 0;           // of the sequences of the rounds before
        bool refused = false;
        for (int b0 = 0; b0 < a.B; b0 += PT) {
            const int b = b0 + tid, want = b < a.B ? a.tok_off[b] : 0;
            uint32_t need = b < a.B ? (uint32_t)a.n_got[b] : 0u;
            int n = min(want, a.T);                // (1024 of at most 2^21 fit)
            const BlockScan::Sum at = scan((uint32_t)n);
            const int off = (int)min(tokens + at.before, (uint32_t)a.T);
            n = min(n, a.T - off);
            tokens = min(tokens + at.all, (uint32_t)a.T);
            // beyond the batch's rows: no tokens, or fewer, whose pages are counted again
            if (tid < 2) cut_s[tid] = -1;
            __syncthreads();
            if (n < want) {
                if (pass) a.flag(MOA_DEV_BAD_LENGTH);
                need = 0;
                if (n > 0) {
                    cut_s[0] = b;
                    cut_s[1] = n;
                }
            }
            __syncthreads();
            if (cut_s[0] >= 0) {
                const int lacks = count_lacking(a, cut_s[0], a.length(cut_s[0], false), cut_s[1]);
                if (b == cut_s[0]) need = (uint32_t)lacks;
                __syncthreads();
            }
            const BlockScan::Sum lack = scan(need);
            const bool got = need == 0 || needed + lack.before + need <= (uint32_t)left;
            if (!pass) taken += scan(got ? need : 0u).all;
            else {
                if (b < a.B) {
                    a.tok_off[b] = off;
                    a.n_got[b] = !got ? -1 : need == 0 ? 0 : (int)(taken - 1 - needed - lack.before);
                }
                refused |= !got;
            }
            needed += lack.all;
        }
        if (!pass) continue;
        if (refused) a.flag(MOA_DEV_CACHE_FULL);
        if (tid == 0) {
            a.tok_off[a.B] = (int)tokens;
            *a.n_free = left - (int)taken;
        }
    }
}

// A workgroup a sequence: its pages, then its tokens' positions and slots; those behind the B-th the batch's rows behind the last token.
__global__ __launch_bounds__(PT) void k_kv_reserve_write(ReserveArgs a)
{
    __shared__ uint32_t sums[2][PW];
    const int tid = threadIdx.x, step = (int)blockDim.x;
    if ((int)blockIdx.x >= a.B) {
        for (int t = ((int)blockIdx.x - a.B) * step + tid; t < a.T; t += ((int)gridDim.x - a.B) * step)
            if (t >= a.tok_off[a.B]) a.no_token(t);
        return;
    }
    const int b = blockIdx.x, off = a.tok_off[b], n = a.tok_off[b + 1] - off, top = a.n_got[b], len = a.length(b, false);
    __syncthreads();                               // everybody has read n_got
    if (tid == 0) a.n_got[b] = top < 0 ? 0 : n;
    BlockScan scan{sums};
    const int pages = a.pages_of(len, n), from = *a.n_free + top;
    int32_t *row = a.table + (int64_t)b * a.max_pages + (int)a.page((uint32_t)len);
    uint32_t rank = 0;
    bool bad = false;                              // (said here: of the batch's rows, which the count did not know)
    for (int p0 = 0; p0 < pages; p0 += step) {
        const int p = p0 + tid;
        const int32_t id = p < pages ? row[p] : 0;
        bad |= id >= a.n_pages;
        if (top < 0) continue;
        const BlockScan::Sum r = scan(id < 0 ? 1u : 0u);
        if (id < 0) row[p] = a.page_from(from - (int)(rank + r.before));
        rank += r.all;
    }
    if (bad) a.flag(MOA_DEV_BAD_PAGE);
    if (!a.pos && !a.slot) return;
    __syncthreads();                               // the table is written
    for (int i = tid; i < n; i += step) a.token(off + i, b, off, top >= 0);
}

// ---------------------------------------------------------------- pages that go back
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

// The same by a launch that writes the list and one that takes the pages out of the table, where that is large: a workgroup has some of the
// sequences, and counts for itself what goes back of the ones behind them, whose pages lie deeper: one compute unit's reads of most of the table
// bound it.  805 sequences of 425 entries 121 us by one workgroup, 40 + 4 so; 745 of 823 60 + 5; 128 of 501 9.7 + 4.1; 128 or 64 workgroups instead of 256
// (805 of 425): 42, 46.
constexpr int FEW_ENTRIES = 16384;
__device__ __forceinline__ int first_gone(const ReleaseArgs &a, int b, bool report)
{
    int n = a.len[b];
    if ((uint32_t)n > (uint32_t)a.cap) {
        if (report && a.dev_status) atomicOr(a.dev_status, MOA_DEV_BAD_LENGTH);
        n = n < 0 ? 0 : a.cap;
    }
    return n > 0 ? (int)a.page((uint32_t)(n - 1)) + 1 : 0;
}

__global__ __launch_bounds__(PT) void k_kv_release_list(ReleaseArgs a, int per)          // sequences of a workgroup
{
    __shared__ uint32_t sums[2][PW];
    const int tid = threadIdx.x, lane = tid & 63, b0 = (int)blockIdx.x * per, b1 = min(b0 + per, a.B);
    BlockScan scan{sums};
    int have = *a.n_free;
    if ((uint32_t)have > (uint32_t)a.n_pages) {
        if (blockIdx.x == 0 && tid == 0 && a.dev_status) atomicOr(a.dev_status, MOA_DEV_BAD_LENGTH);
        have = have < 0 ? 0 : a.n_pages;
    }
    // a wavefront takes up to 64 of the rows behind at a time, whose first entries that go its lanes look up together
    uint32_t behind = 0;
    const int share = min((a.B - b1 + PW - 1) / PW, 64);
    for (int w0 = b1 + share * __builtin_amdgcn_readfirstlane(tid >> 6); w0 < a.B; w0 += share * PW) {
        const int rows = min(share, a.B - w0), mine = lane < rows ? first_gone(a, w0 + lane, false) : a.max_pages;
        int lowest = mine;
#pragma unroll
        for (int o = 32; o >= 1; o >>= 1) lowest = min(lowest, __shfl_xor(lowest, o));
        for (int e0 = 0; e0 < a.max_pages - lowest; e0 += 256)
            for (int k = 0; k < rows; ++k) {
                const int32_t *row = a.table + (int64_t)(w0 + k) * a.max_pages;
                const int p0 = __builtin_amdgcn_readlane(mine, k) + e0 + lane;
                int32_t id[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) id[u] = p0 + 64 * u < a.max_pages ? row[p0 + 64 * u] : -1;
#pragma unroll
                for (int u = 0; u < 4; ++u) behind += (uint32_t)id[u] < (uint32_t)a.n_pages;
            }
    }
    uint32_t count = (uint32_t)have + scan(behind).all;
    for (int b = b1 - 1; b >= b0; --b) {
        const int32_t *row = a.table + (int64_t)b * a.max_pages;
        const int p0 = first_gone(a, b, false);
        for (int top = a.max_pages - 1; top >= p0; top -= PT) {
            const int p = top - tid;
            const int32_t id = p >= p0 ? row[p] : -1;
            const bool goes = (uint32_t)id < (uint32_t)a.n_pages;
            const BlockScan::Sum s = scan(goes ? 1u : 0u);
            const uint32_t at = count + s.before;
            if (goes && at < (uint32_t)a.n_pages) a.free_pages[at] = id;
            count += s.all;
        }
    }
}

__global__ __launch_bounds__(PT) void k_kv_release_table(ReleaseArgs a)
{
    __shared__ uint32_t all_s;
    const int b = __builtin_amdgcn_readfirstlane((int)(blockIdx.x * PW + (threadIdx.x >> 6))), lane = threadIdx.x & 63;
    auto flag = [&](int bit) {
        if (a.dev_status) atomicOr(a.dev_status, bit);
    };
    if (threadIdx.x == 0) all_s = 0;
    __syncthreads();
    if (b < a.B) {
        int32_t *row = a.table + (int64_t)b * a.max_pages;
        uint32_t count = 0;
        bool bad = false;
#pragma unroll 4
        for (int p = first_gone(a, b, lane == 0) + lane; p < a.max_pages; p += 64) {
            const int32_t id = row[p];
            if (id < 0) continue;
            row[p] = -1;
            bad |= id >= a.n_pages;
            count += id < a.n_pages;
        }
        if (bad) flag(MOA_DEV_BAD_PAGE);
        count = from_last_lane(wave_scan(count));
        if (lane == 0 && count) atomicAdd(&all_s, count);
    }
    __syncthreads();
    // Whole numbers: their order is of no account.  A list that claimed to hold less than nothing holds nothing, and no list holds more than
    // there are pages, whoever comes last.
    const int all = (int)all_s;
    if (threadIdx.x || (all == 0 && blockIdx.x)) return;
    // (Within its bounds before anything is added: a claim near 2^31 would come out below zero.)
    (void)atomicMax(a.n_free, 0);
    (void)atomicMin(a.n_free, a.n_pages);
    if (atomicAdd(a.n_free, all) + all > a.n_pages) {
        if (all) flag(MOA_DEV_BAD_PAGE);
        (void)atomicMin(a.n_free, a.n_pages);
    }
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
    prof_set_site(S_KV_PAGES);
    hipStream_t st = (hipStream_t)stream;
    if (B <= PT && (T <= FEW_ROWS || (!pos && !slot && (int64_t)B * max_pages <= FEW_ENTRIES))) {
        prof_begin(K_KV_RESERVE, st);
        MOA_KLAUNCH(k_kv_reserve, dim3(1), dim3(PT), 0, st, a);
        prof_end(st);
    } else {
        prof_begin(K_KV_RESERVE_COUNT, st);
        MOA_KLAUNCH(k_kv_reserve_count, dim3((B + 3) / 4), dim3(256), 0, st, a);
        prof_end(st);
        prof_begin(K_KV_RESERVE_SUM, st);
        MOA_KLAUNCH(k_kv_reserve_sum, dim3(1), dim3(PT), 0, st, a);
        prof_end(st);
        // (a sequence's threads by what it has on average; rows behind the last token by as many workgroups as they may want)
        const int threads = T / B > 512 ? PT : 256, behind = pos || slot ? (T + 8 * threads - 1) / (8 * threads) : 0;
        prof_begin(K_KV_RESERVE_WRITE, st);
        MOA_KLAUNCH(k_kv_reserve_write, dim3(B + behind), dim3(threads), 0, st, a);
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
    if (B == 1 || (int64_t)B * max_pages <= FEW_ENTRIES) {
        prof_begin(K_KV_RELEASE, st);
        MOA_KLAUNCH(k_kv_release, dim3(1), dim3(PT), 0, st, a);
        prof_end(st);
    } else {
        const int per = (B + 255) / 256;
        prof_begin(K_KV_RELEASE_LIST, st);
        MOA_KLAUNCH(k_kv_release_list, dim3((B + per - 1) / per), dim3(PT), 0, st, a, per);
        prof_end(st);
        prof_begin(K_KV_RELEASE_TABLE, st);
        MOA_KLAUNCH(k_kv_release_table, dim3((B + PW - 1) / PW), dim3(PT), 0, st, a);
        prof_end(st);
    }
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? MOA_OK : api_fail(MOA_ERR_HIP, hipGetErrorString(e));
}

}  // extern "C"
