// The cache of pages that moa_kv_append, moa_decode_attn and moa_kv_evict share: what the kernels are given of it and how a
// slot of a sequence is found.
#ifndef MOA_KV_DEVICE_H
#define MOA_KV_DEVICE_H
#include "moa_common.h"
#include "../../include/moa.h"

namespace moa {

// n / d for 0 <= n < 2^31 and 1 <= d < 2^31: with l = ceil(log2 d) and mul = floor(2^(31+l) / d) + 1 the product n mul exceeds
// n 2^(31+l) / d by at most n < 2^31 parts in 2^(31+l) each, too little to reach the next whole number.
struct FastDiv {
    uint32_t d, mul, shift;
    explicit FastDiv(uint32_t div) : d(div), mul(0), shift(31)
    {
        while (shift < 62 && (1ull << (shift - 31)) < div) ++shift;
        mul = (uint32_t)((1ull << shift) / div + 1);
    }
    __host__ __device__ __forceinline__ uint32_t operator()(uint32_t n) const { return (uint32_t)(((uint64_t)n * mul) >> shift); }
};

struct KvDev {
    char *k, *v;             // [n_pages, Hkv, page_size, dh]
    const int32_t *table;    // [B, max_pages]
    int32_t *len;            // [B]
    int32_t *pos, *seen;     // [B, Hkv, cap], [B]; may be NULL
    float *score;            // [B, Hkv, cap]; may be NULL
    int32_t *dev_status;
    int B, Hkv, dh, n_pages, max_pages, cap;
    FastDiv page;
    KvDev(const moa_kv_cache_t &c, int32_t *status)
        : k((char *)c.k), v((char *)c.v), table(c.table), len(c.len), pos(c.pos), seen(c.seen), score(c.score), dev_status(status),
          B(c.B), Hkv(c.n_kv_heads), dh(c.head_dim), n_pages(c.n_pages), max_pages(c.max_pages), cap(c.max_pages * c.page_size),
          page((uint32_t)c.page_size)
    {
    }
    // The row, in the pool seen as rows, of a slot in [0, cap) of KV head h; -1 where the table names no page.  (Rows of a pool
    // fit 31 bits: check_kv_cache.)
    __host__ __device__ __forceinline__ int row(int b, int h, int slot) const
    {
        const int pg = (int)page((uint32_t)slot);
        return row_in(table[(int64_t)b * max_pages + pg], pg, h, slot);
    }
    // the same where the entry of the slot's page pg is at hand
    __host__ __device__ __forceinline__ int row_in(int id, int pg, int h, int slot) const
    {
        return (uint32_t)id < (uint32_t)n_pages ? (id * Hkv + h) * (int)page.d + (slot - pg * (int)page.d) : -1;
    }
    __device__ __forceinline__ void flag(int bit) const
    {
        if (dev_status) atomicOr(dev_status, bit);
    }
    // rows that sequence b holds, within the capacity; `report`: the one thread that says when they were not
    __device__ __forceinline__ int length(int b, bool report) const
    {
        const int n = len[b];
        if ((uint32_t)n <= (uint32_t)cap) return n;
        if (report) flag(MOA_DEV_BAD_LENGTH);
        return n < 0 ? 0 : cap;
    }
};

// inclusive sums over the wavefront's lanes by moves inside the vector unit: within rows of 16, then across them
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t dpp_from(uint32_t x)
{
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, ROWS, 0xf, false);
}
__device__ __forceinline__ uint32_t wave_scan(uint32_t x)
{
    x += dpp_from<0x111, 0xf>(x);     // row_shr 1, 2, 4, 8: from the lane so many below, 0 where there is none
    x += dpp_from<0x112, 0xf>(x);
    x += dpp_from<0x114, 0xf>(x);
    x += dpp_from<0x118, 0xf>(x);
    x += dpp_from<0x142, 0xa>(x);     // row_bcast 15: lane 15 of the row before, to rows 1 and 3
    x += dpp_from<0x143, 0xc>(x);     // row_bcast 31: lane 31, to rows 2 and 3
    return x;
}

// the description's own consistency; `who` for the message
int32_t check_kv_cache(const moa_kv_cache_t *c, const char *who);

inline size_t kv_esize(const moa_kv_cache_t &c) { return c.dtype == MOA_BF16 ? 2 : 4; }
// rows can be read and written 16 bytes at a time
inline bool kv_rows16(const moa_kv_cache_t &c, std::initializer_list<const void *> also)
{
    uintptr_t a = (uintptr_t)c.k | (uintptr_t)c.v | (uintptr_t)(c.head_dim * kv_esize(c));
    for (const void *p : also) a |= (uintptr_t)p;
    return (a & 15) == 0;
}

}  // namespace moa
#endif
