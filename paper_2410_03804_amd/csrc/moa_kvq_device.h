// The cache of pages held in 8 bits that moa_kvq_append, moa_kvq_read and moa_kvq_decode_attn share: e4m3 codes with a scale for every
// MOA_KVQ_BLOCK rows of a page and KV head.
#ifndef MOA_KVQ_DEVICE_H
#define MOA_KVQ_DEVICE_H
#include "moa_kv_device.h"

namespace moa {

// the geometry, as that of a cache that is not held in 8 bits; k and v only stand for whether they are there
inline moa_kv_cache_t kvq_geometry(const moa_kvq_cache_t &c)
{
    return {c.dtype, c.n_kv_heads, c.head_dim, c.B, c.n_pages, c.page_size, c.max_pages, c.k, c.v, c.table, c.len, nullptr, nullptr, nullptr};
}
inline int kvq_blocks(int page_size) { return (page_size + MOA_KVQ_BLOCK - 1) / MOA_KVQ_BLOCK; }

// where a KV head's rows and scales lie: row and block numbers in the pool seen as rows and as blocks
struct KvqDev {
    KvDev c;                     // k, v: [n_pages, Hkv, page_size, dh] codes
    float *k_scale, *v_scale;    // [n_pages, Hkv, blocks of a page]
    FastDiv blocks;              // of a page
    KvqDev(const moa_kvq_cache_t &q, int32_t *status)
        : c(kvq_geometry(q), status), k_scale(q.k_scale), v_scale(q.v_scale), blocks((uint32_t)kvq_blocks(q.page_size))
    {
    }
    __device__ __forceinline__ bool is_page(int id) const { return (uint32_t)id < (uint32_t)c.n_pages; }
    // of page id, KV head h, row r of the page
    __device__ __forceinline__ int block_in(int id, int h, int r) const { return (id * c.Hkv + h) * (int)blocks.d + r / MOA_KVQ_BLOCK; }
};

// codes to numbers and back: e4m3 has a sign, 4 bits of exponent and 3 of mantissa, 448 as its largest number, NaN and no infinity.
// Both by the hardware's own conversions, which round to nearest even, and give NaN for what is infinite (or beyond 464: nothing here is).
__device__ __forceinline__ uint32_t code_pair(float lo, float hi, uint32_t old, bool upper)
{
    return upper ? __builtin_amdgcn_cvt_pk_fp8_f32(lo, hi, old, true) : __builtin_amdgcn_cvt_pk_fp8_f32(lo, hi, old, false);
}
template <int BYTE>
__device__ __forceinline__ float code_value(uint32_t codes) { return __builtin_amdgcn_cvt_f32_fp8(codes, BYTE); }

// the description's own consistency; `who` for the message
int32_t check_kvq_cache(const moa_kvq_cache_t *c, const char *who);

}  // namespace moa
#endif
