// A cache of pages held in 8 bits: rows encoded into it (moa_kvq_append, moa_kvq_append_rows) and read back as values (moa_kvq_read).
//
// A block is MOA_KVQ_BLOCK rows of one page and KV head; keys and values have a scale each.  A code c stands for c * scale.  The scale of
// a block is the smallest power of two 2^e, -120 <= e <= 120, with absmax <= 448 2^e, 448 being the largest e4m3 number.  Powers of two
// because rows come one at a time: x / scale is then exact, so that a row is rounded once, to 4 significant bits, and a row that was
// encoded by a smaller scale keeps all of them when the scale grows, but where it falls below 2^-6 of the new one.  A scale that is no
// power of two would round every earlier row of the block again each time.  The bits lost to it are few: e4m3 is a floating format, its
// precision does not depend on where in its range the values lie.
#include "moa_kvq_device.h"

#include <stdio.h>

namespace moa {

int32_t check_kvq_cache(const moa_kvq_cache_t *c, const char *who)
{
    char msg[160];
    auto refuse = [&](int32_t code, const char *what) {
        snprintf(msg, sizeof msg, "%s: %s", who, what);
        return api_fail(code, msg);
    };
    if (!c) return refuse(MOA_ERR_NULL, "cache is NULL");
    moa_kv_cache_t g = kvq_geometry(*c);
    if (g.k) g.k = (void *)16;           // (codes are aligned to their byte anywhere)
    if (g.v) g.v = (void *)16;
    const int32_t rc = check_kv_cache(&g, who);
    if (rc) return rc;
    if (!c->k_scale || !c->v_scale) return refuse(MOA_ERR_NULL, "cache k_scale / v_scale is NULL");
    if (((uintptr_t)c->k_scale | (uintptr_t)c->v_scale) & 3) return refuse(MOA_ERR_SHAPE, "cache pointers must be aligned to their elements");
    return MOA_OK;
}

namespace {

constexpr int BLK = MOA_KVQ_BLOCK;

// ---------------------------------------------------------------- append
struct KvqAppendArgs {
    KvqDev c;
    const char *k_new, *v_new;
    int64_t seq_stride, head_stride, k_row_stride, v_row_stride;     // elements; rows of sequence b and head h: b seq + h head + (first + i) row
    int M;                           // rows of a sequence's slab, or of the whole batch where they are packed
    const int32_t *path, *n_new;     // [B, M], [B]; may be NULL
    const int32_t *tok_off;          // [B + 1], where rows are packed; else NULL
    FastDiv pieces;                  // of a row, VE elements each
};

struct NewRows { int first, n; };    // in the packed batch (0 in a slab), rows that sequence b gets

__device__ __forceinline__ NewRows new_rows(const KvqAppendArgs &a, int b, int held, bool report)
{
    int first = 0, most = a.M;
    if (a.tok_off) {
        const int o = a.tok_off[b], e = a.tok_off[b + 1];
        first = min(max(o, 0), a.M);
        most = min(max(e, first), a.M) - first;
        if (report && (o != first || e != first + most)) a.c.c.flag(MOA_DEV_BAD_LENGTH);
    }
    int n = a.n_new ? a.n_new[b] : most;
    if ((uint32_t)n > (uint32_t)most) {
        if (report) a.c.c.flag(MOA_DEV_BAD_LENGTH);
        n = n < 0 ? 0 : most;
    }
    if (n > a.c.c.cap - held) {
        if (report) a.c.c.flag(MOA_DEV_CACHE_FULL);
        n = a.c.c.cap - held;
    }
    return {first, n};
}

// e of the smallest scale 2^e that holds numbers of up to this size: 448 = 1.75 2^8, so that 1.m 2^x takes x - 8, or x - 7 where 1.m > 1.75
__device__ __forceinline__ float smallest_scale(float absmax)
{
    const uint32_t u = __float_as_uint(absmax);
    const int e = (int)(u >> 23) - 127 - 8 + ((u & 0x7fffffu) > 0x600000u);
    return __uint_as_float((uint32_t)(min(max(e, -120), 120) + 127) << 23);
}

__device__ __forceinline__ float wave_max(float x)
{
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) x = fmaxf(x, __shfl_xor(x, o));
    return x;
}

// One wavefront encodes what a call brings of one block of one KV head, of the keys or of the values: its rows are read once, into registers,
// while the table's entry and the block's scale are on their way.
// VE: elements that are read and encoded at a time, 16 bytes' worth, or 1 where rows are not in such pieces; IT: such pieces that a lane has at
// most, 0: rows are read twice instead.
template <typename T, int VE, int IT>
__device__ __forceinline__ void encode_block(const KvqAppendArgs &a, int b, int h, bool values, int held, NewRows in, int gb)
{
    const KvDev &c = a.c.c;
    const int lane = threadIdx.x & 63, ps = (int)c.page.d, dh = c.dh;
    const int pg = (int)a.c.blocks((uint32_t)gb), r0 = (gb - pg * (int)a.c.blocks.d) * BLK;
    const int s0 = pg * ps + r0, from = max(s0, held), rows = min(min(s0 + BLK, (pg + 1) * ps), held + in.n) - from;
    const int id = c.table[(int64_t)b * c.max_pages + pg];
    const T *src = (const T *)(values ? a.v_new : a.k_new) + b * a.seq_stride + h * a.head_stride;
    const int64_t row_stride = values ? a.v_row_stride : a.k_row_stride;
    const int pieces = (int)a.pieces.d, items = rows * pieces;
    auto load = [&](int it, u32x4 &x) {
        const int i = (int)a.pieces((uint32_t)it), p = it - i * pieces, at = from - held + i;
        int row = at;
        if (a.path) {
            row = a.path[(int64_t)b * a.M + at];
            if ((uint32_t)row >= (uint32_t)a.M) {
                c.flag(MOA_DEV_BAD_PARENT);
                row = row < 0 ? 0 : a.M - 1;
            }
        }
        const T *p0 = src + (in.first + row) * row_stride + p * VE;
        if constexpr (VE == 1) x[0] = __float_as_uint(ld(p0));
        else x = *(const u32x4 *)p0;
    };
    auto value = [](const u32x4 &x, int e) {
        return VE == 1 || sizeof(T) == 4 ? __uint_as_float(x[e]) : __uint_as_float(e & 1 ? x[e / 2] & 0xffff0000u : x[e / 2] << 16);
    };
    float most = 0.f;
    auto measure = [&](const u32x4 &x) {
#pragma unroll
        for (int e = 0; e < VE; ++e) {
            const float v = fabsf(value(x, e));
            most = fmaxf(most, v < INFINITY ? v : 0.f);                       // (NaN and infinity are held as NaN by any scale)
        }
    };
    u32x4 held_x[IT ? IT : 1];
    if constexpr (IT > 0) {
#pragma unroll
        for (int k = 0; k < IT; ++k) {
            held_x[k] = u32x4{0u, 0u, 0u, 0u};
            if (64 * k < items && lane + 64 * k < items) load(lane + 64 * k, held_x[k]);
        }
    }
    if (!a.c.is_page(id)) {
        if (lane == 0) c.flag(MOA_DEV_BAD_PAGE);
        return;
    }
    float *const scale_at = (values ? a.c.v_scale : a.c.k_scale) + a.c.block_in(id, h, r0);
    const float old = s0 < held ? *scale_at : 0.f;
    if constexpr (IT > 0) {
#pragma unroll
        for (int k = 0; k < IT; ++k) measure(held_x[k]);
    } else
#pragma unroll 1
        for (int it = lane; it < items; it += 64) {
            u32x4 x;
            load(it, x);
            measure(x);
        }
    char *const pool = values ? c.v : c.k;
    const int64_t row0 = (int64_t)(id * c.Hkv + h) * ps;
    float scale = smallest_scale(wave_max(most));
    if (s0 < held) {
        if (scale > old) {
            // rows that the block holds already, in the new scale
            const float f = old / scale;
            unsigned char *p = (unsigned char *)pool + (row0 + r0) * dh;
#pragma unroll 1
            for (int i = lane; i < (from - s0) * dh; i += 64) p[i] = (unsigned char)code_pair(code_value<0>(p[i]) * f, 0.f, 0, false);
        } else scale = old;
    }
    if (lane == 0) *scale_at = scale;
    // (a scale that this call did not make may be no power of two)
    const bool exact = (__float_as_uint(scale) & 0x807fffffu) == 0 && scale >= 0x1p-126f && scale <= 0x1p126f;
    const float inv = exact ? 1.f / scale : 0.f;
    unsigned char *const to0 = (unsigned char *)pool + (row0 + r0 + from - s0) * dh;
    auto store = [&](int it, const u32x4 &v, bool divide) {
        float x[VE];
#pragma unroll
        for (int e = 0; e < VE; ++e) x[e] = divide ? value(v, e) / scale : value(v, e) * inv;
        unsigned char *to = to0 + (int64_t)it * VE;                             // (rows of a block lie behind each other)
        if constexpr (VE == 1) *to = (unsigned char)code_pair(x[0], 0.f, 0, false);
        else {
            uint32_t w[VE / 4];
#pragma unroll
            for (int q = 0; q < VE / 4; ++q) w[q] = code_pair(x[4 * q + 2], x[4 * q + 3], code_pair(x[4 * q], x[4 * q + 1], 0, false), true);
            if constexpr (VE == 8) *(u32x2 *)to = u32x2{w[0], w[1]};
            else *(uint32_t *)to = w[0];
        }
    };
    if (IT > 0 && exact) {
#pragma unroll
        for (int k = 0; k < IT; ++k)
            if (lane + 64 * k < items) store(lane + 64 * k, held_x[k], false);
    } else
#pragma unroll 1
        for (int it = lane; it < items; it += 64) {
            u32x4 x;
            load(it, x);
            store(it, x, !exact);
        }
}

// ONE: a workgroup per sequence, which may then also move its length on.  Else gridDim.x of them per sequence, and a launch for the lengths.
// What bounds it is the chain of a wavefront's loads (length, table and rows, scale), then its maximum over lanes: by trace 4.9 us for a token of
// each of 64 sequences in slabs, 8.2 for up to seven nodes of each of 16, 11.9 + 3.9 for 5100 rows of four prompts (31 MB, 6 us by the copy rate;
// wavefronts wait 54 % of their time, vector units are busy 53 %).  A page of fewer than 16 rows is a block of its own: pages of one row, 41000
// of them, 285 us (252 MB, 49 us by the copy rate).
template <typename T, int VE, int IT, int THREADS, bool ONE>
__global__ __launch_bounds__(THREADS) void k_kvq_append(KvqAppendArgs a)
{
    const KvDev &c = a.c.c;
    const int b = blockIdx.z;
    const bool first = blockIdx.x == 0 && threadIdx.x == 0;
    const int held = c.length(b, first);
    const NewRows in = new_rows(a, b, held, first);
    if (in.n > 0) {
        const int ps = (int)c.page.d, bps = (int)a.c.blocks.d;
        auto block_of = [&](int slot) {
            const int pg = (int)c.page((uint32_t)slot);
            return pg * bps + (slot - pg * ps) / BLK;
        };
        const int gb0 = block_of(held), units = (block_of(held + in.n - 1) - gb0 + 1) * c.Hkv * 2;
        for (int u = blockIdx.x * (THREADS / 64) + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); u < units; u += gridDim.x * (THREADS / 64)) {
            const int j = u / (2 * c.Hkv), hv = u - j * 2 * c.Hkv;
            encode_block<T, VE, IT>(a, b, hv >> 1, hv & 1, held, in, gb0 + j);
        }
    }
    if (ONE) {
        __syncthreads();                     // every thread has read the length
        if (threadIdx.x == 0) c.len[b] = held + in.n;
    }
}

__global__ __launch_bounds__(256) void k_kvq_append_len(KvqAppendArgs a)
{
    const int b = blockIdx.x * 256 + threadIdx.x;
    if (b >= a.c.c.B) return;
    const int held = a.c.c.length(b, false);
    a.c.c.len[b] = held + new_rows(a, b, held, false).n;
}

template <typename T, int VE, int IT>
hipError_t launch_append(const KvqAppendArgs &a, hipStream_t st)
{
    // blocks that the rows of a sequence can be in (of packed rows any number may be one's: a token for each of 64 sequences so takes two launches, 6.4 + 4.9
    // us by events, where slabs take one, 7.1)
    const int64_t units = ((int64_t)a.M * (int)a.c.blocks.d / (int)a.c.c.page.d + 3) * a.c.c.Hkv * 2;
    // A workgroup's round of 16 blocks is about 2.5 us, the other launch 4; of a path's nodes few are accepted.
    const bool one = units <= (a.path ? 128 : 48);
    prof_begin(K_KVQ_APPEND, st);
    if (one) MOA_KLAUNCH((k_kvq_append<T, VE, IT, 1024, true>), dim3(1, 1, a.c.c.B), dim3(1024), 0, st, a);
    else {
        const int64_t blocks = (units + 3) / 4, most = 4096 / a.c.c.B + 1;
        MOA_KLAUNCH((k_kvq_append<T, VE, IT, 256, false>), dim3((unsigned)(blocks < most ? blocks : most), 1, a.c.c.B), dim3(256), 0, st, a);
    }
    prof_end(st);
    if (!one) {
        prof_begin(K_KVQ_APPEND_LEN, st);
        MOA_KLAUNCH(k_kvq_append_len, dim3((a.c.c.B + 255) / 256), dim3(256), 0, st, a);
        prof_end(st);
    }
    return hipGetLastError();
}

// `strides`: what the rows' addresses are made of besides k_new and v_new, in elements
int32_t append(KvqAppendArgs &a, int64_t strides, hipStream_t st, int dtype)
{
    const int es = dtype == MOA_BF16 ? 2 : 4, ve = 16 / es, dh = a.c.c.dh;
    const bool pieces = dh % ve == 0 && strides % ve == 0 && !(((uintptr_t)a.k_new | (uintptr_t)a.v_new) & 15) &&
                        !(((uintptr_t)a.c.c.k | (uintptr_t)a.c.c.v) & (ve - 1));
    a.pieces = FastDiv((uint32_t)(pieces ? dh / ve : dh));
    prof_set_site(S_KVQ);
    // pieces of a block's new rows a lane.  (One where it can be: the kernel's code is fetched while it runs, once.)
    const int per_lane = ((a.M < BLK ? a.M : BLK) * (int)a.pieces.d + 63) / 64;
    const hipError_t e = dtype == MOA_BF16 ? !pieces         ? launch_append<bf16_t, 1, 0>(a, st)
                                             : per_lane <= 1 ? launch_append<bf16_t, 8, 1>(a, st)
                                             : per_lane <= 4 ? launch_append<bf16_t, 8, 4>(a, st)
                                                             : launch_append<bf16_t, 8, 0>(a, st)
                         : !pieces         ? launch_append<float, 1, 0>(a, st)
                         : per_lane <= 1   ? launch_append<float, 4, 1>(a, st)
                         : per_lane <= 4   ? launch_append<float, 4, 4>(a, st)
                                           : launch_append<float, 4, 0>(a, st);
    return e == hipSuccess ? MOA_OK : api_fail(MOA_ERR_HIP, hipGetErrorString(e));
}

// ---------------------------------------------------------------- read
struct KvqReadArgs {
    KvqDev c;
    int P;                           // rows of k_out and v_out per sequence and KV head
    char *k_out, *v_out;             // [B, Hkv, P, dh]
    FastDiv pieces;
};

// VE codes at a time, 16 bytes of results, or 1 where rows are not in such pieces.  HBM bounds it: 16 sequences of 100 to 1500 tokens, 79 MB, 23 us
// with 16 codes a load and 32 bytes of results behind each other, 21.8 with 16 bytes, 16.8 when the stores say that nothing of it is read
// again soon, 15 with two of them a thread instead of four.
// (64 sequences of up to 251 tokens, 53 MB, 12.8 us by trace: 4.1 TB/s.)
constexpr int READ_U = 2;
template <typename T, int VE>
__global__ __launch_bounds__(256) void k_kvq_read(KvqReadArgs a)
{
    constexpr int U = READ_U;
    const KvDev &c = a.c.c;
    const int b = blockIdx.z, h = blockIdx.y >> 1, pieces = (int)a.pieces.d;
    const bool values = blockIdx.y & 1, first = blockIdx.x + blockIdx.y == 0 && threadIdx.x == 0;
    const int held = c.length(b, first), n = min(held, a.P);
    if (first && held > a.P) c.flag(MOA_DEV_CACHE_FULL);
    const unsigned char *pool = (const unsigned char *)(values ? c.v : c.k);
    const float *scales = values ? a.c.v_scale : a.c.k_scale;
    T *out = (T *)(values ? a.v_out : a.k_out) + ((int64_t)b * c.Hkv + h) * a.P * c.dh;
    const uint32_t items = (uint32_t)n * pieces;
    for (uint32_t it0 = blockIdx.x * (256 * U) + threadIdx.x; it0 < items; it0 += gridDim.x * (256 * U)) {
        int id[U], r[U];
        u32x2 w[U];
        float scale[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint32_t it = min(it0 + 256 * u, items - 1);
            const int s = (int)a.pieces(it), pg = (int)c.page((uint32_t)s);
            r[u] = s - pg * (int)c.page.d;
            id[u] = c.table[(int64_t)b * c.max_pages + pg];
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint32_t it = it0 + 256 * u;
            if (it >= items || !a.c.is_page(id[u])) continue;
            const int p = (int)(it - a.pieces(it) * pieces);
            const unsigned char *from = pool + ((int64_t)(id[u] * c.Hkv + h) * c.page.d + r[u]) * c.dh + p * VE;
            scale[u] = scales[a.c.block_in(id[u], h, r[u])];
            if constexpr (VE == 8) w[u] = *(const u32x2 *)from;
            else if constexpr (VE == 4) w[u][0] = *(const uint32_t *)from;
            else w[u][0] = *from;
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint32_t it = it0 + 256 * u;
            if (it >= items) continue;
            if (!a.c.is_page(id[u])) {
                c.flag(MOA_DEV_BAD_PAGE);
                continue;
            }
            T *to = out + (int64_t)it * VE;                                     // (rows of a head lie behind each other)
            const float sc = scale[u];
            if constexpr (VE == 1) st(to, code_value<0>(w[u][0]) * sc);
            else if constexpr (VE == 4)
                __builtin_nontemporal_store(f32x4{code_value<0>(w[u][0]) * sc, code_value<1>(w[u][0]) * sc, code_value<2>(w[u][0]) * sc, code_value<3>(w[u][0]) * sc}, (f32x4 *)to);
            else
                __builtin_nontemporal_store(u32x4{pack_bf16x2(code_value<0>(w[u][0]) * sc, code_value<1>(w[u][0]) * sc), pack_bf16x2(code_value<2>(w[u][0]) * sc, code_value<3>(w[u][0]) * sc),
                                     pack_bf16x2(code_value<0>(w[u][1]) * sc, code_value<1>(w[u][1]) * sc), pack_bf16x2(code_value<2>(w[u][1]) * sc, code_value<3>(w[u][1]) * sc)}, (u32x4 *)to);
        }
    }
}

template <typename T, int VE>
hipError_t launch_read(const KvqReadArgs &a, hipStream_t st)
{
    const int64_t blocks = ((int64_t)a.P * a.pieces.d + 256 * READ_U - 1) / (256 * READ_U);
    prof_begin(K_KVQ_READ, st);
    MOA_KLAUNCH((k_kvq_read<T, VE>), dim3((unsigned)(blocks < 1024 ? blocks : 1024), a.c.c.Hkv * 2, a.c.c.B), dim3(256), 0, st, a);
    prof_end(st);
    return hipGetLastError();
}

int32_t check_append(const moa_kvq_cache_t *c, const void *k_new, const void *v_new, const char *who)
{
    const int32_t rc = check_kvq_cache(c, who);
    if (rc) return rc;
    char msg[160];
    auto refuse = [&](int32_t code, const char *what) {
        snprintf(msg, sizeof msg, "%s: %s", who, what);
        return api_fail(code, msg);
    };
    if (!k_new || !v_new) return refuse(MOA_ERR_NULL, "k_new / v_new is NULL");
    if (((uintptr_t)k_new | (uintptr_t)v_new) & (c->dtype == MOA_BF16 ? 1 : 3)) return refuse(MOA_ERR_SHAPE, "k_new / v_new not aligned to their elements");
    if (c->B > 65535 || c->n_kv_heads > 32767) return refuse(MOA_ERR_SHAPE, "more than 65535 sequences or 32767 KV heads");
    return MOA_OK;
}

}  // namespace
}  // namespace moa

using namespace moa;

extern "C" {

int32_t moa_kvq_append(const moa_kvq_cache_t *cache, const void *k_new, const void *v_new, int32_t M, const int32_t *path,
                       const int32_t *n_new, int32_t *dev_status, void *stream)
{
    const int32_t rc = check_append(cache, k_new, v_new, "kvq_append");
    if (rc) return rc;
    if (M < 1 || M > (1 << 24) || (int64_t)M * cache->head_dim > INT32_MAX || (int64_t)M * cache->n_kv_heads > (1 << 29))
        return api_fail(MOA_ERR_SHAPE, "kvq_append: M outside [1, 2^24], M * head_dim above 2^31 - 1, or M * n_kv_heads above 2^29");
    const int64_t dh = cache->head_dim;
    KvqAppendArgs a = {KvqDev(*cache, dev_status), (const char *)k_new, (const char *)v_new, cache->n_kv_heads * M * dh, M * dh, dh, dh, M, path, n_new, nullptr, FastDiv(1)};
    return append(a, 0, (hipStream_t)stream, cache->dtype);
}

int32_t moa_kvq_append_rows(const moa_kvq_cache_t *cache, const void *k_new, int64_t k_stride, const void *v_new, int64_t v_stride, int32_t T,
                            const int32_t *tok_off, const int32_t *n_new, int32_t *dev_status, void *stream)
{
    if (T == 0) return check_kvq_cache(cache, "kvq_append_rows");        // nothing to do, and an empty batch has no address
    const int32_t rc = check_append(cache, k_new, v_new, "kvq_append_rows");
    if (rc) return rc;
    if (!tok_off) return api_fail(MOA_ERR_NULL, "kvq_append_rows: tok_off is NULL");
    const int64_t dh = cache->head_dim, width = cache->n_kv_heads * dh;
    if (T < 0 || T > (1 << 24) || (int64_t)T * cache->n_kv_heads > (1 << 29))
        return api_fail(MOA_ERR_SHAPE, "kvq_append_rows: T outside [0, 2^24], or T * n_kv_heads above 2^29");
    if (k_stride < width || v_stride < width) return api_fail(MOA_ERR_SHAPE, "kvq_append_rows: rows closer to each other than n_kv_heads * head_dim elements");
    if (k_stride > INT64_MAX / 8 / (T + 1) || v_stride > INT64_MAX / 8 / (T + 1)) return api_fail(MOA_ERR_SHAPE, "kvq_append_rows: strides beyond the address space");
    KvqAppendArgs a = {KvqDev(*cache, dev_status), (const char *)k_new, (const char *)v_new, 0, dh, k_stride, v_stride, T, nullptr, n_new, tok_off, FastDiv(1)};
    return append(a, k_stride | v_stride, (hipStream_t)stream, cache->dtype);
}

int32_t moa_kvq_read(const moa_kvq_cache_t *cache, int32_t P_cap, void *k_out, void *v_out, int32_t *dev_status, void *stream)
{
    const int32_t rc = check_kvq_cache(cache, "kvq_read");
    if (rc) return rc;
    if (!k_out || !v_out) return api_fail(MOA_ERR_NULL, "kvq_read: k_out / v_out is NULL");
    const int es = cache->dtype == MOA_BF16 ? 2 : 4;
    if (((uintptr_t)k_out | (uintptr_t)v_out) & (es - 1)) return api_fail(MOA_ERR_SHAPE, "kvq_read: k_out / v_out not aligned to their elements");
    if (P_cap < 1 || P_cap > (1 << 30) || (int64_t)P_cap * cache->head_dim > INT32_MAX) return api_fail(MOA_ERR_SHAPE, "kvq_read: P_cap outside [1, 2^30], or P_cap * head_dim above 2^31 - 1");
    if (cache->B > 65535 || cache->n_kv_heads > 32767) return api_fail(MOA_ERR_SHAPE, "kvq_read: more than 65535 sequences or 32767 KV heads");
    const int ve = 16 / es;
    const bool pieces = cache->head_dim % ve == 0 && !(((uintptr_t)k_out | (uintptr_t)v_out) & 15) && !(((uintptr_t)cache->k | (uintptr_t)cache->v) & (ve - 1));
    const KvqReadArgs a = {KvqDev(*cache, dev_status), P_cap, (char *)k_out, (char *)v_out, FastDiv((uint32_t)(pieces ? cache->head_dim / ve : cache->head_dim))};
    prof_set_site(S_KVQ);
    hipStream_t st = (hipStream_t)stream;
    const hipError_t e = cache->dtype == MOA_BF16 ? pieces ? launch_read<bf16_t, 8>(a, st) : launch_read<bf16_t, 1>(a, st)
                                                  : pieces ? launch_read<float, 4>(a, st) : launch_read<float, 1>(a, st);
    return e == hipSuccess ? MOA_OK : api_fail(MOA_ERR_HIP, hipGetErrorString(e));
}

}  // extern "C"
