// Attention of one new token per sequence over its cache of pages held in 8 bits (moa_kvq_decode_attn).
//
// As moa_decode_attn.hip, with keys and values code * scale, a scale for each block of rows of a page and KV head:
//   s_j = (q . c_j) ks_j log2(e) / sqrt(dh),  l = sum 2^(s_j - m),  o = sum (2^(s_j - m) vs_j) d_j / l,
// c_j, d_j the codes of key and value j and ks_j, vs_j their blocks' scales: a scale is multiplied into the score or the weight, once
// a key, and not into every element.  On the matrix cores the codes are widened to bf16, which holds every one of them: a product of two e4m3
// numbers would need queries and weights in 8 bits too.
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
// For head dims that are not in sixteens and for codes or queries that are not aligned: a row of keys or values is spread over LPR lanes, four codes
// each; 64 / LPR keys at a time.  WORDS: they can be read as one word.  (Sums over lanes bound it: at 128 dims, where it is not used otherwise, 8 x
// 32768 tokens with 64 heads 1040 us.)
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

// ---------------------------------------------------------------- on the matrix cores: head_dim a multiple of 16
// tiles that a wavefront holds in LDS, and the bytes of that
constexpr int kvq_stages(int DH) { return DH == 64 ? 4 : 2; }
constexpr uint32_t kvq_wave_bytes(int DH) { return kvq_stages(DH) * (2 * WK * DH + 512) + 128; }

// x as the sum of N bf16 numbers, each the rounding of what the ones before leave: to 2^-8, 2^-16, 2^-24 of x
template <int N>
__device__ __forceinline__ void split_pair(float x0, float x1, uint32_t (&part)[N])
{
#pragma unroll
    for (int i = 0; i < N; ++i) {
        part[i] = pack_bf16x2(x0, x1);
        x0 -= __uint_as_float(part[i] << 16);
        x1 -= __uint_as_float(part[i] & 0xffff0000u);
    }
}

typedef union { uint32_t w[4]; bf16x8 v; } Frag;

// eight codes as bf16, which holds every one of them
__device__ __forceinline__ bf16x8 widen(uint32_t c0, uint32_t c1)
{
    Frag f;
    f.w[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c0, 1.f, false));
    f.w[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c0, 1.f, true));
    f.w[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c1, 1.f, false));
    f.w[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c1, 1.f, true));
    return f.v;
}

typedef int i32x2 __attribute__((ext_vector_type(2)));

// The list of all tiles of 32 keys of all pairs, dealt to the runs so that none has more than one more than another.  A pair takes up one more
// place than it has tiles, since going on to it costs a wavefront up to a tile's time (its queries are waited for, its predecessor's result is
// written): 64 ragged sequences up to 8192, some of which are short, 105 us without and 94 with.  (At least two or four places a run: one
// sequence of 1084 5.6 us without, 7.5 and 10; of 27000 with 2 KV heads 6.9, 10.8 and 14.4.)  Every run goes over the lengths of all sequences to find its
// first, and so does every workgroup of the second launch: 8b heads, lengths up to 32, 64 sequences 5.5 + 4.6 us, 512 12.7 + 21.7, 4096 98.5 + 783.
struct PlaceList {
    uint32_t total, log2;                // places; runs that they are dealt to: a.runs, or as many as leave none without
    static __device__ __forceinline__ uint32_t of(int len) { return tiles_of<WK>(len) + (len > 0); }
    __device__ __forceinline__ void set(const DecodeArgs &a, uint32_t all)       // all: places of the sequences, for one KV head
    {
        total = all * (uint32_t)a.HB;
        log2 = min((uint32_t)a.runs_log2, 31u - (uint32_t)__clz((int)max(total, 1u)));
    }
    // the first place of run w (of the one behind the last: total), and the run of place f
    __device__ __forceinline__ uint32_t first(uint32_t w) const { return (uint32_t)((uint64_t)w * total >> log2); }
    __device__ __forceinline__ uint32_t run_of(uint32_t f) const { return (uint32_t)((((uint64_t)(f + 1) << log2) - 1) / total); }
    // the sequence that place f of run w's first is in, its length and its first place; false where the run has none
    __device__ __forceinline__ bool find(const DecodeArgs &a, uint32_t w, int &b, int &len, uint32_t &begin, uint32_t &f, uint32_t &n)
    {
        const int lane = threadIdx.x & 63;
        int mine = lane < a.c.B ? a.c.length(lane, false) : 0;
        uint32_t upto = wave_scan(of(mine)), all = from_lane(upto, 63);
        for (int i = lane + 64; i < (a.c.B + 63) / 64 * 64; i += 64) all += from_lane(wave_scan(i < a.c.B ? of(a.c.length(i, false)) : 0u), 63);
        set(a, all);
        f = first(w);
        n = first(w + 1) - f;
        if (w >> log2 || n == 0) return false;
        uint32_t base = 0;
        for (int b0 = 0;; b0 += 64) {
            const uint64_t past = __ballot(f < (base + upto) * (uint32_t)a.HB);
            if (past) {
                const int at = __ffsll((unsigned long long)past) - 1;
                b = b0 + at;
                len = (int)from_lane((uint32_t)mine, at);
                begin = (base + from_lane(upto, at) - of(len)) * (uint32_t)a.HB;
                return true;
            }
            base += from_lane(upto, 63);
            mine = b0 + 64 + lane < a.c.B ? a.c.length(b0 + 64 + lane, false) : 0;
            upto = wave_scan(of(mine));
        }
    }
};

// Where a wavefront's tile lies, and what is to be done behind it.
enum { GOES_ON = 0, PART_ENDS = 1, PAIR_ENDS = 2, NO_TILE = 3 };
struct Place {
    int b, hb, len, key0;
    int ends;
};

// The tiles of a wavefront's run, pair after pair.  Lengths of 64 sequences lie in a register, so that going on to the next sequence waits
// for nothing.
struct Walk {
    const DecodeArgs &a;
    int b, hb, len, lens_b, lens;
    uint32_t t, nt, left;                // the next tile of the pair, its tiles, places of the list that are left of the run
    bool from_start;                     // the run has had the pair's first tile
    __device__ __forceinline__ int length(int of)
    {
        if (of - lens_b >= 64) {
            lens_b = of;
            const int i = of + ((int)threadIdx.x & 63);
            lens = i < a.c.B ? a.c.length(i, false) : 0;
        }
        return (int)from_lane((uint32_t)lens, of - lens_b);
    }
    __device__ __forceinline__ void next(Place &p)
    {
        // (behind the last tile: table entries are read as if it were the pair's next one, and not used)
        p = Place{b, hb, len, (int)t * WK, NO_TILE};
        if (left == 0) return;
        --left;
        ++t;
        p.ends = t == nt ? from_start ? PAIR_ENDS : PART_ENDS : left == 0 ? PART_ENDS : GOES_ON;
        if (t < nt || left <= 1) {
            left = t < nt ? left : 0;    // (the one that is left is the next pair's beginning)
            return;
        }
        --left;
        t = 0;
        from_start = true;
        if (++hb < a.HB) return;
        hb = 0;
        do len = length(++b);
        while (len == 0);                // (left > 0: there is one)
        nt = tiles_of<WK>(len);
    }
};

// Sixteen query heads of a KV head are the columns of a tile of 32 keys: S^T = K Q^T, O^T += V^T P^T, codes widened to bf16 on their way into the
// matrix cores.  A wavefront has LDS of its own for NST tiles, and no barrier.  Codes go straight into LDS: a tile's keys take the place of
// those NST tiles before as soon as these have been used, their scales and its values likewise, and its table entries come another NST tiles
// before that.
// HBM bounds it: 8 sequences of 32768 tokens, 64 heads, 538 MB, 90 us (6.0 TB/s over all of it, 5 us of which are its beginning; FETCH_SIZE is the
// bytes of the codes and scales); vector units are busy 51 % of SIMD time, the matrix pipe 14 %, no LDS bank is waited for.  At 64 dims the
// vector units bound it, whose work is per key and not per byte: 64 x 4000 tokens, 131 MB, 31 us.  With more than 16 query heads a KV head, keys and
// values are read once for every 16: 32 on one, 64 x 32000 tokens, 526 MB, 148 us.  (Four wavefronts a run, as moa_decode_attn: 64
// ragged sequences up to 8192 125 us, now 95.)
// ONE: a workgroup of four wavefronts per pair, a quarter of its tiles each, joined in LDS.  Else a wavefront per run, which is a workgroup: what
// is fetched goes on from one pair to the next.
// DH: head_dim as it lies in LDS; the rows in the pool may be shorter (PAD, a multiple of 16): their last pieces are then zeros.
template <typename T, int DH, bool PAD, bool ONE>
__global__ __launch_bounds__(ONE ? 256 : 64, DH == 256 ? 1 : 2) void k_kvq_decode_mfma(KvqDecodeArgs k)
{
    constexpr int PIECES = DH / 16, RPI = 64 / PIECES, NL = WK / RPI;      // 16-byte pieces of a row; rows of a load, loads of K (or V)
    constexpr int NST = kvq_stages(DH), NKS = DH / 32, NDB = DH / 16;
    constexpr int QP = sizeof(T) == 4 ? 3 : 1, WP = sizeof(T) == 4 ? 3 : 2;    // bf16 numbers that a query's element, a weight is the sum of
    constexpr uint32_t HALFB = WK * DH, STAGEB = 2 * HALFB, IDB = 256, WAVEB = kvq_wave_bytes(DH);
    constexpr int PERTILE = 2 * NL + 2;                          // loads of a tile: keys, scales, table entries for NST tiles later, values
    constexpr int BEHIND_K = (NST - 1) * PERTILE + NL, BEHIND_V = (NST - 1) * PERTILE + NL + 2;
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    __shared__ float ml_s[ONE ? WAVES * 16 * 2 : 1], fin[ONE ? 16 * 2 : 1];
    const DecodeArgs &a = k.d;
    const int lane = threadIdx.x & 63, n16 = lane & 15, quad = lane >> 4;
    const int wave = ONE ? __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6) : 0;
    const int dh = PAD ? a.c.dh : DH;
    // [stages: K rows, V rows][table entries][scales][row numbers] of this wavefront.  Rows lie in LDS in the order in which the loads
    // bring them: load j has the keys g (32 / RPI) + j of its lane groups g, so that a lane's keys are neighbours.
    char *mine = smem + wave * WAVEB;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)smem + (uint32_t)wave * WAVEB;
    const uint32_t ids0 = lds0 + NST * STAGEB, scales0 = ids0 + NST * IDB, rows0 = scales0 + NST * IDB;
    const int grp = lane / PIECES;
    // key of a tile that lies in row p = lane % 32 in LDS
    const int key_p = (lane & 31) % RPI * NL + (lane & 31) / RPI;
    const float *const my_scales = lane < 32 ? k.k_scale : k.v_scale;
    const uint64_t zeros = (uint64_t)(uintptr_t)zero_row;
    // A piece of row p lies at position piece ^ f(p): reads of K touch 16 rows of one column, the transposing reads of V eight rows of
    // one column in each of two groups, 16 of 256 bytes in every case.
    auto swz = [](int p) {
        return DH == 64 ? ((p >> 2) & 3) ^ ((p >> 4) * 2) : DH == 128 ? ((p >> 1) & 7) ^ ((p >> 4) * 4) : (p & 15) ^ ((p >> 4) * 8);
    };

    // ---- the run
    Walk walk{a, 0, 0, 0, 0, 0, 0, 0, 0, true};
    uint32_t tile_one = (uint32_t)wave;
    if (ONE) {
        walk.b = (int)blockIdx.x / a.HB;
        walk.hb = (int)blockIdx.x - walk.b * a.HB;
        walk.len = (int)uniform((uint32_t)a.c.length(walk.b, walk.hb == 0 && threadIdx.x == 0));
        walk.nt = tiles_of<WK>(walk.len);
    } else {
        PlaceList list;
        uint32_t begin = 0, f = 0;
        if (!list.find(a, blockIdx.x, walk.b, walk.len, begin, f, walk.left)) return;
        const uint32_t in = f - begin, places = PlaceList::of(walk.len);
        walk.nt = tiles_of<WK>(walk.len);
        walk.hb = (int)uniform(in / places);
        walk.t = in - (uint32_t)walk.hb * places;
        if (walk.t == 0) --walk.left;                       // the pair's beginning
        else --walk.t;
        walk.from_start = walk.t == 0;
        if (walk.left == 0) return;
        walk.lens_b = walk.b - 64;                          // (nothing there yet)
        (void)walk.length(walk.b);
    }
    auto next_place = [&](Place &p) {
        if (!ONE) return walk.next(p);
        p = Place{walk.b, walk.hb, walk.len, (int)min(tile_one, walk.nt - 1) * WK, tile_one < walk.nt ? GOES_ON : NO_TILE};
        tile_one += WAVES;                                  // (tiles wave, wave + WAVES ..)
    };
    const bool some = !ONE || tile_one < walk.nt;           // whether there is a tile at all

    Place ahead[NST] = {}, cur[NST] = {};                   // of the tiles whose table entries are, whose rows are on their way
    auto fetch_ids = [&](int st) {
        next_place(ahead[st]);
        const Place &p = ahead[st];
        const int s = min(p.key0 + key_p, p.len - 1);       // in the order of rows, lanes 32 .. 63 as lanes 0 .. 31
        lds_gather4(uniform(ids0 + (uint32_t)st * IDB), (uint64_t)(uintptr_t)(a.c.table + (int64_t)p.b * a.c.max_pages + a.c.page((uint32_t)s)));
    };
    uint32_t row[NL];                                       // rows of the pool that this lane reads of the tile that is being fetched
    uint64_t scale_at = 0;                                  // and the scale that it brings
    // from the table entries in stage st, which are there; returns which of its rows count
    auto find_rows = [&](int st) -> uint32_t {
        cur[st] = ahead[st];
        const Place &p = cur[st];
        const int h = a.rtiles == 1 ? p.hb : p.hb / a.rtiles;
        const int s = p.key0 + key_p;
        const int id = *(const __attribute__((address_space(3))) int32_t *)(uintptr_t)(ids0 + (uint32_t)st * IDB + lane * 4);
        int r = -1;
        scale_at = zeros;
        if (s < p.len) {
            const int pg = (int)a.c.page((uint32_t)s);
            r = a.c.row_in(id, pg, h, s);
            if (r < 0) a.c.flag(MOA_DEV_BAD_PAGE);
            else scale_at = (uint64_t)(uintptr_t)(my_scales + (id * a.c.Hkv + h) * k.blocks + (s - pg * (int)a.c.page.d) / MOA_KVQ_BLOCK);
        }
        if (lane < 32) *(__attribute__((address_space(3))) int32_t *)(uintptr_t)(rows0 + key_p * 4) = r;
        const uint32_t ok = (uint32_t)__ballot(r >= 0);
#pragma unroll
        for (int j = 0; j < NL; ++j) row[j] = *(const __attribute__((address_space(3))) uint32_t *)(uintptr_t)(rows0 + (grp * NL + j) * 4);
        return ok;
    };
    auto fetch = [&](const char *pool, uint32_t at) {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");                      // nobody reads the place any more that is filled now
#pragma unroll
        for (int j = 0; j < NL; ++j) {
            const int piece = (lane % PIECES) ^ swz(RPI * j + grp);
            const bool in = (int)row[j] >= 0 && (!PAD || 16 * piece < dh);
            const uint64_t from = in ? (uint64_t)(uintptr_t)pool + (uint64_t)row[j] * (uint32_t)dh + 16 * piece : zeros + 16 * piece;
            lds_gather16<!PAD>(uniform(at + j * 1024), from);
        }
    };
    if (some) {
#pragma unroll
        for (int st = 0; st < NST; ++st) fetch_ids(st);
    }

    // ---- queries: the codes that a lane reads of a key, 16 behind each other, are the operands of two instructions
    Frag qf[NKS][QP];
    auto load_queries = [&](int b, int hb) {
        const int h = a.rtiles == 1 ? hb : hb / a.rtiles, r0 = (hb - h * a.rtiles) * 16, rows = min(16, a.G - r0);
        const T *q0 = (const T *)a.q + ((int64_t)b * a.H + h * a.G + r0 + min(n16, rows - 1)) * dh;
#pragma unroll
        for (int ks = 0; ks < NKS; ++ks) {
            const int d = 64 * (ks / 2) + 16 * quad + 8 * (ks & 1);
            if constexpr (QP == 1) {
                u32x4 x = {0u, 0u, 0u, 0u};
                if (!PAD || d < dh) x = *(const u32x4 *)(q0 + d);
                qf[ks][0].v = __builtin_bit_cast(bf16x8, x);
            } else {
                f32x4 x[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
                if (!PAD || d < dh) {
                    x[0] = *(const f32x4 *)(q0 + d);
                    x[1] = *(const f32x4 *)(q0 + d + 4);
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    uint32_t part[QP];
                    split_pair<QP>(x[e / 2][e % 2 * 2], x[e / 2][e % 2 * 2 + 1], part);
#pragma unroll
                    for (int i = 0; i < QP; ++i) qf[ks][i].w[e] = part[i];
                }
            }
        }
#pragma unroll
        for (int ks = 0; ks < NKS; ++ks)
#pragma unroll
            for (int i = 0; i < QP; ++i) asm volatile("" : "+v"(qf[ks][i].v));       // waited for here, not among the loads behind
    };
    load_queries(ONE ? walk.b : ahead[0].b, ONE ? walk.hb : ahead[0].hb);

    f32x4 acc[NDB];
    float mref = -INFINITY, lsum = 0.f;                     // reference of the exponent (log2 domain); this lane's part of the sum
    uint32_t ok[NST], any = 0;                              // rows of the tiles that count; whether any did
#pragma unroll
    for (int d = 0; d < NDB; ++d) acc[d] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int st = 0; st < NST; ++st) {
        ok[st] = 0;
        cur[st].ends = NO_TILE;
    }
    if (some) {
        wait_loads<0>();
#pragma unroll
        for (int st = 0; st < NST; ++st) {
            if (ahead[st].ends != NO_TILE) {
                ok[st] = find_rows(st);
                fetch(a.c.k, lds0 + st * STAGEB);
                lds_gather4(uniform(scales0 + st * IDB), scale_at);
                fetch_ids(st);
                fetch(a.c.v, lds0 + st * STAGEB + HALFB);
            }
        }
    }
    while (cur[0].ends != NO_TILE)
#pragma unroll
        for (int st = 0; st < NST; ++st) {
            if (cur[st].ends == NO_TILE) break;
            const uint32_t kb = lds0 + st * STAGEB, vb = kb + HALFB, sb = scales0 + st * IDB, count = ok[st];
            const Place at = cur[st];
            const bool next = ahead[st].ends != NO_TILE;         // the tile that takes this one's place
            any |= count;
            if (cur[(st + NST - 1) % NST].ends != NO_TILE) wait_loads<BEHIND_K>();
            else wait_loads<0>();
            f32x4 s[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
            for (int kp = 0; kp < NKS / 2; ++kp)
#pragma unroll
                for (int hf = 0; hf < 2; ++hf) {
                    const int p = 16 * hf + n16;
                    const u32x4 c = *(const __attribute__((address_space(3))) u32x4 *)(uintptr_t)(kb + p * DH + 16 * ((4 * kp + quad) ^ swz(p)));
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        const bf16x8 kf = widen(c[2 * half], c[2 * half + 1]);
#pragma unroll
                        for (int x = QP - 1; x >= 0; --x) s[hf] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[2 * kp + half][x].v, s[hf], 0, 0, 0);
                    }
                }
            // score element e: row 16 (e >> 2) + 4 quad + (e & 3) in LDS
            f32x4 ks[2], vs[2];
#pragma unroll
            for (int hf = 0; hf < 2; ++hf) {
                ks[hf] = *(const __attribute__((address_space(3))) f32x4 *)(uintptr_t)(sb + (16 * hf + 4 * quad) * 4);
                vs[hf] = *(const __attribute__((address_space(3))) f32x4 *)(uintptr_t)(sb + 128 + (16 * hf + 4 * quad) * 4);
            }
            float x[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = s[e >> 2][e & 3] * (ks[e >> 2][e & 3] * a.scale);
            if (count != 0xffffffffu) {
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    if (!(count >> (16 * (e >> 2) + 4 * quad + (e & 3)) & 1u)) x[e] = -INFINITY;
            }
            if (next) {
                ok[st] = find_rows(st);
                fetch(a.c.k, kb);
                lds_gather4(uniform(sb), scale_at);
                fetch_ids(st);
            } else cur[st].ends = NO_TILE;
            // A weight (times its value's scale) as the sum of two or three bf16 numbers: one alone (2^-8) would double the rounding of a
            // bf16 result.
            Frag w[WP];
            float tm = -INFINITY;
#pragma unroll
            for (int e = 0; e < 8; ++e) tm = fmaxf(tm, x[e]);
            if (__ballot(tm > mref)) {
                tm = over_lanes<4>(tm, fmaxf);
                const float mnew = fmaxf(mref, tm), corr = mnew == -INFINITY ? 1.f : fast_exp2(mref - mnew);
                mref = mnew;
                lsum *= corr;
#pragma unroll
                for (int d = 0; d < NDB; ++d)
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[d][e] *= corr;
            }
            const float ms = mref == -INFINITY ? 0.f : mref;
#pragma unroll
            for (int e = 0; e < 8; e += 2) {
                const float p0 = fast_exp2(x[e] - ms), p1 = fast_exp2(x[e + 1] - ms);
                lsum += p0 + p1;
                uint32_t part[WP];
                split_pair<WP>(p0 * vs[e >> 2][e & 3], p1 * vs[e >> 2][(e & 3) + 1], part);
#pragma unroll
                for (int i = 0; i < WP; ++i) w[i].w[e / 2] = part[i];
            }
            if (next) wait_loads<BEHIND_V>();
            else wait_loads<0>();
#pragma unroll
            for (int d = 0; d < NDB; ++d) {
                // transposing read: lane j of a group of 16 addresses row j >> 1 of the group's eight and dims 8 (j & 1) .. of the 16
                const int r = n16 >> 1, p = r < 4 ? 4 * quad + r : 12 + 4 * quad + r;
                const i32x2 c = __builtin_amdgcn_ds_read_tr8_b64_v2i32((__attribute__((address_space(3))) i32x2 *)(uintptr_t)(vb + p * DH + 16 * (d ^ swz(p)) + 8 * (n16 & 1)));
                const bf16x8 vf = widen((uint32_t)c[0], (uint32_t)c[1]);
#pragma unroll
                for (int i = WP - 1; i >= 0; --i) acc[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, w[i].v, acc[d], 0, 0, 0);
            }
            if (next) fetch(a.c.v, vb);
            if (ONE || at.ends == GOES_ON) continue;
            // ---- the pair, or the run's part of it, ends: a lane has 4 dims of every 16 of one head
            const int h = a.rtiles == 1 ? at.hb : at.hb / a.rtiles, r0 = (at.hb - h * a.rtiles) * 16, rows = min(16, a.G - r0);
            const float l = over_lanes<4>(lsum, add), m = max_of_keys(mref, any != 0);
            if (n16 < rows) {
                if (at.ends == PAIR_ENDS) {
                    const float inv = inverse_sum(m, l);
                    T *out = (T *)a.out + ((int64_t)at.b * a.H + h * a.G + r0 + n16) * dh;
#pragma unroll
                    for (int d = 0; d < NDB; ++d)
                        if (!PAD || 16 * d < dh) {
#pragma unroll
                            for (int e = 0; e < 4; ++e) moa::st(out + 16 * d + 4 * quad + e, acc[d][e] * inv);
                        }
                    if (m == -INFINITY && l == 0.f) a.c.flag(MOA_DEV_EMPTY_KEYS);
                } else {
                    const int64_t slot = ((int64_t)blockIdx.x + (int64_t)at.b * a.HB + at.hb) * a.HG + n16;
#pragma unroll
                    for (int d = 0; d < NDB; ++d)
                        if (!PAD || 16 * d < dh) *(f32x4 *)(a.part_o + slot * dh + 16 * d + 4 * quad) = acc[d];
                    if (quad == 0) {
                        a.part_ml[slot * 2] = m;
                        a.part_ml[slot * 2 + 1] = l;
                    }
                }
            }
            if (cur[(st + 1) % NST].ends == NO_TILE) return;
#pragma unroll
            for (int d = 0; d < NDB; ++d) acc[d] = f32x4{0.f, 0.f, 0.f, 0.f};
            mref = -INFINITY;
            lsum = 0.f;
            any = 0;
            load_queries(cur[(st + 1) % NST].b, cur[(st + 1) % NST].hb);
        }
    if (!ONE) return;
    wait_loads<0>();
    const int h = a.rtiles == 1 ? walk.hb : walk.hb / a.rtiles, rows = min(16, a.G - (walk.hb - h * a.rtiles) * 16);
    float *acc_s = (float *)mine;                                  // the stages are free again
    const float l = over_lanes<4>(lsum, add);
    if (n16 < rows) {
#pragma unroll
        for (int d = 0; d < NDB; ++d)
            if (!PAD || 16 * d < dh) *(f32x4 *)(acc_s + n16 * dh + 16 * d + 4 * quad) = acc[d];
        if (quad == 0) {
            ml_s[(wave * a.HG + n16) * 2] = max_of_keys(mref, any != 0);
            ml_s[(wave * a.HG + n16) * 2 + 1] = l;
        }
    }
    finish<T, PAD ? 0 : DH>(a, walk.b, walk.len, walk.hb, true, 0, (const float *)smem, WAVEB / 4, ml_s, fin);
}

// ---------------------------------------------------------------- the second launch
// A workgroup joins the partial results of one or more query heads of a pair: as many as leave 512 workgroups, where there are so many.
// Us, a workgroup a head against one a pair: 512 pairs of 4 heads, five parts each, 8.4 and 4.8; 64 pairs of 8 heads, 32 parts, 5.2 and 9.0.  Where
// parts are many, maxima and sums by one wavefront a head bound it: 2 pairs of 3 heads, 845 parts, 23 us; by all of them, and of the 512 parts that
// there now are, 8.
constexpr int JT = 512;
template <typename T>
__global__ __launch_bounds__(JT) void k_kvq_join(DecodeArgs a, int per, int chunks)      // heads of a workgroup; such workgroups of a pair
{
    __shared__ __attribute__((aligned(16))) float part[4 * JT];
    __shared__ float m_s[16], inv_s[16], parts_s[2][16];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, dh = a.c.dh;
    const int pair = (int)blockIdx.x / chunks, first = ((int)blockIdx.x - pair * chunks) * per;          // of the tile's heads
    const int b = pair / a.HB, hb = pair - b * a.HB, h = hb / a.rtiles, t0 = (hb - h * a.rtiles) * 16, r0 = t0 + first, rows = min(per, min(16, a.G - t0) - first);
    if (rows <= 0) return;
    uint32_t all = 0, before = 0;
    for (int b0 = 0; b0 < a.c.B; b0 += 64) {
        const uint32_t upto = wave_scan(b0 + lane < a.c.B ? PlaceList::of(a.c.length(b0 + lane, false)) : 0u);
        if (b > b0) before = all + from_lane(upto, min(b - b0, 64) - 1);
        all += from_lane(upto, 63);
    }
    PlaceList list;
    list.set(a, all);
    const int len = a.c.length(b, hb + first == 0 && tid == 0);
    const uint32_t nt = tiles_of<WK>(len);
    T *const out = (T *)a.out + ((int64_t)b * a.H + h * a.G + r0) * dh;
    if (nt == 0) {
        for (int i = tid; i < rows * dh; i += JT) st(out + i, 0.f);
        if (tid == 0) a.c.flag(MOA_DEV_EMPTY_KEYS);
        return;
    }
    // the runs that its tiles are in, and the first one's place among the partial results
    const uint32_t f0 = before * (uint32_t)a.HB + (uint32_t)hb * (nt + 1) + 1, w0 = list.run_of(f0), ns = list.run_of(f0 + nt - 1) - w0 + 1;
    if (ns == 1) return;                                         // the first launch had all of it
    const int64_t slot0 = (int64_t)w0 + (int64_t)b * a.HB + hb;
    const float *ml = a.part_ml + (slot0 * a.HG + first) * 2, *po = a.part_o + (slot0 * a.HG + first) * dh;
    // a group of E threads adds up every so many-th of them, four elements a thread; the first ones are loaded while the sums are unknown
    const uint32_t E = (uint32_t)(rows * dh) / 4, groups = E < JT ? JT / E : 1, step = groups;
    const uint32_t g = (uint32_t)tid / E;
    constexpr int U = 4;
    const bool on = g < groups;
    uint32_t c = (uint32_t)tid - g * E;
    auto load = [&](uint32_t s) { return on && c < E && s < ns ? *(const f32x4 *)(po + (int64_t)s * a.HG * dh + 4 * c) : f32x4{0.f, 0.f, 0.f, 0.f}; };
    f32x4 x[U];
#pragma unroll
    for (int u = 0; u < U; ++u) x[u] = load(g + u * step);
    // maxima and sums, by as many wavefronts a head as there are
    constexpr int JW = JT / 64;
    const int share = rows < JW ? JW / rows : 1;                 // wavefronts of a head
    for (int rw = wave; rw < rows * share; rw += JW) {
        const int r = rw / share;
        float m = -INFINITY, l = 0.f;
        for (uint32_t s = (uint32_t)(rw - r * share) * 64 + lane; s < ns; s += 64 * share) {
            const float mn = ml[(s * a.HG + r) * 2], ln = ml[(s * a.HG + r) * 2 + 1], top = fmaxf(m, mn), ms = top == -INFINITY ? 0.f : top;
            l = l * fast_exp2(m - ms) + ln * fast_exp2(mn - ms);
            m = top;
        }
        const float top = over_lanes<0>(m, fmaxf), ms = top == -INFINITY ? 0.f : top;
        l = over_lanes<0>(l * fast_exp2(m - ms), add);
        if (lane == 0) {
            parts_s[0][rw] = top;
            parts_s[1][rw] = l;
        }
    }
    __syncthreads();
    if (tid < rows) {
        float m = -INFINITY, l = 0.f;
        for (int k = 0; k < share; ++k) m = fmaxf(m, parts_s[0][tid * share + k]);
        const float ms = m == -INFINITY ? 0.f : m;
        for (int k = 0; k < share; ++k) l += parts_s[1][tid * share + k] * fast_exp2(parts_s[0][tid * share + k] - ms);
        if (m == -INFINITY && l == 0.f) a.c.flag(MOA_DEV_EMPTY_KEYS);
        m_s[tid] = ms;
        inv_s[tid] = inverse_sum(m, l);
    }
    __syncthreads();
    for (;;) {                                                   // (more than once where a pair has more than 4 JT elements)
        const int r = min((int)(4 * c) / dh, rows - 1);
        const float ms = m_s[r];
        f32x4 o = {0.f, 0.f, 0.f, 0.f};
        auto top_of = [&](uint32_t s) { return s < ns ? ml[(s * a.HG + r) * 2] : -INFINITY; };
        float t[U];
#pragma unroll
        for (int u = 0; u < U; ++u) t[u] = top_of(g + u * step);
        for (uint32_t s = g; s < ns; s += U * step) {
            f32x4 y[U];
            float w[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                w[u] = fast_exp2(t[u] - ms);
                y[u] = x[u];
                t[u] = top_of(s + (U + u) * step);
                x[u] = load(s + (U + u) * step);
            }
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int i = 0; i < 4; ++i) o[i] = fmaf(y[u][i], w[u], o[i]);
        }
        if (groups > 1) {
            *(f32x4 *)(part + 4 * tid) = o;
            __syncthreads();
            if ((uint32_t)tid >= E) return;
            for (uint32_t k = 1; k < groups; ++k) {
                const f32x4 y = *(const f32x4 *)(part + 4 * (k * E + tid));
#pragma unroll
                for (int i = 0; i < 4; ++i) o[i] += y[i];
            }
        }
        if (on && c < E) {
            const float inv = inv_s[r];
            if constexpr (sizeof(T) == 4) {
#pragma unroll
                for (int i = 0; i < 4; ++i) out[4 * c + i] = o[i] * inv;
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) st(out + 4 * c + i, o[i] * inv);
            }
        }
        if (groups > 1 || (c += JT) >= E) return;
#pragma unroll
        for (int u = 0; u < U; ++u) x[u] = load(g + u * step);
    }
}

// ---------------------------------------------------------------- host
template <typename T, int DH, bool PAD, bool ONE>
hipError_t launch_mfma(const KvqDecodeArgs &k, hipStream_t st)
{
    constexpr size_t lds = (size_t)(ONE ? WAVES : 1) * kvq_wave_bytes(DH);
    static bool raised[16] = {};
    const hipError_t e = raise_lds_limit_once(raised, (const void *)k_kvq_decode_mfma<T, DH, PAD, ONE>, lds);
    if (e != hipSuccess) return e;
    prof_begin(K_KVQ_DECODE_MFMA, st);
    MOA_KLAUNCH((k_kvq_decode_mfma<T, DH, PAD, ONE>), dim3(ONE ? k.d.c.B * k.d.HB : k.d.runs), dim3(ONE ? 64 * WAVES : 64), lds, st, k);
    prof_end(st);
    return hipGetLastError();
}

template <typename T, int DH>
hipError_t launch_mfma(const KvqDecodeArgs &k, hipStream_t st)
{
    if (k.d.c.dh == DH) return k.d.runs ? launch_mfma<T, DH, false, false>(k, st) : launch_mfma<T, DH, false, true>(k, st);
    return k.d.runs ? launch_mfma<T, DH, true, false>(k, st) : launch_mfma<T, DH, true, true>(k, st);
}

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
hipError_t launch_decode(const KvqDecodeArgs &k, const KvqPlan &p, hipStream_t st)
{
    const DecodeArgs &a = k.d;
    const int grid = a.runs ? a.runs : a.c.B * a.HB;
    hipError_t e;
    if (p.mfma) e = a.c.dh <= 64 ? launch_mfma<T, 64>(k, st) : a.c.dh <= 128 ? launch_mfma<T, 128>(k, st) : launch_mfma<T, 256>(k, st);
    else e = a.c.dh <= 64 ? launch_elements<T, 16>(k, grid, st) : a.c.dh <= 128 ? launch_elements<T, 32>(k, grid, st) : launch_elements<T, 64>(k, grid, st);
    if (e != hipSuccess || !a.runs) return e;
    if (!p.mfma) return launch_decode_join(a, sizeof(T) == 2, st);
    prof_begin(K_KVQ_JOIN, st);
    MOA_KLAUNCH(k_kvq_join<T>, dim3(a.c.B * a.HB * p.chunks), dim3(JT), 0, st, a, p.per, p.chunks);
    prof_end(st);
    return hipGetLastError();
}

// whether the matrix cores' form takes such a cache (and queries q, which it also reads 16 bytes at a time)
bool takes_mfma(const moa_kvq_cache_t &c, const void *q)
{
    return c.head_dim % 16 == 0 && !(((uintptr_t)c.k | (uintptr_t)c.v | (uintptr_t)q) & 15);
}
KvqPlan plan_of(const moa_kvq_cache_t &c, int H, bool mfma) { return kvq_plan(c.B, c.n_kv_heads, c.head_dim, c.max_pages * c.page_size, H, mfma); }

// enough for either form
size_t workspace_bytes(const moa_kvq_cache_t &c, int H)
{
    const size_t one = plan_of(c, H, false).total(), two = plan_of(c, H, takes_mfma(c, nullptr)).total();
    return one > two ? one : two;
}

int32_t check_decode(const moa_kvq_cache_t *c, int32_t H, const char *who)
{
    int32_t rc = check_kvq_cache(c, who);
    if (rc) return rc;
    if (H < 1 || H % c->n_kv_heads) return api_fail(MOA_ERR_SHAPE, "kvq_decode_attn: n_q_heads must be a multiple of the cache's n_kv_heads");
    if ((int64_t)c->B * H > (1 << 20)) return api_fail(MOA_ERR_SHAPE, "kvq_decode_attn: more than 2^20 pairs of sequence and query head");
    const int64_t cap = (int64_t)c->max_pages * c->page_size;
    // tiles are counted in 32 bits
    if ((int64_t)c->B * H * ((cap + WK - 1) / WK) > INT32_MAX / 2)
        return api_fail(MOA_ERR_SHAPE, "kvq_decode_attn: B * n_q_heads * ceil(capacity / 32) above 2^30");
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
    *bytes_host = workspace_bytes(*cache, n_q_heads);
    return MOA_OK;
}

int32_t moa_kvq_decode_attn(const moa_kvq_cache_t *cache, int32_t n_q_heads, const void *q, void *out, int32_t *dev_status, void *ws,
                            size_t ws_bytes, void *stream)
{
    const int32_t rc = check_decode(cache, n_q_heads, "kvq_decode_attn");
    if (rc) return rc;
    if (!q || !out) return api_fail(MOA_ERR_NULL, "kvq_decode_attn: q / out is NULL");
    if (((uintptr_t)q | (uintptr_t)out) & (cache->dtype == MOA_BF16 ? 1 : 3)) return api_fail(MOA_ERR_SHAPE, "kvq_decode_attn: q / out not aligned to their elements");
    const KvqPlan p = plan_of(*cache, n_q_heads, takes_mfma(*cache, q));
    const size_t need = workspace_bytes(*cache, n_q_heads);
    if (need && (!ws || (((uintptr_t)ws) & 255) || ws_bytes < need))
        return api_fail(MOA_ERR_WORKSPACE, "kvq_decode_attn: workspace NULL, misaligned or smaller than moa_kvq_decode_attn_workspace_bytes");
    const KvqDecodeArgs k = {{KvDev(kvq_geometry(*cache), dev_status), q, out, n_q_heads, n_q_heads / cache->n_kv_heads, p.HG, p.rtiles, cache->n_kv_heads * p.rtiles,
                              p.runs, p.runs ? 31 - __builtin_clz((unsigned)p.runs) : 0, 1.4426950408889634f / sqrtf((float)cache->head_dim),
                              (float *)ws, (float *)((char *)ws + p.part_o), 0, nullptr},
                             cache->k_scale, cache->v_scale, kvq_blocks(cache->page_size)};
    prof_set_site(S_KVQ);
    hipStream_t st = (hipStream_t)stream;
    const hipError_t e = cache->dtype == MOA_BF16 ? launch_decode<bf16_t>(k, p, st) : launch_decode<float>(k, p, st);
    return e == hipSuccess ? MOA_OK : api_fail(MOA_ERR_HIP, hipGetErrorString(e));
}

}  // extern "C"
