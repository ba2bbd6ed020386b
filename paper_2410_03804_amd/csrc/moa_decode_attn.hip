// Attention of one new token per sequence over its cache of pages (moa_decode_attn).
//
// One pass over the keys and values with the running maximum m and sum l of a softmax per query head, scores in the log2 domain:
//   s_j = q . k_j log2(e) / sqrt(dh),  l = sum 2^(s_j - m),  o = sum 2^(s_j - m) v_j / l.
// The work is the list of all tiles of TK keys of all (sequence, KV head) pairs, in that order, cut into runs of equally many whole
// tiles, one per workgroup: lengths are only known on the device, and a batch of very different ones is then as fast as an even
// one.  (Rounding up leaves the last runs without any: 2070 tiles in 512 runs are five for each of 414.)  A run
// that has all tiles of a pair writes its result; other pairs leave m, l and the unnormalised o (single precision) of each run
// that touched them in the workspace for a second launch to join.
#include "moa_decode_device.h"

namespace moa {

namespace {

// ---------------------------------------------------------------- element by element: single precision, and rows of bf16 that are not in 16 bytes
template <int LPR>
__device__ __forceinline__ float sum_over_lanes(float x)
{
    x += dpp_move_f32<0xB1>(x);     // quad_perm [1, 0, 3, 2]
    x += dpp_move_f32<0x4E>(x);     // quad_perm [2, 3, 0, 1]
    x += dpp_move_f32<0x141>(x);    // row_half_mirror
    if (LPR >= 16) x += dpp_move_f32<0x140>(x);    // row_mirror
    if (LPR >= 32) x = with_lane16(x, add);
    if (LPR >= 64) x = with_lane32(x, add);
    return x;
}

// A row of keys or values is spread over LPR lanes, VE = 16 bytes' worth of elements each; 64 / LPR keys at a time.
// WIDE: rows (of single precision: those of bf16 are then taken by the matrix cores) can be read 16 bytes at a time.
template <typename T, int LPR, int HG, bool WIDE>
__global__ __launch_bounds__(256, HG == 2 && sizeof(T) == 4 ? 4 : 2) void k_decode_attn(DecodeArgs a)
{
    constexpr int VE = 16 / sizeof(T), KPW = 64 / LPR, U = KPW < 8 ? 4 : 2;
    static_assert(WK % (KPW * U) == 0, "rounds of a tile");
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    float *acc_s = (float *)smem, *ml_s = acc_s + WAVES * HG * a.c.dh, *fin = ml_s + WAVES * HG * 2;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, c = lane % LPR, grp = lane / LPR, dh = a.c.dh;
    const int e0 = c * VE, ne = min(max(dh - e0, 0), VE);
    for_each_pair(a, [&](int b, int len, int hb, uint32_t t0, uint32_t nt, bool whole, int64_t slot) {
        const int h = hb / a.rtiles, r0 = (hb - h * a.rtiles) * HG, rows = min(HG, a.G - r0);
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
        auto load = [&](const char *pool, int row, u32x4 &x) {
            const T *p = (const T *)pool + (int64_t)row * dh + e0;
            x = u32x4{0u, 0u, 0u, 0u};
            if (row < 0 || ne == 0) return;
            // (whole lines where rows are not short: as lds_gather16, 64 sequences of up to 4000 keys 47 us without and 42 with; 16
            // heads on one KV head, which are two tiles, 8 x 8000 keys 59 and 62)
            if (WIDE) x = __builtin_nontemporal_load((const u32x4 *)p);
            else
#pragma unroll
                for (int e = 0; e < VE; ++e) {
                    const uint32_t one = e < ne ? sizeof(T) == 4 ? ((const uint32_t *)p)[e] : ((const uint16_t *)p)[e] : 0u;
                    if (sizeof(T) == 4) x[e] = one;
                    else x[e / 2] |= one << 16 * (e & 1);
                }
        };
        auto value = [](const u32x4 &x, int e) {
            return sizeof(T) == 4 ? __uint_as_float(x[e]) : __uint_as_float(e & 1 ? x[e / 2] & 0xffff0000u : x[e / 2] << 16);
        };
        // rounds of KPW U keys of this wavefront; the rows of one are looked up while the one before is computed
        constexpr int RT = WK / (KPW * U);
        int row_next[U];
        auto slot_of = [&](uint32_t t, int u) { return (int)(t * WAVES + wave) * KPW * U + u * KPW + grp; };
        auto look_up = [&](uint32_t t) {
#pragma unroll
            for (int u = 0; u < U; ++u) row_next[u] = a.c.row(b, h, min(slot_of(t, u), a.c.cap - 1));   // (what is there only counts below len)
        };
        look_up(t0 * RT);
#pragma unroll 1
        for (uint32_t t = t0 * RT; t < (t0 + nt) * RT && slot_of(t, 0) - grp < len; ++t) {
            int slots[U], row[U];
            u32x4 k[U], v[U];
            float s[U][HG];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                slots[u] = slot_of(t, u);
                row[u] = slots[u] < len ? row_next[u] : -1;
                if (slots[u] < len && row[u] < 0) a.c.flag(MOA_DEV_BAD_PAGE);
                any |= __ballot(row[u] >= 0);
            }
            look_up(t + 1);
#pragma unroll
            for (int u = 0; u < U; ++u) load(a.c.k, row[u], k[u]);
#pragma unroll
            for (int u = 0; u < U; ++u) load(a.c.v, row[u], v[u]);
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int r = 0; r < HG; ++r) {
                    float d = 0.f;
#pragma unroll
                    for (int e = 0; e < VE; ++e) d = fmaf(qf[r][e], value(k[u], e), d);
                    d = sum_over_lanes<LPR>(d);
                    s[u][r] = row[u] >= 0 ? d : -INFINITY;
                    if (a.raw && c == 0 && slots[u] < len && r < rows)
                        a.raw[(((int64_t)b * a.HB + hb) * a.cap32 + slots[u]) * HG + r] = s[u][r];
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
                    const float p = fast_exp2(s[u][r] - ms);
                    l[r] += p;
#pragma unroll
                    for (int e = 0; e < VE; ++e) acc[r][e] = fmaf(p, value(v[u], e), acc[r][e]);
                }
            }
        }
        // the lane groups' parts of a head, then one per wavefront into LDS
#pragma unroll
        for (int r = 0; r < HG; ++r) {
            constexpr int FROM = LPR == 8 ? 3 : LPR == 16 ? 4 : LPR == 32 ? 5 : 6;
            const float mn = over_lanes<FROM>(m[r], fmaxf), ms = mn == -INFINITY ? 0.f : mn, corr = fast_exp2(m[r] - ms);
            l[r] = over_lanes<FROM>(l[r] * corr, add);
#pragma unroll
            for (int e = 0; e < VE; ++e) {
                const float o = over_lanes<FROM>(acc[r][e] * corr, add);
                if (grp == 0 && e < ne) acc_s[(wave * HG + r) * dh + e0 + e] = o;
            }
            if (lane == 0) {
                ml_s[(wave * HG + r) * 2] = max_of_keys(mn, any != 0);
                ml_s[(wave * HG + r) * 2 + 1] = l[r];
            }
        }
        finish<T, 0>(a, b, len, hb, whole, slot, acc_s, HG * dh, ml_s, fin);
    });
}

// ---------------------------------------------------------------- on the matrix cores: bf16, head_dim a multiple of 8
// tiles that a wavefront holds in LDS, and the bytes of that
constexpr int decode_stages(int DH) { return DH == 64 ? 2 : 1; }
constexpr uint32_t decode_wave_bytes(int DH, int CT, bool accounts)
{
    return decode_stages(DH) * (2 * WK * DH * 2 + 256) + 128 + (accounts ? WK * 16 * CT * 4 : 0);      // (the last: a tile's scores)
}

// Sixteen query heads of a KV head are the columns of a tile, CT of which are computed side by side from the same keys and values:
// S^T = K Q^T, O^T += V^T P^T.  Every wavefront walks its own 32 keys of each tile of the run, with LDS of its own for NST tiles, so
// that there is no barrier before the run's end.  Keys and values go straight into LDS: a tile's keys take the place of those NST
// tiles before as soon as these have been used, its values likewise, and its table entries come another NST tiles before that.  Two
// workgroups share a compute unit, so that one loads while the other begins or ends a run; at 256 dims, and at 128 with two column
// tiles, the registers fit once only.  (At 64 dims with two column tiles they would fit twice, 227 of 256; it is launched as at
// 128.)  (Rings of two tiles and one workgroup a compute unit: 8 x 32768 keys 181 us against 180, 64 ragged
// sequences up to 8192 207 against 192, 96 of up to 100 16.7 against 11.1.)
// DH: head_dim as it lies in LDS; the rows in the pool may be shorter (PAD, a multiple of 8): their last pieces are then zeros.
template <int DH, int CT, bool PAD, bool ACC>
__global__ __launch_bounds__(256, DH == 256 || CT == 2 ? 1 : 2) void k_decode_attn_mfma(DecodeArgs a)
{
    constexpr int ROWB = DH * 2, PIECES = ROWB / 16, RPI = 64 / PIECES, NL = WK / RPI;   // bytes and 16-byte pieces of a row; rows of a load, loads of K (or V)
    constexpr int NST = decode_stages(DH), NKS = DH / 32, NDB = DH / 16;
    constexpr uint32_t HALFB = WK * ROWB, STAGEB = 2 * HALFB, IDB = 256, WAVEB = decode_wave_bytes(DH, CT, ACC);
    constexpr int PERTILE = 2 * NL + 1;                          // loads of a tile: keys, table entries for NST tiles later, values
    constexpr int BEHIND_K = (NST - 1) * PERTILE + NL, BEHIND_V = (NST - 1) * PERTILE + NL + 1;
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    __shared__ float ml_s[WAVES * 16 * CT * 2], fin[16 * CT * 2];
    const int tid = threadIdx.x, lane = tid & 63, n16 = lane & 15, quad = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int dh = PAD ? a.c.dh : DH;
    // [stages: K rows, V rows][table entries][row numbers][scores] of this wavefront.  Rows lie in LDS in the order in which the loads
    // bring them: load j has the keys g (32 / RPI) + j of its lane groups g, so that a lane's keys are neighbours.
    char *mine = smem + wave * WAVEB;
    const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)smem + (uint32_t)wave * WAVEB;
    const uint32_t ids0 = lds0 + NST * STAGEB, rows0 = ids0 + NST * IDB, raw0 = rows0 + 128;
    const int grp = lane / PIECES;
    // A piece of row p lies at position piece ^ f(p): reads of K touch 16 rows of one column, the transposing reads of V four
    // rows of 32 bytes.
    auto swz = [](int p) { return DH >= 128 ? 4 * (p & 3) + ((p >> 2) & 3) : (((p >> 1) & 3) << 1) | ((p >> 3) & 1); };

    for_each_pair(a, [&](int b, int len, int hb, uint32_t t0, uint32_t nt, bool whole, int64_t slot) {
        const int h = hb / a.rtiles, r0 = (hb - h * a.rtiles) * 16 * CT, rows = min(16 * CT, a.G - r0);
        const int cnt = (int)nt, key0 = (int)t0 * TK + wave * WK;
        const int32_t *table = a.c.table + (int64_t)b * a.c.max_pages;
        const bf16_t *q0 = (const bf16_t *)a.q + ((int64_t)b * a.H + h * a.G + r0) * dh;
        const uint64_t zeros = (uint64_t)(uintptr_t)zero_row;
        // table entries of the keys of tile i (lanes 32 .. 63 as lanes 0 .. 31)
        auto fetch_ids = [&](int i) {
            const int s = min(key0 + i * TK + (lane & 31), len - 1);
            lds_gather4(ids0 + (uint32_t)(i % NST) * IDB, (uint64_t)(uintptr_t)(table + a.c.page((uint32_t)s)));
        };
        u32x4 row[NL / 4];                                  // rows of the pool that this lane reads of the tile that is being fetched
        // from the table entries of tile i, which are there; returns which of its keys count
        auto find_rows = [&](int i) -> uint32_t {
            const int s = key0 + i * TK + (lane & 31);
            const int id = *(const __attribute__((address_space(3))) int32_t *)(uintptr_t)(ids0 + (uint32_t)(i % NST) * IDB + lane * 4);
            int r = -1;
            if (s < len) {
                r = a.c.row_in(id, (int)a.c.page((uint32_t)s), h, s);
                if (r < 0) a.c.flag(MOA_DEV_BAD_PAGE);
            }
            if (lane < 32) *(__attribute__((address_space(3))) int32_t *)(uintptr_t)(rows0 + lane * 4) = r;
            const uint32_t ok = (uint32_t)__ballot(r >= 0);
#pragma unroll
            for (int j = 0; j < NL / 4; ++j) row[j] = *(const __attribute__((address_space(3))) u32x4 *)(uintptr_t)(rows0 + (grp * NL + 4 * j) * 4);
            return ok;
        };
        auto fetch = [&](const char *pool, uint32_t at) {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");                  // nobody reads the place any more that is filled now
#pragma unroll
            for (int j = 0; j < NL; ++j) {
                const int piece = (lane % PIECES) ^ swz(RPI * j + grp);
                const uint32_t r = row[j / 4][j % 4];
                const bool in = (int)r >= 0 && (!PAD || 8 * piece < dh);
                const uint64_t from = in ? (uint64_t)(uintptr_t)pool + (uint64_t)r * (uint32_t)(2 * dh) + 16 * piece : zeros + 16 * piece;
                lds_gather16<!PAD>(at + j * 1024, from);
            }
        };
        // key of the tile that score element e (row 16 (e >> 2) + 4 quad + (e & 3) in LDS) belongs to
        auto key_of = [&](int e) {
            const int p = 16 * (e >> 2) + 4 * quad + (e & 3);
            return (p % RPI) * NL + p / RPI;
        };
        if (cnt > 0) {
#pragma unroll
            for (int i = 0; i < NST; ++i) fetch_ids(i);
        }
        bf16x8 qf[CT][NKS];
#pragma unroll
        for (int ct = 0; ct < CT; ++ct)
#pragma unroll
            for (int ks = 0; ks < NKS; ++ks) {
                const int d = 32 * ks + 8 * quad;
                union { u32x4 u; bf16x8 v; } x;
                x.u = u32x4{0u, 0u, 0u, 0u};
                if (!PAD || d < dh) x.u = *(const u32x4 *)(q0 + min(16 * ct + n16, rows - 1) * dh + d);
                qf[ct][ks] = x.v;
            }
#pragma unroll
        for (int ct = 0; ct < CT; ++ct)
#pragma unroll
            for (int ks = 0; ks < NKS; ++ks) asm volatile("" : "+v"(qf[ct][ks]));       // waited for here, not among the loads below
        f32x4 acc[CT][NDB];
        float mref[CT], lsum[CT];                           // reference of the exponent (log2 domain); this lane's part of the sum
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
#pragma unroll
            for (int d = 0; d < NDB; ++d) acc[ct][d] = f32x4{0.f, 0.f, 0.f, 0.f};
            mref[ct] = -INFINITY;
            lsum[ct] = 0.f;
        }

        uint32_t ok[NST], any = 0;                          // keys of the tiles that count; whether any did
        if (cnt > 0) {
            wait_loads<0>();
#pragma unroll
            for (int i = 0; i < NST; ++i) {
                ok[i] = 0;
                if (i < cnt) {
                    ok[i] = find_rows(i);
                    fetch(a.c.k, lds0 + i * STAGEB);
                    fetch_ids(i + NST);
                    fetch(a.c.v, lds0 + i * STAGEB + HALFB);
                }
            }
        }
        for (int i0 = 0; i0 < cnt; i0 += NST)
#pragma unroll
            for (int st = 0; st < NST; ++st) {
                const int i = i0 + st;
                if (i >= cnt) break;
                const uint32_t kb = lds0 + st * STAGEB, vb = kb + HALFB, count = ok[st];
                const bool next = i + NST < cnt;
                any |= count;
                if (i + NST <= cnt) wait_loads<BEHIND_K>();
                else wait_loads<0>();
                f32x4 s[CT][2];
#pragma unroll
                for (int ct = 0; ct < CT; ++ct) s[ct][0] = s[ct][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int ks = 0; ks < NKS; ++ks)
#pragma unroll
                    for (int hf = 0; hf < 2; ++hf) {
                        const int p = 16 * hf + n16;
                        const bf16x8 kf = *(const __attribute__((address_space(3))) bf16x8 *)(uintptr_t)(kb + p * ROWB + 16 * ((4 * ks + quad) ^ swz(p)));
#pragma unroll
                        for (int ct = 0; ct < CT; ++ct) s[ct][hf] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[ct][ks], s[ct][hf], 0, 0, 0);
                    }
                float x[CT][8];
#pragma unroll
                for (int ct = 0; ct < CT; ++ct) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) x[ct][e] = s[ct][e >> 2][e & 3] * a.scale;
                    if (count != 0xffffffffu) {
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            if (!(count >> key_of(e) & 1u)) x[ct][e] = -INFINITY;
                    }
                }
                // (in front of the next loads, so that nobody waits for these with the stores.  The stores are most of what accounts
                // cost: 8 x 8192 keys, 8 query heads per KV head, 49.5 us without, 59.5 with, 52 with all but the stores.)
                if (ACC && key0 + i * TK < len) {
                    // through LDS, where a tile's scores lie as they do in memory
#pragma unroll
                    for (int ct = 0; ct < CT; ++ct)
                        if (16 * ct + n16 < rows) {
#pragma unroll
                            for (int e = 0; e < 8; ++e)
                                *(__attribute__((address_space(3))) float *)(uintptr_t)(raw0 + (key_of(e) * a.HG + 16 * ct + n16) * 4) = x[ct][e];
                        }
                    float *raw = a.raw + (((int64_t)b * a.HB + hb) * a.cap32 + key0 + i * TK) * a.HG;
                    for (int at = 4 * lane; at < WK * a.HG; at += 256)
                        *(u32x4 *)(raw + at) = *(const __attribute__((address_space(3))) u32x4 *)(uintptr_t)(raw0 + at * 4);
                }
                if (next) {
                    ok[st] = find_rows(i + NST);
                    fetch(a.c.k, kb);
                    fetch_ids(i + 2 * NST);
                }
                // A weight as the sum of two bf16 numbers, so that it counts with 2^-16 like in single precision: the matrix
                // cores have nothing else to do, and one bf16 alone (2^-8) would double the result's own rounding.
                union { uint32_t w[4]; bf16x8 v; } hi[CT], lo[CT];
#pragma unroll
                for (int ct = 0; ct < CT; ++ct) {
                    float tm = -INFINITY;
#pragma unroll
                    for (int e = 0; e < 8; ++e) tm = fmaxf(tm, x[ct][e]);
                    if (__ballot(tm > mref[ct])) {
                        tm = over_lanes<4>(tm, fmaxf);
                        const float mnew = fmaxf(mref[ct], tm), corr = mnew == -INFINITY ? 1.f : fast_exp2(mref[ct] - mnew);
                        mref[ct] = mnew;
                        lsum[ct] *= corr;
#pragma unroll
                        for (int d = 0; d < NDB; ++d)
#pragma unroll
                            for (int e = 0; e < 4; ++e) acc[ct][d][e] *= corr;
                    }
                    const float ms = mref[ct] == -INFINITY ? 0.f : mref[ct];
#pragma unroll
                    for (int e = 0; e < 8; e += 2) {
                        const float p0 = fast_exp2(x[ct][e] - ms), p1 = fast_exp2(x[ct][e + 1] - ms);
                        lsum[ct] += p0 + p1;
                        const uint32_t w = pack_bf16x2(p0, p1);
                        hi[ct].w[e / 2] = w;
                        lo[ct].w[e / 2] = pack_bf16x2(p0 - __uint_as_float(w << 16), p1 - __uint_as_float(w & 0xffff0000u));
                    }
                }
                if (next) wait_loads<BEHIND_V>();
                else wait_loads<0>();
#pragma unroll
                for (int d = 0; d < NDB; ++d) {
                    // transposing read: lane j of a group of 16 addresses key j >> 2 and dims 4 (j & 3) .. of the group's 16
                    union { i16x4 h[2]; bf16x8 v; } u;
#pragma unroll
                    for (int hf = 0; hf < 2; ++hf) {
                        const int p = 16 * hf + 4 * quad + (n16 >> 2);
                        u.h[hf] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4 *)(uintptr_t)(
                            vb + p * ROWB + 16 * ((2 * d + ((n16 & 3) >> 1)) ^ swz(p)) + 8 * (n16 & 1)));
                    }
#pragma unroll
                    for (int ct = 0; ct < CT; ++ct) {
                        acc[ct][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(u.v, hi[ct].v, acc[ct][d], 0, 0, 0);
                        acc[ct][d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(u.v, lo[ct].v, acc[ct][d], 0, 0, 0);
                    }
                }
                if (next) fetch(a.c.v, vb);
            }
        wait_loads<0>();
        float *acc_s = (float *)mine;                              // the stages are free again
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
            const float l = over_lanes<4>(lsum[ct], add);
            const int r = 16 * ct + n16;
            if (r < rows) {
#pragma unroll
                for (int d = 0; d < NDB; ++d)
                    if (!PAD || 16 * d + 4 * quad < dh) *(f32x4 *)(acc_s + r * dh + 16 * d + 4 * quad) = acc[ct][d];
                if (quad == 0) {
                    ml_s[(wave * a.HG + r) * 2] = max_of_keys(mref[ct], any != 0);
                    ml_s[(wave * a.HG + r) * 2 + 1] = l;
                }
            }
        }
        finish<bf16_t, PAD ? 0 : DH>(a, b, len, hb, whole, slot, (const float *)smem, WAVEB / 4, ml_s, fin);
    });
}

// ---------------------------------------------------------------- the second launch
// Workgroups 0 .. B H - 1 join the partial results of one query head; the others bring the accounts of 256 slots of a (sequence,
// KV head) up to date from its scores, now that the sums are known.  Either leaves alone what the first launch finished.
// The latter are as many as the capacity has, and read their scores before they know the length, which hides the one behind the other
// where most slots are in use and is paid for where few are.  16 sequences of 2048 tokens, 8b heads, us: 7.2 in a capacity of
// 2112, 19.3 of 16384, 48.5 of 65536; 64 of 1000: none in a capacity of 1024, 36 of 8192, 91 of 32768.  (Without accounts 4 in any.)
constexpr int ACC_SLOTS = 256;
template <typename T>
__global__ __launch_bounds__(256) void k_decode_join(DecodeArgs a)
{
    __shared__ float sm[2][32][8], fin[32][2];
    __shared__ __attribute__((aligned(16))) float part[1024];
    const int tid = threadIdx.x, lane = tid & 63, dh = a.c.dh;
    const int nb = a.c.B * a.H;
    const bool accounts = (int)blockIdx.x >= nb;
    int b, h, r = 0, chunk = 0;                              // r: query head within its KV head
    if (!accounts) {
        if (blockIdx.y) return;
        b = (int)blockIdx.x / a.H;
        h = ((int)blockIdx.x - b * a.H) / a.G;
        r = (int)blockIdx.x - b * a.H - h * a.G;
    } else {
        const int chunks = (a.c.cap + ACC_SLOTS - 1) / ACC_SLOTS, i = (int)(blockIdx.x + blockIdx.y * (gridDim.x - nb)) - nb, bh = i / chunks;
        if (bh >= a.c.B * a.c.Hkv) return;
        chunk = i - bh * chunks;
        b = bh / a.c.Hkv;
        h = bh - b * a.c.Hkv;
    }
    // this thread's account and scores, while the lengths are on their way (where there are several row tiles, those of the first)
    const int mine = chunk * ACC_SLOTS + tid;
    float score = 0.f, weight = 0.f, raw[32];
    auto load_raw = [&](int rt) {
        const float *p = a.raw + ((((int64_t)b * a.HB + h * a.rtiles + rt)) * a.cap32 + mine) * a.HG;
        if ((a.HG & 3) == 0) {
#pragma unroll
            for (int q = 0; q < 8; ++q)
                if (4 * q < a.HG) *(f32x4 *)(raw + 4 * q) = *(const f32x4 *)(p + 4 * q);
        } else {
#pragma unroll
            for (int q = 0; q < 32; ++q)
                if (q < a.HG) raw[q] = p[q];
        }
    };
    float *const account = a.c.score + ((int64_t)b * a.c.Hkv + h) * a.c.cap + mine;
    if (accounts && mine < a.c.cap) {
        score = *account;
        load_raw(0);
    }
    uint32_t all = 0, before = 0;
    for (int b0 = 0; b0 < a.c.B; b0 += 64) {
        const uint32_t upto = wave_scan(b0 + lane < a.c.B ? tiles_of(a.c.length(b0 + lane, false)) : 0u);
        if (b > b0) before = all + from_lane(upto, min(b - b0, 64) - 1);
        all += from_lane(upto, 63);
    }
    TileList list;
    list.set(a, all);
    const int len = a.c.length(b, !accounts && h + r == 0 && tid == 0);
    const uint32_t nt = tiles_of(len);
    // the runs that tiles of row tile rt of this KV head are in, and the first's place among the partial results
    auto runs_of = [&](int rt, uint32_t &w0, uint32_t &ns, int64_t &slot0) {
        const uint32_t hb = (uint32_t)(h * a.rtiles + rt), f0 = before * (uint32_t)a.HB + hb * nt;
        w0 = f0 / list.per;
        ns = nt ? (f0 + nt - 1) / list.per - w0 + 1 : 0;
        slot0 = (int64_t)w0 + (int64_t)b * a.HB + hb;
    };
    uint32_t w0, ns;
    int64_t slot0;
    if (!accounts) {
        const int rt = r / a.HG, rr = r - rt * a.HG;
        runs_of(rt, w0, ns, slot0);
        T *out = (T *)a.out + ((int64_t)b * a.H + h * a.G + r) * dh;
        if (ns == 0) {
            for (int d = tid; d < dh; d += 256) st(out + d, 0.f);
            if (tid == 0) a.c.flag(MOA_DEV_EMPTY_KEYS);
        }
        if (ns <= 1) return;
        const float *ml = a.part_ml + (slot0 * a.HG + rr) * 2, *po = a.part_o + (slot0 * a.HG + rr) * dh;
        const int64_t ml_step = (int64_t)a.HG * 2, po_step = (int64_t)a.HG * dh;
        // each group of `lanes` threads adds up every so many-th partial result, four elements a thread; the first ones are loaded
        // while the sums are still unknown
        const int lanes = dh <= 64 ? 16 : dh <= 128 ? 32 : 64, c = tid & (lanes - 1), groups = 256 / lanes, d0 = 4 * c, g0 = tid / lanes;
        auto load = [&](uint32_t s) {
            f32x4 x = {0.f, 0.f, 0.f, 0.f};
            if (s < ns && d0 < dh) {
                if ((dh & 3) == 0) x = *(const f32x4 *)(po + s * po_step + d0);
                else
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (d0 + i < dh) x[i] = po[s * po_step + d0 + i];
            }
            return x;
        };
        constexpr int U = 4;
        f32x4 x[U];
#pragma unroll
        for (int u = 0; u < U; ++u) x[u] = load(g0 + u * groups);
        float m = -INFINITY, l = 0.f;
        for (uint32_t s = lane; s < ns; s += 64) m = fmaxf(m, ml[s * ml_step]);
        m = over_lanes<0>(m, fmaxf);
        const float ms = m == -INFINITY ? 0.f : m;
        for (uint32_t s = lane; s < ns; s += 64) l += ml[s * ml_step + 1] * fast_exp2(ml[s * ml_step] - ms);
        l = over_lanes<0>(l, add);
        if (tid == 0 && m == -INFINITY && l == 0.f) a.c.flag(MOA_DEV_EMPTY_KEYS);
        const float inv = inverse_sum(m, l);
        f32x4 o = {0.f, 0.f, 0.f, 0.f};
        for (uint32_t s = g0; s < ns; s += U * groups) {
            f32x4 y[U];
            float w[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const uint32_t su = s + u * groups;
                w[u] = su < ns ? fast_exp2(ml[su * ml_step] - ms) : 0.f;
                y[u] = x[u];
                x[u] = load(su + U * groups);
            }
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int i = 0; i < 4; ++i) o[i] = fmaf(y[u][i], w[u], o[i]);
        }
        *(f32x4 *)(part + 4 * tid) = o;
        __syncthreads();
        if (tid < dh) {
            float x = 0.f;
            for (int g = 0; g < groups; ++g) x += part[g * 4 * lanes + tid];
            st(out + tid, x * inv);
        }
        return;
    }
    if (chunk * ACC_SLOTS >= len) return;
    for (int rt = 0; rt < a.rtiles; ++rt) {
        const int r0 = rt * a.HG, rows = min(a.HG, a.G - r0);
        runs_of(rt, w0, ns, slot0);
        if (ns == 1 && a.rtiles == 1) return;                // the first launch had all of it
        // of each row the maximum and the sum: eight threads a row
        const int row = tid & 31, p = tid >> 5;
        float m = -INFINITY, l = 0.f;
        if (row < rows)
            for (uint32_t s = p; s < ns; s += 8) m = fmaxf(m, a.part_ml[((slot0 + s) * a.HG + row) * 2]);
        __syncthreads();
        sm[0][row][p] = m;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 8; ++i) m = fmaxf(m, sm[0][row][i]);
        const float ms = m == -INFINITY ? 0.f : m;
        if (row < rows)
            for (uint32_t s = p; s < ns; s += 8) {
                const float *ml = a.part_ml + ((slot0 + s) * a.HG + row) * 2;
                l += ml[1] * fast_exp2(ml[0] - ms);
            }
        sm[1][row][p] = l;
        __syncthreads();
        if (p == 0) {
            l = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) l += sm[1][row][i];
            fin[row][0] = ms;
            fin[row][1] = inverse_sum(m, l);
        }
        __syncthreads();
        if (mine < len) {
            if (rt > 0) load_raw(rt);
#pragma unroll
            for (int q = 0; q < 32; ++q)
                if (q < rows) weight += fast_exp2(raw[q] - fin[q][0]) * fin[q][1];
        }
    }
    if (mine < len) *account = score + weight;
}

// ---------------------------------------------------------------- host
// whether the matrix cores' form takes such a cache (and queries q, which it also reads 16 bytes at a time)
bool takes_mfma(const moa_kv_cache_t &c, const void *q)
{
    return c.dtype == MOA_BF16 && kv_rows16(c, {q});
}

DecodePlan plan_of(const moa_kv_cache_t &c, int H, bool accounts, bool mfma)
{
    return decode_plan(c.B, c.n_kv_heads, c.head_dim, c.max_pages * c.page_size, H, accounts, mfma, c.dtype == MOA_F32 && kv_rows16(c, {}));
}

// enough for either form, and for accounts where the cache keeps them
size_t workspace_bytes(const moa_kv_cache_t &c, int H)
{
    size_t most = 0;
    for (const bool mfma : {false, takes_mfma(c, nullptr)})
        for (const bool accounts : {false, c.score != nullptr}) {
            const size_t n = plan_of(c, H, accounts, mfma).total();
            if (n > most) most = n;
        }
    return most;
}

template <typename T, int LPR, int HG, bool WIDE>
hipError_t launch_one(const DecodeArgs &a, int grid, hipStream_t st)
{
    const size_t lds = ((size_t)WAVES * HG * (a.c.dh + 2) + HG * 2) * 4;
    prof_begin(K_DECODE_ATTN, st);
    MOA_KLAUNCH((k_decode_attn<T, LPR, HG, WIDE>), dim3(grid), dim3(64 * WAVES), lds, st, a);
    prof_end(st);
    return hipGetLastError();
}

template <int DH, int CT, bool PAD, bool ACC>
hipError_t launch_mfma(const DecodeArgs &a, int grid, hipStream_t st)
{
    constexpr size_t lds = (size_t)WAVES * decode_wave_bytes(DH, CT, ACC);
    static bool raised[16] = {};
    hipError_t e = raise_lds_limit_once(raised, (const void *)k_decode_attn_mfma<DH, CT, PAD, ACC>, lds);
    if (e != hipSuccess) return e;
    prof_begin(K_DECODE_ATTN_MFMA, st);
    MOA_KLAUNCH((k_decode_attn_mfma<DH, CT, PAD, ACC>), dim3(grid), dim3(64 * WAVES), lds, st, a);
    prof_end(st);
    return hipGetLastError();
}

template <int DH, int CT>
hipError_t launch_mfma(const DecodeArgs &a, int grid, hipStream_t st)
{
    if (a.c.dh == DH) return a.raw ? launch_mfma<DH, CT, false, true>(a, grid, st) : launch_mfma<DH, CT, false, false>(a, grid, st);
    return a.raw ? launch_mfma<DH, CT, true, true>(a, grid, st) : launch_mfma<DH, CT, true, false>(a, grid, st);
}

template <int DH>
hipError_t launch_mfma(const DecodeArgs &a, int grid, hipStream_t st)
{
    if constexpr (DH <= 128)
        if (a.HG > 16) return launch_mfma<DH, 2>(a, grid, st);
    return launch_mfma<DH, 1>(a, grid, st);
}

template <typename T, int HG, bool WIDE>
hipError_t launch_rows(const DecodeArgs &a, int grid, hipStream_t st)
{
    constexpr int L1 = 4 * sizeof(T);            // lanes of a row of 64 elements
    return a.c.dh <= 64 ? launch_one<T, L1, HG, WIDE>(a, grid, st) : a.c.dh <= 128 ? launch_one<T, 2 * L1, HG, WIDE>(a, grid, st) : launch_one<T, 4 * L1, HG, WIDE>(a, grid, st);
}

template <typename T>
hipError_t launch_decode(const DecodeArgs &a, bool mfma, bool wide, hipStream_t st)
{
    const int grid = a.runs ? a.runs : a.c.B * a.HB;
    hipError_t e = hipErrorInvalidValue;
    if (mfma) e = a.c.dh <= 64 ? launch_mfma<64>(a, grid, st) : a.c.dh <= 128 ? launch_mfma<128>(a, grid, st) : launch_mfma<256>(a, grid, st);
    else if (!wide) e = launch_rows<T, 2, false>(a, grid, st);
    else if constexpr (sizeof(T) == 4)
        e = a.HG == 2 ? launch_rows<T, 2, true>(a, grid, st) : a.HG == 4 ? launch_rows<T, 4, true>(a, grid, st) : launch_rows<T, 8, true>(a, grid, st);
    if (e != hipSuccess || !a.runs) return e;
    return launch_decode_join(a, sizeof(T) == 2, st);
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

hipError_t launch_decode_join(const DecodeArgs &a, bool bf16, hipStream_t st)
{
    // (a dimension of a launch has less than 2^32 threads)
    const int64_t accounts = a.raw ? (int64_t)a.c.B * a.c.Hkv * ((a.c.cap + ACC_SLOTS - 1) / ACC_SLOTS) : 0;
    const int64_t wide_x = accounts < (1 << 20) ? accounts : 1 << 20, y = accounts > wide_x ? (accounts + wide_x - 1) / wide_x : 1;
    const dim3 grid((unsigned)(a.c.B * a.H + wide_x), (unsigned)y);
    prof_begin(K_DECODE_JOIN, st);
    if (bf16) MOA_KLAUNCH(k_decode_join<bf16_t>, grid, dim3(256), 0, st, a);
    else MOA_KLAUNCH(k_decode_join<float>, grid, dim3(256), 0, st, a);
    prof_end(st);
    return hipGetLastError();
}

}  // namespace moa

using namespace moa;

extern "C" {

int32_t moa_decode_attn_workspace_bytes(const moa_kv_cache_t *cache, int32_t n_q_heads, size_t *bytes_host)
{
    if (!bytes_host) return api_fail(MOA_ERR_NULL, "decode_attn_workspace_bytes: bytes_host is NULL");
    int32_t rc = check_decode(cache, n_q_heads, "decode_attn_workspace_bytes");
    if (rc) return rc;
    *bytes_host = workspace_bytes(*cache, n_q_heads);
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
    const DecodePlan p = plan_of(*cache, n_q_heads, accumulate != 0, takes_mfma(*cache, q));
    const size_t need = workspace_bytes(*cache, n_q_heads);
    if (need && (!ws || (((uintptr_t)ws) & 255) || ws_bytes < need))
        return api_fail(MOA_ERR_WORKSPACE, "decode_attn: workspace NULL, misaligned or smaller than moa_decode_attn_workspace_bytes");
    DecodeArgs a = {KvDev(*cache, dev_status), q, out, n_q_heads, n_q_heads / cache->n_kv_heads, p.HG, p.rtiles, cache->n_kv_heads * p.rtiles,
                    p.runs, p.runs ? 31 - __builtin_clz((unsigned)p.runs) : 0, 1.4426950408889634f / sqrtf((float)cache->head_dim),
                    (float *)ws, (float *)((char *)ws + p.part_o), p.cap32, p.raw ? (float *)((char *)ws + p.part_o + p.part_ml) : nullptr};
    prof_set_site(S_DECODE);
    hipStream_t st = (hipStream_t)stream;
    const hipError_t e = es == 2 ? launch_decode<bf16_t>(a, p.mfma, p.wide, st) : launch_decode<float>(a, false, p.wide, st);
    if (e != hipSuccess) return api_fail(MOA_ERR_HIP, hipGetErrorString(e));
    return MOA_OK;
}

}  // extern "C"
