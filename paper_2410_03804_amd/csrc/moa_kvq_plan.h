// Which form the attention of one token per sequence over a cache held in 8 bits takes (moa_kvq_decode.hip) and what workspace it
// needs.  Host arithmetic only, so that a test on a machine without a GPU can go through it.
#pragma once
#include "moa_decode_plan.h"

namespace moa {

constexpr int KVQ_JOINS = 512;         // workgroups that the second launch is to have

struct KvqPlan {
    bool mfma;                         // on the matrix cores, else element by element
    int HG, rtiles, runs;              // query heads in a tile; tiles per KV head; workgroups, 0: one per pair
    int per, chunks;                   // of the second launch behind the matrix cores' runs: query heads of a workgroup, such workgroups of a pair
    size_t part_o, part_ml;            // bytes
    size_t total() const { return part_o + part_ml; }
};

// mfma: rows of codes and queries can be read 16 bytes at a time.
// One workgroup of four wavefronts per pair, without a second launch (5 us), where that is a short walk, or not a long one and there are pairs
// enough.  Else 2048 runs of a wavefront each, eight a compute unit, on the matrix cores (at 256 dims 1024, whose registers fit once a
// SIMD), 1024 of four wavefronts element by element.  Measured, us, 8b heads: per pair 1 x 300 7.3, 1 x 512 9.5, 64 x 500 14.9, 64 x 1000
// 24.9; runs + join 1 x 1084 6.2 + 5.9, 1 x 2000 5.1 + 5.2.  4096 and 8192 runs: 8 x 32768 with 64 heads 98 and 105 against 92, 64 ragged
// sequences up to 8192 105 and 112 against 105.
inline KvqPlan kvq_plan(int B, int Hkv, int dh, int cap, int H, bool mfma)
{
    auto align256 = [](size_t n) { return (n + 255) & ~(size_t)255; };
    KvqPlan p;
    const int G = H / Hkv, most = mfma ? 16 : 4;
    p.mfma = mfma;
    p.HG = G < most ? G : most;
    p.rtiles = (G + p.HG - 1) / p.HG;
    const int64_t pairs = (int64_t)B * Hkv * p.rtiles;
    const int64_t walk = pairs >= 512 ? 1024 : 512;
    p.runs = cap <= walk ? 0 : !mfma ? 1024 : dh <= 128 ? 2048 : 1024;
    p.part_o = p.runs ? align256((size_t)(p.runs + pairs) * p.HG * dh * 4) : 0;
    p.part_ml = p.runs ? align256((size_t)(p.runs + pairs) * p.HG * 2 * 4) : 0;
    // As many heads a workgroup as leave 512 of them, where there are so many.
    const int64_t heads = pairs * p.HG / KVQ_JOINS;
    p.per = heads < 1 ? 1 : heads < p.HG ? (int)heads : p.HG;
    p.chunks = (p.HG + p.per - 1) / p.per;
    return p;
}

}  // namespace moa
