// Which form the attention of one token per sequence takes (moa_decode_attn.hip) and what workspace it needs.  Host arithmetic only,
// so that a test on a machine without a GPU can go through it.
#pragma once
#include <stddef.h>
#include <stdint.h>

namespace moa {

constexpr int TK = 128;                // keys of a tile

struct DecodePlan {
    bool mfma, wide;                   // on the matrix cores; element by element, rows read 16 bytes at a time
    int HG, rtiles, runs, cap32;       // query heads in a tile; tiles per KV head; workgroups, 0: one per pair; capacity in whole blocks of 32
    size_t part_o, part_ml, raw;       // bytes
    size_t total() const { return part_o + part_ml + raw; }
};

// mfma: rows and queries are bf16 and can be read 16 bytes at a time; wide: rows are single precision and can be.
// The host knows the capacity, not the lengths, so that short sequences in a wide table get the form that long ones want.  Us, in a
// capacity of their length against one of 65536: 32 heads on one KV head, 1 x 8000 keys 8.4 + 5.9, 12.5 + 6.1; 8b heads, 1 x 400 9.2, 6.3 +
// 4.3; 64 x 1000 in 1024 42.0, in 32768 42.1 + 4.0.
inline DecodePlan decode_plan(int B, int Hkv, int dh, int cap, int H, bool accounts, bool mfma, bool wide)
{
    auto align256 = [](size_t n) { return (n + 255) & ~(size_t)255; };
    DecodePlan p;
    const int G = H / Hkv;
    p.mfma = mfma;
    p.wide = wide;
    // On the matrix cores 32 query heads share a pass over the keys where there is enough of it, and 16 where more runs are wanted (or,
    // beyond 128 dims, two tiles of columns do not fit the registers).  32 heads on one KV head, us, 16 a pass against 32: 1 x 8000 keys 8.6, 12.8; 16 x
    // 8000 25.7, 26.0, and with 64 heads 39.4, 33; 64 x 8000 68.5, 45.5; 64 x 32000 312, 168.
    const int most = dh <= 128 && (int64_t)B * Hkv * ((cap + TK - 1) / TK) >= 512 ? 32 : 16;
    p.HG = p.mfma ? (G < most ? G : most) : G <= 2 || !p.wide ? 2 : G <= 4 ? 4 : 8;
    p.rtiles = (G + p.HG - 1) / p.HG;
    const int64_t pairs = (int64_t)B * Hkv * p.rtiles;
    // One workgroup per pair, without a second launch (4 us), where that is a short walk, or not a long one and there are pairs
    // enough for two workgroups a compute unit.  Else two runs per compute unit on the matrix cores, four element by element.
    // Measured, us, per pair against runs + join, 8b heads: 1 x 512 tokens 8.7, 6.9 + 4.0; 1 x 1024 12.5, 5.8 + 4.1; 64 x 1024
    // 38.9, 40.7 + 6.4; 64 x 17 .. 2048 55.3, 50.6 + 7.3.  Single precision: 1 x 256 11.4, 8.2 + 4.1; 1 x 512 19.3, 8.8 + 4.2.
    // Half and twice as many runs: 64 ragged sequences up to 8192 181 and 176 against 173, 8 x 32768 158 and 164 against 158; single
    // precision 4 x 32000 28.1 and 27.3 against 23.7.
    const int64_t walk = p.mfma ? pairs >= 512 ? 1024 : 512 : 256;
    p.runs = cap <= walk && !(accounts && p.rtiles > 1) ? 0 : !p.mfma ? 1024 : dh <= 128 && p.HG <= 16 ? 512 : 256;
    p.part_o = p.runs ? align256((size_t)(p.runs + pairs) * p.HG * dh * 4) : 0;
    p.part_ml = p.runs ? align256((size_t)(p.runs + pairs) * p.HG * 2 * 4) : 0;
    p.cap32 = (cap + 31) & ~31;
    p.raw = accounts ? align256((size_t)pairs * p.cap32 * p.HG * 4) : 0;
    return p;
}

}  // namespace moa
