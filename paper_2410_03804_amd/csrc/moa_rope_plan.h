// Which form the norm and rotation of queries and keys takes (moa_qk_norm_rope.hip).  Host arithmetic only, so that a test on a machine
// without a GPU can go through it.
#pragma once
#include <stdint.h>

#include <initializer_list>

namespace moa {

struct RopePlan {
    int words, lanes, tokens;          // of a piece, 0: element by element; of a head; of a workgroup
    bool apart;                        // queries and keys in workgroups of their own
};

// size: of an element; addresses, strides (in elements): the bits of all of them; heads: of queries or keys, whichever are more
inline RopePlan rope_plan(int size, int dh, int half, uint64_t addresses, uint64_t strides, int64_t T, int heads)
{
    // pieces of 16 bytes, else of 8 (16145 tokens of 8 heads of 80 dims, 40 of them rotated: 44 us in the kernel for any sizes, 18 so)
    for (const int words : {4, 2}) {
        const int elems = 4 * words / size;
        if (dh % (2 * elems) || half % elems || (addresses & (uint64_t)(4 * words - 1)) || strides % (uint64_t)elems) continue;
        int lanes = 4;
        while (lanes < dh / (2 * elems)) lanes *= 2;
        // Four tokens a workgroup where there are many, so that its threads' angles are one each; sixteen where four have too few heads for its
        // threads (16000 tokens of 8 heads of 80 dims: 20.0 us and 14.6; 8192 of 40 of 128 31.0 and 36.0).  Of few, one, queries and keys apart (16: 7.5 us
        // one behind the other, 4.9).  40 heads, one token a workgroup against four: 512 tokens 6.4 us and 8.6, 1024 10.3 and 8.9, 1536 14.5 and 10.4.
        const bool many = T >= 1024, few = T >= 4096 && (int64_t)heads * 4 * lanes < 512;
        return {words, lanes, few ? 16 : many ? 4 : 1, !many};
    }
    return {0, 64, 1, false};
}

}  // namespace moa
