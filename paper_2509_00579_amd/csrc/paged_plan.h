// How work over the paged cache is dealt to workgroups: plain arithmetic without HIP types, so that it also compiles (and is
// checked) on the CPU.
#pragma once

#include <stdint.h>

#ifdef __HIPCC__
#define KVC_BOTH __host__ __device__ __forceinline__
#else
#define KVC_BOTH inline
#endif

namespace kvc {

constexpr int kPBT = 64;  // tokens of a block and page

// `total` units dealt evenly, in order, to `ways` owners: the first total % ways get one more.
struct Deal {
    uint32_t each, more;
    KVC_BOTH Deal(uint32_t total, uint32_t ways) : each(total / ways), more(total - each * ways) {}
    KVC_BOTH uint32_t begin(uint32_t w) const { return each * w + (w < more ? w : more); }
    KVC_BOTH uint32_t owner(uint32_t unit) const {
        const uint32_t longer = more * (each + 1);
        return unit < longer ? unit / (each + 1) : more + (unit - longer) / each;  // each = 0: every unit is in the first part
    }
};

// Division of numbers below 2^31 by one that the host knows: m is 2^(31 + s) / d rounded up, s the bits of d - 1, so m has 32 bits and is
// too large by less than 2^s / 2^(31 + s) of itself.  (A division by a number in a register is some twenty instructions one after the other.)
struct Divide {
    uint32_t m, shift;
    Divide() = default;
    KVC_BOTH explicit Divide(uint32_t d) : m(0), shift(31) {
        while ((1ull << (shift - 31)) < d) shift++;
        m = (uint32_t)(((1ull << shift) + d - 1) / d);
    }
    KVC_BOTH uint32_t of(uint32_t n) const { return (uint32_t)(((uint64_t)n * m) >> shift); }
};

// Tiles of 64 tokens that query rows at positions len - q_len .. len - 1 have to look at: from `first`, `count` of them.
struct TileRange {
    int first, count;
};
KVC_BOTH TileRange tiles_of(int len, int q_len, int window) {
    TileRange r;
    const int low = len - q_len + 1 - window;  // the first key that the first row sees
    r.first = window > 0 && low > 0 ? low / kPBT : 0;
    r.count = (len + kPBT - 1) / kPBT - r.first;
    return r;
}

}  // namespace kvc
