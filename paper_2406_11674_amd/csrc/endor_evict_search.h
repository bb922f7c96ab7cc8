// Which tokens an eviction keeps: the search for the key of the last one, apart from the kernel so that it can be run on
// the host against a sort. A pass over the keys counts them; what follows from the counts is plain arithmetic.
#ifndef ENDOR_EVICT_SEARCH_H_
#define ENDOR_EVICT_SEARCH_H_

#include <cstdint>

namespace endor_evict_search {

constexpr int kBinBits = 11, kBins = 1 << kBinBits;  // of a pass over the keys
constexpr uint32_t kFew = 64;                        // keys that a wave ranks among each other

// Keys in question: those in [low, high]; the `need` largest of them stay, and all above high do.
struct Range {
    uint32_t low, high, need;
    constexpr bool holds(uint32_t key) const { return key - low <= high - low; }
    // A bin of a pass: 2^shift keys, the first from low on.
    constexpr uint32_t shift() const {
        const uint32_t range = high - low;
        return range >> kBinBits ? 32 - __builtin_clz(range) - kBinBits : 0;
    }
    constexpr uint32_t bin_of(uint32_t key, uint32_t bits) const { return (key - low) >> bits; }
    // From now on the keys of one bin. The topmost bin may reach past high, where keys lie that have been counted as kept:
    // the upper end stays below them.
    constexpr void take_bin(uint32_t bin, uint32_t bits) {
        low += bin << bits;
        const uint32_t top = low + ((1u << bits) - 1);  // keys are at most those of infinity: no overflow
        high = top < high ? top : high;
    }
};

// The last that stay: keys above `key`, and of those equal to it the first `ties` in the order of slots.
struct Last {
    uint32_t key, ties;
};
struct Bin {
    uint32_t at, above, in;  // the bin that the last kept key is in, the keys in higher ones, the keys in it
};

// The last key of r.need in the range; P does what takes a pass over the keys:
//   Bin count(const Range &, bits)    of bins of 2^bits keys the one that holds the last key to stay
//   Last rank(const Range &, count)   of the keys in the range, that many and at most kFew
//   void ends(Range *)                narrows the range to the least and the largest key in it
// Many keys in one of so many bins are often one and the same: the bin's own ends are looked for where it holds more than
// `many`.
template <class P>
constexpr Last last_to_stay(Range r, uint32_t many, P &&passes) {
    for (;;) {
        const uint32_t bits = r.shift();
        const Bin bin = passes.count(r, bits);
        r.take_bin(bin.at, bits);
        r.need -= bin.above;
        if (bits == 0) return {r.low, r.need};
        if (r.need == bin.in) return {r.low, 0xffffffffu};  // all of the bin stay: those from its lower end on
        if (bin.in <= kFew) return passes.rank(r, bin.in);
        if (bin.in < many) continue;
        passes.ends(&r);
        if (r.low == r.high) return {r.low, r.need};
    }
}

}  // namespace endor_evict_search

#endif  // ENDOR_EVICT_SEARCH_H_
