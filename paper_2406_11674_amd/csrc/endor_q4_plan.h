// How a product with a 4-bit weight is laid out on the chip: plain arithmetic on its sizes.
#ifndef ENDOR_Q4_PLAN_H_
#define ENDOR_Q4_PLAN_H_

#include <cstddef>
#include <cstdint>

namespace endor_q4_plan {

struct Plan {
    int tiles;           // row tiles of a workgroup whose x comes from the caches; 0: one row tile, and x in LDS
    uint32_t waves;      // of a workgroup
    int depth;           // blocks a wave has on their way (x in LDS)
    uint32_t splits;     // parts of the columns, a workgroup each
    uint32_t per_split;  // blocks of one
};

// Bytes of x in LDS: blocks of 128 columns of 16 bits.
inline size_t x_bytes(uint32_t blocks, uint32_t nb) { return size_t(blocks) * 256 * nb; }

inline Plan make_plan(uint32_t tiles, uint32_t blocks, uint32_t nb) {
    Plan p{};
    // Few row tiles leave compute units empty: the columns are split over several workgroups, where that saves more
    // than the second launch that adds them up costs (2.5 us). A block takes a workgroup some 0.04 us with x in LDS,
    // 0.1 otherwise.
    p.splits = 1;
    if (tiles <= 128) {
        uint32_t most = 256 / tiles;
        if (most > blocks / 32) most = blocks / 32;
        const bool in_lds = x_bytes(blocks, nb) <= (128u << 10);
        if (most > 1 && (in_lds ? 1 : 2) * (blocks - blocks / most) > 80) p.splits = most;
    }
    p.per_split = (blocks + p.splits - 1) / p.splits;
    p.splits = (blocks + p.per_split - 1) / p.per_split;
    const size_t x = x_bytes(p.per_split, nb);
    const uint32_t groups = tiles * p.splits;
    if (groups <= 256 ? x <= (128u << 10) : x <= (nb <= 2 ? 64u << 10 : nb <= 4 ? 32u << 10 : 0)) {
        p.waves = groups <= 512 ? 16 : 8;
        while (p.waves > 4 && p.waves > p.per_split) p.waves /= 2;
        p.depth = p.per_split >= 4 * p.waves ? 2 : 1;
        return p;
    }
    p.tiles = groups >= 800 ? 4 : groups > 256 ? 2 : 1;
    p.waves = p.tiles == 4 && groups >= 1600 ? 4 : 8;
    p.depth = 1;
    return p;
}

}  // namespace endor_q4_plan

#endif  // ENDOR_Q4_PLAN_H_
