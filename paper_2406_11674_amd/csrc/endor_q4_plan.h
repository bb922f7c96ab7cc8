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

inline Plan make_plan(uint32_t tiles, uint32_t blocks, uint32_t nb, int group) {
    Plan p{};
    // Few row tiles leave compute units empty: the columns are split over several workgroups, where that saves more
    // than the second launch that adds them up costs (2.5 us). A block takes a workgroup some 0.04 us with x in LDS,
    // 0.1 otherwise. (1024 x 28672 with two right-hand sides 11.5 us, split 8.3; 2048 x 20000 with four 18 and 10.)
    p.splits = 1;
    if (tiles <= 128) {
        uint32_t most = 256 / tiles;
        if (most > blocks / 32) most = blocks / 32;
        const bool in_lds = x_bytes(blocks, nb) <= (128u << 10);
        if (most > 1 && (in_lds ? 1 : 2) * (blocks - blocks / most) > 80) p.splits = most;
    }
    p.per_split = (blocks + p.splits - 1) / p.splits;
    p.splits = (blocks + p.per_split - 1) / p.per_split;
    // x in LDS is read from L2 once and costs a workgroup the wait for it; from the caches it is read for every
    // workgroup's row tiles, and these share it. Measured, microseconds in LDS | from the caches, fp16, groups of 128:
    // 8192 x 8192 with three right-hand sides 9.6 | 10.2, with four 10.5 | 10.1; 28672 x 8192 with one 21.7 | 23.0, with
    // two 23.2 | 23.0; 28672 x 2048 with four 10.1 | 8.4; 60000 x 1200 with three 11.8 | 12.3, with six 14.8 | 12.7.
    const size_t x = x_bytes(p.per_split, nb);
    const uint32_t groups = tiles * p.splits;
    const size_t in_lds = groups <= 256   ? 128u << 10
                          : groups <= 512 ? (nb <= 2 ? 128u : 48u) << 10
                                          : (nb <= 1 ? 64u : 10u) << 10;
    if (x <= in_lds) {
        // Workgroups that fit on the chip at once have as many waves as they can, of more and shorter ones each CU takes
        // several: 28672 x 4096 in eight waves 13.4 us, in four 12.6; 28672 x 8192 21.7 and 22.4.
        p.waves = groups <= 512 ? 16 : groups <= 1024 || p.per_split > 40 ? 8 : 4;
        while (p.waves > 4 && p.waves > p.per_split) p.waves /= 2;
        // (the scales of groups of 32 leave no registers for a second block: 8192 x 8192 15.9 us, 12.3 with one)
        p.depth = group > 32 && p.per_split >= 4 * p.waves ? 2 : 1;
        return p;
    }
    // As many row tiles for a workgroup as give every compute unit one, or two smaller ones, in as few rounds as a
    // wave's registers allow: 12000 x 8192 (750 tiles, 16 right-hand sides) in threes 14.4 us, twos 23.7, fours 15.9;
    // 28672 x 8192 (1792) in sevens 23.8, fours 28.1; 40000 x 4096 (2500) in fives of four waves 19.1, of eight 20.4.
    const uint32_t most = group == 32 ? 5 : 7;
    p.waves = groups <= 256 * most ? 8 : 4;
    const uint32_t places = 256 * (8 / p.waves), rounds = (groups - 1) / (places * most) + 1;
    p.tiles = static_cast<int>((groups - 1) / (places * rounds) + 1);
    p.depth = 1;
    return p;
}

}  // namespace endor_q4_plan

#endif  // ENDOR_Q4_PLAN_H_
