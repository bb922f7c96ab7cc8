// How the attention of one token is laid out on the chip, from what the host knows: plain arithmetic.
#ifndef ENDOR_ATTN_PLAN_H_
#define ENDOR_ATTN_PLAN_H_

#include <cstddef>
#include <cstdint>

namespace endor_attn_plan {

constexpr int kQueries = 16;  // query heads that share a pass over the keys: the width of an instruction's result

struct Plan {
    int group;           // query heads of a kv head
    int qtiles;          // passes over the keys of a kv head
    uint32_t units;      // of a sequence: kv_heads * qtiles
    int32_t row;         // logits of a query head: max_len, rounded up to whole tiles
    int waves;           // of a workgroup
    int32_t least;       // slots of a part of a sequence at least,
    int32_t chunk;       // at most where the lengths differ,
    int32_t even;        // and parts where they are alike: which it is the device sees
    uint32_t heads;      // query heads that a workgroup joins
    int32_t splits;      // parts of the longest sequence; 0: a workgroup for every unit, and no scratch
    size_t partial, ml, logits, bytes;  // scratch: sums of parts of units, their maxima and totals, logits
};

inline size_t round256(size_t n) { return (n + 255) & ~size_t(255); }

inline Plan make_plan(int batch, int kv_heads, int q_heads, int dim, int32_t max_len, bool with_weights) {
    Plan p{};
    p.group = q_heads / kv_heads;
    p.qtiles = (p.group + kQueries - 1) / kQueries;
    p.units = static_cast<uint32_t>(kv_heads) * p.qtiles;
    p.row = static_cast<int32_t>((int64_t(max_len) + 63) / 64 * 64);
    const int64_t units = int64_t(batch) * p.units;
    if (units == 0) return p;  // no sequences
    // One launch where a compute unit reads its share in about the time of the second one (1024 slots of one head of
    // 64, or 512 of 128: 8.6 us in one launch, 8.8 in two; 1024 of 128 17.8 and 10.8), or where the units fill half of
    // the chip by themselves (256 of 1000 slots: 24.7 and 29.5).
    if (max_len <= 1024 && units <= 512 && (int64_t(max_len) * dim <= 65536 || units >= 128) && (p.qtiles == 1 || !with_weights)) return p;
    // Where four waves to a compute unit would have less than two tiles each, two of them.
    p.waves = int64_t(max_len) * units >= 256 * 256 ? 4 : 2;
    p.least = 64 * p.waves;
    // Sequences of like lengths are cut where that fills the chip more evenly than it costs: the compute units with the
    // most workgroups take `turns` of them, each the time that 40 KB/us take for its slots and some 1.5 us to begin and
    // to join. (19 sequences of 4001 slots, 8 heads of 64: uncut 43.7 us, in three 34.8, in five 34.1; 8 of 2048, 72
    // heads of 128: 118, in two 111; 64 of 2048, 8 heads of 64: 49.5, in two 54; one of 131072, 8 heads of 128: in 32
    // 87, in 27 92, in 128 98.)
    constexpr int64_t kMostGroups = 1536;
    const double uncut = static_cast<double>(max_len) * dim * 4 / 40e3;
    double least_time = 0;
    p.even = 1;
    for (int64_t turns = (units + 255) / 256; turns * 256 <= kMostGroups; ++turns) {
        const int64_t parts = 256 * turns / units;
        const double time = static_cast<double>(turns) * (uncut / static_cast<double>(parts) + 1.5);
        if (least_time > 0 && time >= least_time) continue;
        least_time = time;
        p.even = static_cast<int32_t>(parts);
    }
    // Others: workgroups that have no part hold up others, and a part costs what its start and its join take: some six
    // workgroups for every compute unit (of widest heads one, for the registers of one fill it), and four tiles of 64
    // slots or more for two waves.
    const int64_t groups = dim <= 128 ? kMostGroups : 256;
    int64_t chunk = ((int64_t(max_len) * units + groups - 1) / groups + 63) / 64 * 64;
    if (chunk > p.row) chunk = p.row;
    if (chunk < 2 * p.least) chunk = 2 * p.least;
    while ((int64_t(max_len) + chunk - 1) / chunk > 65535) chunk *= 2;  // a grid's third dimension
    p.chunk = static_cast<int32_t>(chunk);
    p.splits = batch > 1 ? static_cast<int32_t>((int64_t(max_len) + chunk - 1) / chunk) : 1;
    if (p.splits < p.even) p.splits = p.even;
    const int64_t most = (int64_t(max_len) + p.least - 1) / p.least;
    if (p.splits > most) p.splits = static_cast<int32_t>(most);
    if (p.splits < 1) p.splits = 1;
    p.heads = p.splits <= 16 ? 8 : 1;
    // Scratch is what the largest plan up to max_len takes, so that scratch for a bound serves every lower one too.
    const int64_t ceiling = (kMostGroups + units - 1) / units;
    int64_t parts = (int64_t(max_len) + 127) / 128;
    if (parts > ceiling) parts = ceiling;
    const size_t rows = size_t(batch) * q_heads;
    p.partial = parts > 1 ? round256(rows * parts * dim * 4) : 0;
    p.ml = round256(rows * parts * 8);
    p.logits = with_weights ? round256(rows * p.row * 4) : 0;
    p.bytes = p.partial + p.ml + p.logits;
    return p;
}

}  // namespace endor_attn_plan

#endif  // ENDOR_ATTN_PLAN_H_
