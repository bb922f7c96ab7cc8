// How the attention of one token is laid out on the chip, from what the host knows: plain arithmetic.
#ifndef ENDOR_ATTN_PLAN_H_
#define ENDOR_ATTN_PLAN_H_

#include <cstddef>
#include <cstdint>

namespace endor_attn_plan {

constexpr int kWaves = 4;       // of a workgroup
constexpr int kTile = 32;       // slots a wave takes at a time: the inner length of the second product's instruction
constexpr int kQueries = 16;    // query heads that share a pass over the keys: the width of an instruction's result
constexpr int kStep = kWaves * kTile;

struct Plan {
    int group;           // query heads of a kv head
    int qtiles;          // passes over the keys of a kv head
    int32_t chunk;       // slots of a workgroup
    int32_t splits;      // workgroups over the longest sequence
    int32_t row;         // logits of a query head kept for the weights: max_len, rounded up to whole tiles
    size_t partial, ml, logits, bytes;  // scratch: sums of the splits, their maxima and totals, logits
};

inline size_t round256(size_t n) { return (n + 255) & ~size_t(255); }

inline Plan make_plan(int batch, int kv_heads, int q_heads, int dim, int32_t max_len, bool with_weights) {
    Plan p{};
    p.group = q_heads / kv_heads;
    p.qtiles = (p.group + kQueries - 1) / kQueries;
    const int64_t units = int64_t(batch) * kv_heads * p.qtiles;
    int64_t chunk = (int64_t(max_len) * units / 1024 + kStep - 1) / kStep * kStep;
    if (chunk < 2 * kStep) chunk = 2 * kStep;
    if (chunk > 1024) chunk = 1024;
    p.chunk = static_cast<int32_t>(chunk);
    p.splits = static_cast<int32_t>((int64_t(max_len) + p.chunk - 1) / p.chunk);
    if (p.splits < 1) p.splits = 1;
    p.row = static_cast<int32_t>((int64_t(max_len) + kTile - 1) / kTile * kTile);
    const size_t rows = size_t(batch) * q_heads;
    p.partial = p.splits > 1 ? round256(rows * p.splits * dim * 4) : 0;
    p.ml = p.splits > 1 || with_weights ? round256(rows * p.splits * 8) : 0;
    p.logits = with_weights ? round256(rows * p.row * 4) : 0;
    p.bytes = p.partial + p.ml + p.logits;
    return p;
}

}  // namespace endor_attn_plan

#endif  // ENDOR_ATTN_PLAN_H_
