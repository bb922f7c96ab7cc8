// How the decode side lays its work out (endor_attn_plan.h, endor_q4_plan.h), checked on the host over sizes of every kind.  Built and run by
// tests/test_decode_plan.py; not part of the library.
#include <cstdint>
#include <cstdio>

#include "endor_attn_plan.h"
#include "endor_q4_plan.h"

static uint64_t state = 0x243F6A8885A308D3ull;
static uint64_t rnd() {
    state ^= state << 13;
    state ^= state >> 7;
    state ^= state << 17;
    return state;
}
static int64_t size(int bits) {  // spread over its logarithm
    const int b = static_cast<int>(rnd() % (bits + 1));
    return 1 + static_cast<int64_t>(rnd() % (uint64_t(1) << b));
}

// The parts of a sequence, as the kernels cut it.
static int64_t parts(int64_t length, int64_t chunk) { return (length + chunk - 1) / chunk; }

static const char *check_attn(int batch, int kv, int group, int dim, int32_t most, bool weights) {
    using namespace endor_attn_plan;
    const Plan p = make_plan(batch, kv, kv * group, dim, most, weights);
    if (p.group != group || p.qtiles != (group + 15) / 16 || int64_t(p.units) != int64_t(kv) * p.qtiles) return "units";
    if (p.row < most || p.row % 64) return "a row of logits";
    const int queries = group < 16 ? group : 16, wide = dim <= 64 ? 64 : dim <= 128 ? 128 : 256, waves = p.splits ? p.waves : wide == 256 ? 4 : 8;
    const size_t lds = size_t(queries) * waves * (wide + 2) * 4 + (p.splits ? 0 : 16 * 4 + (weights ? size_t(queries) * p.row * 4 : 0));
    if (lds > (160u << 10)) return "more LDS than there is";
    if (p.splits == 0) return p.bytes ? "scratch for one launch" : weights && p.qtiles > 1 ? "two workgroups add to the same weights" : nullptr;
    if (p.splits < 1 || p.splits > 65535) return "parts";
    if (p.chunk < p.least || p.least < 64 || p.chunk % 64 || p.least % 64 || p.even < 1) return "slots of a part";
    const size_t rows = size_t(batch) * kv * group;
    if (p.splits > 1 && p.partial < rows * p.splits * dim * 4) return "room for sums";
    if (p.ml < rows * p.splits * 8 || (weights && p.logits < rows * p.row * 4) || p.bytes != p.partial + p.ml + p.logits) return "room";
    // a sequence never has more parts than the grid: lengths alike and not
    for (int i = 0; i < 8; ++i) {
        const int64_t longest = i ? 1 + static_cast<int64_t>(rnd() % most) : most, length = i & 1 ? longest : 1 + static_cast<int64_t>(rnd() % longest);
        int64_t chunk = ((longest + p.even - 1) / p.even + 63) / 64 * 64;
        if (chunk < p.least) chunk = p.least;
        if (parts(length, chunk) > p.splits) return "more parts of like lengths than workgroups";
        if (batch > 1 && parts(length, p.chunk) > p.splits) return "more parts than workgroups";
    }
    // scratch for a bound serves the lower ones
    for (int i = 0; i < 8; ++i) {
        const int32_t lower = static_cast<int32_t>(rnd() % (uint64_t(most) + 1));
        if (make_plan(batch, kv, kv * group, dim, lower, weights).bytes > p.bytes) return "a lower bound takes more scratch";
        if (make_plan(batch, kv, kv * group, dim, most, false).bytes > p.bytes) return "no weights take more scratch";
    }
    return nullptr;
}

static const char *check_q4(uint32_t tiles, uint32_t blocks, uint32_t nb, int group) {
    using namespace endor_q4_plan;
    const Plan p = make_plan(tiles, blocks, nb, group);
    if (p.splits < 1 || p.splits > 65535 || uint64_t(p.splits) * p.per_split < blocks) return "columns left out";
    if (uint64_t(p.splits - 1) * p.per_split >= blocks) return "a part without columns";
    if (p.tiles == 0) {
        if (p.waves != 4 && p.waves != 8 && p.waves != 16) return "waves";
        if (p.depth != 1 && (p.depth != 2 || group == 32)) return "depth";
        if (x_bytes(p.per_split, nb) > (128u << 10)) return "x takes more LDS than it may";
        if (size_t(p.waves) * nb * 64 > (160u << 10)) return "sums take more LDS than there is";
    } else {
        if (p.tiles < 1 || p.tiles > (group == 32 ? 5 : 7)) return "tiles";
        if (p.waves != 4 && p.waves != 8) return "waves";
        if (size_t(p.waves) * nb * p.tiles * 64 > (160u << 10)) return "sums take more LDS than there is";
    }
    return nullptr;
}

int main() {
    for (int i = 0; i < 200000; ++i) {
        const int batch = static_cast<int>(size(i % 3 ? 7 : 16)), kv = static_cast<int>(size(7)), group = static_cast<int>(size(6)), dim = 8 * static_cast<int>(1 + rnd() % 32);
        const int32_t most = static_cast<int32_t>(size(i % 5 ? 17 : 30));
        if (const char *what = check_attn(batch > 65535 ? 65535 : batch, kv, group, dim, most, rnd() & 1)) {
            std::printf("attention of %d x %d x %d heads of %d, %d slots: %s\n", batch, kv, group, dim, most, what);
            return 1;
        }
    }
    for (int i = 0; i < 200000; ++i) {
        const uint32_t tiles = static_cast<uint32_t>(size(20)), blocks = static_cast<uint32_t>(size(18)), nb = 1 + rnd() % 16;
        const int group = 32 << rnd() % 4;
        if (const char *what = check_q4(tiles, blocks, nb, group)) {
            std::printf("4-bit product of %u row tiles and %u blocks, %u right-hand sides: %s\n", tiles, blocks, nb, what);
            return 1;
        }
    }
    std::printf("ok\n");
    return 0;
}
