// Products with 4-bit weights that carry a scale, and if wanted a zero point, per row and group of columns.
//
// PACKED FORM. Rows go in tiles of 16, columns in blocks of 128, both padded with codes and scales of zero, so that no
// kernel has an edge in W. Codes: [tile][block][lane 0..63][16 bytes]; lane l has row l & 15 of the tile, and its
// 32-bit word j the columns 32 j + 8 (l >> 4) + 0..7 of the block, the even ones in the lower half and the odd ones in
// the upper, 4 bits each. Then the scales, fp16, for a tile and a block (or a group that holds blocks): [4
// quarters][groups of the block][4 rows], as the lanes of a product's result want them; then, if there are any, the
// zeros, bytes [16 rows][groups of the block], as the lanes of its operand do. A block and a group that holds several
// blocks end at the same column.
#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "endor.h"
#include "endor_device.h"
#include "endor_kv.h"
#include "endor_q4_plan.h"

namespace {

using endor_device::u32x4;
using endor_kv::aligned;
using endor_q4_plan::make_plan;
using endor_q4_plan::Plan;

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

struct Layout {
    int64_t tiles, blocks, groups;  // groups: of a padded row
    size_t codes, scales, zeros, bytes;
};

inline bool sizes_ok(int64_t rows, int64_t cols, int group) {
    return rows >= 0 && cols >= 0 && rows < (int64_t(1) << 26) && cols < (int64_t(1) << 26) && group >= 32 && group <= 32768 &&
           (group & (group - 1)) == 0 && (rows == 0 || cols < ((int64_t(1) << 34) + rows - 1) / rows);
}

inline Layout layout_of(int64_t rows, int64_t cols, int group, bool with_zeros) {
    Layout l;
    l.tiles = (rows + 15) / 16;
    l.blocks = (cols + 127) / 128;
    l.groups = (l.blocks * 128 + group - 1) / group;
    l.codes = size_t(l.tiles) * l.blocks * 1024;
    l.scales = size_t(l.tiles) * l.groups * 32;
    l.zeros = with_zeros ? size_t(l.tiles) * l.groups * 16 : 0;
    l.bytes = (l.codes + l.scales + l.zeros + 255) & ~size_t(255);
    return l;
}

struct PackParams {
    const uint8_t *codes;
    const uint16_t *scales;
    const uint8_t *zeros;
    uint32_t *out_codes;
    uint16_t *out_scales;
    uint8_t *out_zeros;
    int64_t rows, cols, group, groups, tiles, blocks, padded_groups;
};

// Eight columns' codes as a checkpoint has them, column c in bits 4c, with the even columns in the lower half: pairs of
// columns lie 16 bits apart then, where packed 16-bit arithmetic takes them.
__device__ __forceinline__ uint32_t even_below_odd(uint32_t x) {
    auto squeeze = [](uint32_t v) {  // the low halves of four bytes side by side
        v &= 0x0f0f0f0fu;
        v = (v | v >> 4) & 0x00ff00ffu;
        return (v | v >> 8) & 0xffffu;
    };
    return squeeze(x) | squeeze(x >> 4) << 16;
}

// A thread makes a lane's 16 bytes of a block; the first ones of a workgroup the scales and zeros. 28672 x 8192 in groups
// of 64: 242 MB read and written in 67 to 74 us, 3.3 to 3.6 TB/s, half of what a copy reaches: a load takes 16 bytes each of
// 16 rows. Done once for a weight.
__global__ __launch_bounds__(256) void endor_q4_pack_kernel(PackParams P) {
    const int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x, units = P.tiles * P.blocks * 64;
    if (i < units) {
        const uint32_t lane = i & 63;
        const int64_t block = (i >> 6) % P.blocks, row = (i >> 6) / P.blocks * 16 + (lane & 15), pitch = (P.cols + 1) / 2;
        u32x4 words = {0, 0, 0, 0};
        if (row < P.rows) {
            const uint8_t *from = P.codes + row * pitch;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int64_t col = block * 128 + 32 * j + 8 * (lane >> 4);
                uint32_t x = 0;
                if (col + 8 <= P.cols) {
                    typedef uint32_t u32_any __attribute__((aligned(1)));
                    x = *reinterpret_cast<const u32_any *>(from + col / 2);
                } else {
                    for (int64_t c = col; c < P.cols; ++c) x |= ((c & 1 ? from[c / 2] >> 4 : from[c / 2] & 15u)) << (4 * (c - col));  // col is even
                }
                words[j] = even_below_odd(x);
            }
        }
        reinterpret_cast<u32x4 *>(P.out_codes)[i] = words;
    }
    const int64_t entries = P.tiles * P.padded_groups * 16;
    if (i < entries) {
        const int64_t of_tile = 16 * P.padded_groups, tile = i / of_tile, parts = P.group < 128 ? 128 / P.group : 1;
        const int64_t base = i % of_tile / (16 * parts) * parts;  // the first group of the block, or the group
        const int64_t in = i % (16 * parts);
        auto source = [&](int64_t r, int64_t g) { return 16 * tile + r < P.rows && g < P.groups ? (16 * tile + r) * P.groups + g : -1; };
        const int64_t s = source(in / (4 * parts) * 4 + in % 4, base + in / 4 % parts), z = source(in / parts, base + in % parts);
        P.out_scales[i] = s >= 0 ? P.scales[s] : 0;
        if (P.out_zeros) P.out_zeros[i] = z >= 0 ? P.zeros[z] & 15 : 0;
    }
}

typedef u32x4 u32x4_any __attribute__((aligned(2)));

// kLanes lanes for a row's group, eight columns to a lane at a time: a group of up to 512 in one go. The scale is rounded
// to fp16 before the codes are taken, so that they are the nearest to what they stand for. 8192 x 8192 in groups of 128 52 to 56 us,
// 28672 x 8192 of 64 with zeros 199: 595 MB read and written at 3.0 TB/s, less than half of what a copy reaches. Done once for a
// weight.
template <uint32_t kLanes>
__global__ __launch_bounds__(256) void endor_q4_quantize_kernel(const _Float16 *dense, uint32_t first, uint32_t count, int64_t cols, int64_t group,
                                                                uint32_t groups, uint8_t *codes, _Float16 *scales, uint8_t *zeros) {
    const uint32_t i = first + blockIdx.x * (256 / kLanes) + threadIdx.x / kLanes, lane = threadIdx.x % kLanes;
    if (i >= count) return;  // all lanes of a group
    const int64_t row = i / groups, from = (i % groups) * group, to = from + group < cols ? from + group : cols;
    const _Float16 *w = dense + row * cols;
    auto eight = [&](int64_t c) {
        if (c + 8 <= to) return __builtin_bit_cast(f16x8, *reinterpret_cast<const u32x4_any *>(w + c));
        f16x8 x = {0, 0, 0, 0, 0, 0, 0, 0};  // which change neither end
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (c + e < to) x[e] = w[c + e];
        return x;
    };
    const int64_t mine = from + 8 * lane;
    const f16x8 begin = eight(mine);
    float lo = 0, hi = 0;
    for (int64_t c = mine; c < to; c += 8 * kLanes) {
        const f16x8 x = c == mine ? begin : eight(c);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            lo = fminf(lo, x[e]);
            hi = fmaxf(hi, x[e]);
        }
    }
#pragma unroll
    for (int d = kLanes / 2; d; d >>= 1) {
        lo = fminf(lo, __shfl_xor(lo, d));
        hi = fmaxf(hi, __shfl_xor(hi, d));
    }
    const _Float16 scale = static_cast<_Float16>(zeros ? (hi - lo) / 15.0f : fmaxf(hi, -lo) / 7.0f);
    const float s = scale, inverse = s > 0 ? 1.0f / s : 0.0f;
    const float zero = zeros ? fminf(fmaxf(rintf(-lo * inverse), 0.0f), 15.0f) : 8.0f;
    if (lane == 0) {
        scales[i] = scale;
        if (zeros) zeros[i] = static_cast<uint8_t>(zero);
    }
    for (int64_t c = mine; c < to; c += 8 * kLanes) {
        const f16x8 x = c == mine ? begin : eight(c);
        uint32_t word = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (c + e < to) word |= static_cast<uint32_t>(fminf(fmaxf(rintf(float(x[e]) * inverse) + zero, 0.0f), 15.0f)) << (4 * e);
        uint8_t *out = codes + row * ((cols + 1) / 2) + c / 2;  // a group begins at an even column
        if (c + 8 <= to) {
            typedef uint32_t u32_any __attribute__((aligned(1)));
            *reinterpret_cast<u32_any *>(out) = word;
        } else {
            for (int b = 0; c + 2 * b < to; ++b) out[b] = static_cast<uint8_t>(word >> (8 * b));
        }
    }
}

struct Q4Params {
    const uint32_t *codes;
    const _Float16 *scales;
    const uint8_t *zeros;
    const uint16_t *x;
    float *y;
    int64_t rows, cols, ldx;
    float *partial;  // [split][nb][rows], where there are several
    uint32_t tiles, blocks, groups, per_group_shift, nb;  // per_group_shift: blocks of a group, where those are whole
    uint32_t splits, per_split;  // parts of the columns, and blocks of one
};

// Eight codes as pairs of the type's numbers code - zero, which are exact: columns (0, 1), (2, 3), (4, 5), (6, 7).
struct Pairs {  // fp16
    f16x2 near, far;
    uint32_t mask, one;  // kept in registers, so that a pair takes one instruction
    // z: the zero in both halves; -(1024 + z) and -(64 + z), whose last bits stand for 1 and for a sixteenth
    __device__ __forceinline__ explicit Pairs(uint32_t z) : mask(0x000f000fu), one(0x64006400u) {
        near = __builtin_bit_cast(f16x2, z | 0xe400e400u);
        far = __builtin_bit_cast(f16x2, z << 4 | 0xd400d400u);
        asm("" : "+s"(mask));
        asm("" : "+v"(one));
    }
    // A code in the low bits of 0x6400 is the number 1024 + code, in the next four 1024 + 16 code.
    __device__ __forceinline__ void get(uint32_t w, f16x2 p[4]) const {
        const f16x2 sixteenth = {static_cast<_Float16>(0.0625f), static_cast<_Float16>(0.0625f)};
        uint32_t high = mask << 4;
        const uint32_t v = w >> 8;
        p[0] = __builtin_bit_cast(f16x2, (w & mask) | one) + near;
        p[1] = __builtin_elementwise_fma(__builtin_bit_cast(f16x2, (w & high) | one), sixteenth, far);
        p[2] = __builtin_bit_cast(f16x2, (v & mask) | one) + near;
        p[3] = __builtin_elementwise_fma(__builtin_bit_cast(f16x2, (v & high) | one), sixteenth, far);
    }
};
template <bool kBf16, bool kZeros>
struct Operand;  // of a row and group; what it makes of a code, times kUnit, is the number wanted
template <bool kZeros>
struct Operand<false, kZeros> {
    static constexpr float kUnit = 1.0f;
    Pairs pairs;
    __device__ __forceinline__ explicit Operand(uint32_t z) : pairs(z) {}
    __device__ __forceinline__ u32x4 of(uint32_t w) const {
        f16x2 p[4];
        pairs.get(w, p);
        return u32x4{__builtin_bit_cast(uint32_t, p[0]), __builtin_bit_cast(uint32_t, p[1]), __builtin_bit_cast(uint32_t, p[2]), __builtin_bit_cast(uint32_t, p[3])};
    }
};
template <>
struct Operand<true, true> {
    static constexpr float kUnit = 1.0f;
    Pairs pairs;
    __device__ __forceinline__ explicit Operand(uint32_t z) : pairs(z) {}
    __device__ __forceinline__ u32x4 of(uint32_t w) const {
        f16x2 p[4];
        pairs.get(w, p);
        u32x4 out;
#pragma unroll
        for (int i = 0; i < 4; ++i) {  // whole numbers below 16 have their bits in the upper half of a float
            const float x = static_cast<float>(p[i][0]), y = static_cast<float>(p[i][1]);
            out[i] = __builtin_amdgcn_perm(__float_as_uint(y), __float_as_uint(x), 0x07060302u);
        }
        return out;
    }
};
template <>
struct Operand<true, false> {  // code - 8, of which the instruction makes a sixteenth
    static constexpr float kUnit = 16.0f;
    __device__ __forceinline__ explicit Operand(uint32_t) {}
    __device__ __forceinline__ u32x4 of(uint32_t w) const {
        const uint32_t low = w ^ 0x88888888u, high = low >> 4;
        auto pair = [&](uint32_t v, int a) {
            const float x = __builtin_amdgcn_cvt_off_f32_i4(v >> (8 * a)), y = __builtin_amdgcn_cvt_off_f32_i4(v >> (8 * a + 16));
            return __builtin_amdgcn_perm(__float_as_uint(y), __float_as_uint(x), 0x07060302u);
        };
        return u32x4{pair(low, 0), pair(high, 0), pair(low, 1), pair(high, 1)};
    }
};

// Scales of four rows, zeros of one, of a block's groups.
template <int kParts>
using Scales = _Float16 __attribute__((ext_vector_type(4 * kParts)));
template <int kParts>
using Bytes = std::conditional_t<kParts == 4, uint32_t, std::conditional_t<kParts == 2, uint16_t, uint8_t>>;

template <bool kBf16>
__device__ __forceinline__ f32x4 product(u32x4 a, u32x4 b, f32x4 c) {
    if constexpr (kBf16)
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// What a wave has of W on its way: a block of 128 columns of kTiles row tiles, with the scales and zeros of its groups
// (kParts of them).
template <int kTiles, int kParts, bool kZeros>
struct Block {
    u32x4 codes[kTiles];
    Scales<kParts> scales[kTiles];
    Bytes<kParts> zeros[kZeros ? kTiles : 1];

    // Tiles past the last one and blocks past `last` stand for it; what is loaded of them is not used.
    __device__ __forceinline__ void load(const Q4Params &Q, uint32_t tile0, uint32_t wanted, uint32_t last, uint32_t lane) {
        const uint32_t n = lane & 15, g = lane >> 4, block = wanted < last ? wanted : last;
        const uint32_t group = kParts > 1 ? block * kParts : block >> Q.per_group_shift;
#pragma unroll
        for (int r = 0; r < kTiles; ++r) {
            const uint32_t tile = tile0 + r < Q.tiles ? tile0 + r : Q.tiles - 1;
            codes[r] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(Q.codes) + (uint64_t(tile) * Q.blocks + block) * 64 +
                                                  (wanted <= last ? lane : 0));
            const uint64_t at = (uint64_t(tile) * Q.groups + group) * 16;
            scales[r] = *reinterpret_cast<const Scales<kParts> *>(Q.scales + at + 4 * kParts * g);
            if constexpr (kZeros) zeros[r] = *reinterpret_cast<const Bytes<kParts> *>(Q.zeros + at + kParts * n);
        }
    }
};

// total += the block's products with x, the operands of its four instructions.
template <int kTiles, int kParts, bool kZeros, bool kBf16>
__device__ __forceinline__ void add_block(f32x4 (&total)[kTiles], const Block<kTiles, kParts, kZeros> &B, const u32x4 (&x)[4]) {
#pragma unroll
    for (int r = 0; r < kTiles; ++r)
#pragma unroll
        for (int p = 0; p < kParts; ++p) {
            const Operand<kBf16, kZeros> operand(kZeros ? __builtin_amdgcn_perm(0, B.zeros[r], 0x0c000c00u | p << 16 | p) : 0x00080008u);
            f32x4 sum = {0, 0, 0, 0};
#pragma unroll
            for (int j = 4 / kParts * p; j < 4 / kParts * (p + 1); ++j) sum = product<kBf16>(operand.of(B.codes[r][j]), x[j], sum);
#pragma unroll
            for (int i = 0; i < 4; ++i) total[r][i] += sum[i] * (static_cast<float>(B.scales[r][4 * p + i]) * Operand<kBf16, kZeros>::kUnit);
        }
}

// The waves' sums are added in their order; a lane has rows 4g + 0..3 of every tile for the right-hand side of its
// column.
template <int kTiles>
__device__ __forceinline__ void join_waves(const Q4Params &Q, float *s_part, uint32_t tile0, const f32x4 (&total)[kTiles]) {
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6, n = lane & 15, g = lane >> 4;
    if (n < Q.nb)
#pragma unroll
        for (int r = 0; r < kTiles; ++r) *reinterpret_cast<f32x4 *>(s_part + ((wave * Q.nb + n) * kTiles + r) * 16 + 4 * g) = total[r];
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < Q.nb * kTiles * 16; i += blockDim.x) {
        float sum = 0;
        for (uint32_t w = 0; w < waves; ++w) sum += s_part[w * Q.nb * kTiles * 16 + i];
        const uint32_t b = i / (kTiles * 16);
        const int64_t row = int64_t(tile0) * 16 + i % (kTiles * 16);
        if (row < Q.rows) (Q.splits > 1 ? Q.partial + int64_t(blockIdx.y) * Q.nb * Q.rows : Q.y)[b * Q.rows + row] = sum;
    }
}

// Elements c to c + 7 of a vector of x, zeros past the last column.
__device__ __forceinline__ u32x4 columns_of(const uint16_t *x, int64_t c, int64_t cols) {
    if (c + 8 <= cols) return *reinterpret_cast<const u32x4_any *>(x + c);
    u32x4 v = {0, 0, 0, 0};
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (c + e < cols) v[e / 2] |= uint32_t(x[c + e]) << (16 * (e & 1));
    return v;
}

// Few right-hand sides: all of x lies in LDS, in the order of the operands, [block][32 columns][quarter][right-hand
// side][8 columns]. A workgroup has one row tile, its waves take the blocks in turn, kDepth of them on their way. Bound by
// memory: 8192 x 28672 with groups of 128 and one right-hand side 22 to 24 us, 121 MB at 5.0 to 5.5 TB/s; small ones by what comes
// before the first product, 1024 x 8192 5.6 us.
template <int kDepth, int kParts, bool kZeros, bool kBf16>
__global__ __launch_bounds__(1024) void endor_q4_gemv_kernel(Q4Params Q) {
    extern __shared__ u32x4 s_x[];
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6, n = lane & 15, g = lane >> 4;
    const uint32_t first = blockIdx.y * Q.per_split, end = first + Q.per_split < Q.blocks ? first + Q.per_split : Q.blocks;
    const uint32_t units = (end - first) * 16 * Q.nb, column = n < Q.nb ? n : Q.nb - 1;  // columns past the last right-hand side are not stored
    for (uint32_t u = threadIdx.x; u < units; u += blockDim.x)
        s_x[u] = columns_of(Q.x + int64_t(u % Q.nb) * Q.ldx, int64_t(first) * 128 + u / Q.nb * 8, Q.cols);
    Block<1, kParts, kZeros> ring[kDepth];
#pragma unroll
    for (int d = 0; d < kDepth; ++d) ring[d].load(Q, blockIdx.x, first + wave + d * waves, end - 1, lane);
    // a barrier for LDS alone: the blocks on their way are not waited for
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
    f32x4 total[1] = {{0, 0, 0, 0}};
    for (uint32_t block = first + wave; block < end; block += kDepth * waves) {
#pragma unroll
        for (int d = 0; d < kDepth; ++d) {
            const uint32_t at = block + d * waves;
            if (at >= end) break;
            u32x4 x[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) x[j] = s_x[(((at - first) * 4 + j) * 4 + g) * Q.nb + column];
            add_block<1, kParts, kZeros, kBf16>(total, ring[d], x);
            ring[d].load(Q, blockIdx.x, at + kDepth * waves, end - 1, lane);
        }
    }
    __syncthreads();
    join_waves<1>(Q, reinterpret_cast<float *>(s_x), blockIdx.x, total);
}

// More right-hand sides: x comes from the caches, once for kTiles row tiles. Bound by memory and by the vector ALUs
// together, which make numbers of codes (9 instructions for 8 codes of fp16, 13 or 21 of bf16) and scale the sums: 28672 x
// 8192 with 16 right-hand sides, groups of 64 and zeros 25 to 27 us, 131 MB at 4.9 to 5.2 TB/s; bf16 with groups of 32 42. A second
// block on its way takes as long or longer (8192 x 8192 12.5 us, 13.8 with two), so it is not latency that it waits for.
template <int kTiles, int kParts, bool kZeros, bool kBf16>
__global__ __launch_bounds__(512) void endor_q4_gemm_kernel(Q4Params Q) {
    extern __shared__ float s_part[];
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6, n = lane & 15, g = lane >> 4;
    const uint32_t first = blockIdx.y * Q.per_split, end = first + Q.per_split < Q.blocks ? first + Q.per_split : Q.blocks;
    const uint32_t tile0 = blockIdx.x * kTiles, last = end - 1;
    const uint16_t *row = Q.x + int64_t(n < Q.nb ? n : Q.nb - 1) * Q.ldx;  // columns past the last right-hand side are not stored
    struct {
        Block<kTiles, kParts, kZeros> w;
        u32x4 x[4];
    } held;
    auto load = [&](uint32_t wanted) {
        held.w.load(Q, tile0, wanted, last, lane);
        const uint32_t block = wanted < last ? wanted : last;
        const int64_t c = int64_t(block) * 128 + 8 * g;
        if (block < Q.blocks - 1 || Q.cols % 128 == 0) {
#pragma unroll
            for (int j = 0; j < 4; ++j) held.x[j] = *reinterpret_cast<const u32x4_any *>(row + c + 32 * j);
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) held.x[j] = columns_of(row, c + 32 * j, Q.cols);
        }
    };
    f32x4 total[kTiles];
#pragma unroll
    for (int r = 0; r < kTiles; ++r) total[r] = f32x4{0, 0, 0, 0};
    load(first + wave);
    for (uint32_t block = first + wave; block < end; block += waves) {
        add_block<kTiles, kParts, kZeros, kBf16>(total, held.w, held.x);
        load(block + waves);
    }
    join_waves<kTiles>(Q, s_part, tile0, total);
}

// Adds the parts of the columns, in their order: a launch and its trip to memory, 2.5 us.
__global__ __launch_bounds__(256) void endor_q4_join_kernel(const float *partial, float *y, int64_t count, uint32_t splits) {
    const int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x;
    if (i >= count) return;
    float sum = 0;
    for (uint32_t s = 0; s < splits; ++s) sum += partial[s * count + i];
    y[i] = sum;
}

template <int kParts, bool kZeros, bool kBf16>
void (*gemm_kernel(const Plan &p))(Q4Params) {
    if (p.tiles == 0) {
        if constexpr (kParts < 4)  // with a group of 32 one block is on its way
            if (p.depth == 2) return endor_q4_gemv_kernel<2, kParts, kZeros, kBf16>;
        return endor_q4_gemv_kernel<1, kParts, kZeros, kBf16>;
    }
    if constexpr (kParts < 4) {  // and there are at most five row tiles
        if (p.tiles == 7) return endor_q4_gemm_kernel<7, kParts, kZeros, kBf16>;
        if (p.tiles == 6) return endor_q4_gemm_kernel<6, kParts, kZeros, kBf16>;
    }
    return p.tiles == 5   ? endor_q4_gemm_kernel<5, kParts, kZeros, kBf16>
           : p.tiles == 4 ? endor_q4_gemm_kernel<4, kParts, kZeros, kBf16>
           : p.tiles == 3 ? endor_q4_gemm_kernel<3, kParts, kZeros, kBf16>
           : p.tiles == 2 ? endor_q4_gemm_kernel<2, kParts, kZeros, kBf16>
                          : endor_q4_gemm_kernel<1, kParts, kZeros, kBf16>;
}
template <int kParts, bool kZeros, bool kBf16>
void launch(const Q4Params &Q, const Plan &p, hipStream_t s) {
    const uint32_t tiles = p.tiles ? p.tiles : 1;
    size_t lds = size_t(p.waves) * Q.nb * tiles * 16 * sizeof(float);
    if (!p.tiles && lds < endor_q4_plan::x_bytes(p.per_split, Q.nb)) lds = endor_q4_plan::x_bytes(p.per_split, Q.nb);
    const auto kernel = gemm_kernel<kParts, kZeros, kBf16>(p);
    hipLaunchKernelGGL(kernel, dim3((Q.tiles + tiles - 1) / tiles, p.splits), dim3(64 * p.waves), lds, s, Q);
}
template <int kParts>
void launch_kind(const Q4Params &Q, const Plan &p, bool bf16, hipStream_t s) {
    if (Q.zeros)
        bf16 ? launch<kParts, true, true>(Q, p, s) : launch<kParts, true, false>(Q, p, s);
    else
        bf16 ? launch<kParts, false, true>(Q, p, s) : launch<kParts, false, false>(Q, p, s);
}
void launch_group(Q4Params Q, const Plan &p, int group, bool bf16, hipStream_t s) {
    Q.splits = p.splits;
    Q.per_split = p.per_split;
    if (group == 32)
        launch_kind<4>(Q, p, bf16, s);
    else if (group == 64)
        launch_kind<2>(Q, p, bf16, s);
    else
        launch_kind<1>(Q, p, bf16, s);
    if (p.splits > 1) {
        const int64_t count = Q.rows * Q.nb;
        hipLaunchKernelGGL(endor_q4_join_kernel, dim3(static_cast<uint32_t>((count + 255) / 256)), dim3(256), 0, s, Q.partial, Q.y, count, p.splits);
    }
}

}  // namespace

extern "C" size_t endor_q4_bytes(int64_t rows, int64_t cols, int group, int with_zeros) {
    return sizes_ok(rows, cols, group) ? layout_of(rows, cols, group, with_zeros != 0).bytes : 0;
}

extern "C" size_t endor_q4_scratch_bytes(int64_t rows, int64_t cols, int group, int nb) {
    if (!sizes_ok(rows, cols, group) || nb < 1 || nb > ENDOR_GEMM_MAX_BATCH || rows == 0 || cols == 0) return 0;
    const Layout l = layout_of(rows, cols, group, false);
    const Plan p = make_plan(static_cast<uint32_t>(l.tiles), static_cast<uint32_t>(l.blocks), static_cast<uint32_t>(nb), group);
    return p.splits > 1 ? (size_t(p.splits) * nb * rows * sizeof(float) + 255) & ~size_t(255) : 0;
}

extern "C" endor_status endor_q4_pack(int64_t rows, int64_t cols, int group, const uint8_t *d_codes, const uint16_t *d_scales,
                                      const uint8_t *d_zeros, void *d_packed, size_t packed_bytes, void *stream) {
    if (rows < 0 || cols < 0) return ENDOR_ERR_INVALID_ARG;
    if (!sizes_ok(rows, cols, group)) return ENDOR_ERR_UNSUPPORTED;
    if (rows == 0 || cols == 0) return ENDOR_OK;
    if (!d_codes || !aligned(d_scales, 2) || !aligned(d_packed, 256)) return ENDOR_ERR_INVALID_ARG;
    const Layout l = layout_of(rows, cols, group, d_zeros != nullptr);
    if (packed_bytes < l.bytes) return ENDOR_ERR_BUFFER_TOO_SMALL;
    PackParams P{};
    P.codes = d_codes;
    P.scales = d_scales;
    P.zeros = d_zeros;
    P.out_codes = static_cast<uint32_t *>(d_packed);
    P.out_scales = reinterpret_cast<uint16_t *>(static_cast<char *>(d_packed) + l.codes);
    P.out_zeros = d_zeros ? static_cast<uint8_t *>(d_packed) + l.codes + l.scales : nullptr;
    P.rows = rows;
    P.cols = cols;
    P.group = group;
    P.groups = (cols + group - 1) / group;
    P.tiles = l.tiles;
    P.blocks = l.blocks;
    P.padded_groups = l.groups;
    // 64 units of codes a tile and block, and at most 64 scales
    hipLaunchKernelGGL(endor_q4_pack_kernel, dim3(static_cast<uint32_t>((l.tiles * l.blocks + 3) / 4)), dim3(256), 0, static_cast<hipStream_t>(stream), P);
    return hipGetLastError() == hipSuccess ? ENDOR_OK : ENDOR_ERR_HIP;
}

extern "C" endor_status endor_q4_quantize(int64_t rows, int64_t cols, int group, const uint16_t *d_dense, uint8_t *d_codes, uint16_t *d_scales,
                                          uint8_t *d_zeros, void *stream) {
    if (rows < 0 || cols < 0) return ENDOR_ERR_INVALID_ARG;
    if (!sizes_ok(rows, cols, group)) return ENDOR_ERR_UNSUPPORTED;
    if (rows == 0 || cols == 0) return ENDOR_OK;
    if (!aligned(d_dense, 2) || !d_codes || !aligned(d_scales, 2)) return ENDOR_ERR_INVALID_ARG;
    const int64_t groups = (cols + group - 1) / group;
    // below 2^30 groups, for a matrix has less than 2^34 elements and 2^26 rows
    const uint32_t count = static_cast<uint32_t>(rows * groups);
    const uint32_t lanes = group >= 512 ? 64 : static_cast<uint32_t>(group / 8), each = 256 / lanes;
    const auto kernel = lanes == 4    ? endor_q4_quantize_kernel<4>
                        : lanes == 8  ? endor_q4_quantize_kernel<8>
                        : lanes == 16 ? endor_q4_quantize_kernel<16>
                        : lanes == 32 ? endor_q4_quantize_kernel<32>
                                      : endor_q4_quantize_kernel<64>;
    constexpr uint32_t kMost = 1 << 23;  // workgroups of a launch: its threads are counted in 32 bits
    for (uint32_t first = 0; first < count; first += kMost * each) {
        const uint32_t left = (count - first + each - 1) / each;
        hipLaunchKernelGGL(kernel, dim3(left < kMost ? left : kMost), dim3(256), 0, static_cast<hipStream_t>(stream),
                           reinterpret_cast<const _Float16 *>(d_dense), first, count, cols, int64_t(group), static_cast<uint32_t>(groups), d_codes,
                           reinterpret_cast<_Float16 *>(d_scales), d_zeros);
        if (hipGetLastError() != hipSuccess) return ENDOR_ERR_HIP;
    }
    return ENDOR_OK;
}

namespace {
__global__ __launch_bounds__(256) void endor_q4_zero_kernel(float *y, int64_t count) {
    const int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x;
    if (i < count) y[i] = 0.0f;
}
}  // namespace

extern "C" endor_status endor_q4_gemm(int64_t rows, int64_t cols, int group, int with_zeros, const void *d_packed, size_t packed_bytes, int dtype,
                                      const void *d_x, int64_t ldx, int nb, float *d_y, void *d_scratch, size_t scratch_bytes, void *stream) {
    if (rows < 0 || cols < 0 || nb < 0 || nb > ENDOR_GEMM_MAX_BATCH) return ENDOR_ERR_INVALID_ARG;
    if (!sizes_ok(rows, cols, group) || (dtype != ENDOR_F16 && dtype != ENDOR_BF16)) return ENDOR_ERR_UNSUPPORTED;
    if (rows == 0 || nb == 0) return ENDOR_OK;
    if (!aligned(d_y, 4)) return ENDOR_ERR_INVALID_ARG;
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (cols == 0) {  // an empty sum
        hipLaunchKernelGGL(endor_q4_zero_kernel, dim3(static_cast<uint32_t>((nb * rows + 255) / 256)), dim3(256), 0, s, d_y, nb * rows);
        return hipGetLastError() == hipSuccess ? ENDOR_OK : ENDOR_ERR_HIP;
    }
    if (!aligned(d_packed, 256) || !aligned(d_x, 2) || ldx < cols) return ENDOR_ERR_INVALID_ARG;
    const Layout l = layout_of(rows, cols, group, with_zeros != 0);
    if (packed_bytes < l.bytes) return ENDOR_ERR_BUFFER_TOO_SMALL;
    Q4Params Q{};
    Q.codes = static_cast<const uint32_t *>(d_packed);
    Q.scales = reinterpret_cast<const _Float16 *>(static_cast<const char *>(d_packed) + l.codes);
    Q.zeros = with_zeros ? static_cast<const uint8_t *>(d_packed) + l.codes + l.scales : nullptr;
    Q.x = static_cast<const uint16_t *>(d_x);
    Q.y = d_y;
    Q.rows = rows;
    Q.cols = cols;
    Q.ldx = ldx;
    Q.tiles = static_cast<uint32_t>(l.tiles);
    Q.blocks = static_cast<uint32_t>(l.blocks);
    Q.groups = static_cast<uint32_t>(l.groups);
    Q.per_group_shift = group > 128 ? static_cast<uint32_t>(__builtin_ctz(static_cast<unsigned>(group))) - 7 : 0;
    Q.nb = static_cast<uint32_t>(nb);
    const Plan p = make_plan(Q.tiles, Q.blocks, Q.nb, group);
    if (p.splits > 1) {
        if (!aligned(d_scratch, 256)) return ENDOR_ERR_INVALID_ARG;
        if (scratch_bytes < endor_q4_scratch_bytes(rows, cols, group, nb)) return ENDOR_ERR_BUFFER_TOO_SMALL;
        Q.partial = static_cast<float *>(d_scratch);
    }
    launch_group(Q, p, group, dtype == ENDOR_BF16, s);
    return hipGetLastError() == hipSuccess ? ENDOR_OK : ENDOR_ERR_HIP;
}
