// Products with 4-bit weights that carry a scale, and if wanted a zero point, per row and group of columns.
//
// PACKED FORM.  Rows go in tiles of 16, columns in blocks of 128, both padded with codes and scales of zero, so that no
// kernel has an edge in W.  Codes: [tile][block][lane 0..63][16 bytes]; lane l has row l & 15 of the tile, and its 32-bit word j the
// columns 32 j + 8 (l >> 4) + 0..7 of the block, column c in bits 4 * kNibble[c].  Then the scales, fp16 [tile][group][16 rows],
// then, if there are any, the zeros, a byte [tile][group][16 rows].  A block and a group that holds several blocks end
// at the same column.
#include <hip/hip_runtime.h>

#include <cstdint>

#include "endor.h"
#include "endor_device.h"
#include "endor_kv.h"

namespace {

using endor_device::u32x4;
using endor_kv::aligned;

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

// The 4-bit place of a word's column: pairs of columns lie 16 bits apart, where packed 16-bit arithmetic takes them.
__device__ __forceinline__ uint32_t place_of(uint32_t c) { return (c >> 1) + 4 * (c & 1); }

__global__ __launch_bounds__(256) void endor_q4_pack_kernel(PackParams P) {
    const int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x, words = P.tiles * P.blocks * 256;
    if (i < words) {
        const uint32_t j = i & 3, lane = (i >> 2) & 63;
        const int64_t block = (i >> 8) % P.blocks, row = (i >> 8) / P.blocks * 16 + (lane & 15), col = block * 128 + 32 * j + 8 * (lane >> 4);
        uint32_t word = 0;
        if (row < P.rows)
            for (uint32_t c = 0; c < 8; ++c)
                if (col + c < P.cols) {
                    const uint32_t two = P.codes[row * ((P.cols + 1) / 2) + (col + c) / 2];
                    word |= ((c & 1) ? two >> 4 : two & 15u) << (4 * place_of(c));  // col is even
                }
        P.out_codes[i] = word;
    }
    const int64_t entries = P.tiles * P.padded_groups * 16;
    if (i < entries) {
        const int64_t row = i / (16 * P.padded_groups) * 16 + (i & 15), g = (i >> 4) % P.padded_groups;
        const bool in = row < P.rows && g < P.groups;
        P.out_scales[i] = in ? P.scales[row * P.groups + g] : 0;
        if (P.out_zeros) P.out_zeros[i] = in ? P.zeros[row * P.groups + g] & 15 : 0;
    }
}

// One wave per row and group.  The scale is rounded to fp16 before the codes are taken, so that they are the nearest to what they stand for.
__global__ __launch_bounds__(64) void endor_q4_quantize_kernel(const _Float16 *dense, int64_t first, int64_t cols, int64_t group, int64_t groups,
                                                               uint8_t *codes, _Float16 *scales, uint8_t *zeros) {
    const int64_t i = first + blockIdx.x, row = i / groups, g = i % groups, from = g * group;
    const int64_t to = from + group < cols ? from + group : cols;
    const uint32_t lane = threadIdx.x;
    const _Float16 *w = dense + row * cols;
    float lo = 0, hi = 0;
    for (int64_t c = from + lane; c < to; c += 64) {
        const float x = w[c];
        lo = fminf(lo, x);
        hi = fmaxf(hi, x);
    }
    for (int d = 32; d; d >>= 1) {
        lo = fminf(lo, __shfl_xor(lo, d));
        hi = fmaxf(hi, __shfl_xor(hi, d));
    }
    const _Float16 scale = static_cast<_Float16>(zeros ? (hi - lo) / 15.0f : fmaxf(hi, -lo) / 7.0f);
    const float s = scale, inverse = s > 0 ? 1.0f / s : 0.0f;
    const float zero = zeros ? fminf(fmaxf(rintf(-lo * inverse), 0.0f), 15.0f) : 8.0f;
    if (lane == 0) {
        scales[row * groups + g] = scale;
        if (zeros) zeros[row * groups + g] = static_cast<uint8_t>(zero);
    }
    for (int64_t c = from + 2 * lane; c < to; c += 128) {  // a group begins at an even column
        uint32_t two = 0;
        for (int k = 0; k < 2; ++k)
            if (c + k < to) two |= static_cast<uint32_t>(fminf(fmaxf(rintf(float(w[c + k]) * inverse) + zero, 0.0f), 15.0f)) << (4 * k);
        codes[row * ((cols + 1) / 2) + c / 2] = static_cast<uint8_t>(two);
    }
}

struct Q4Params {
    const uint32_t *codes;
    const _Float16 *scales;
    const uint8_t *zeros;
    const uint16_t *x;
    float *y;
    int64_t rows, cols, ldx;
    uint32_t tiles, blocks, groups, per_group_shift, nb;  // per_group_shift: blocks of a group, where those are whole
};

// Eight codes as pairs of the type's numbers code - zero, which are exact: columns (0, 1), (2, 3), (4, 5), (6, 7).
template <bool kBf16>
struct Zero;  // what is taken off: prepared once per row and group
template <>
struct Zero<false> {
    f16x2 near, far;
    __device__ __forceinline__ explicit Zero(float z) {
        near = f16x2{static_cast<_Float16>(-1024.0f - z), static_cast<_Float16>(-1024.0f - z)};
        far = f16x2{static_cast<_Float16>(-64.0f - z), static_cast<_Float16>(-64.0f - z)};
    }
    // A code in the low bits of 0x6400 is the number 1024 + code, in the next four 1024 + 16 code.
    __device__ __forceinline__ u32x4 operand(uint32_t w) const {
        auto low = [](uint32_t v) { return __builtin_bit_cast(f16x2, (v & 0x000f000fu) | 0x64006400u); };
        auto high = [](uint32_t v) { return __builtin_bit_cast(f16x2, (v & 0x00f000f0u) | 0x64006400u); };
        const f16x2 sixteenth = {static_cast<_Float16>(0.0625f), static_cast<_Float16>(0.0625f)};
        const uint32_t v = w >> 8;
        return u32x4{__builtin_bit_cast(uint32_t, low(w) + near), __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(high(w), sixteenth, far)),
                     __builtin_bit_cast(uint32_t, low(v) + near), __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(high(v), sixteenth, far))};
    }
};
template <>
struct Zero<true> {
    float z;
    __device__ __forceinline__ explicit Zero(float zero) : z(zero) {}
    __device__ __forceinline__ u32x4 operand(uint32_t w) const {
        const uint32_t low = w & 0x0f0f0f0fu, high = (w >> 4) & 0x0f0f0f0fu;  // columns 0, 4, 1, 5 and 2, 6, 3, 7
        auto pair = [&](uint32_t v, int a) {  // a whole number below 16 has its bits in the upper half of a float
            const float x = static_cast<float>((v >> (8 * a)) & 0xffu) - z, y = static_cast<float>((v >> (8 * a + 16)) & 0xffu) - z;
            return __builtin_amdgcn_perm(__float_as_uint(y), __float_as_uint(x), 0x07060302u);
        };
        return u32x4{pair(low, 0), pair(high, 0), pair(low, 1), pair(high, 1)};
    }
};

template <bool kBf16>
__device__ __forceinline__ f32x4 product(u32x4 a, u32x4 b, f32x4 c) {
    if constexpr (kBf16)
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// A workgroup has kTiles row tiles; its waves take the blocks of 128 columns in turn and are joined in LDS.  kParts: groups of a block.
// kAligned: rows of x begin at 16-byte boundaries.
template <int kTiles, int kParts, bool kZeros, bool kBf16, bool kAligned>
__global__ __launch_bounds__(512) void endor_q4_gemm_kernel(Q4Params Q) {
    extern __shared__ float s_part[];  // [wave][right-hand side][16 kTiles rows]
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6, n = lane & 15, g = lane >> 4;
    const uint32_t tile0 = blockIdx.x * kTiles;
    const uint16_t *x = Q.x + int64_t(n < Q.nb ? n : Q.nb - 1) * Q.ldx + 8 * g;  // columns past the last right-hand side are not stored

    struct Block {
        u32x4 codes[kTiles], x[4];
        f16x4 scales[kTiles][kParts];
        uint8_t zeros[kTiles][kZeros ? kParts : 1];
    };
    const uint32_t last = Q.blocks - 1;
    auto load = [&](uint32_t block, Block &B) {
        const uint32_t group = kParts > 1 ? block * kParts : block >> Q.per_group_shift;
#pragma unroll
        for (int r = 0; r < kTiles; ++r) {
            const uint32_t tile = tile0 + r < Q.tiles ? tile0 + r : Q.tiles - 1;
            B.codes[r] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(Q.codes) + (uint64_t(tile) * Q.blocks + block) * 64 + lane);
#pragma unroll
            for (int p = 0; p < kParts; ++p) {
                const uint64_t at = (uint64_t(tile) * Q.groups + group + p) * 16;
                B.scales[r][p] = *reinterpret_cast<const f16x4 *>(Q.scales + at + 4 * g);
                if constexpr (kZeros) B.zeros[r][p] = Q.zeros[at + n];
            }
        }
        const uint16_t *from = x + int64_t(block) * 128;
        if (block < last || Q.cols % 128 == 0) {
            typedef u32x4 u32x4_any __attribute__((aligned(2)));
#pragma unroll
            for (int j = 0; j < 4; ++j)
                B.x[j] = kAligned ? *reinterpret_cast<const u32x4 *>(from + 32 * j) : *reinterpret_cast<const u32x4_any *>(from + 32 * j);
        } else {  // zeros past the last column
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int e = 0; e < 8; e += 2) {
                    const int64_t c = int64_t(block) * 128 + 32 * j + 8 * g + e;
                    const uint32_t a = c < Q.cols ? from[32 * j + e] : 0, z = c + 1 < Q.cols ? from[32 * j + e + 1] : 0;
                    B.x[j][e / 2] = a | z << 16;
                }
        }
    };
    f32x4 total[kTiles];
#pragma unroll
    for (int r = 0; r < kTiles; ++r) total[r] = f32x4{0, 0, 0, 0};
    auto add = [&](const Block &B) {
#pragma unroll
        for (int r = 0; r < kTiles; ++r)
#pragma unroll
            for (int p = 0; p < kParts; ++p) {
                const Zero<kBf16> zero(kZeros ? static_cast<float>(B.zeros[r][p]) : 8.0f);
                f32x4 sum = {0, 0, 0, 0};
#pragma unroll
                for (int j = 4 / kParts * p; j < 4 / kParts * (p + 1); ++j) sum = product<kBf16>(zero.operand(B.codes[r][j]), B.x[j], sum);
#pragma unroll
                for (int i = 0; i < 4; ++i) total[r][i] += sum[i] * static_cast<float>(B.scales[r][p][i]);
            }
    };
    if (wave < Q.blocks) {
        Block a, z;
        uint32_t block = wave;
        load(block, a);
        for (;;) {
            const uint32_t second = block + waves, third = second + waves;
            load(second < last ? second : last, z);
            add(a);
            if (second >= Q.blocks) break;
            load(third < last ? third : last, a);
            add(z);
            if (third >= Q.blocks) break;
            block = third;
        }
    }
    if (n < Q.nb)
#pragma unroll
        for (int r = 0; r < kTiles; ++r) *reinterpret_cast<f32x4 *>(s_part + ((wave * Q.nb + n) * kTiles + r) * 16 + 4 * g) = total[r];
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < Q.nb * kTiles * 16; i += blockDim.x) {
        float sum = 0;
        for (uint32_t w = 0; w < waves; ++w) sum += s_part[w * Q.nb * kTiles * 16 + i];
        const uint32_t b = i / (kTiles * 16);
        const int64_t row = int64_t(tile0) * 16 + i % (kTiles * 16);
        if (row < Q.rows) Q.y[b * Q.rows + row] = sum;
    }
}

template <int kTiles, int kParts, bool kZeros, bool kBf16>
void launch_aligned(const Q4Params &Q, uint32_t waves, hipStream_t s) {
    const bool even = (reinterpret_cast<uintptr_t>(Q.x) & 15) == 0 && (Q.ldx % 8 == 0 || Q.nb == 1);
    hipLaunchKernelGGL((even ? endor_q4_gemm_kernel<kTiles, kParts, kZeros, kBf16, true> : endor_q4_gemm_kernel<kTiles, kParts, kZeros, kBf16, false>),
                       dim3((Q.tiles + kTiles - 1) / kTiles), dim3(64 * waves), waves * Q.nb * kTiles * 16 * sizeof(float), s, Q);
}
template <int kTiles, int kParts>
void launch_kind(const Q4Params &Q, bool bf16, uint32_t waves, hipStream_t s) {
    if (Q.zeros)
        bf16 ? launch_aligned<kTiles, kParts, true, true>(Q, waves, s) : launch_aligned<kTiles, kParts, true, false>(Q, waves, s);
    else
        bf16 ? launch_aligned<kTiles, kParts, false, true>(Q, waves, s) : launch_aligned<kTiles, kParts, false, false>(Q, waves, s);
}
template <int kTiles>
void launch_parts(const Q4Params &Q, int group, bool bf16, uint32_t waves, hipStream_t s) {
    if (group == 32)
        launch_kind<kTiles, 4>(Q, bf16, waves, s);
    else if (group == 64)
        launch_kind<kTiles, 2>(Q, bf16, waves, s);
    else
        launch_kind<kTiles, 1>(Q, bf16, waves, s);
}
void launch(const Q4Params &Q, int group, bool bf16, int tiles, uint32_t waves, hipStream_t s) {
    if (tiles == 4)
        launch_parts<4>(Q, group, bf16, waves, s);
    else if (tiles == 2)
        launch_parts<2>(Q, group, bf16, waves, s);
    else
        launch_parts<1>(Q, group, bf16, waves, s);
}

}  // namespace

extern "C" size_t endor_q4_bytes(int64_t rows, int64_t cols, int group, int with_zeros) {
    return sizes_ok(rows, cols, group) ? layout_of(rows, cols, group, with_zeros != 0).bytes : 0;
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
    // 256 words of codes a tile and block, and at most 64 scales
    hipLaunchKernelGGL(endor_q4_pack_kernel, dim3(static_cast<uint32_t>(l.tiles * l.blocks)), dim3(256), 0, static_cast<hipStream_t>(stream), P);
    return hipGetLastError() == hipSuccess ? ENDOR_OK : ENDOR_ERR_HIP;
}

extern "C" endor_status endor_q4_quantize(int64_t rows, int64_t cols, int group, const uint16_t *d_dense, uint8_t *d_codes, uint16_t *d_scales,
                                          uint8_t *d_zeros, void *stream) {
    if (rows < 0 || cols < 0) return ENDOR_ERR_INVALID_ARG;
    if (!sizes_ok(rows, cols, group)) return ENDOR_ERR_UNSUPPORTED;
    if (rows == 0 || cols == 0) return ENDOR_OK;
    if (!aligned(d_dense, 2) || !d_codes || !aligned(d_scales, 2)) return ENDOR_ERR_INVALID_ARG;
    const int64_t groups = (cols + group - 1) / group;
    constexpr int64_t kMost = 1 << 24;  // workgroups of a launch: its threads are counted in 32 bits
    for (int64_t first = 0; first < rows * groups; first += kMost) {
        const int64_t left = rows * groups - first;
        hipLaunchKernelGGL(endor_q4_quantize_kernel, dim3(static_cast<uint32_t>(left < kMost ? left : kMost)), dim3(64), 0,
                           static_cast<hipStream_t>(stream), reinterpret_cast<const _Float16 *>(d_dense), first, cols, int64_t(group), groups,
                           d_codes, reinterpret_cast<_Float16 *>(d_scales), d_zeros);
        if (hipGetLastError() != hipSuccess) return ENDOR_ERR_HIP;
    }
    return ENDOR_OK;
}

__global__ __launch_bounds__(256) void endor_q4_zero_kernel(float *y, int64_t count) {
    const int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x;
    if (i < count) y[i] = 0.0f;
}

extern "C" endor_status endor_q4_gemm(int64_t rows, int64_t cols, int group, int with_zeros, const void *d_packed, size_t packed_bytes, int dtype,
                                      const void *d_x, int64_t ldx, int nb, float *d_y, void *stream) {
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
    launch(Q, group, dtype == ENDOR_BF16, l.tiles >= 1024 ? 2 : 1, 8, s);
    return hipGetLastError() == hipSuccess ? ENDOR_OK : ENDOR_ERR_HIP;
}
