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
#include "endor_kv.h"

namespace {

using endor_kv::aligned;

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
    int64_t rows, cols, ldx, blocks, groups;
    uint32_t group_shift;
};

template <bool kBf16>
__device__ __forceinline__ float widen(uint16_t x) {
    if constexpr (kBf16) return __uint_as_float(uint32_t(x) << 16);
    return static_cast<float>(__builtin_bit_cast(_Float16, x));
}

// One wave per row and right-hand side.
template <bool kBf16>
__global__ __launch_bounds__(64) void endor_q4_gemm_kernel(Q4Params Q) {
    const int64_t row = blockIdx.x, tile = row / 16;
    const uint16_t *x = Q.x + blockIdx.y * Q.ldx;
    const uint32_t r = row & 15, lane = threadIdx.x;
    float total = 0;
    for (int64_t g = 0; g < Q.groups; ++g) {
        float sum = 0;
        const int64_t from = g << Q.group_shift, to = from + (int64_t(1) << Q.group_shift) < Q.cols ? from + (int64_t(1) << Q.group_shift) : Q.cols;
        const float zero = Q.zeros ? Q.zeros[(tile * Q.groups + g) * 16 + r] : 8.0f;
        for (int64_t c = from + lane; c < to; c += 64) {
            const uint32_t in = c & 127, word = Q.codes[((tile * Q.blocks + c / 128) * 64 + (in / 8 % 4) * 16 + r) * 4 + in / 32];
            sum += (float(word >> (4 * place_of(in & 7)) & 15u) - zero) * widen<kBf16>(x[c]);
        }
        total += sum * float(Q.scales[(tile * Q.groups + g) * 16 + r]);
    }
    for (int d = 32; d; d >>= 1) total += __shfl_xor(total, d);
    if (lane == 0) Q.y[blockIdx.y * Q.rows + row] = total;
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
    Q.blocks = l.blocks;
    Q.groups = l.groups;
    Q.group_shift = static_cast<uint32_t>(__builtin_ctz(static_cast<unsigned>(group)));
    hipLaunchKernelGGL(dtype == ENDOR_BF16 ? endor_q4_gemm_kernel<true> : endor_q4_gemm_kernel<false>, dim3(static_cast<uint32_t>(rows), nb), dim3(64),
                       0, s, Q);
    return hipGetLastError() == hipSuccess ? ENDOR_OK : ENDOR_ERR_HIP;
}
