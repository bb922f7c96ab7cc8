// Attention of one new token per sequence over a paged key-value cache.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "endor.h"
#include "endor_device.h"
#include "endor_kv.h"

namespace {

using endor_kv::aligned;
using endor_kv::Cache;
using endor_kv::capacity_of;
using endor_kv::clamp_length;
using endor_kv::page_of;
using endor_kv::read_cache;
using endor_kv::slot_at;

struct AttnParams {
    Cache C;
    const uint16_t *q;
    int64_t q_seq_stride, q_head_stride;
    const int32_t *lengths;
    const uint64_t *mask;
    int64_t mask_stride;
    uint16_t *out;
    float *lse;
    const float *weights;
    float *weights_out;
    float scale;
    int32_t q_heads, most_len, capacity;
};

template <bool kBf16>
__device__ __forceinline__ float widen(uint16_t x) {
    if constexpr (kBf16) return __uint_as_float(uint32_t(x) << 16);
    return static_cast<float>(__builtin_bit_cast(_Float16, x));
}
template <bool kBf16>
__device__ __forceinline__ uint16_t narrow(float x) {
    if constexpr (kBf16) return __builtin_bit_cast(uint16_t, static_cast<__bf16>(x));
    return __builtin_bit_cast(uint16_t, static_cast<_Float16>(x));
}

__device__ __forceinline__ bool visible(const AttnParams &A, uint32_t b, uint32_t t) {
    return !A.mask || (A.mask[b * A.mask_stride + (t >> 6)] >> (t & 63) & 1);
}

__device__ __forceinline__ float sum_of_wave(float x) {
    for (int d = 32; d; d >>= 1) x += __shfl_xor(x, d);
    return x;
}

// One wave per query head and sequence; a lane holds elements lane, 64 + lane, ... of q and of the output.
template <bool kBf16>
__global__ __launch_bounds__(64) void endor_attn_kernel(AttnParams A) {
    const uint32_t b = blockIdx.y, h = blockIdx.x, lane = threadIdx.x, kv = h / (A.q_heads / A.C.kv_heads), dim = A.C.dim;
    const int32_t length = clamp_length(A.lengths[b], A.most_len);
    const int32_t *table = A.C.pages + b * A.C.pages_stride;
    float q[4], o[4] = {0, 0, 0, 0}, top = -INFINITY, total = 0;
    for (uint32_t i = 0; i < 4; ++i)
        q[i] = 64 * i + lane < dim ? widen<kBf16>(A.q[b * A.q_seq_stride + h * A.q_head_stride + 64 * i + lane]) : 0.0f;
    for (int32_t t = 0; t < length; ++t) {
        uint32_t page;
        if (!visible(A, b, t) || !page_of(A.C, table, t, &page)) continue;
        const int64_t at = slot_at(A.C, page, kv, t);
        float s = 0;
        for (uint32_t i = 0; i < 4; ++i)
            if (64 * i + lane < dim) s += q[i] * widen<kBf16>(A.C.k[at + 64 * i + lane]);
        s = sum_of_wave(s) * A.scale;
        const float next = fmaxf(top, s), keep = top == -INFINITY ? 0.0f : expf(top - next), p = next == -INFINITY ? 0.0f : expf(s - next);
        for (uint32_t i = 0; i < 4; ++i)
            if (64 * i + lane < dim) o[i] = o[i] * keep + p * widen<kBf16>(A.C.v[at + 64 * i + lane]);
        total = total * keep + p;
        top = next;
    }
    const int64_t row = int64_t(b) * A.q_heads + h;
    for (uint32_t i = 0; i < 4; ++i)
        if (64 * i + lane < dim) A.out[row * dim + 64 * i + lane] = narrow<kBf16>(total > 0 ? o[i] / total : 0.0f);
    if (lane == 0) A.lse[row] = total > 0 ? top + logf(total) : -INFINITY;
}

// One wave per slot: the logits of the heads that share it once more, from the rows' lse.
template <bool kBf16>
__global__ __launch_bounds__(64) void endor_attn_weights_kernel(AttnParams A) {
    const uint32_t b = blockIdx.z, kv = blockIdx.y, lane = threadIdx.x, group = A.q_heads / A.C.kv_heads, dim = A.C.dim;
    const int32_t length = clamp_length(A.lengths[b], A.most_len);
    const int32_t *table = A.C.pages + b * A.C.pages_stride;
    for (int32_t t = blockIdx.x; t < length; t += gridDim.x) {
        uint32_t page;
        float sum = 0;
        if (visible(A, b, t) && page_of(A.C, table, t, &page)) {
            const int64_t at = slot_at(A.C, page, kv, t);
            for (uint32_t g = 0; g < group; ++g) {
                const uint32_t h = kv * group + g;
                float s = 0;
                for (uint32_t i = 0; i < 4; ++i)
                    if (64 * i + lane < dim)
                        s += widen<kBf16>(A.q[b * A.q_seq_stride + h * A.q_head_stride + 64 * i + lane]) * widen<kBf16>(A.C.k[at + 64 * i + lane]);
                sum += expf(sum_of_wave(s) * A.scale - A.lse[int64_t(b) * A.q_heads + h]);
            }
        }
        const int64_t w = (int64_t(b) * A.C.kv_heads + kv) * A.capacity + t;
        if (lane == 0) A.weights_out[w] = (A.weights ? A.weights[w] : 0.0f) + sum;
    }
}

}  // namespace

extern "C" size_t endor_attn_scratch_bytes(const endor_kv_cache *cache, int q_heads, int32_t max_len, int with_weights) {
    Cache C;
    if (read_cache(cache, &C) != ENDOR_OK || q_heads < 1 || q_heads % C.kv_heads != 0 || max_len < 0) return 0;
    (void)with_weights;
    return (size_t(C.batch) * q_heads * 4 + 255) & ~size_t(255);
}

extern "C" endor_status endor_attn_decode(const endor_kv_cache *cache, int q_heads, const void *d_q, int64_t q_seq_stride, int64_t q_head_stride,
                                          const int32_t *d_lengths, int32_t max_len, const uint64_t *d_mask, int64_t mask_stride, float scale,
                                          void *d_out, float *d_lse, const float *d_weights, float *d_weights_out, void *d_scratch,
                                          size_t scratch_bytes, void *stream) {
    AttnParams A{};
    if (const endor_status st = read_cache(cache, &A.C)) return st;
    if (q_heads < 1 || q_heads > 65535 || q_heads % A.C.kv_heads != 0 || max_len < 0 || q_seq_stride < 0 || q_head_stride < 0) return ENDOR_ERR_INVALID_ARG;
    if (A.C.batch == 0) return ENDOR_OK;
    A.capacity = capacity_of(*cache);
    A.most_len = max_len < A.capacity ? max_len : A.capacity;
    if (!aligned(d_q, 2) || !aligned(d_out, 2) || !aligned(d_lengths, 4) || (d_lse && !aligned(d_lse, 4))) return ENDOR_ERR_INVALID_ARG;
    if (d_mask && (!aligned(d_mask, 8) || mask_stride < (int64_t(A.most_len) + 63) / 64)) return ENDOR_ERR_INVALID_ARG;
    if ((d_weights && !aligned(d_weights, 4)) || (d_weights_out && !aligned(d_weights_out, 4)) || (d_weights && !d_weights_out)) return ENDOR_ERR_INVALID_ARG;
    const size_t need = endor_attn_scratch_bytes(cache, q_heads, max_len, d_weights_out != nullptr);
    if (need && !aligned(d_scratch, 256)) return ENDOR_ERR_INVALID_ARG;
    if (scratch_bytes < need) return ENDOR_ERR_BUFFER_TOO_SMALL;
    A.q = static_cast<const uint16_t *>(d_q);
    A.q_seq_stride = q_seq_stride;
    A.q_head_stride = q_head_stride;
    A.lengths = d_lengths;
    A.mask = d_mask;
    A.mask_stride = mask_stride;
    A.out = static_cast<uint16_t *>(d_out);
    A.lse = d_lse ? d_lse : static_cast<float *>(d_scratch);
    A.weights = d_weights;
    A.weights_out = d_weights_out;
    A.scale = scale;
    A.q_heads = q_heads;
    hipStream_t s = static_cast<hipStream_t>(stream);
    const bool bf16 = cache->dtype == ENDOR_BF16;
    hipLaunchKernelGGL(bf16 ? endor_attn_kernel<true> : endor_attn_kernel<false>, dim3(q_heads, A.C.batch), dim3(64), 0, s, A);
    if (hipGetLastError() != hipSuccess) return ENDOR_ERR_HIP;
    if (d_weights_out && A.most_len > 0) {
        hipLaunchKernelGGL(bf16 ? endor_attn_weights_kernel<true> : endor_attn_weights_kernel<false>,
                           dim3(A.most_len < 1024 ? A.most_len : 1024, A.C.kv_heads, A.C.batch), dim3(64), 0, s, A);
        if (hipGetLastError() != hipSuccess) return ENDOR_ERR_HIP;
    }
    return ENDOR_OK;
}
