// Writes into a paged key-value cache, and eviction from it by accumulated attention weight.
#include <hip/hip_runtime.h>

#include <cstdint>

#include "endor.h"
#include "endor_device.h"
#include "endor_kv.h"

namespace {

using endor_device::u32x4;
using endor_device::wave_inclusive_scan;
using endor_kv::aligned;
using endor_kv::Cache;
using endor_kv::capacity_of;
using endor_kv::clamp_length;
using endor_kv::page_of;
using endor_kv::read_cache;
using endor_kv::slot_at;

// ---------------------------------------------------------------- append

struct AppendParams {
    Cache C;
    const uint16_t *k, *v;
    int64_t seq_stride, token_stride, head_stride;
    const int32_t *counts, *lengths, *seen;
    int32_t *lengths_out, *seen_out;
    float *weights;
    int32_t *positions;
    int32_t tokens, capacity;
};

// One workgroup per sequence and token; a separate launch advances the lengths behind it.
__global__ __launch_bounds__(256) void endor_kv_append_kernel(AppendParams A) {
    const uint32_t b = blockIdx.y, t = blockIdx.x;
    const int32_t length = clamp_length(A.lengths[b], A.capacity);
    const int32_t count = A.counts ? clamp_length(A.counts[b], A.tokens) : A.tokens;
    if (static_cast<int32_t>(t) >= count || length + int64_t(t) >= A.capacity) return;
    const uint32_t slot = length + t, heads = A.C.kv_heads, dim = A.C.dim;
    uint32_t page;
    if (page_of(A.C, A.C.pages + b * A.C.pages_stride, slot, &page)) {
        for (uint32_t i = threadIdx.x; i < heads * dim; i += 256) {
            const uint32_t h = i / dim, d = i % dim;
            const int64_t from = int64_t(b) * A.seq_stride + int64_t(t) * A.token_stride + int64_t(h) * A.head_stride + d;
            const int64_t to = slot_at(A.C, page, h, slot) + d;
            A.C.k[to] = A.k[from];
            A.C.v[to] = A.v[from];
        }
    }
    for (uint32_t h = threadIdx.x; h < heads; h += 256) {
        const int64_t at = (int64_t(b) * heads + h) * A.capacity + slot;
        if (A.weights) A.weights[at] = 0.0f;
        if (A.positions) A.positions[at] = A.seen[b] + static_cast<int32_t>(t);
    }
}

__global__ __launch_bounds__(256) void endor_kv_advance_kernel(AppendParams A) {
    const int32_t b = blockIdx.x * 256 + threadIdx.x;
    if (b >= A.C.batch) return;
    const int32_t length = clamp_length(A.lengths[b], A.capacity);
    const int32_t count = A.counts ? clamp_length(A.counts[b], A.tokens) : A.tokens;
    const int32_t stored = count < A.capacity - length ? count : A.capacity - length;
    A.lengths_out[b] = length + stored;
    A.seen_out[b] = A.seen[b] + stored;
}

// ---------------------------------------------------------------- evict

struct EvictParams {
    Cache C;
    const int32_t *lengths, *seen;
    const float *weights;
    const int32_t *positions;
    int32_t *lengths_out;
    float *weights_out;
    int32_t *positions_out;
    int32_t *count, *holes, *movers;  // scratch: [batch * kv_heads], and [batch * kv_heads][most] each
    int32_t budget, recent, most_len, capacity, most;
};

// Weights as unsigned numbers in the same order: NaN below all, -0 with +0; what must stay above all.
__device__ __forceinline__ uint32_t key_of(float w, int32_t position, int64_t newest) {
    if (position >= newest) return 0xffffffffu;
    if (w != w) return 0;
    const uint32_t bits = __float_as_uint(w + 0.0f);
    return bits >> 31 ? ~bits : bits | 0x80000000u;
}

constexpr int kSelectThreads = 1024;

// Sum over the workgroup; every thread gets it.
__device__ __forceinline__ uint32_t group_sum(uint32_t x, uint32_t *s_part) {
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint32_t upto = wave_inclusive_scan(x);
    __syncthreads();
    if (lane == 63) s_part[wave] = upto;
    __syncthreads();
    uint32_t sum = 0;
    for (int w = 0; w < kSelectThreads / 64; ++w) sum += s_part[w];
    return sum;
}
// Exclusive prefix over the workgroup, and the total.
__device__ __forceinline__ uint32_t group_scan(uint32_t x, uint32_t *s_part, uint32_t *total) {
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint32_t upto = wave_inclusive_scan(x);
    __syncthreads();
    if (lane == 63) s_part[wave] = upto;
    __syncthreads();
    uint32_t before = 0, sum = 0;
    for (uint32_t w = 0; w < kSelectThreads / 64; ++w) {
        before += w < wave ? s_part[w] : 0;
        sum += s_part[w];
    }
    *total = sum;
    return before + upto - x;
}

// One workgroup per sequence and kv head: the key of the budget-th largest, bit by bit; then the slots that come free below the
// budget and the kept ones past it, in order.
__global__ __launch_bounds__(kSelectThreads) void endor_kv_select_kernel(EvictParams E) {
    __shared__ uint32_t s_part[kSelectThreads / 64];
    const uint32_t b = blockIdx.y, h = blockIdx.x;
    const int64_t row = int64_t(b) * E.C.kv_heads + h, base = row * E.capacity;
    const float *w = E.weights + base;
    const int32_t *pos = E.positions + base;
    float *w_out = E.weights_out + base;
    int32_t *pos_out = E.positions_out + base;
    const int32_t length = clamp_length(E.lengths[b], E.most_len), budget = E.budget;
    if (length <= budget) {
        for (int32_t t = threadIdx.x; t < length; t += kSelectThreads) {
            w_out[t] = w[t];
            pos_out[t] = pos[t];
        }
        if (threadIdx.x == 0) E.count[row] = 0;
        return;
    }
    const int64_t newest = int64_t(E.seen[b]) - E.recent;
    // the largest threshold that at least `budget` keys reach
    uint32_t least = 0;
    for (int bit = 31; bit >= 0; --bit) {
        const uint32_t trial = least | (1u << bit);
        uint32_t n = 0;
        for (int32_t t = threadIdx.x; t < length; t += kSelectThreads) n += key_of(w[t], pos[t], newest) >= trial;
        if (group_sum(n, s_part) >= static_cast<uint32_t>(budget)) least = trial;
    }
    uint32_t above = 0;
    for (int32_t t = threadIdx.x; t < length; t += kSelectThreads) above += key_of(w[t], pos[t], newest) > least;
    uint32_t ties = budget - group_sum(above, s_part);  // of the keys equal to `least`, the first so many stay
    int32_t *holes = E.holes + row * E.most, *movers = E.movers + row * E.most;
    uint32_t nholes = 0, nmovers = 0;
    for (int32_t t0 = 0; t0 < length; t0 += kSelectThreads) {
        const int32_t t = t0 + threadIdx.x;
        const uint32_t key = t < length ? key_of(w[t], pos[t], newest) : 0;
        uint32_t total;
        const uint32_t tie = t < length && key == least;
        const uint32_t rank = group_scan(tie, s_part, &total);
        const bool keep = t < length && (key > least || (tie && rank < ties));
        ties -= total < ties ? total : ties;
        const uint32_t hole = t < budget && !keep, mover = t >= budget && keep;
        const uint32_t before = group_scan(hole | mover << 16, s_part, &total);  // at most 1024 of each
        if (hole) holes[nholes + (before & 0xffffu)] = t;
        if (mover) movers[nmovers + (before >> 16)] = t;
        nholes += total & 0xffffu;
        nmovers += total >> 16;
        if (t < budget && keep) {
            w_out[t] = w[t];
            pos_out[t] = pos[t];
        }
    }
    __threadfence_block();
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < nholes; i += kSelectThreads) {
        w_out[holes[i]] = w[movers[i]];
        pos_out[holes[i]] = pos[movers[i]];
    }
    if (threadIdx.x == 0) E.count[row] = nholes;
}

// Keys and values of the kept tokens past the budget; and the lengths.
__global__ __launch_bounds__(256) void endor_kv_move_kernel(EvictParams E) {
    const uint32_t b = blockIdx.z, h = blockIdx.y;
    const int64_t row = int64_t(b) * E.C.kv_heads + h;
    if (blockIdx.x == 0 && h == 0 && threadIdx.x == 0) {
        const int32_t length = clamp_length(E.lengths[b], E.most_len);
        E.lengths_out[b] = length < E.budget ? length : E.budget;
    }
    const int32_t count = E.count[row];
    const int32_t *table = E.C.pages + b * E.C.pages_stride;
    for (int32_t i = blockIdx.x; i < count; i += gridDim.x) {
        const uint32_t to = E.holes[row * E.most + i], from = E.movers[row * E.most + i];
        uint32_t to_page, from_page;
        if (!page_of(E.C, table, to, &to_page) || !page_of(E.C, table, from, &from_page)) continue;
        const int64_t dst = slot_at(E.C, to_page, h, to), src = slot_at(E.C, from_page, h, from);
        for (int32_t d = threadIdx.x; d < E.C.dim; d += 256) {
            E.C.k[dst + d] = E.C.k[src + d];
            E.C.v[dst + d] = E.C.v[src + d];
        }
    }
}

// The most tokens of a sequence and head that move: as many as come free below the budget, or lie past it.
int32_t most_moves(int32_t budget, int32_t len) {
    const int32_t past = len > budget ? len - budget : 0;
    return past < budget ? past : budget;
}

}  // namespace

extern "C" endor_status endor_kv_append(const endor_kv_cache *cache, const void *d_k_new, const void *d_v_new, int64_t seq_stride,
                                        int64_t token_stride, int64_t head_stride, int tokens, const int32_t *d_counts,
                                        const int32_t *d_lengths, const int32_t *d_seen, int32_t *d_lengths_out, int32_t *d_seen_out,
                                        float *d_weights, int32_t *d_positions, void *stream) {
    AppendParams A{};
    if (const endor_status st = read_cache(cache, &A.C)) return st;
    if (tokens < 0 || seq_stride < 0 || token_stride < 0 || head_stride < 0) return ENDOR_ERR_INVALID_ARG;
    if (A.C.batch == 0) return ENDOR_OK;
    if (!aligned(d_lengths, 4) || !aligned(d_seen, 4) || !aligned(d_lengths_out, 4) || !aligned(d_seen_out, 4)) return ENDOR_ERR_INVALID_ARG;
    if (tokens > 0 && (!aligned(d_k_new, 2) || !aligned(d_v_new, 2))) return ENDOR_ERR_INVALID_ARG;
    for (const void *p : {static_cast<const void *>(d_counts), static_cast<const void *>(d_weights), static_cast<const void *>(d_positions)})
        if (p && !aligned(p, 4)) return ENDOR_ERR_INVALID_ARG;
    A.k = static_cast<const uint16_t *>(d_k_new);
    A.v = static_cast<const uint16_t *>(d_v_new);
    A.seq_stride = seq_stride;
    A.token_stride = token_stride;
    A.head_stride = head_stride;
    A.counts = d_counts;
    A.lengths = d_lengths;
    A.seen = d_seen;
    A.lengths_out = d_lengths_out;
    A.seen_out = d_seen_out;
    A.weights = d_weights;
    A.positions = d_positions;
    A.tokens = tokens;
    A.capacity = capacity_of(*cache);
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (tokens > 0 && A.capacity > 0) {
        hipLaunchKernelGGL(endor_kv_append_kernel, dim3(tokens, A.C.batch), dim3(256), 0, s, A);
        if (hipGetLastError() != hipSuccess) return ENDOR_ERR_HIP;
    }
    hipLaunchKernelGGL(endor_kv_advance_kernel, dim3((A.C.batch + 255) / 256), dim3(256), 0, s, A);
    return hipGetLastError() == hipSuccess ? ENDOR_OK : ENDOR_ERR_HIP;
}

extern "C" size_t endor_kv_evict_scratch_bytes(const endor_kv_cache *cache, int32_t budget, int32_t max_len) {
    Cache C;
    if (read_cache(cache, &C) != ENDOR_OK || budget < 0 || max_len < 0) return 0;
    const int32_t cap = capacity_of(*cache);
    const size_t rows = size_t(C.batch) * C.kv_heads;
    const size_t n = 4 * rows * (1 + 2 * size_t(most_moves(budget, max_len < cap ? max_len : cap)));
    return (n + 255) & ~size_t(255);
}

extern "C" endor_status endor_kv_evict(const endor_kv_cache *cache, int32_t budget, int32_t recent, int32_t max_len, const int32_t *d_lengths,
                                       const int32_t *d_seen, const float *d_weights, const int32_t *d_positions, int32_t *d_lengths_out,
                                       float *d_weights_out, int32_t *d_positions_out, void *d_scratch, size_t scratch_bytes, void *stream) {
    EvictParams E{};
    if (const endor_status st = read_cache(cache, &E.C)) return st;
    if (budget < 0 || recent < 0 || recent > budget || max_len < 0) return ENDOR_ERR_INVALID_ARG;
    if (E.C.batch == 0) return ENDOR_OK;
    if (!aligned(d_lengths, 4) || !aligned(d_seen, 4) || !aligned(d_lengths_out, 4)) return ENDOR_ERR_INVALID_ARG;
    E.capacity = capacity_of(*cache);
    E.most_len = max_len < E.capacity ? max_len : E.capacity;
    if (E.capacity > 0 && (!aligned(d_weights, 4) || !aligned(d_positions, 4) || !aligned(d_weights_out, 4) || !aligned(d_positions_out, 4)))
        return ENDOR_ERR_INVALID_ARG;
    const size_t need = endor_kv_evict_scratch_bytes(cache, budget, max_len);
    if (!aligned(d_scratch, 256)) return ENDOR_ERR_INVALID_ARG;
    if (scratch_bytes < need) return ENDOR_ERR_BUFFER_TOO_SMALL;
    E.lengths = d_lengths;
    E.seen = d_seen;
    E.weights = d_weights;
    E.positions = d_positions;
    E.lengths_out = d_lengths_out;
    E.weights_out = d_weights_out;
    E.positions_out = d_positions_out;
    E.budget = budget;
    E.recent = recent;
    E.most = most_moves(budget, E.most_len);
    const int64_t rows = int64_t(E.C.batch) * E.C.kv_heads;
    E.count = static_cast<int32_t *>(d_scratch);
    E.holes = E.count + rows;
    E.movers = E.holes + rows * E.most;
    hipStream_t s = static_cast<hipStream_t>(stream);
    hipLaunchKernelGGL(endor_kv_select_kernel, dim3(E.C.kv_heads, E.C.batch), dim3(kSelectThreads), 0, s, E);
    if (hipGetLastError() != hipSuccess) return ENDOR_ERR_HIP;
    const int64_t want = E.most < 1 ? 1 : E.most;
    hipLaunchKernelGGL(endor_kv_move_kernel, dim3(static_cast<uint32_t>(want < 256 ? want : 256), E.C.kv_heads, E.C.batch), dim3(256), 0, s, E);
    return hipGetLastError() == hipSuccess ? ENDOR_OK : ENDOR_ERR_HIP;
}
