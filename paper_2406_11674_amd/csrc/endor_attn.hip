// Attention of one new token per sequence over a paged key-value cache (Section 3.1's generation, one token at a time):
//     s_t = scale <q, k_t>,  out = sum_t exp(s_t - lse) v_t,  lse = log sum_t exp(s_t),
// for all query heads that share a kv head in one pass over its keys and values.
//
// A wave takes 32 slots at a time.  Both products go to the matrix cores, with up to 16 query heads as the result's columns; one
// head alone leaves 15 of 16 columns empty, which costs nothing: an instruction takes 16 clocks for 1 KB of keys that memory
// brings in some 100.  S^T = K Q^T: a lane loads 16 bytes of the key of its row, straight into the operand's
// registers.  Its result has a lane hold, for the query of its column, slots 4g + 0..3 and 16 + 4g + 0..3 (g: its quarter of the wave), which
// is, with the slots in that order, the operand that O^T = V^T P^T wants: P never leaves the lane.  For V^T a lane loads, of those
// 8 slots, 16 bytes each at dims 8n.. (n: its place in the quarter, so a quarter reads whole rows) and turns the 8 x 8
// elements around in its registers (v_perm_b32): instruction j has dims 8m + j for rows m, and a lane ends up with 32 neighbouring
// dims of its query.  Neither operand passes through LDS.
//
// Softmax: the running maximum m is raised only when a logit passes it by 4 (in powers of two), so that sums are
// rescaled a few times in all; p = 2^(s - m + 11) then fills fp16's range (at most 2^15, and a p of 2^-35 of the largest still counts).
// P enters the second product in two parts of the type, high and remainder, so that of 32 bits 2^-16 (bf16) or 2^-20 (fp16) is
// lost and not 2^-9 or 2^-11: matrix instructions are not what bounds this.  m, the totals and all sums are fp32.
//
// A workgroup is four waves on one chunk of a sequence, joined in LDS; chunks are joined by a second kernel, which also
// adds the tokens' weights from the logits that the first one left behind.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "endor.h"
#include "endor_attn_plan.h"
#include "endor_device.h"
#include "endor_kv.h"

namespace {

using endor_attn_plan::kQueries;
using endor_attn_plan::kStep;
using endor_attn_plan::kTile;
using endor_attn_plan::kWaves;
using endor_attn_plan::make_plan;
using endor_attn_plan::Plan;
using endor_device::u32x4;
using endor_kv::aligned;
using endor_kv::Cache;
using endor_kv::capacity_of;
using endor_kv::clamp_length;
using endor_kv::read_cache;

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

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
    float *partial;   // [batch][q head][split][dim]: sums, relative to the split's maximum
    float2 *ml;       // [batch][q head][split]: maximum and total
    float *logits;    // [batch][q head][row], in powers of two; or NULL
    float scale2;     // scale * log2(e)
    int32_t q_heads, group, qtiles, most_len, capacity, chunk, splits, row;
};

constexpr float kShift = 11.0f;  // see the top
constexpr float kSlack = 4.0f;
constexpr float kLn2 = 0.69314718055994530942f;

template <bool kBf16>
__device__ __forceinline__ f32x4 product(u32x4 a, u32x4 b, f32x4 c) {
    if constexpr (kBf16)
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
}

// Two numbers as a pair of the type, cut off, and what that leaves of each.
template <bool kBf16>
__device__ __forceinline__ uint32_t high_part(float x, float y, float *rx, float *ry) {
    if constexpr (kBf16) {
        const uint32_t a = __float_as_uint(x), b = __float_as_uint(y);
        *rx = x - __uint_as_float(a & 0xffff0000u);
        *ry = y - __uint_as_float(b & 0xffff0000u);
        return __builtin_amdgcn_perm(b, a, 0x07060302u);
    } else {
        const auto h = __builtin_amdgcn_cvt_pkrtz(x, y);
        *rx = x - static_cast<float>(h[0]);
        *ry = y - static_cast<float>(h[1]);
        return __builtin_bit_cast(uint32_t, h);
    }
}
template <bool kBf16>
__device__ __forceinline__ uint32_t pair_of(float x, float y) {
    if constexpr (kBf16) {
        typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
        bf16x2 h;
        h[0] = static_cast<__bf16>(x);
        h[1] = static_cast<__bf16>(y);
        return __builtin_bit_cast(uint32_t, h);
    } else {
        typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
        f16x2 h;
        h[0] = static_cast<_Float16>(x);
        h[1] = static_cast<_Float16>(y);
        return __builtin_bit_cast(uint32_t, h);
    }
}
template <bool kBf16>
__device__ __forceinline__ uint16_t narrow(float x) {
    return static_cast<uint16_t>(pair_of<kBf16>(x, 0.0f));
}

// Over the four quarters of a wave, for every place in them.
__device__ __forceinline__ float quarters_max(float x) {
    x = fmaxf(x, __shfl_xor(x, 16));
    return fmaxf(x, __shfl_xor(x, 32));
}
__device__ __forceinline__ float quarters_sum(float x) {
    x += __shfl_xor(x, 16);
    return x + __shfl_xor(x, 32);
}

// kDim: 64, 128 or 256; a narrower head is treated as the next of them: lanes past it read its first elements instead, which meet zeros in q or
// end up in dims that nobody writes.
template <int kDim, bool kBf16>
__global__ __launch_bounds__(64 * kWaves, kDim == 256 ? 1 : kDim == 128 ? 2 : 4) void endor_attn_kernel(AttnParams A) {
    constexpr int kChunks = kDim / 32;                  // instructions of a key's dot product
    constexpr int kPer = kDim >= 128 ? 8 : 4;           // dims a lane loads of a value at once
    constexpr int kParts = kDim / (16 * kPer);          // such loads
    extern __shared__ float s_join[];                   // [wave][query][dim], then [wave][query][2]
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n = lane & 15, g = lane >> 4;
    const uint32_t split = blockIdx.x, b = blockIdx.z;
    const uint32_t kv = blockIdx.y / A.qtiles, qt = blockIdx.y % A.qtiles;
    const int32_t length = clamp_length(A.lengths[b], A.most_len);
    const int32_t first = static_cast<int32_t>(split) * A.chunk;
    if (first >= length && split > 0) return;  // the first workgroup writes an empty sequence's outputs
    const int32_t past = first + A.chunk < length ? first + A.chunk : length;
    const int32_t end = A.C.num_pages ? past : first;  // without a pool there is nothing to read
    const int32_t queries = A.group - static_cast<int32_t>(qt) * kQueries < kQueries ? A.group - static_cast<int32_t>(qt) * kQueries : kQueries;
    const int32_t head0 = static_cast<int32_t>(kv) * A.group + static_cast<int32_t>(qt) * kQueries;  // the query head of column 0
    const uint32_t dim = A.C.dim;

    u32x4 q[kChunks];
#pragma unroll
    for (int c = 0; c < kChunks; ++c) {
        typedef u32x4 u32x4_any __attribute__((aligned(2)));
        q[c] = u32x4{0, 0, 0, 0};
        if (static_cast<int32_t>(n) < queries && 32 * c + 8 * g < dim)
            q[c] = *reinterpret_cast<const u32x4_any *>(A.q + int64_t(b) * A.q_seq_stride + int64_t(head0 + n) * A.q_head_stride + 32 * c + 8 * g);
    }

    f32x4 o[kParts][kPer];  // row 4g + i of instruction j: dim 16 kPer part + kPer (4g + i) + j
#pragma unroll
    for (int p = 0; p < kParts; ++p)
#pragma unroll
        for (int j = 0; j < kPer; ++j) o[p][j] = f32x4{0, 0, 0, 0};
    float top = -INFINITY, total = 0;

    const int32_t tiles = (end - first + kTile - 1) / kTile;  // of the chunk; this wave's: wave, wave + kWaves, ...
    if (static_cast<int32_t>(wave) < tiles) {
        const int32_t *table = A.C.pages + int64_t(b) * A.C.pages_stride;
        const uint64_t *mask = A.mask ? A.mask + int64_t(b) * A.mask_stride : nullptr;
        const uint16_t *kbase = A.C.k + int64_t(kv) * A.C.head_stride, *vbase = A.C.v + int64_t(kv) * A.C.head_stride;
        const uint32_t in_page = (1u << A.C.page_shift) - 1;
        uint32_t kdim[kChunks], vdim[kParts];
#pragma unroll
        for (int c = 0; c < kChunks; ++c) kdim[c] = 32 * c + 8 * g < dim ? 32 * c + 8 * g : 0;
#pragma unroll
        for (int p = 0; p < kParts; ++p) vdim[p] = 16 * kPer * p + kPer * n < dim ? 16 * kPer * p + kPer * n : 0;

        struct Pages {
            uint32_t k0, k1, v0, v1;  // of slots n, 16 + n, 4g and 16 + 4g of a tile
        };
        // Slots past the end stand for the last one, whose page is there to be looked up.
        auto pages_of = [&](int32_t t0) {
            auto at = [&](uint32_t t) { return static_cast<uint32_t>(table[(static_cast<int32_t>(t) < end ? t : end - 1) >> A.C.page_shift]); };
            return Pages{at(t0 + n), at(t0 + 16 + n), at(t0 + 4 * g), at(t0 + 16 + 4 * g)};
        };
        // A page that is not there is read as page 0, which is, and its slots are not visible.
        auto row_of = [&](uint32_t page, uint32_t t) {
            const uint32_t slot = static_cast<int32_t>(t) < end ? t : end - 1;
            return int64_t(page < A.C.num_pages ? page : 0) * A.C.page_stride + int64_t(slot & in_page) * A.C.slot_stride;
        };
        u32x4 k[2][kChunks];
        auto load_keys = [&](int32_t t0, const Pages &p) {
            const uint16_t *r0 = kbase + row_of(p.k0, t0 + n), *r1 = kbase + row_of(p.k1, t0 + 16 + n);
#pragma unroll
            for (int c = 0; c < kChunks; ++c) {
                k[0][c] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(r0 + kdim[c]));
                k[1][c] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(r1 + kdim[c]));
            }
        };
        typedef uint32_t Value __attribute__((ext_vector_type(kPer / 2)));
        Value v[8][kParts];
        auto load_values = [&](int32_t t0, const Pages &p) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {  // four slots lie on one page: pages hold a multiple of 8
                const uint32_t t = t0 + 4 * g + (e & 3) + (e & 4) * 4;
                const uint16_t *r = vbase + row_of(e < 4 ? p.v0 : p.v1, t);
#pragma unroll
                for (int part = 0; part < kParts; ++part)
                    v[e][part] = __builtin_nontemporal_load(reinterpret_cast<const Value *>(r + vdim[part]));
            }
        };

        int32_t t0 = first + kTile * static_cast<int32_t>(wave);
        Pages now = pages_of(t0), next = pages_of(t0 + kStep);
        load_keys(t0, now);
        for (; t0 < end; t0 += kStep) {
            // Loads come back in order, so what is wanted first goes out first: the pages of the tile after the next one, this tile's values; the
            // next tile's keys follow when this one's have been used.
            const Pages later = pages_of(t0 + 2 * kStep);
            load_values(t0, now);
            uint32_t seen;  // bit i: slot t0 + i is visible
            {
                const uint64_t a = __ballot(static_cast<int32_t>(t0 + n) < end && now.k0 < A.C.num_pages);
                const uint64_t z = __ballot(static_cast<int32_t>(t0 + 16 + n) < end && now.k1 < A.C.num_pages);
                seen = static_cast<uint32_t>(a & 0xffffu) | static_cast<uint32_t>(z & 0xffffu) << 16;
                if (mask) seen &= static_cast<uint32_t>(mask[t0 >> 6] >> (t0 & 32));
            }
            f32x4 s[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
#pragma unroll
            for (int c = 0; c < kChunks; ++c) {
                s[0] = product<kBf16>(k[0][c], q[c], s[0]);
                s[1] = product<kBf16>(k[1][c], q[c], s[1]);
            }
            load_keys(t0 + kStep, next);
#pragma unroll
            for (int j = 0; j < 2; ++j) s[j] *= A.scale2;
            if (seen != 0xffffffffu) {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const bool in = seen >> (4 * g + (e & 3) + (e & 4) * 4) & 1;
                    if (!in) s[e >> 2][e & 3] = -INFINITY;
#pragma unroll
                    for (int part = 0; part < kParts; ++part) v[e][part] = in ? v[e][part] : Value(0);  // not even a NaN may count
                }
            }
            if (A.logits && static_cast<int32_t>(n) < queries) {
                float *to = A.logits + (int64_t(b) * A.q_heads + head0 + n) * A.row + t0 + 4 * g;
                *reinterpret_cast<f32x4 *>(to) = s[0];
                *reinterpret_cast<f32x4 *>(to + 16) = s[1];
            }
            float most = fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3])), fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3])));
            if (__ballot(most > top + kSlack)) {
                const float raised = fmaxf(top, quarters_max(most));
                const float keep = top == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(top - raised);
                top = raised;
                total *= keep;
#pragma unroll
                for (int p = 0; p < kParts; ++p)
#pragma unroll
                    for (int j = 0; j < kPer; ++j) o[p][j] *= keep;
            }
            const float base = top == -INFINITY ? 0.0f : top - kShift;
            float p[8], rest[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                p[e] = __builtin_amdgcn_exp2f(s[e >> 2][e & 3] - base);
                total += p[e];
            }
            u32x4 hi, lo;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                hi[e] = high_part<kBf16>(p[2 * e], p[2 * e + 1], &rest[2 * e], &rest[2 * e + 1]);
                lo[e] = pair_of<kBf16>(rest[2 * e], rest[2 * e + 1]);
            }
#pragma unroll
            for (int part = 0; part < kParts; ++part)
#pragma unroll
                for (int j = 0; j < kPer; ++j) {
                    u32x4 a;
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        a[e] = __builtin_amdgcn_perm(v[2 * e + 1][part][j / 2], v[2 * e][part][j / 2], j & 1 ? 0x07060302u : 0x05040100u);
                    o[part][j] = product<kBf16>(a, hi, o[part][j]);
                    o[part][j] = product<kBf16>(a, lo, o[part][j]);
                }
            now = next;
            next = later;
        }
    }
    total = quarters_sum(total);

    // Join the waves: every wave leaves its sums and its maximum; a thread then adds up single elements of the result.
    float *s_ml = s_join + kWaves * queries * kDim;
    if (static_cast<int32_t>(n) < queries) {
        float *mine = s_join + (wave * queries + n) * kDim;
#pragma unroll
        for (int p = 0; p < kParts; ++p)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < kPer; ++j) mine[16 * kPer * p + kPer * (4 * g + i) + j] = o[p][j][i];
        if (g == 0) {
            s_ml[2 * (wave * queries + n)] = top;
            s_ml[2 * (wave * queries + n) + 1] = total;
        }
    }
    __syncthreads();
    for (int32_t i = threadIdx.x; i < queries * kDim; i += 64 * kWaves) {
        const int32_t h = i / kDim, d = i % kDim;
        float m = -INFINITY, sum = 0, all = 0;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) m = fmaxf(m, s_ml[2 * (w * queries + h)]);
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const float its = s_ml[2 * (w * queries + h)], share = its == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(its - m);
            all += share * s_ml[2 * (w * queries + h) + 1];
            sum += share * s_join[(w * queries + h) * kDim + d];
        }
        if (d >= static_cast<int32_t>(dim)) continue;
        const int64_t row = int64_t(b) * A.q_heads + head0 + h;
        if (A.splits == 1) {
            A.out[row * dim + d] = narrow<kBf16>(all == 0 ? 0.0f : sum / all);
            if (d == 0 && A.lse) A.lse[row] = all == 0 ? -INFINITY : (m - kShift + log2f(all)) * kLn2;
        } else {
            A.partial[(row * A.splits + split) * dim + d] = sum;
        }
        if (d == 0 && A.ml) A.ml[row * A.splits + split] = make_float2(m, all);
    }
}

// Maximum and total of a query head over its sequence's splits; every lane of the wave gets them.
__device__ __forceinline__ float2 joined(const float2 *ml, int32_t splits, uint32_t lane) {
    float m = -INFINITY, all = 0;
    for (int32_t s0 = 0; s0 < splits; s0 += 256) {  // four splits of every lane on their way
        float2 x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int32_t s = s0 + 64 * i + static_cast<int32_t>(lane);
            x[i] = ml[s < splits ? s : splits - 1];
            if (s >= splits) x[i] = make_float2(-INFINITY, 0.0f);
        }
        float most = m;
#pragma unroll
        for (int i = 0; i < 4; ++i) most = fmaxf(most, x[i].x);
        all = m == -INFINITY ? 0.0f : all * __builtin_amdgcn_exp2f(m - most);
        m = most;
#pragma unroll
        for (int i = 0; i < 4; ++i) all += x[i].x == -INFINITY ? 0.0f : x[i].y * __builtin_amdgcn_exp2f(x[i].x - m);
    }
    float most = m;
    for (int d = 32; d; d >>= 1) most = fmaxf(most, __shfl_xor(most, d));
    all = m == -INFINITY ? 0.0f : all * __builtin_amdgcn_exp2f(m - most);
    for (int d = 32; d; d >>= 1) all += __shfl_xor(all, d);
    return make_float2(most, all);
}

constexpr int kJoinThreads = 512;
constexpr int kSlots = 2048;  // slots of a workgroup that adds weights

// Workgroups below batch * q_heads join a head's splits (if there are several): a thread takes four dims of every so many splits.  The others add the
// weights of kSlots slots of a kv head.
template <bool kBf16>
__global__ __launch_bounds__(kJoinThreads) void endor_attn_join_kernel(AttnParams A, uint32_t joins, uint32_t pieces) {
    __shared__ f32x4 s_sum[kJoinThreads];
    __shared__ float s_off[256];
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if (blockIdx.x < joins) {
        const int64_t row = blockIdx.x, b = row / A.q_heads;
        const int32_t length = clamp_length(A.lengths[b], A.most_len), dim = A.C.dim;
        const int32_t splits = length > 0 ? (length + A.chunk - 1) / A.chunk : 1;
        const float2 *ml = A.ml + row * A.splits;
        const int32_t units = dim / 4, lines = kJoinThreads / units, line = threadIdx.x / units, d = 4 * (threadIdx.x % units);
        const float *from = A.partial + row * A.splits * dim + d;
        const float2 all = joined(ml, splits, lane);
        f32x4 sum = {0, 0, 0, 0};
        if (line < lines)
            for (int32_t s0 = line; s0 < splits; s0 += 4 * lines) {
                f32x4 x[4];
                float share[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int32_t s = s0 + i * lines < splits ? s0 + i * lines : s0;
                    x[i] = *reinterpret_cast<const f32x4 *>(from + int64_t(s) * dim);
                    share[i] = ml[s].x;
                }
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (s0 + i * lines < splits && share[i] != -INFINITY) sum += __builtin_amdgcn_exp2f(share[i] - all.x) * x[i];
            }
        s_sum[threadIdx.x] = sum;
        __syncthreads();
        if (static_cast<int32_t>(threadIdx.x) < dim) {
            const float *part = reinterpret_cast<const float *>(s_sum) + threadIdx.x;
            float x = 0;
            for (int32_t l = 0; l < lines && l < splits; ++l) x += part[l * dim];
            A.out[row * dim + threadIdx.x] = narrow<kBf16>(all.y == 0 ? 0.0f : x / all.y);
        }
        if (threadIdx.x == 0 && A.lse) A.lse[row] = all.y == 0 ? -INFINITY : (all.x - kShift + log2f(all.y)) * kLn2;
        return;
    }
    const uint32_t unit = (blockIdx.x - joins) / pieces, piece = (blockIdx.x - joins) % pieces;
    const uint32_t b = unit / A.C.kv_heads, kv = unit % A.C.kv_heads;
    const int32_t length = clamp_length(A.lengths[b], A.most_len);
    const int32_t t0 = static_cast<int32_t>(piece) * kSlots;
    if (t0 >= length) return;
    const int32_t splits = (length + A.chunk - 1) / A.chunk;
    const int64_t row0 = int64_t(b) * A.q_heads + int64_t(kv) * A.group;
    // four slots to a thread; rows of logits are whole tiles, so that a unit that begins below the length can be read
    const int32_t t = t0 + 4 * static_cast<int32_t>(threadIdx.x);
    const bool in = t < length;
    typedef f32x4 f32x4_any __attribute__((aligned(4)));
    const int64_t at = (int64_t(b) * A.C.kv_heads + kv) * A.capacity + t;
    f32x4 sum = {0, 0, 0, 0};
    if (in && A.weights) sum = *reinterpret_cast<const f32x4_any *>(A.weights + at);  // the capacity is whole pages, of 8 slots at least
    f32x4 added = {0, 0, 0, 0};
    for (int32_t h0 = 0; h0 < A.group && A.C.num_pages; h0 += 256) {
        const int32_t heads = A.group - h0 < 256 ? A.group - h0 : 256;
        __syncthreads();
        for (int32_t h = wave; h < heads; h += kJoinThreads / 64) {
            const float2 all = joined(A.ml + (row0 + h0 + h) * A.splits, splits, lane);
            // what is taken off a logit: all of them are -infinity where nothing is visible
            if (lane == 0) s_off[h] = all.y == 0 ? 0.0f : all.x - kShift + log2f(all.y);
        }
        __syncthreads();
        if (in) {
            const float *logit = A.logits + (row0 + h0) * A.row + t;
#pragma unroll 4
            for (int32_t h = 0; h < heads; ++h) {
                const f32x4 s = *reinterpret_cast<const f32x4 *>(logit + int64_t(h) * A.row);
#pragma unroll
                for (int i = 0; i < 4; ++i) added[i] += __builtin_amdgcn_exp2f(s[i] - s_off[h]);
            }
        }
    }
    sum += added;
    if (t + 4 <= length) {
        *reinterpret_cast<f32x4_any *>(A.weights_out + at) = sum;
    } else if (in) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (t + i < length) A.weights_out[at + i] = sum[i];
    }
}

template <int kDim, bool kBf16>
void launch_attn(const AttnParams &A, hipStream_t s) {
    const int queries = A.group < kQueries ? A.group : kQueries;
    hipLaunchKernelGGL((endor_attn_kernel<kDim, kBf16>), dim3(A.splits, A.C.kv_heads * A.qtiles, A.C.batch), dim3(64 * kWaves),
                       kWaves * queries * (kDim + 2) * sizeof(float), s, A);
}
template <bool kBf16>
void launch_dim(const AttnParams &A, hipStream_t s) {
    if (A.C.dim <= 64)
        launch_attn<64, kBf16>(A, s);
    else if (A.C.dim <= 128)
        launch_attn<128, kBf16>(A, s);
    else
        launch_attn<256, kBf16>(A, s);
}

}  // namespace

extern "C" size_t endor_attn_scratch_bytes(const endor_kv_cache *cache, int q_heads, int32_t max_len, int with_weights) {
    Cache C;
    if (read_cache(cache, &C) != ENDOR_OK || q_heads < 1 || q_heads % C.kv_heads != 0 || max_len < 0) return 0;
    const int32_t cap = capacity_of(*cache);
    return make_plan(C.batch, C.kv_heads, q_heads, C.dim, max_len < cap ? max_len : cap, with_weights != 0).bytes;
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
    const Plan p = make_plan(A.C.batch, A.C.kv_heads, q_heads, A.C.dim, A.most_len, d_weights_out != nullptr);
    if (p.bytes && !aligned(d_scratch, 256)) return ENDOR_ERR_INVALID_ARG;
    if (scratch_bytes < p.bytes) return ENDOR_ERR_BUFFER_TOO_SMALL;
    A.q = static_cast<const uint16_t *>(d_q);
    A.q_seq_stride = q_seq_stride;
    A.q_head_stride = q_head_stride;
    A.lengths = d_lengths;
    A.mask = d_mask;
    A.mask_stride = mask_stride;
    A.out = static_cast<uint16_t *>(d_out);
    A.lse = d_lse;
    A.weights = d_weights;
    A.weights_out = d_weights_out;
    char *scratch = static_cast<char *>(d_scratch);
    A.partial = reinterpret_cast<float *>(scratch);
    A.ml = p.ml ? reinterpret_cast<float2 *>(scratch + p.partial) : nullptr;
    A.logits = p.logits ? reinterpret_cast<float *>(scratch + p.partial + p.ml) : nullptr;
    A.scale2 = scale * 1.44269504088896340736f;
    A.q_heads = q_heads;
    A.group = p.group;
    A.qtiles = p.qtiles;
    A.chunk = p.chunk;
    A.splits = p.splits;
    A.row = p.row;
    hipStream_t s = static_cast<hipStream_t>(stream);
    const bool bf16 = cache->dtype == ENDOR_BF16;
    if (bf16)
        launch_dim<true>(A, s);
    else
        launch_dim<false>(A, s);
    if (hipGetLastError() != hipSuccess) return ENDOR_ERR_HIP;
    const uint32_t joins = p.splits > 1 ? static_cast<uint32_t>(A.C.batch) * q_heads : 0;
    const uint32_t pieces = d_weights_out ? (A.most_len + kSlots - 1) / kSlots : 0;
    const uint32_t groups = joins + pieces * static_cast<uint32_t>(A.C.batch) * A.C.kv_heads;
    if (groups) {
        hipLaunchKernelGGL(bf16 ? endor_attn_join_kernel<true> : endor_attn_join_kernel<false>, dim3(groups), dim3(kJoinThreads), 0, s, A, joins, pieces);
        if (hipGetLastError() != hipSuccess) return ENDOR_ERR_HIP;
    }
    return ENDOR_OK;
}
