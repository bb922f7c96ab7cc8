// Attention of one new token per sequence over a paged key-value cache (Section 3.1's generation, one token at a time):
//     s_t = scale <q, k_t>,  out = sum_t exp(s_t - lse) v_t,  lse = log sum_t exp(s_t),
// for all query heads that share a kv head in one pass over its keys and values.
//
// A wave takes 32 slots at a time. Both products go to the matrix cores, with up to 16 query heads as the result's
// columns; one head alone leaves 15 of 16 columns empty, which costs nothing: an instruction takes 16 clocks for 1 KB
// of keys that memory brings in some 100. S^T = K Q^T: a lane loads 16 bytes of the key of its row, straight into the
// operand's registers. Its result has a lane hold, for the query of its column, slots 4g + 0..3 and 16 + 4g + 0..3 (g:
// its quarter of the wave), which is, with the slots in that order, the operand that O^T = V^T P^T wants: P never
// leaves the lane. For V^T a lane loads, of those 8 slots, 16 bytes each at dims 8n.. (n: its place in the quarter, so
// a quarter reads whole rows) and turns the 8 x 8 elements around in its registers (v_perm_b32): instruction j has dims
// 8m + j for rows m, and a lane ends up with 32 neighbouring dims of its query. Neither operand passes through LDS.
//
// Softmax: the running maximum m is raised only when a logit passes it by 4 (in powers of two), so that sums are
// rescaled a few times in all; p = 2^(s - m + 11) then fills fp16's range (at most 2^15, and a p of 2^-35 of the
// largest still counts). P enters the second product in two parts of the type, high and remainder, so that of 32 bits
// 2^-16 (bf16) or 2^-20 (fp16) is lost and not 2^-9 or 2^-11: matrix instructions are not what bounds this. m, the
// totals and all sums are fp32.
//
// Short sequences take one launch, a workgroup for a kv head's queries; longer ones are cut into parts, a workgroup
// each, which a second kernel joins; it also adds the tokens' weights, from the logits that the first one left behind.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "endor.h"
#include "endor_attn_plan.h"
#include "endor_device.h"
#include "endor_kv.h"

namespace {

using endor_attn_plan::kQueries;
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
    float *partial;   // [batch][q head][part][dim]: sums, relative to the part's maximum
    float2 *ml;       // [batch][q head][part]: maximum and total
    float *logits;    // [batch][q head][row], in powers of two; or NULL
    float scale2;     // scale * log2(e)
    int32_t q_heads, group, qtiles, most_len, capacity, row;
    uint32_t units, least, chunk, even, splits;  // units of a sequence; slots of a part: at least, where lengths differ; parts where they are alike, at most
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

// What a wave does with a tile, and what it has of one on its way.
//
// kDim: 64, 128 or 256; a narrower head is treated as the next of them: lanes past it read its first elements instead,
// which are cleared before they meet the zeros in q, or end up in dims that nobody writes. kSub: runs of 32 slots that a wave takes at a time, so
// that narrow heads keep as many bytes on their way.
template <int kDim, int kSub, bool kBf16>
struct Tiles {
    static constexpr int kChunks = kDim / 32;          // instructions of a key's dot product
    static constexpr int kPer = kDim >= 128 ? 8 : 4;   // dims a lane loads of a value at once
    static constexpr int kParts = kDim / (16 * kPer);  // such loads
    static constexpr uint32_t kSlots = 32 * kSub;
    typedef uint32_t Value __attribute__((ext_vector_type(kPer / 2)));

    // One unit of work: a sequence's kv head and up to 16 of the query heads that read it.
    struct Unit {
        const int32_t *table;
        const uint64_t *mask;
        int64_t head;              // element offset of the kv head in a page
        uint32_t length;           // slots of the sequence, 0 without a pool
        int32_t queries, head0;    // the query heads: how many, and the first of the sequence's
        int64_t row;               // of the first one's outputs
    };
    static __device__ __forceinline__ Unit unit_of(const AttnParams &A, uint32_t b, uint32_t of_sequence, uint32_t length) {
        const uint32_t kv = of_sequence / A.qtiles, qt = of_sequence % A.qtiles;
        Unit u;
        u.table = A.C.pages + int64_t(b) * A.C.pages_stride;
        u.mask = A.mask ? A.mask + int64_t(b) * A.mask_stride : nullptr;
        u.head = int64_t(kv) * A.C.head_stride;
        u.length = length;
        u.queries = A.group - static_cast<int32_t>(qt) * kQueries < kQueries ? A.group - static_cast<int32_t>(qt) * kQueries : kQueries;
        u.head0 = static_cast<int32_t>(kv) * A.group + static_cast<int32_t>(qt) * kQueries;
        u.row = int64_t(b) * A.q_heads + u.head0;
        return u;
    }

    struct Pages {
        uint32_t k[2 * kSub], v[2 * kSub];  // of slots n and 4g of every 16 of a tile
    };
    const AttnParams &A;
    const uint32_t n, g;  // place in the quarter of the wave, quarter
    uint32_t kdim[kChunks], vdim[kParts];
    u32x4 q[kChunks], k[2 * kSub][kChunks];
    Value v[kSub][8][kParts];
    f32x4 o[kParts][kPer];  // row 4g + i of instruction j: dim 16 kPer part + kPer (4g + i) + j
    float top, total;

    __device__ __forceinline__ Tiles(const AttnParams &a, uint32_t lane) : A(a), n(lane & 15), g(lane >> 4) {
        const uint32_t dim = A.C.dim;
#pragma unroll
        for (int c = 0; c < kChunks; ++c) kdim[c] = 32 * c + 8 * g < dim ? 32 * c + 8 * g : 0;
#pragma unroll
        for (int p = 0; p < kParts; ++p) vdim[p] = 16 * kPer * p + kPer * n < dim ? 16 * kPer * p + kPer * n : 0;
    }
    // Nothing added up yet.
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int p = 0; p < kParts; ++p)
#pragma unroll
            for (int j = 0; j < kPer; ++j) o[p][j] = f32x4{0, 0, 0, 0};
        top = -INFINITY;
        total = 0;
    }
    __device__ __forceinline__ void load_query(const Unit &u, uint32_t b) {
        typedef u32x4 u32x4_any __attribute__((aligned(2)));
#pragma unroll
        for (int c = 0; c < kChunks; ++c) {
            q[c] = u32x4{0, 0, 0, 0};
            if (static_cast<int32_t>(n) < u.queries && 32 * c + 8 * g < static_cast<uint32_t>(A.C.dim))
                q[c] = *reinterpret_cast<const u32x4_any *>(A.q + int64_t(b) * A.q_seq_stride + int64_t(u.head0 + n) * A.q_head_stride + 32 * c + 8 * g);
        }
    }
    // Slots from `most` on stand for the one below it, whose page is there to be looked up, if not to be read.
    __device__ __forceinline__ Pages pages_of(const int32_t *table, uint32_t t0, uint32_t most) const {
        Pages p;
#pragma unroll
        for (int j = 0; j < 2 * kSub; ++j) {
            const uint32_t a = t0 + 16 * j + n, z = t0 + 16 * j + 4 * g;
            p.k[j] = table[(a < most ? a : most - 1) >> A.C.page_shift];
            p.v[j] = table[(z < most ? z : most - 1) >> A.C.page_shift];
        }
        return p;
    }
    // A page that is not there is read as page 0, which is, and its slots are not visible; so are those past the
    // length.
    __device__ __forceinline__ int64_t row_of(uint32_t page, uint32_t t, uint32_t length) const {
        const uint32_t slot = (t < length ? t : length - 1) & ((1u << A.C.page_shift) - 1);
        return int64_t(page < A.C.num_pages ? page : 0) * A.C.page_stride + int64_t(slot) * A.C.slot_stride;
    }
    __device__ __forceinline__ void load_keys(const Unit &u, uint32_t t0, const Pages &p) {
#pragma unroll
        for (int j = 0; j < 2 * kSub; ++j) {
            const uint16_t *r = A.C.k + u.head + row_of(p.k[j], t0 + 16 * j + n, u.length);
#pragma unroll
            for (int c = 0; c < kChunks; ++c) k[j][c] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(r + kdim[c]));
        }
    }
    __device__ __forceinline__ void load_values(const Unit &u, uint32_t t0, const Pages &p) {
#pragma unroll
        for (int s = 0; s < kSub; ++s)
#pragma unroll
            for (int e = 0; e < 8; ++e) {  // four slots lie on one page: pages hold a multiple of 8
                const uint16_t *r = A.C.v + u.head + row_of(p.v[2 * s + e / 4], t0 + 32 * s + 16 * (e / 4) + 4 * g + (e & 3), u.length);
#pragma unroll
                for (int part = 0; part < kParts; ++part)
                    v[s][e][part] = __builtin_nontemporal_load(reinterpret_cast<const Value *>(r + vdim[part]));
            }
    }
    static __device__ __forceinline__ uint64_t mask_of(const Unit &u, uint32_t t0) {
        return u.mask ? u.mask[(t0 < u.length ? t0 : u.length - 1) >> 6] : ~uint64_t(0);
    }
    // The logits of the tile whose keys are loaded, in powers of two; `next` puts out the next tile's keys once these
    // are used.
    template <class Next>
    __device__ __forceinline__ void logits_of(f32x4 (&s)[2 * kSub], Next next) {
        // What lanes past a narrower head have read of its beginning may be an infinity, of which zeros in q make NaN.
        // (Heads of 40, 80, 96 and 200 take as long as without.)
        if (A.C.dim < kDim)
#pragma unroll
            for (int j = 0; j < 2 * kSub; ++j)
#pragma unroll
                for (int c = 0; c < kChunks; ++c) k[j][c] = 32 * c + 8 * g < static_cast<uint32_t>(A.C.dim) ? k[j][c] : u32x4{0, 0, 0, 0};
#pragma unroll
        for (int j = 0; j < 2 * kSub; ++j) {
            s[j] = f32x4{0, 0, 0, 0};
#pragma unroll
            for (int c = 0; c < kChunks; ++c) s[j] = product<kBf16>(k[j][c], q[c], s[j]);
        }
        next();
#pragma unroll
        for (int j = 0; j < 2 * kSub; ++j) s[j] *= A.scale2;
    }
    // Hides slots: past the length, on pages that are not there, or by the mask's word.
    __device__ __forceinline__ void hide(f32x4 (&s)[2 * kSub], uint32_t t0, uint32_t length, const Pages &p, uint64_t word) {
        uint32_t seen[kSub];  // bit i: slot t0 + 32 u + i is visible
        bool all_seen = true;
#pragma unroll
        for (int u = 0; u < kSub; ++u) {
            const uint32_t at = t0 + 32 * u;
            const uint64_t a = __ballot(at + n < length && p.k[2 * u] < A.C.num_pages);
            const uint64_t z = __ballot(at + 16 + n < length && p.k[2 * u + 1] < A.C.num_pages);
            seen[u] = (static_cast<uint32_t>(a & 0xffffu) | static_cast<uint32_t>(z & 0xffffu) << 16) & static_cast<uint32_t>(word >> (at & 32));
            all_seen = all_seen && seen[u] == 0xffffffffu;
        }
        if (all_seen) return;
#pragma unroll
        for (int u = 0; u < kSub; ++u)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const bool in = seen[u] >> (4 * g + (e & 3) + (e & 4) * 4) & 1;
                if (!in) s[2 * u + e / 4][e & 3] = -INFINITY;
#pragma unroll
                for (int part = 0; part < kParts; ++part) v[u][e][part] = in ? v[u][e][part] : Value(0);  // not even a NaN may count
            }
    }
    // Adds the tile whose logits and values these are.
    __device__ __forceinline__ void add(const f32x4 (&s)[2 * kSub]) {
        float highest = s[0][0];
#pragma unroll
        for (int j = 0; j < 2 * kSub; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) highest = fmaxf(highest, s[j][i]);
        if (__ballot(highest > top + kSlack)) {
            const float raised = fmaxf(top, quarters_max(highest));
            const float keep = top == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(top - raised);
            top = raised;
            total *= keep;
#pragma unroll
            for (int p = 0; p < kParts; ++p)
#pragma unroll
                for (int j = 0; j < kPer; ++j) o[p][j] *= keep;
        }
        const float base = top == -INFINITY ? 0.0f : top - kShift;
#pragma unroll
        for (int u = 0; u < kSub; ++u) {
            float p[8], rest[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                p[e] = __builtin_amdgcn_exp2f(s[2 * u + e / 4][e & 3] - base);
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
                        a[e] = __builtin_amdgcn_perm(v[u][2 * e + 1][part][j / 2], v[u][2 * e][part][j / 2], j & 1 ? 0x07060302u : 0x05040100u);
                    o[part][j] = product<kBf16>(a, hi, o[part][j]);
                    o[part][j] = product<kBf16>(a, lo, o[part][j]);
                }
        }
    }
    // f(dim, four sums from it on) for all that the lane holds of its query
    template <class F>
    __device__ __forceinline__ void each_sum(F f) const {
#pragma unroll
        for (int p = 0; p < kParts; ++p)
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < kPer; j += 4)
                    f(16 * kPer * p + kPer * (4 * g + i) + j, f32x4{o[p][j][i], o[p][j + 1][i], o[p][j + 2][i], o[p][j + 3][i]});
    }
};

__device__ __forceinline__ float lse_of(float top, float total) { return total == 0 ? -INFINITY : (top - kShift + log2f(total)) * kLn2; }
// What is taken off a logit to make it a weight: all of them are -infinity where nothing is visible.
__device__ __forceinline__ float offset_of(float top, float total) { return total == 0 ? 0.0f : top - kShift + log2f(total); }

// Joins a workgroup's waves: every wave leaves its sums and its maximum in LDS, then a thread adds up single elements:
// f(query, dim, sum, maximum, total).
template <class T, int kWaves, class F>
__device__ __forceinline__ void join_waves(const AttnParams &A, const typename T::Unit &u, const T &tiles, float *s_join, F f) {
    constexpr int kDim = 16 * T::kPer * T::kParts;
    const uint32_t wave = threadIdx.x >> 6;
    float *s_ml = s_join + kWaves * u.queries * kDim;
    const float total = quarters_sum(tiles.total);
    if (static_cast<int32_t>(tiles.n) < u.queries) {
        float *mine = s_join + (wave * u.queries + tiles.n) * kDim;
        tiles.each_sum([&](uint32_t d, f32x4 x) { *reinterpret_cast<f32x4 *>(mine + d) = x; });
        if (tiles.g == 0) {
            s_ml[2 * (wave * u.queries + tiles.n)] = tiles.top;
            s_ml[2 * (wave * u.queries + tiles.n) + 1] = total;
        }
    }
    __syncthreads();
    for (int32_t i = threadIdx.x; i < u.queries * kDim; i += 64 * kWaves) {
        const int32_t h = i / kDim, d = i % kDim;
        float m = -INFINITY, sum = 0, all = 0;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) m = fmaxf(m, s_ml[2 * (w * u.queries + h)]);
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const float its = s_ml[2 * (w * u.queries + h)], share = its == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(its - m);
            all += share * s_ml[2 * (w * u.queries + h) + 1];
            sum += share * s_join[(w * u.queries + h) * kDim + d];
        }
        if (d < A.C.dim) f(h, d, sum, m, all);
    }
}

// Short sequences: one workgroup for a unit, its waves take the tiles in turn and are joined in LDS. The weights too
// are added here, from logits in LDS (`pitch` floats a query; a group of more than 16 query heads goes by the other
// form, for two workgroups would add to the same weights). 131 slots, 64 query heads over 8 of 128: 7.2 us, of which the
// dependent trips to memory (the length and the page, the keys, the values) and the launch are nearly all.
template <int kDim, int kWaves, bool kBf16>
__global__ __launch_bounds__(64 * kWaves) void endor_attn_kernel(AttnParams A, uint32_t pitch) {
    typedef Tiles<kDim, 1, kBf16> T;
    constexpr uint32_t kStep = kWaves * T::kSlots;
    extern __shared__ float s_join[];  // [wave][query][dim], [wave][query][2], [query] offsets (whole fours), [query][pitch]
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t b = blockIdx.y, dim = A.C.dim, most = A.most_len;
    T tiles(A, lane);
    tiles.clear();
    uint32_t t0 = T::kSlots * wave;
    typename T::Pages now{}, next{};
    if (most > 0) {  // on their way beside the length
        const int32_t *table = A.C.pages + int64_t(b) * A.C.pages_stride;
        now = tiles.pages_of(table, t0, most);
        next = tiles.pages_of(table, t0 + kStep, most);
    }
    const uint32_t held = clamp_length(A.lengths[b], A.most_len);
    const typename T::Unit u = T::unit_of(A, b, blockIdx.x, A.C.num_pages ? held : 0);
    float *s_ml = s_join + kWaves * u.queries * kDim, *s_off = s_ml + 2 * kWaves * u.queries, *s_logits = s_off + (u.queries + 3) / 4 * 4;
    if (t0 < u.length) {
        tiles.load_keys(u, t0, now);
        tiles.load_query(u, b);
        uint64_t word = T::mask_of(u, t0);
        for (; t0 < u.length; t0 += kStep) {
            // Loads come back in order, so what is wanted first goes out first: the pages of the tile after the next
            // one, this tile's values; the next tile's keys follow when this one's have been used.
            const typename T::Pages later = tiles.pages_of(u.table, t0 + 2 * kStep, most);
            tiles.load_values(u, t0, now);
            const uint64_t next_word = T::mask_of(u, t0 + kStep);
            f32x4 s[2];
            tiles.logits_of(s, [&] { tiles.load_keys(u, t0 + kStep, next); });
            tiles.hide(s, t0, u.length, now, word);
            if (A.weights_out && static_cast<int32_t>(tiles.n) < u.queries) {
                *reinterpret_cast<f32x4 *>(s_logits + tiles.n * pitch + t0 + 4 * tiles.g) = s[0];
                *reinterpret_cast<f32x4 *>(s_logits + tiles.n * pitch + t0 + 16 + 4 * tiles.g) = s[1];
            }
            tiles.add(s);
            now = next;
            next = later;
            word = next_word;
        }
    }
    join_waves<T, kWaves>(A, u, tiles, s_join, [&](int32_t h, int32_t d, float sum, float m, float all) {
        A.out[(u.row + h) * dim + d] = narrow<kBf16>(all == 0 ? 0.0f : sum / all);
        if (d == 0) {
            if (A.lse) A.lse[u.row + h] = lse_of(m, all);
            s_off[h] = offset_of(m, all);
        }
    });
    if (!A.weights_out) return;
    __syncthreads();
    const int64_t base = (int64_t(b) * A.C.kv_heads + blockIdx.x) * A.capacity;
    for (uint32_t t = threadIdx.x; t < held; t += 64 * kWaves) {
        float sum = 0;
        if (A.C.num_pages)
            for (int32_t h = 0; h < u.queries; ++h) sum += __builtin_amdgcn_exp2f(s_logits[h * pitch + t] - s_off[h]);
        A.weights_out[base + t] = (A.weights ? A.weights[base + t] : 0.0f) + sum;
    }
}

// Longer sequences are cut into parts, a workgroup each, of equal numbers of tiles; the waves take a part's tiles in
// turn, so that a workgroup reads neighbouring slots, and workgroups of one sequence's heads, which lie side by side on
// its pages, follow each other.
//
// How long parts are follows from the lengths, which only the device knows. Sequences of like lengths are best cut into
// as many parts as make one workgroup for every compute unit (64 sequences of 2048 slots, 8 heads of 64: 45 us uncut,
// 55 in two parts; 131072 slots of 8 heads of 128: 32 parts 86, 128 parts 98); where lengths differ, several times as
// many let the short ones fill in behind the long (32 sequences of up to 4096: 54 us, 72 uncut). (Workgroups or waves
// that stay and share out all tiles evenly were slower: on pages of their own, or by what finding their places costs.)
//
// Bound by memory where sequences are alike: 131072 slots of 8 heads of 128 take 86 us in a trace, 6.2 TB/s of the 6.6
// that streamed reads reach. Where they are not, by the compute units that have more than the mean at the end, and some 9 us in which
// the first tiles are waited for and the waves joined: 48 sequences of 0 to 4001 slots, 8 heads of 64, 42 us for 158 MB.
struct Part {
    uint32_t count, first, past;  // parts of the sequence; tiles of this one
};
// n / d for n up to 2^30 and d > 0: the float quotient is off by one at most where it is below 2^22, and a sequence has
// no more parts or tiles.
__device__ __forceinline__ uint32_t over(uint32_t n, uint32_t d) {
    uint32_t q = static_cast<uint32_t>(static_cast<float>(n) * __builtin_amdgcn_rcpf(static_cast<float>(d)));
    while (uint64_t(q) * d > n) --q;
    while (uint64_t(q + 1) * d <= n) ++q;
    return q;
}
// Sum and maximum over a wave; every lane gets them.
template <int kCtrl, int kRowMask>
__device__ __forceinline__ float sum_step(float x) {
    return x + __uint_as_float(endor_device::dpp_or_zero<kCtrl, kRowMask>(__float_as_uint(x)));
}
template <int kCtrl, int kRowMask>
__device__ __forceinline__ uint32_t max_step(uint32_t x) {
    const uint32_t y = endor_device::dpp_or_zero<kCtrl, kRowMask>(x);
    return x > y ? x : y;
}
// Slots of a part at most; every lane gets it.
__device__ __forceinline__ uint32_t chunk_of(const AttnParams &A, uint32_t lane, uint32_t length) {
    uint32_t longest = length;
    if (A.C.batch > 1) {
        float sum = 0;
        for (int32_t b0 = 0; b0 < A.C.batch; b0 += 64) {
            const int32_t b = b0 + static_cast<int32_t>(lane);
            const uint32_t n = clamp_length(A.lengths[b < A.C.batch ? b : 0], A.most_len);
            sum += b < A.C.batch ? static_cast<float>(n) : 0.0f;
            longest = n > longest ? n : longest;
        }
        sum = sum_step<0x118, 0xf>(sum_step<0x114, 0xf>(sum_step<0x112, 0xf>(sum_step<0x111, 0xf>(sum))));
        sum = sum_step<0x143, 0xc>(sum_step<0x142, 0xa>(sum));
        longest = max_step<0x118, 0xf>(max_step<0x114, 0xf>(max_step<0x112, 0xf>(max_step<0x111, 0xf>(longest))));
        longest = max_step<0x143, 0xc>(max_step<0x142, 0xa>(longest));
        sum = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(sum), 63));
        longest = __builtin_amdgcn_readlane(longest, 63);
        // alike: the mean is at least four fifths of the longest
        if (sum < 0.8f * static_cast<float>(longest) * static_cast<float>(A.C.batch)) return A.chunk;
    }
    const uint32_t chunk = (over(longest + A.even - 1, A.even) + 63) & ~63u;
    return __builtin_amdgcn_readfirstlane(chunk > A.least ? chunk : A.least);
}
__device__ __forceinline__ uint32_t parts_of(uint32_t length, uint32_t chunk) { return over(length + chunk - 1, chunk); }
__device__ __forceinline__ Part part_of(uint32_t length, uint32_t chunk, uint32_t slots, uint32_t s) {
    if (length == 0) return {0, 0, 0};
    const uint32_t tiles = (length + slots - 1) / slots, count = parts_of(length, chunk);
    const uint32_t each = over(tiles, count), more = tiles - each * count;  // the first `more` parts have one tile more
    const uint32_t first = s * each + (s < more ? s : more);
    return {count, first, first + each + (s < more ? 1 : 0)};
}

// (Three waves to a SIMD leave heads of 65 to 128 three registers too few: two of them are read back in the loop, where
// logits are stored.)
template <int kDim, int kSub, int kWaves, bool kBf16>
__global__ __launch_bounds__(64 * kWaves) __attribute__((amdgpu_waves_per_eu(kDim == 256 ? 1 : 3))) void endor_attn_part_kernel(AttnParams A) {
    typedef Tiles<kDim, kSub, kBf16> T;
    constexpr uint32_t kStep = kWaves * T::kSlots;
    extern __shared__ float s_join[];  // [wave][query][dim], [wave][query][2]
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    // Workgroups go to the eight XCDs in turn: with the parts last, those that short sequences do not have are spread
    // over all of them (with the parts first, four or eight of them, some XCDs had nothing but the ends of long
    // sequences: 72 us for 58).
    const uint32_t split = blockIdx.z, b = blockIdx.y, dim = A.C.dim;
    const uint32_t held = clamp_length(A.lengths[b], A.most_len), length = A.C.num_pages ? held : 0;
    const Part part = part_of(length, chunk_of(A, lane, held), T::kSlots, split);
    if (split > 0 && split >= part.count) return;  // the first workgroup writes an empty sequence's outputs
    const typename T::Unit u = T::unit_of(A, b, blockIdx.x, length);
    T tiles(A, lane);
    tiles.clear();
    uint32_t t0 = (part.first + wave) * T::kSlots;
    const uint32_t end = part.past * T::kSlots < length ? part.past * T::kSlots : length;
    if (t0 < end) {
        typename T::Pages now = tiles.pages_of(u.table, t0, end), next = tiles.pages_of(u.table, t0 + kStep, end);
        tiles.load_keys(u, t0, now);
        tiles.load_query(u, b);
        uint64_t word = T::mask_of(u, t0);
        for (; t0 < end; t0 += kStep) {
            // Loads come back in order, so what is wanted first goes out first: the pages of the tile after the next
            // one, this tile's values; the next tile's keys follow when this one's have been used.
            const typename T::Pages later = tiles.pages_of(u.table, t0 + 2 * kStep, end);
            tiles.load_values(u, t0, now);
            const uint64_t next_word = T::mask_of(u, t0 + kStep);
            f32x4 s[2 * kSub];
            tiles.logits_of(s, [&] { tiles.load_keys(u, t0 + kStep, next); });
            tiles.hide(s, t0, u.length, now, word);
            if (A.logits && static_cast<int32_t>(tiles.n) < u.queries) {
                float *to = A.logits + (u.row + tiles.n) * A.row + t0 + 4 * tiles.g;
#pragma unroll
                for (int j = 0; j < 2 * kSub; ++j) *reinterpret_cast<f32x4 *>(to + 16 * j) = s[j];
            }
            tiles.add(s);
            now = next;
            next = later;
            word = next_word;
        }
    }
    join_waves<T, kWaves>(A, u, tiles, s_join, [&](int32_t h, int32_t d, float sum, float m, float all) {
        const int64_t row = u.row + h;
        if (part.count <= 1) {
            A.out[row * dim + d] = narrow<kBf16>(all == 0 ? 0.0f : sum / all);
            if (d == 0 && A.lse) A.lse[row] = lse_of(m, all);
        } else {
            A.partial[(row * A.splits + split) * dim + d] = sum;
        }
        if (d == 0) A.ml[row * A.splits + split] = make_float2(m, all);
    });
}

// Maximum and total of a query head over its sequence's parts; every lane of the wave gets them.
__device__ __forceinline__ float2 joined(const float2 *ml, uint32_t parts, uint32_t lane) {
    float m = -INFINITY, all = 0;
    for (uint32_t s0 = 0; s0 < parts; s0 += 256) {  // four parts of every lane on their way
        float2 x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t s = s0 + 64 * i + lane;
            x[i] = ml[s < parts ? s : parts - 1];
            if (s >= parts) x[i] = make_float2(-INFINITY, 0.0f);
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

constexpr int kJoinThreads = 512, kJoinWaves = kJoinThreads / 64;
constexpr int kSlots = 2048;  // slots of a workgroup that adds weights

// After the parts: the first `joins` workgroups join those of `heads` query heads each, where there are several,
// kJoinWaves / heads waves a head, a lane four dims of every so many parts. The others add the weights of kSlots slots
// of a kv head. What it reads is little; a launch and three dependent trips to memory take 4.7 to 5.5 us, with the 10 MB
// of logits of 48 sequences and 32 query heads 7.4.
template <bool kBf16>
__global__ __launch_bounds__(kJoinThreads) void endor_attn_join_kernel(AttnParams A, uint32_t joins, uint32_t heads, uint32_t pieces) {
    __shared__ f32x4 s_sum[kJoinThreads];
    __shared__ float s_off[256];
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if (blockIdx.x < joins) {
        const uint32_t waves = kJoinWaves / heads, dim = A.C.dim;
        const int64_t rows = int64_t(A.C.batch) * A.q_heads, mine = int64_t(blockIdx.x) * heads + wave / waves, row = mine < rows ? mine : rows - 1;
        const uint32_t length = clamp_length(A.lengths[row / A.q_heads], A.most_len), chunk = chunk_of(A, lane, length);
        const uint32_t count = A.C.num_pages ? parts_of(length, chunk) : 0;
        const bool idle = mine >= rows || count <= 1;  // one part has written its outputs itself
        const float2 *ml = A.ml + row * A.splits;
        // units of four dims, lines of them in a wave
        const uint32_t units = dim / 4, lines = 64 / units, line = lane / units, d = 4 * (lane % units), of_wave = wave % waves;
        const float *from = A.partial + row * A.splits * dim + d;
        float2 sums = make_float2(-INFINITY, 0.0f);
        f32x4 sum = {0, 0, 0, 0};
        if (!idle) {
            sums = joined(ml, count, lane);
            if (line < lines)
                for (uint32_t s0 = of_wave * lines + line; s0 < count; s0 += 4 * waves * lines) {
                    f32x4 x[4];
                    float part[4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint32_t s = s0 + i * waves * lines < count ? s0 + i * waves * lines : s0;
                        x[i] = *reinterpret_cast<const f32x4 *>(from + int64_t(s) * dim);
                        part[i] = ml[s].x;
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (s0 + i * waves * lines < count && part[i] != -INFINITY) sum += __builtin_amdgcn_exp2f(part[i] - sums.x) * x[i];
                }
        }
        s_sum[threadIdx.x] = sum;
        __syncthreads();
        if (idle) return;
        const float *part = reinterpret_cast<const float *>(s_sum + 64 * waves * (wave / waves));
        for (uint32_t e = 64 * of_wave + lane; e < dim; e += 64 * waves) {
            float x = 0;
            for (uint32_t w = 0; w < waves; ++w)
                for (uint32_t l = 0; l < lines; ++l) x += part[256 * w + l * dim + e];
            A.out[row * dim + e] = narrow<kBf16>(sums.y == 0 ? 0.0f : x / sums.y);
            if (e == 0 && A.lse) A.lse[row] = lse_of(sums.x, sums.y);
        }
        return;
    }
    const uint32_t piece = (blockIdx.x - joins) % pieces, group = (blockIdx.x - joins) / pieces, b = group / A.C.kv_heads;
    const uint32_t length = clamp_length(A.lengths[b], A.most_len);
    if (piece * kSlots >= length) return;
    const uint32_t chunk = chunk_of(A, lane, length), count = A.C.num_pages ? parts_of(length, chunk) : 0;
    const uint32_t kv = group % A.C.kv_heads;
    const int64_t row0 = int64_t(b) * A.q_heads + int64_t(kv) * A.group;
    // four slots to a thread; rows of logits are whole tiles, so that a unit that begins below the length can be read
    const uint32_t t = piece * kSlots + 4 * threadIdx.x;
    const bool in = t < length;
    typedef f32x4 f32x4_any __attribute__((aligned(4)));
    const int64_t at = (int64_t(b) * A.C.kv_heads + kv) * A.capacity + t;
    f32x4 sum = {0, 0, 0, 0}, added = {0, 0, 0, 0};
    if (in && A.weights) sum = *reinterpret_cast<const f32x4_any *>(A.weights + at);  // the capacity is whole pages, of 8 slots at least
    for (int32_t h0 = 0; h0 < A.group && count > 0; h0 += 256) {
        const int32_t heads = A.group - h0 < 256 ? A.group - h0 : 256;
        __syncthreads();
        for (int32_t h = wave; h < heads; h += kJoinThreads / 64) {
            const float2 sums = joined(A.ml + (row0 + h0 + h) * A.splits, count, lane);
            if (lane == 0) s_off[h] = offset_of(sums.x, sums.y);
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

template <int kDim, int kWaves>
void launch_short(const AttnParams &A, const Plan &p, bool bf16, hipStream_t s) {
    const int queries = A.group < kQueries ? A.group : kQueries;
    const size_t floats = size_t(queries) * (kWaves * (kDim + 2) + (A.weights_out ? p.row : 0)) + (queries + 3) / 4 * 4;
    hipLaunchKernelGGL((bf16 ? endor_attn_kernel<kDim, kWaves, true> : endor_attn_kernel<kDim, kWaves, false>), dim3(p.units, A.C.batch),
                       dim3(64 * kWaves), floats * sizeof(float), s, A, static_cast<uint32_t>(p.row));
}
template <int kDim, int kSub, int kWaves>
void launch_parts(const AttnParams &A, bool bf16, hipStream_t s) {
    hipLaunchKernelGGL((bf16 ? endor_attn_part_kernel<kDim, kSub, kWaves, true> : endor_attn_part_kernel<kDim, kSub, kWaves, false>),
                       dim3(A.units, A.C.batch, A.splits), dim3(64 * kWaves),
                       size_t(kWaves) * (A.group < kQueries ? A.group : kQueries) * (kDim + 2) * sizeof(float), s, A);
}
template <int kWaves>
void launch_waves(const AttnParams &A, bool bf16, hipStream_t s) {
    if (A.C.dim <= 64)
        launch_parts<64, 2, kWaves>(A, bf16, s);
    else if (A.C.dim <= 128)
        launch_parts<128, 1, kWaves>(A, bf16, s);
    else
        launch_parts<256, 1, kWaves>(A, bf16, s);
}

// The kernels of a plan; false if a launch failed.
bool launch(AttnParams A, const Plan &p, void *d_scratch, bool bf16, hipStream_t s) {
    char *scratch = static_cast<char *>(d_scratch);
    A.group = p.group;
    A.qtiles = p.qtiles;
    A.units = p.units;
    if (p.splits == 0) {
        if (A.C.dim <= 64)
            launch_short<64, 8>(A, p, bf16, s);
        else if (A.C.dim <= 128)
            launch_short<128, 8>(A, p, bf16, s);
        else
            launch_short<256, 4>(A, p, bf16, s);
        return hipGetLastError() == hipSuccess;
    }
    A.partial = reinterpret_cast<float *>(scratch);
    A.ml = reinterpret_cast<float2 *>(scratch + p.partial);
    A.logits = p.logits ? reinterpret_cast<float *>(scratch + p.partial + p.ml) : nullptr;
    A.row = p.row;
    A.least = p.least;
    A.chunk = p.chunk;
    A.even = p.even;
    A.splits = p.splits;
    if (p.waves == 4)
        launch_waves<4>(A, bf16, s);
    else
        launch_waves<2>(A, bf16, s);
    if (hipGetLastError() != hipSuccess) return false;
    const uint32_t joins = p.splits > 1 ? (static_cast<uint32_t>(A.C.batch) * A.q_heads + p.heads - 1) / p.heads : 0;
    const uint32_t pieces = A.weights_out ? (A.most_len + kSlots - 1) / kSlots : 0;
    const uint32_t groups = joins + pieces * static_cast<uint32_t>(A.C.batch) * A.C.kv_heads;
    if (groups == 0) return true;
    hipLaunchKernelGGL(bf16 ? endor_attn_join_kernel<true> : endor_attn_join_kernel<false>, dim3(groups), dim3(kJoinThreads), 0, s, A, joins, p.heads, pieces);
    return hipGetLastError() == hipSuccess;
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
    // a launch counts its threads in 32 bits
    const int64_t groups = int64_t(A.C.batch) * q_heads + (d_weights_out ? (int64_t(A.most_len) / kSlots + 1) * A.C.batch * A.C.kv_heads : 0);
    if (groups > (int64_t(1) << 32) / kJoinThreads - 1) return ENDOR_ERR_UNSUPPORTED;
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
    A.scale2 = scale * 1.44269504088896340736f;
    A.q_heads = q_heads;
    return launch(A, p, d_scratch, cache->dtype == ENDOR_BF16, static_cast<hipStream_t>(stream)) ? ENDOR_OK : ENDOR_ERR_HIP;
}
