// Writes into a paged key-value cache, and eviction from it by accumulated attention weight.
#include <hip/hip_runtime.h>

#include <cstdint>

#include "endor.h"
#include "endor_device.h"
#include "endor_evict_search.h"
#include "endor_kv.h"

namespace {

using endor_device::u32x4;
using endor_device::wave_inclusive_scan;
using endor_device::wave_sum;
using endor_evict_search::Bin;
using endor_evict_search::kBins;
using endor_evict_search::kFew;
using endor_evict_search::Last;
using endor_evict_search::last_to_stay;
using endor_evict_search::Range;
using endor_kv::aligned;
using endor_kv::Cache;
using endor_kv::capacity_of;
using endor_kv::clamp_length;
using endor_kv::page_of;
using endor_kv::read_cache;
using endor_kv::slot_at;

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int32_t i32x4 __attribute__((ext_vector_type(4)));

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
    bool advances;  // a prompt's kernel the lengths, for nothing else reads them
};

// Tokens first to first + count of heads head0 to head0 + heads of a sequence. Threads: x the 16-byte units of a head's
// key or value, y the keys and then the values of the heads and on to the next token, four of them on their way.
__device__ __forceinline__ void store_tokens(const AppendParams &A, uint32_t b, uint32_t head0, uint32_t heads, uint32_t length, uint32_t seen,
                                             uint32_t first, uint32_t count) {
    typedef u32x4 u32x4_any __attribute__((aligned(2)));
    const uint32_t rows = 2 * heads, d = 8 * threadIdx.x;
    const int32_t *table = A.C.pages + int64_t(b) * A.C.pages_stride;
    uint32_t t = first, r = threadIdx.y;
    auto settle = [&] {
        while (r >= rows) {
            r -= rows;
            ++t;
        }
    };
    settle();
    while (t < first + count) {
        u32x4 held[4];
        uint16_t *dst[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            dst[k] = nullptr;
            uint32_t page;
            if (t < first + count && page_of(A.C, table, length + t, &page)) {
                const uint32_t h = head0 + (r < heads ? r : r - heads);
                held[k] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_any *>(
                    (r < heads ? A.k : A.v) + int64_t(b) * A.seq_stride + int64_t(t) * A.token_stride + int64_t(h) * A.head_stride + d));
                dst[k] = (r < heads ? A.C.k : A.C.v) + slot_at(A.C, page, h, length + t) + d;
            }
            r += blockDim.y;
            settle();
        }
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (dst[k]) *reinterpret_cast<u32x4 *>(dst[k]) = held[k];
    }
    const uint32_t thread = threadIdx.y * blockDim.x + threadIdx.x, threads = blockDim.x * blockDim.y;
    if (A.weights || A.positions)
        for (uint32_t i = thread; i < heads * count; i += threads) {
            const uint32_t at = first + i % count;
            const int64_t to = (int64_t(b) * A.C.kv_heads + head0 + i / count) * A.capacity + length + at;
            if (A.weights) A.weights[to] = 0.0f;
            if (A.positions) A.positions[to] = static_cast<int32_t>(seen + at);
        }
}

// How many tokens of the sequence are stored.
__device__ __forceinline__ uint32_t stored_of(const AppendParams &A, uint32_t b, uint32_t length) {
    const uint32_t count = A.counts ? clamp_length(A.counts[b], A.tokens) : A.tokens, room = A.capacity - length;
    return count < room ? count : room;
}

// A few tokens: one workgroup per sequence, which also advances its length. One token each for 32 sequences, 8 heads of
// 128: 3.4 us, a launch and two dependent trips to memory; what a caller waits for is its own 7.5 us in the host.
__global__ __launch_bounds__(1024) void endor_kv_append_kernel(AppendParams A) {
    const uint32_t b = blockIdx.x, length = clamp_length(A.lengths[b], A.capacity), seen = A.seen[b], stored = stored_of(A, b, length);
    if (stored) store_tokens(A, b, 0, A.C.kv_heads, length, seen, 0, stored);
    __syncthreads();  // the lengths may be changed in place
    if (threadIdx.x == 0 && threadIdx.y == 0) {
        A.lengths_out[b] = length + stored;
        A.seen_out[b] = seen + stored;
    }
}

constexpr uint32_t kTokensEach = 8;

// Prompts: kTokensEach tokens of a few heads a workgroup, so that a thread has four units of a head's. A second launch
// advances the lengths where they may be read and written in one place. 1777 tokens at most for each of 4
// sequences, 72 heads of 128: 299 MB read and written in 66 us, 4.5 TB/s. A large copy by streamed loads and stores
// reaches 6.6; the stores here are plain.
__global__ __launch_bounds__(256) void endor_kv_append_many_kernel(AppendParams A, uint32_t heads_each) {
    const uint32_t b = blockIdx.z, first = blockIdx.x * kTokensEach, head0 = blockIdx.y * heads_each;
    const uint32_t length = clamp_length(A.lengths[b], A.capacity), stored = stored_of(A, b, length), heads = A.C.kv_heads;
    if (A.advances && blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0 && threadIdx.y == 0) {
        A.lengths_out[b] = length + stored;
        A.seen_out[b] = A.seen[b] + stored;
    }
    if (first < stored)
        store_tokens(A, b, head0, heads - head0 < heads_each ? heads - head0 : heads_each, length, A.seen[b], first,
                     stored - first < kTokensEach ? stored - first : kTokensEach);
}

__global__ __launch_bounds__(256) void endor_kv_advance_kernel(AppendParams A) {
    const int32_t b = blockIdx.x * 256 + threadIdx.x;
    if (b >= A.C.batch) return;
    // both before either is stored: all four may be one array
    const uint32_t length = clamp_length(A.lengths[b], A.capacity), seen = A.seen[b], stored = stored_of(A, b, length);
    A.lengths_out[b] = length + stored;
    A.seen_out[b] = seen + stored;
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
    bool shortens;  // the lengths here, for nothing else reads them
};

// Weights as unsigned numbers in the same order: NaN 1, below all, -0 with +0; what must stay is above all. 0 is no
// token.
__device__ __forceinline__ uint32_t key_of(float w, int32_t position, int64_t newest) {
    if (position >= newest) return 0xffffffffu;
    if (w != w) return 1;
    const uint32_t bits = __float_as_uint(w + 0.0f);
    return bits >> 31 ? ~bits : bits | 0x80000000u;
}

constexpr int kMostWaves = 16;  // of a workgroup that selects

// Where a token's keys and values are and go: element offsets from the pools' beginnings; -1 where a page is not there.
struct Move {
    int64_t from, to;
};
__device__ __forceinline__ Move move_of(const Cache &C, const int32_t *table, uint32_t h, uint32_t to, uint32_t from) {
    uint32_t a, z;
    const bool here = page_of(C, table, to, &a), there = page_of(C, table, from, &z);
    return here && there ? Move{slot_at(C, z, h, from), slot_at(C, a, h, to)} : Move{-1, -1};
}

// A workgroup moves so many tokens by itself sooner than a second launch begins.
constexpr int kFewMoves = 64;

struct SelectShared {
    uint32_t bins[kBins];
    uint32_t part[2][kMostWaves];
    uint32_t low[kMostWaves], high[kMostWaves];
    uint32_t found[3];  // the bin that the last kept key is in, the keys above it, the keys in it
    uint32_t left, last[kFew], over[kFew], same[kFew];  // the keys in question, when a wave can hold them; the keys above each and its equals
    int32_t holes[kFewMoves], movers[kFewMoves];
    Move moves[kFewMoves];
};

// The passes of the search for the last key that stays.
template <class Count, class Rank, class Ends>
struct Passes {
    Count count;
    Rank rank;
    Ends ends;
};

// Exclusive prefix over the workgroup, and the total. `turn` changes from one call to the next, so that one barrier
// does.
template <uint32_t kWaves>
__device__ __forceinline__ uint32_t group_scan(uint32_t x, SelectShared &S, uint32_t turn, uint32_t *total) {
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint32_t upto = wave_inclusive_scan(x);
    if (lane == 63) S.part[turn & 1][wave] = upto;
    __syncthreads();
    uint32_t before = 0, sum = 0;
#pragma unroll
    for (uint32_t w = 0; w < kWaves; ++w) {
        before += w < wave ? S.part[turn & 1][w] : 0;
        sum += S.part[turn & 1][w];
    }
    *total = sum;
    return before + upto - x;
}

// Moves tokens, 16 bytes a lane, keys and values side by side, four loads of a thread on their way.
__device__ __forceinline__ void move_tokens(const Cache &C, const Move *moves, uint32_t count, uint32_t threads) {
    const uint32_t half = C.dim / 8, per = 2 * half, lines = threads / per, line = threadIdx.x / per, part = threadIdx.x % per;
    uint16_t *pool = (part < half ? C.k : C.v) + 8 * (part < half ? part : part - half);
    if (line >= lines || C.num_pages == 0) return;  // a pool without pages may be no memory at all
    for (uint32_t i0 = line; i0 < count; i0 += 4 * lines) {
        u32x4 held[4];
        int64_t to[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const uint32_t i = i0 + k * lines;
            const Move m = moves[i < count ? i : i0];
            to[k] = i < count ? m.to : -1;
            held[k] = *reinterpret_cast<const u32x4 *>(pool + (m.from < 0 ? 0 : m.from));  // the first page is there
        }
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (to[k] >= 0) *reinterpret_cast<u32x4 *>(pool + to[k]) = held[k];
    }
}

// One workgroup per sequence and kv head finds the key of the last token that stays, then the slots that come free
// below the budget and the kept ones past it, in order.
//
// The keys are looked at 11 bits at a time from the highest bit in which they differ: a histogram in LDS, and a scan of
// it from the top, until a wave can hold what is left and count for each key those above it. (Weights of one row share
// most of their leading bits: a fixed first digit would have nearly all keys in a few bins, where LDS adds them one
// after the other.) A wave has a contiguous piece of the slots, 256 of them at a time, four to a lane: loads are whole
// lines, and ranks in the order of slots need wave scans only. kChunks: such chunks of a wave that it keeps as keys in
// registers; 0: the keys are formed anew in every pass, for rows past 32768 slots. kMove: the moves are few and done
// here.
//
// Bound by the passes one after the other, each of which the slowest wave ends, not by the 8 bytes a slot that it reads:
// 16 x 8 rows of 16000 tokens 17 us, a third of it until the keys are there, a third the histograms, a third ranks and
// lists; 13 x 16 of 6600 11.3, 8 x 72 of 3457 13.6.
template <int kThreads, int kChunks, bool kMove>
__global__ __launch_bounds__(kThreads) void endor_kv_select_kernel(EvictParams E) {
    constexpr uint32_t kWaves = kThreads / 64;
    constexpr int kOwn = kBins / kThreads;  // bins that a thread reads
    __shared__ SelectShared S;
    const uint32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t b = blockIdx.y, h = blockIdx.x;
    const int64_t row = int64_t(b) * E.C.kv_heads + h, base = row * E.capacity;
    const float *w = E.weights + base;
    const int32_t *pos = E.positions + base;
    float *w_out = E.weights_out + base;
    int32_t *pos_out = E.positions_out + base;
    const uint32_t length = clamp_length(E.lengths[b], E.most_len), budget = E.budget;
    const bool copies = w_out != w || pos_out != pos;  // what stays where it is has to be written
    if (E.shortens && h == 0 && threadIdx.x == 0) E.lengths_out[b] = length < budget ? length : budget;
    if (length <= budget || budget == 0) {
        const uint32_t kept = length < budget ? length : budget;
        if (copies)
            for (uint32_t t = threadIdx.x; t < kept; t += kThreads) {
                w_out[t] = w[t];
                pos_out[t] = pos[t];
            }
        if (!kMove && threadIdx.x == 0) E.count[row] = 0;
        return;
    }
    const int64_t newest = int64_t(E.seen[b]) - E.recent;
    const uint32_t chunks = kChunks ? kChunks : (length + 256 * kWaves - 1) / (256 * kWaves);
    const uint32_t mine = wave * chunks * 256 + 4 * lane;  // slot of this lane's first key
    typedef f32x4 f32x4_any __attribute__((aligned(4)));
    typedef i32x4 i32x4_any __attribute__((aligned(4)));
    constexpr uint32_t kStay = 0xffffffffu;
    // Four keys from slot t on; of a slot past the length, 0.
    auto keys_at = [&](uint32_t t) {
        u32x4 key = {0, 0, 0, 0};
        if (t + 4 <= length) {
            const f32x4 x = *reinterpret_cast<const f32x4_any *>(w + t);
            const i32x4 p = *reinterpret_cast<const i32x4_any *>(pos + t);
#pragma unroll
            for (int e = 0; e < 4; ++e) key[e] = key_of(x[e], p[e], newest);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (t + e < length) key[e] = key_of(w[t + e], pos[t + e], newest);
        }
        return key;
    };
#pragma unroll
    for (int i = 0; i < kOwn; ++i) S.bins[threadIdx.x + i * kThreads] = 0;
    if (threadIdx.x < kFew) S.over[threadIdx.x] = S.same[threadIdx.x] = 0;
    if (threadIdx.x == 0) S.left = 0;
    u32x4 held[kChunks ? kChunks : 1];
    if constexpr (kChunks > 0)
#pragma unroll
        for (int i = 0; i < kChunks; ++i) held[i] = keys_at(mine + 256 * i);
    // Slots below the budget as they are; those that come free are written again behind several barriers.
    if (copies)
        for (uint32_t t = mine, i = 0; i < chunks; ++i, t += 256) {
            if (t + 4 <= budget) {  // which is below the length
                *reinterpret_cast<f32x4_any *>(w_out + t) = *reinterpret_cast<const f32x4_any *>(w + t);
                *reinterpret_cast<i32x4_any *>(pos_out + t) = *reinterpret_cast<const i32x4_any *>(pos + t);
            } else {
                for (uint32_t e = 0; e < 4 && t + e < budget; ++e) {
                    w_out[t + e] = w[t + e];
                    pos_out[t + e] = pos[t + e];
                }
            }
        }
    // f(slot of four keys, the keys) for all of the lane's
    auto each = [&](auto f) {
        if constexpr (kChunks > 0) {
#pragma unroll
            for (int i = 0; i < kChunks; ++i) f(mine + 256 * i, held[i]);
        } else {
            for (uint32_t i = 0; i < chunks; ++i) f(mine + 256 * i, keys_at(mine + 256 * i));
        }
    };

    uint32_t turn = 0, total;
    // What stays whatever it weighs; the least and the largest key of the others.
    // One is taken off or added so that neither what stays nor what is no token is the least or the largest.
    uint32_t staying = 0, low = 0xffffffffu, high = 0;
    auto leave_ends = [&] {  // the wave's, for all
#pragma unroll
        for (int d = 32; d; d >>= 1) {
            const uint32_t l = __shfl_xor(low, d), u = __shfl_xor(high, d);
            low = l < low ? l : low;
            high = u > high ? u : high;
        }
        if (lane == 0) {
            S.low[wave] = low;
            S.high[wave] = high;
        }
    };
    auto take_ends = [&] {
#pragma unroll
        for (uint32_t v = 0; v < kWaves; ++v) {
            low = S.low[v] < low ? S.low[v] : low;
            high = S.high[v] > high ? S.high[v] : high;
        }
    };
    each([&](uint32_t, u32x4 key) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            staying += key[e] == kStay;
            low = key[e] - 1 < low ? key[e] - 1 : low;
            high = key[e] + 1 > high ? key[e] + 1 : high;
        }
    });
    leave_ends();
    group_scan<kWaves>(staying, S, turn++, &total);  // its barrier is for both
    staying = total;
    take_ends();
    ++low;
    --high;
    uint32_t least = kStay, ties = budget;  // keys above `least` stay, and the first `ties` of those equal to it
    // An eviction at every step has one token too many: the least key is known by now. 4 x 8 rows of 2049 tokens 5.8 us,
    // 7.9 by the histograms.
    const bool one_goes = staying < budget && length - budget == 1;
    if (one_goes) {
        least = low;  // and the last of its equals goes, once they are counted
    } else if (staying < budget) {
        auto count = [&](const Range &r, uint32_t bits) {
            const uint32_t range = r.high - r.low;
            uint32_t least_ones = 0;  // often many, weights of zero say, which would be added one after the other
            each([&](uint32_t, u32x4 key) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    least_ones += key[e] == r.low;
                    if (key[e] - r.low - 1 < range) atomicAdd(&S.bins[r.bin_of(key[e], bits)], 1u);
                }
            });
            least_ones = wave_sum(least_ones);
            if (lane == 0) atomicAdd(&S.bins[0], least_ones);
            __syncthreads();
            // from the top down
            const uint32_t top = kBins - 1 - kOwn * threadIdx.x;
            uint32_t own[kOwn], sum = 0;
#pragma unroll
            for (int i = 0; i < kOwn; ++i) {
                own[i] = S.bins[top - i];
                S.bins[top - i] = 0;
                sum += own[i];
            }
            uint32_t above = group_scan<kWaves>(sum, S, turn++, &total);
            if (above < r.need && above + sum >= r.need)
#pragma unroll
                for (int i = 0; i < kOwn; ++i) {
                    if (above < r.need && above + own[i] >= r.need) {
                        S.found[0] = top - i;
                        S.found[1] = above;
                        S.found[2] = own[i];
                    }
                    above += own[i];
                }
            __syncthreads();
            return Bin{S.found[0], S.found[1], S.found[2]};
        };
        auto rank = [&](const Range &r, uint32_t in_bin) {
            each([&](uint32_t, u32x4 key) {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (r.holds(key[e])) S.last[atomicAdd(&S.left, 1u)] = key[e];
            });
            __syncthreads();
            const uint32_t key = lane < in_bin ? S.last[lane] : 0;
            uint32_t over = 0, same = 0;
            for (uint32_t i = wave; i < in_bin; i += kWaves) {
                const uint32_t other = S.last[i];
                over += other > key;
                same += other == key;
            }
            atomicAdd(&S.over[lane], over);
            atomicAdd(&S.same[lane], same);
            __syncthreads();
            over = S.over[lane];
            same = S.same[lane];
            // the lanes that hold the last key to stay; all waves find the same
            const uint64_t at = __ballot(lane < in_bin && over < r.need && over + same >= r.need);
            const uint32_t from = __builtin_ctzll(at);
            return Last{uint32_t(__builtin_amdgcn_readlane(key, from)), r.need - __builtin_amdgcn_readlane(over, from)};
        };
        auto ends = [&](Range *r) {
            low = 0xffffffffu;
            high = 0;
            each([&](uint32_t, u32x4 key) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const bool in = r->holds(key[e]);
                    low = in && key[e] < low ? key[e] : low;
                    high = in && key[e] > high ? key[e] : high;
                }
            });
            leave_ends();
            __syncthreads();
            take_ends();
            r->low = low;
            r->high = high;
        };
        // More keys are left than are needed, so low <= high. A bin's own ends cost a pass: a fifth of the weights zero and
        // the last kept one among them, 6 rows of 23823 tokens 22.7 us, by the bins alone 32.1; 4 x 8 of 2050 7.8 and 9.1;
        // where bins hold less it would cost 0.8.
        const Last last = last_to_stay(Range{low, high, budget - staying}, length / 16, Passes<decltype(count), decltype(rank), decltype(ends)>{count, rank, ends});
        least = last.key;
        ties = last.ties;
    }

    // Which stay: above, or equal and among the first. Of the waves before this one: equal keys, then slots that come
    // free and tokens that move.
    auto waves_before = [&](uint32_t x, uint32_t *all) {
        const uint32_t sum = wave_sum(x);
        if (lane == 0) S.part[turn & 1][wave] = sum;
        __syncthreads();
        uint32_t before = 0;
        *all = 0;
#pragma unroll
        for (uint32_t v = 0; v < kWaves; ++v) {
            before += v < wave ? S.part[turn & 1][v] : 0;
            *all += S.part[turn & 1][v];
        }
        ++turn;
        return before;
    };
    uint32_t equal = 0;
    each([&](uint32_t, u32x4 key) {
#pragma unroll
        for (int e = 0; e < 4; ++e) equal += key[e] == least;
    });
    const uint32_t equal_before = waves_before(equal, &total);
    if (one_goes) ties = total - 1;
    uint32_t ranked;
    // The bits of the four slots that stay; called for the wave's chunks in order.
    auto kept_of = [&](u32x4 key) {
        uint32_t same = 0, more = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            same |= uint32_t(key[e] == least) << e;
            more |= uint32_t(key[e] > least) << e;
        }
        if (__ballot(same != 0)) {
            const uint32_t upto = wave_inclusive_scan(__popc(same));
            uint32_t rank = ranked + upto - __popc(same);
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (same >> e & 1) more |= uint32_t(rank++ < ties) << e;
            ranked += __builtin_amdgcn_readlane(upto, 63);
        }
        return more;
    };
    // the bits of the four slots from t on that lie below the budget
    auto below = [&](uint32_t t) { return t >= budget ? 0u : budget - t >= 4 ? 15u : (1u << (budget - t)) - 1; };
    ranked = equal_before;
    uint32_t bits = 0, holes_mine = 0, movers_mine = 0, at = 0;  // bits: of all chunks, where they are registers
    each([&](uint32_t t, u32x4 key) {
        const uint32_t kept = kept_of(key);
        bits |= kChunks ? kept << (4 * at++) : 0;
        holes_mine += __popc(below(t) & ~kept);
        movers_mine += __popc(kept & ~below(t));
    });
    uint32_t holes = waves_before(holes_mine, &total), movers = waves_before(movers_mine, &total);
    int32_t *hole_list = kMove ? S.holes : E.holes + row * E.most, *mover_list = kMove ? S.movers : E.movers + row * E.most;
    ranked = equal_before;
    at = 0;
    each([&](uint32_t t, u32x4 key) {
        const uint32_t kept = kChunks ? bits >> (4 * at++) & 15u : kept_of(key);
        const uint32_t free = below(t) & ~kept, past = kept & ~below(t);
        if (!__ballot((free | past) != 0)) return;
        const uint32_t mine_of = __popc(free) | __popc(past) << 16, upto = wave_inclusive_scan(mine_of);  // at most 256 of each
        uint32_t hole = holes + ((upto - mine_of) & 0xffffu), mover = movers + ((upto - mine_of) >> 16);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (free >> e & 1) hole_list[hole++] = t + e;
            if (past >> e & 1) mover_list[mover++] = t + e;
        }
        const uint32_t all = __builtin_amdgcn_readlane(upto, 63);
        holes += all & 0xffffu;
        movers += all >> 16;
    });
    if (threadIdx.x == kThreads - 1) S.found[0] = holes;
    __threadfence_block();
    __syncthreads();  // the lists are whole, and nobody reads the slots that come free any more
    const uint32_t count = S.found[0];
    for (uint32_t i = threadIdx.x; i < count; i += kThreads) {
        const int32_t to = hole_list[i], from = mover_list[i];
        w_out[to] = w[from];
        pos_out[to] = pos[from];
        if constexpr (kMove) S.moves[i] = move_of(E.C, E.C.pages + b * E.C.pages_stride, h, to, from);
    }
    if constexpr (kMove) {
        __syncthreads();
        move_tokens(E.C, S.moves, count, kThreads);
    } else if (threadIdx.x == 0) {
        E.count[row] = count;
    }
}

constexpr int kMovesEach = 64;  // of a workgroup of the move kernel

// Keys and values of the kept tokens past the budget. 8 x 72 rows that move 860 tokens of 64 dims each: 255 MB read and
// written in 59 us, 4.3 TB/s, where a large copy by streamed loads and stores reaches 6.6. Rows are of 128 to 512 bytes in
// no order, and loads and stores are plain; how much either costs was not measured.
__global__ __launch_bounds__(256) void endor_kv_move_kernel(EvictParams E) {
    __shared__ Move s_moves[kMovesEach];
    const uint32_t b = blockIdx.z, h = blockIdx.y, first = blockIdx.x * kMovesEach;
    const int64_t row = int64_t(b) * E.C.kv_heads + h;
    const uint32_t all = E.count[row];
    if (first >= all) return;
    const uint32_t count = all - first < kMovesEach ? all - first : kMovesEach;
    if (threadIdx.x < count)
        s_moves[threadIdx.x] = move_of(E.C, E.C.pages + b * E.C.pages_stride, h, E.holes[row * E.most + first + threadIdx.x],
                                       E.movers[row * E.most + first + threadIdx.x]);
    __syncthreads();
    move_tokens(E.C, s_moves, count, 256);
}

// The lengths in place, once nobody reads the old ones any more.
__global__ __launch_bounds__(256) void endor_kv_shorten_kernel(EvictParams E) {
    const int32_t b = blockIdx.x * 256 + threadIdx.x;
    if (b >= E.C.batch) return;
    const int32_t length = clamp_length(E.lengths[b], E.most_len);
    E.lengths_out[b] = length < E.budget ? length : E.budget;
}

// The chunks are the fewest that hold the tokens in registers. Small workgroups have fewer waves to
// wait for at each barrier, and two of them share a compute unit better than two large ones do; large
// ones hold more tokens and work longer rows off sooner where there is one for each unit at most.
// Measured with 512 | 1024 threads: 1 x 8 rows of 1026 tokens 6.5 | 8.0 us, 4 x 8 of 2050 7.9 | 8.3, 8 x 72 of 3457
// 13.6 | 23.3, 64 x 8 of 8000 22.9 | 27.4, of 16000 39.1 | 45.0; but 13 x 16 of 6600 12.3 | 11.2 and 16 x 8 of 16000
// 22 | 17. 256 threads take longer for all but the shortest rows.
template <bool kMove>
void launch_select(const EvictParams &E, hipStream_t s) {
    constexpr int kUnits = 256;
    const int64_t rows = int64_t(E.C.batch) * E.C.kv_heads;
    const bool small = E.most_len <= 4096 || (rows > kUnits && E.most_len <= 16384);
    const int threads = small ? 512 : 1024, chunks = (E.most_len - 1) / (4 * threads) + 1;
    const auto kernel = small ? chunks <= 1   ? endor_kv_select_kernel<512, 1, kMove>
                                : chunks <= 2 ? endor_kv_select_kernel<512, 2, kMove>
                                : chunks <= 4 ? endor_kv_select_kernel<512, 4, kMove>
                                              : endor_kv_select_kernel<512, 8, kMove>
                        : chunks <= 2 ? endor_kv_select_kernel<1024, 2, kMove>
                        : chunks <= 4 ? endor_kv_select_kernel<1024, 4, kMove>
                        : chunks <= 8 ? endor_kv_select_kernel<1024, 8, kMove>
                                      : endor_kv_select_kernel<1024, 0, kMove>;
    hipLaunchKernelGGL(kernel, dim3(E.C.kv_heads, E.C.batch), dim3(threads), 0, s, E);
}

// Whether a kernel may write the one while its other workgroups read the other, n numbers each.
bool apart(const int32_t *in, const int32_t *out, size_t n) {
    const uintptr_t a = reinterpret_cast<uintptr_t>(in), z = reinterpret_cast<uintptr_t>(out);
    return a >= z + 4 * n || z >= a + 4 * n;
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
    const size_t n = A.C.batch;
    A.advances = apart(d_lengths, d_lengths_out, n) && apart(d_lengths, d_seen_out, n) && apart(d_seen, d_lengths_out, n) && apart(d_seen, d_seen_out, n) &&
                 (!d_counts || (apart(d_counts, d_lengths_out, n) && apart(d_counts, d_seen_out, n)));
    hipStream_t s = static_cast<hipStream_t>(stream);
    const uint32_t units = A.C.dim / 8;
    if (tokens <= static_cast<int>(kTokensEach)) {
        const uint32_t rows = 2 * A.C.kv_heads * (tokens ? tokens : 1), most = 1024 / units;
        hipLaunchKernelGGL(endor_kv_append_kernel, dim3(A.C.batch), dim3(units, rows < most ? rows : most), 0, s, A);
        return hipGetLastError() == hipSuccess ? ENDOR_OK : ENDOR_ERR_HIP;
    }
    const uint32_t lines = 256 / units, each = 4 * lines / (2 * kTokensEach) ? 4 * lines / (2 * kTokensEach) : 1, heads = A.C.kv_heads;
    hipLaunchKernelGGL(endor_kv_append_many_kernel, dim3((static_cast<uint32_t>(tokens) + kTokensEach - 1) / kTokensEach, (heads + each - 1) / each, A.C.batch),
                       dim3(units, lines), 0, s, A, each);
    if (hipGetLastError() != hipSuccess) return ENDOR_ERR_HIP;
    if (!A.advances) hipLaunchKernelGGL(endor_kv_advance_kernel, dim3((A.C.batch + 255) / 256), dim3(256), 0, s, A);
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
    E.shortens = apart(d_lengths, d_lengths_out, E.C.batch) && apart(d_seen, d_lengths_out, E.C.batch);
    const int64_t rows = int64_t(E.C.batch) * E.C.kv_heads;
    E.count = static_cast<int32_t *>(d_scratch);
    E.holes = E.count + rows;
    E.movers = E.holes + rows * E.most;
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (E.most <= kFewMoves) {
        launch_select<true>(E, s);
    } else {
        launch_select<false>(E, s);
        if (hipGetLastError() != hipSuccess) return ENDOR_ERR_HIP;
        hipLaunchKernelGGL(endor_kv_move_kernel, dim3((E.most + kMovesEach - 1) / kMovesEach, E.C.kv_heads, E.C.batch), dim3(256), 0, s, E);
    }
    if (hipGetLastError() != hipSuccess) return ENDOR_ERR_HIP;
    if (!E.shortens) hipLaunchKernelGGL(endor_kv_shorten_kernel, dim3((E.C.batch + 255) / 256), dim3(256), 0, s, E);
    return hipGetLastError() == hipSuccess ? ENDOR_OK : ENDOR_ERR_HIP;
}
