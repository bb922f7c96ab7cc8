// The search for the last key that an eviction keeps (endor_evict_search.h), with the kernel's passes done one key after the other,
// against a sort.  Built and run by tests/test_evict_search.py; not part of the library.
#include <algorithm>
#include <cstdint>
#include <cstdio>
#include <cstring>
#include <vector>

#include "endor_evict_search.h"

using namespace endor_evict_search;

static uint64_t state = 0x243F6A8885A308D3ull;
static uint64_t rnd() {
    state ^= state << 13;
    state ^= state >> 7;
    state ^= state << 17;
    return state;
}
static double uniform() { return static_cast<double>(rnd() >> 11) * 0x1p-53; }

// As the kernel forms them: the numbers in their order, above 0 and below what stays whatever it weighs.
static uint32_t key_of(float w) {
    uint32_t bits;
    w += 0.0f;
    std::memcpy(&bits, &w, 4);
    return w != w ? 1 : bits >> 31 ? ~bits : bits | 0x80000000u;
}

struct Passes {
    const std::vector<uint32_t> &keys;
    const char *wrong = nullptr;
    int counts = 0;
    Bin count(const Range &r, uint32_t bits) {
        std::vector<uint32_t> bins(kBins);
        for (uint32_t k : keys)
            if (r.holds(k)) ++bins.at(r.bin_of(k, bits));
        if (++counts > 8) wrong = "no end";
        uint32_t above = 0;
        for (int b = kBins - 1; b >= 0; --b) {
            if (above + bins[b] >= r.need) return {static_cast<uint32_t>(b), above, wrong ? r.need - above : bins[b]};
            above += bins[b];
        }
        wrong = "fewer keys in question than are needed";
        return {0, 0, r.need};
    }
    std::vector<uint32_t> in(const Range &r) const {
        std::vector<uint32_t> some;
        for (uint32_t k : keys)
            if (r.holds(k)) some.push_back(k);
        return some;
    }
    Last rank(const Range &r, uint32_t count) {
        std::vector<uint32_t> some = in(r);
        if (some.size() != count || count > kFew || r.need == 0 || r.need > count) {
            wrong = "not the keys of the bin are ranked";
            return {0, 0};
        }
        std::sort(some.begin(), some.end(), [](uint32_t a, uint32_t z) { return a > z; });
        const uint32_t key = some[r.need - 1];
        return {key, r.need - static_cast<uint32_t>(std::count_if(some.begin(), some.end(), [&](uint32_t k) { return k > key; }))};
    }
    void ends(Range *r) {
        const std::vector<uint32_t> some = in(*r);
        r->low = *std::min_element(some.begin(), some.end());
        r->high = *std::max_element(some.begin(), some.end());
    }
};

// `sorted`: the keys from the largest on.
static bool check(const std::vector<uint32_t> &keys, const std::vector<uint32_t> &sorted, uint32_t need, const char *what) {
    Passes passes{keys};
    const Last last = last_to_stay({sorted.back(), sorted.front(), need}, static_cast<uint32_t>(keys.size()) / 16, passes);
    const uint32_t above = static_cast<uint32_t>(std::lower_bound(sorted.begin(), sorted.end(), last.key, [](uint32_t a, uint32_t k) { return a > k; }) - sorted.begin());
    const uint32_t upto = static_cast<uint32_t>(std::upper_bound(sorted.begin(), sorted.end(), last.key, [](uint32_t k, uint32_t a) { return k > a; }) - sorted.begin());
    const uint64_t kept = above + std::min<uint64_t>(last.ties, upto - above);
    if (!passes.wrong && kept != need) passes.wrong = "not as many stay as are wanted";
    if (passes.wrong) std::printf("%s, %zu keys of which %u stay: %s (%llu)\n", what, keys.size(), need, passes.wrong, static_cast<unsigned long long>(kept));
    return !passes.wrong;
}
static bool check_all(const std::vector<float> &weights, const char *what, uint32_t step = 1) {
    std::vector<uint32_t> keys;
    for (float w : weights) keys.push_back(key_of(w));
    std::vector<uint32_t> sorted = keys;
    std::sort(sorted.begin(), sorted.end(), [](uint32_t a, uint32_t z) { return a > z; });
    for (uint32_t need = 1; need < keys.size(); need += step)
        if (!check(keys, sorted, need, what)) return false;
    return true;
}

static float float_of(uint32_t bits) {
    float x;
    std::memcpy(&x, &bits, 4);
    return x;
}

int main() {
    // A cluster that ends just below a power of two, zeros that make it the second bin's, and more beyond its upper end, as many as a wave holds and
    // more.
    for (uint32_t ones : {0u, 1u, 5u, 64u, 65u, 400u}) {
        std::vector<float> w(200, 0.0f);
        w.insert(w.end(), {0.98437488f, 0.99999994f, 0.99999988f});
        for (int i = 0; i < 1500; ++i) w.push_back(static_cast<float>(0.98437488 + uniform() * (0.99999994 - 0.98437488)));
        w.insert(w.end(), ones, 1.0f);
        if (!check_all(w, "a cluster below one")) return 1;
    }
    // Clusters across the boundaries of bins of every width, narrow and wide, with far ones on either side.
    for (int i = 0; i < 400; ++i) {
        const uint32_t bits = 1 + rnd() % 22, center = (0x30000000u + static_cast<uint32_t>(rnd() % 0x10000000u)) >> bits << bits;
        std::vector<float> w;
        const int inside = 100 + rnd() % 900, at_center = rnd() % 200, zeros = rnd() % 300, far = rnd() % 10;
        for (int k = 0; k < inside; ++k) w.push_back(float_of(center - 1 - static_cast<uint32_t>(rnd() % (uint64_t(1) << bits))));
        for (int k = 0; k < at_center; ++k) w.push_back(float_of(center + static_cast<uint32_t>(k % 3 ? rnd() % (1 + rnd() % (uint64_t(1) << bits)) : 0)));
        w.insert(w.end(), zeros, 0.0f);
        for (int k = 0; k < far; ++k) w.push_back(static_cast<float>(k % 2 ? 3e30 : -1e-30 * uniform()));
        if (!check_all(w, "a cluster across a boundary")) return 1;
    }
    for (int i = 0; i < 60; ++i) {
        std::vector<float> even, spread, few, odd;
        const int n = 2 + rnd() % 3000;
        for (int k = 0; k < n; ++k) {
            even.push_back(uniform() < 0.2 ? 0.0f : static_cast<float>(0.9 + 0.2 * uniform()));
            const double u = uniform();
            spread.push_back(u < 0.2 ? 0.0f : static_cast<float>(-__builtin_log(1 - u) * __builtin_log(1 - u) * u));
            few.push_back(static_cast<float>(rnd() % 4));
            odd.push_back(float_of(static_cast<uint32_t>(rnd())));  // every kind of number, NaN and infinities among them
        }
        if (!check_all(even, "around one") || !check_all(spread, "of many sizes") || !check_all(few, "whole numbers") || !check_all(odd, "any")) return 1;
    }
    std::vector<float> many;
    for (int k = 0; k < 40000; ++k) many.push_back(k % 7 ? static_cast<float>(1 + (rnd() % 3000) * 0x1p-23) : k % 2 ? 0.0f : static_cast<float>(1 + 1500 * 0x1p-23));
    if (!check_all(many, "close together", 97)) return 1;
    std::printf("ok\n");
    return 0;
}
