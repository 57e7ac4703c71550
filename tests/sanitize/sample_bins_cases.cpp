// Divides rows of logits as a wave of ds_sample does (paper_1907_07346_amd/csrc/dsq_sample_bins.h), on the host: every division leaves fewer logits than there were, whichever
// of them is looked for, and what is found is the nth of the order.  Built and run by tests/test_sample_bins.py.
#include <algorithm>
#include <cmath>
#include <cstdio>
#include <cstring>
#include <limits>
#include <random>
#include <vector>

#include "dsq_sample_bins.h"

namespace {

int failures = 0;
void fail(const char* what, const char* row, size_t size, size_t nth) {
    if (++failures <= 20) std::printf("FAILED %s: %s, %zu logits, number %zu\n", what, row, size, nth);
}

uint32_t key_of(float z) {
    z += 0.f;
    uint32_t bits;
    std::memcpy(&bits, &z, 4);
    return bits & 0x80000000u ? ~bits : bits | 0x80000000u;
}
float of_key(uint32_t key) {
    const uint32_t bits = key & 0x80000000u ? key & 0x7FFFFFFFu : ~key;
    float z;
    std::memcpy(&z, &bits, 4);
    return z;
}

// The nth (from 1) largest of a row, down to `room` logits that are put in order.
float find(const std::vector<float>& row, const char* name, size_t nth, size_t room) {
    const float max = *std::max_element(row.begin(), row.end());
    dsq::LinearBins bins{(double)max, 0.0, 0.0};
    float lo = *std::min_element(row.begin(), row.end()), hi = max;
    size_t left = nth;
    for (;;) {
        std::vector<float> here;
        for (float x : row)
            if (x >= lo && x <= hi) here.push_back(x);
        if (lo == hi) return lo;
        if (here.size() <= room) {
            std::sort(here.begin(), here.end(), std::greater<float>());
            return here[left - 1];
        }
        if (bins.alike(lo, hi)) {
            for (float x : here)
                if (bins.distance(x) != bins.distance(hi)) fail("not alike", name, row.size(), nth);
            dsq::NthKey keys{key_of(lo), key_of(hi)};
            int tries = 0;
            while (!keys.done()) {
                const uint32_t key = keys.tried();
                keys.counted((size_t)std::count_if(here.begin(), here.end(), [&](float x) { return key_of(x) >= key; }) >= left);
                if (++tries > 32) {
                    fail("more than 32 tries", name, row.size(), nth);
                    break;
                }
            }
            return of_key(keys.low);
        }
        bins.set(lo, hi);
        std::vector<size_t> count(dsq::kWaveBins);
        uint32_t before = 0;
        std::sort(here.begin(), here.end(), std::greater<float>());
        for (float x : here) {
            const uint32_t bin = bins(x);
            if (bin >= dsq::kWaveBins) {
                fail("no such bin", name, row.size(), nth);
                return 0.f;
            }
            if (bin < before) fail("bins out of order", name, row.size(), nth);
            before = bin;
            ++count[bin];
        }
        uint32_t bin = 0;
        while (left > count[bin]) left -= count[bin++];
        if (count[bin] >= here.size()) {                          // the kernel would divide for ever
            fail("a division that leaves all", name, row.size(), nth);
            return 0.f;
        }
        hi = -std::numeric_limits<float>::infinity();
        lo = -hi;
        for (float x : here)
            if (bins(x) == bin) {
                lo = std::min(lo, x);
                hi = std::max(hi, x);
            }
    }
}

void every_one(const char* name, const std::vector<float>& row) {
    std::vector<float> order = row;
    std::sort(order.begin(), order.end(), std::greater<float>());
    const size_t step = row.size() > 100 ? row.size() / 97 : 1;
    for (size_t room : {1, 64})
        for (size_t nth = 1; nth <= row.size(); nth += step)
            if (find(row, name, nth, room) != order[nth - 1]) fail("another number", name, row.size(), nth);
}

float to_bf16(float x) {
    uint32_t bits;
    std::memcpy(&bits, &x, 4);
    bits &= 0xFFFF0000u;
    std::memcpy(&x, &bits, 4);
    return x;
}

}  // namespace

int main() {
    std::mt19937 rng(5);
    std::normal_distribution<float> normal;
    std::uniform_int_distribution<uint32_t> any;
    for (size_t size : {2, 65, 66, 300, 512, 2048}) {
        auto row = [&](auto f) {
            std::vector<float> z(size);
            for (size_t i = 0; i < size; ++i) z[i] = f(i);
            return z;
        };
        for (bool half : {false, true}) {                         // (as numbers of 8 bits, too)
            auto each = [&](const char* name, auto f) { every_one(name, row([&](size_t i) { return half ? to_bf16(f(i)) : f(i); })); };
            each("normal", [&](size_t) { return 3.f * normal(rng); });
            // one logit in front of others that lie closer together than a difference to it is told in 64 bits
            for (float front : {1.f, 3e38f, 1e-3f, 0.f})
                for (float scale : {1e-20f, 1e-30f, 1e-37f, 1e-44f, 1e-10f}) {
                    each("one in front", [&](size_t i) { return i ? scale * normal(rng) : front; });
                    each("one in front of smaller ones", [&](size_t i) { return i ? -scale * std::fabs(normal(rng)) : front; });
                    each("two in front", [&](size_t i) { return i > 1 ? scale * normal(rng) : i ? front / 2 : front; });
                }
            each("half of them tiny", [&](size_t i) { return i & 1 ? normal(rng) : 1e-25f * normal(rng); });
            each("small whole numbers of the least", [&](size_t i) { return i ? (float)((int)(any(rng) % 2001) - 1000) * 1e-45f : 10.f; });
            each("a number and both zeros", [&](size_t i) { return i ? (i & 1 ? 0.f : -0.f) : 2.f; });
            each("zeros among tiny ones", [&](size_t i) { return i ? (i & 1 ? (i & 2 ? 0.f : -0.f) : 1e-20f * normal(rng)) : 2.f; });
            each("any size", [&](size_t) { return std::ldexp(normal(rng), (int)(any(rng) % 250) - 140); });
            each("powers of two", [&](size_t i) { return std::ldexp(i & 1 ? 1.f : -1.f, 100 - (int)(i % 249)); });
            each("masks", [&](size_t i) { return i % 3 ? normal(rng) : -3.4028235e38f; });
        }
    }
    if (failures) return std::printf("%d failures\n", failures), 1;
    std::printf("sample bins ok\n");
    return 0;
}
