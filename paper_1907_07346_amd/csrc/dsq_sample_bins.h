// How a wave divides the logits of a short row (ds_sample): plain arithmetic, so that a program on the host can go through the divisions of any row and see that they end.
#pragma once

#include <stdint.h>

namespace dsq {

constexpr uint32_t kWaveBins = 256;

// Bins of logits from lo to hi by their distance to the row's largest, which is what masses are made of too.  hi is in the first one and lo in the last, so that each of
// them has fewer logits than all have: unless the distances, in 64 bits, are the same (1, 1e-20 and 2e-20).  Such logits are divided no further: they are alike, have one
// mass and are kept by min_p together, so that only their order is left to tell one from another (NthKey).
struct LinearBins {
    double max, from, scale;
    constexpr double distance(float x) const { return max - (double)x; }
    constexpr bool alike(float lo, float hi) const { return distance(lo) == distance(hi); }
    constexpr void set(float lo, float hi) {                      // not alike
        from = distance(hi);
        scale = (kWaveBins - 0.5) / (distance(lo) - from);
    }
    constexpr uint32_t operator()(float x) const { return (uint32_t)((distance(x) - from) * scale); }
};

// The nth largest (from 1) of numbers from low to high, of which there are that many at least: tried() says up to which one to count, until done(), which 32 counts are enough for.
struct NthKey {
    uint32_t low, high;                                           // the last is low
    constexpr bool done() const { return low == high; }
    constexpr uint32_t tried() const { return low + (high - low) / 2 + ((high - low) & 1); }
    constexpr void counted(bool enough) {                          // n of the numbers from tried() on, or more
        if (enough) low = tried();
        else high = tried() - 1;
    }
};

}  // namespace dsq
