// Order keys of logits, and the grid on which sampling (sample.hip) counts them.  Plain arithmetic without a GPU's own functions: a
// host compiler that knows __device__ and __forceinline__ as macros reads this file too.
#pragma once

#include <math.h>
#include <stdint.h>

namespace sushi {

// Unsigned numbers in the order of the logits: larger = earlier.  NaN as -inf, -0 as 0.
constexpr uint32_t KEY_NONE = 0x007FFFFFu;  // of -inf: in no order
__device__ __forceinline__ uint32_t order_key(float z) {
    z = z == z ? z + 0.0f : -INFINITY;
    const uint32_t u = __builtin_bit_cast(uint32_t, z);
    return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float key_value(uint32_t k) { return __builtin_bit_cast(float, k & 0x80000000u ? k ^ 0x80000000u : ~k); }

constexpr int BINS = 1024;
constexpr double BINS_PER_LOG2 = 12.0;  // 1024: down to 2^-85 of the largest weight, the rest in the last one

// The grid: a logit lies in interval floor(place), counted downwards from the largest logit's.
struct Grid {
    double anchor, scale, top;  // place 0; intervals per unit of the logits; the largest logit's interval
    // (rounded by itself: fused with a subtraction it would be another number in each use)
    __device__ __forceinline__ double place(float z) const {
#ifdef __clang__
#pragma clang fp contract(off)
#endif
        return (anchor - (double)z) * scale;
    }
    __device__ __forceinline__ Grid(float best, double inv_t, double anchor_) : anchor(anchor_), scale(inv_t * (1.4426950408889634074 * BINS_PER_LOG2)) { top = floor(place(best)); }
};

// The lowest key in lowest .. highest for which below() holds, where it holds for all above one for which it does; highest if for
// none.  Next to the guess it is found with two calls; elsewhere by doubling steps away from the guess, then by halving: 64 at most.
template <typename F>
__device__ __forceinline__ uint32_t first_key(uint32_t guess, uint32_t lowest, uint32_t highest, F below) {
    uint32_t lo = guess < lowest ? lowest : guess > highest ? highest : guess, hi = lo;
    uint32_t step = 1;
    if (below(lo)) {
        for (;;) {  // below(hi)
            if (hi == lowest) return lowest;
            lo = hi - lowest > step ? hi - step : lowest;
            if (!below(lo)) break;
            hi = lo, step *= 2;
        }
    } else {
        for (;;) {  // not below(lo)
            if (lo == highest) return highest;
            hi = highest - lo > step ? lo + step : highest;
            if (below(hi)) break;
            lo = hi, step *= 2;
        }
    }
    while (hi - lo > 1) {
        const uint32_t middle = lo + (hi - lo) / 2;
        if (below(middle)) hi = middle; else lo = middle;
    }
    return hi;
}

// Key of the smallest logit in intervals 0 .. b.  unit: 1 / scale, about.  The guess is good to a key or two, but for a border next to
// logit 0: anchor - x * unit cancels there, and up to 1.3e9 keys lie between what is left of it, 1e-16 or 0, and the border.
template <typename G>
__device__ __forceinline__ uint32_t lowest_key(const G &grid, int b, float best, double unit) {
    const uint32_t lowest = KEY_NONE + 1;
    const double x = grid.top + (b + 1.0);
    if (b >= BINS - 1 || !(grid.scale > 0.0)) return lowest;
    const uint32_t guess = order_key((float)fmin(fmax(grid.anchor - x * unit, -3.4028234663852886e38), 3.4028234663852886e38));
    return first_key(guess, lowest, order_key(best), [&](uint32_t k) { return grid.place(key_value(k)) < x; });
}

}  // namespace sushi
